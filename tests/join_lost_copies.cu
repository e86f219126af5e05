// The joins' ring kernels with a limit of the caller's for their waits: 0 is a copy that never comes in time.
// The copies themselves are the kernels' own, in bounds, and land before the kernels end.
#include <cmath>

#include "../paper_2003_11666_b200/csrc/tok_join.cuh"

using namespace pb;
using B = __nv_bfloat16;

namespace {
constexpr int kThreads = 256, kDepth = 3;
template <typename K> int go(K kernel, int blocks, int bytes, const JoinParams& p) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 * 1024);
    if (e != cudaSuccess) return (int)e;
    kernel<<<blocks, kThreads, bytes>>>(p);
    e = cudaGetLastError();
    return (int)(e != cudaSuccess ? e : cudaDeviceSynchronize());
}
JoinParams base(int rows, int dim, const void* u, const float* post, const float* pre, float* rstd_post, float* rstd_pre, long long wait_ns) {
    JoinParams p{};
    p.rows = rows; p.dim = dim; p.lanes = kThreads;
    p.u = u; p.ld_u = dim;
    p.by_gate = Quotient(rows);
    p.post = post; p.pre = pre; p.weights_f32 = true;
    p.rstd_post = rstd_post; p.rstd_pre = rstd_pre;
    p.rs = 1.f; p.eps = 1e-6f; p.inv_dim = (float)(1.0 / dim);
    p.keep.scale = 1.f;
    p.depth = kDepth;
    p.wait_ns = wait_ns;
    return p;
}
}  // namespace

// x, u, y, h: bfloat16 [rows, 4096]; post and pre may be NULL (pre and h together).
extern "C" int forward(int rows, int blocks, const void* x, const void* u, const float* post, const float* pre, void* y, void* h, float* rstd_post, float* rstd_pre,
                       long long wait_ns) {
    constexpr int dim = 16 * kThreads;
    JoinParams p = base(rows, dim, u, post, pre, rstd_post, rstd_pre, wait_ns);
    p.x = x; p.ld_x = dim;
    p.y = y; p.ld_y = dim;
    p.h = h; p.ld_h = dim;
    p.row_bytes = dim * 4;
    return go(join_forward_ring_kernel<B, B, kFull, kThreads>, blocks, kDepth * p.row_bytes, p);
}

// u, y, dy, dh, dx, du: bfloat16 [rows, 2048]; gate, dgate: [2048] or NULL; part_pre, part_post: float32 [blocks, 2048].
// One chunk of rows for each block, and of all rows for the gate's sums where there is a single block.
extern "C" int backward(int rows, int blocks, const void* u, const void* y, const void* dy, const void* dh, const void* gate, const float* post, const float* pre,
                        float* rstd_post, float* rstd_pre, void* dx, void* du, void* dgate, float* part_pre, float* part_post, long long wait_ns) {
    constexpr int dim = 8 * kThreads;
    JoinParams p = base(rows, dim, u, post, pre, rstd_post, rstd_pre, wait_ns);
    p.yin = y; p.ld_y = dim;
    p.dy = dy; p.ld_dy = dim;
    p.dh = dh; p.ld_dh = dim;
    p.dx = dx; p.ld_dx = dim;
    p.du = du; p.ld_du = dim;
    p.gate = gate; p.ld_gate = dim;
    p.dgate = dgate; p.ld_dgate = dim;
    p.rows_per_gate = rows;
    p.chunk_rows = (rows + blocks - 1) / blocks;
    p.chunks = p.chunks_per_gate = (rows + p.chunk_rows - 1) / p.chunk_rows;
    if (p.chunks != blocks) return -1;
    p.by_chunks = Quotient(p.chunks_per_gate);
    p.part_pre = part_pre; p.part_post = part_post;
    p.row_bytes = dim * 10;
    return go(join_backward_ring_kernel<B, B, kFull, 1, kThreads>, blocks, kDepth * p.row_bytes, p);
}
