// C entry points of the join of a block to the residual stream and of dropout: argument checks and launches.
// Nothing here allocates, and no state is kept between calls.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "tok_host.h"
#include "tok_join.cuh"

using namespace pb;

namespace {

constexpr int64_t kMaxJoinDim = 16384, kMaxJoinRows = 1 << 30;
constexpr int kJoinTurns = 2;                   // chunks per worker of the backward, where gates are long enough

int refuse(const char* who, const char* what) {
    char text[256];
    snprintf(text, sizeof text, "%s: %s", who, what);
    return fail_text(PB_E_ARG, text);
}

// Threads of a row, eight columns each, or 16 in rows of more than `wide` columns: a power of two up to a warp, else whole warps.
int join_lanes(int64_t dim, int64_t wide, int& units) {
    units = dim > wide ? 2 : 1;
    const int64_t n = (dim + 8 * units - 1) / (8 * units);
    if (n > 32) return (int)((n + 31) / 32 * 32);
    int lanes = 1;
    while (lanes < n) lanes *= 2;
    return lanes;
}
// A block: rows of a warp or less share one.
int join_threads(int lanes) { return lanes > 32 ? lanes : kJoinThreads; }

constexpr int kRingBytes = 220 * 1024;          // of an SM, for the rings of all of its blocks
// Rows of a ring in shared memory, with so many blocks on an SM; below two the ring is no use.
int ring_depth(int row_bytes, int blocks) {
    return std::min(kJoinRing, kRingBytes / blocks / row_bytes);
}
// The limit of a kernel's shared memory is the same in every call: it belongs to the kernel, and another thread's call may come between this one's and its
// launch.
cudaError_t launch_ring(void (*kernel)(JoinParams), int blocks, int threads, size_t shared, cudaStream_t s, const JoinParams& p) {
    if (shared > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t c{};
    c.gridDim = dim3((unsigned)blocks);
    c.blockDim = dim3((unsigned)threads);
    c.dynamicSmemBytes = shared;
    c.stream = s;
    return cudaLaunchKernelEx(&c, (void (*)(const JoinParams))kernel, p);
}

struct JoinPlan {
    int lanes, units, threads, slots, blocks;
    int64_t rows_per_gate, chunk_rows, chunks_per_gate, chunks;
    float *pre, *post, *gate;
    size_t bytes;
};
JoinPlan join_plan(int64_t rows, int64_t dim, int64_t rows_per_gate, char* scratch) {
    JoinPlan e{};
    e.lanes = join_lanes(dim, 8192, e.units);
    e.threads = join_threads(e.lanes);
    e.slots = e.threads / e.lanes;
    e.rows_per_gate = rows_per_gate > 0 ? std::min(rows_per_gate, rows) : rows;
    const int64_t gate = e.rows_per_gate, most = kSms * std::max<int64_t>(1, 768 / e.threads), workers = most * e.slots;      // what is resident
    const int64_t want = std::max<int64_t>(1, (rows + workers * kJoinTurns - 1) / (workers * kJoinTurns));
    e.chunks_per_gate = gate > want ? (gate + want - 1) / want : 1;
    e.chunk_rows = (gate + e.chunks_per_gate - 1) / e.chunks_per_gate;
    e.chunks_per_gate = (gate + e.chunk_rows - 1) / e.chunk_rows;                  // none is empty
    const int64_t whole = rows / gate, rest = rows - whole * gate;
    e.chunks = whole * e.chunks_per_gate + (rest + e.chunk_rows - 1) / e.chunk_rows;
    e.blocks = (int)std::min<int64_t>(most, (e.chunks + e.slots - 1) / e.slots);
    size_t at = 0;
    auto take = [&](int64_t floats) {
        float* p = scratch ? (float*)(scratch + at) : nullptr;
        at += (size_t)(floats * 4 + 255) / 256 * 256;
        return p;
    };
    e.pre = take(e.blocks * dim);
    e.post = take(e.blocks * dim);
    if (rows_per_gate > 0 && e.chunks_per_gate > 1) e.gate = take(e.chunks * dim);
    e.bytes = at;
    return e;
}

// Scratch of a gradient of `rows` rows or fewer, which can need more: their chunks are shorter.
size_t join_bytes(int64_t rows, int64_t dim, int64_t rows_per_gate) {
    const JoinPlan e = join_plan(rows, dim, rows_per_gate, nullptr);
    const int64_t most = kSms * std::max<int64_t>(1, 768 / e.threads), blocks = std::min(most, (rows + e.slots - 1) / e.slots);
    const int64_t turns = most * e.slots * kJoinTurns;
    // Rows of n times `turns` come in chunks of n: as many as turns and one for each gate, no more than rows; none where a gate has no more than n.
    const int64_t split = rows_per_gate > 1 ? std::min(rows, std::min(rows_per_gate, rows) * turns) : 0;
    const int64_t chunks = split > 1 ? std::min(split, turns + (split + rows_per_gate - 1) / rows_per_gate) : 0;
    return (size_t)(2 * ((blocks * dim * 4 + 255) / 256 * 256) + (chunks * dim * 4 + 255) / 256 * 256);
}

// Share of the elements that is dropped, in units of 2^-16; false if p is no such share.
bool share_of(double p, unsigned& drop) {
    if (!(p >= 0.0) || !(p < 1.0)) return false;
    drop = (unsigned)std::nearbyint(p * 65536.0);
    return drop < 65536;
}
Keep keep_of(unsigned drop, uint64_t seed, int64_t offset, const int64_t* dev_offset) {
    return Keep{seed, offset, (const long long*)dev_offset, drop << 16, (float)(65536.0 / (65536.0 - drop))};
}

template <int L> using Layout = std::integral_constant<int, L>;
template <typename F> auto by_types(int dtype, int stream_dtype, F f) {
    using B = __nv_bfloat16;
    using H = __half;
    if (dtype == PB_F32) return f(float(), float());
    if (dtype == PB_BF16) return stream_dtype == PB_F32 ? f(B(), float()) : f(B(), B());
    return stream_dtype == PB_F32 ? f(H(), float()) : f(H(), H());
}

// What both directions ask of the arguments; NULL, or what is wrong.
const char* bad_join(const pb_join_args& a) {
    if (!dtype_ok(a.dtype) || !dtype_ok(a.stream_dtype) || !dtype_ok(a.weight_dtype)) return "unknown element type";
    if (a.stream_dtype != PB_F32 && a.stream_dtype != a.dtype) return "the residual stream is float32 or of the block's type";
    if (a.weight_dtype != PB_F32 && a.weight_dtype != a.dtype) return "the norms' weights are float32 or of the block's type";
    if (a.rows < 0 || a.rows > kMaxJoinRows) return "rows must be between 0 and 2^30";
    if (a.dim < 1 || a.dim > kMaxJoinDim) return "dim must be between 1 and 16384";
    if (a.gate && (a.rows_per_gate < 1 || a.rows_per_gate > kMaxCount)) return "rows_per_gate must be at least 1";
    if (a.gate && a.ld_gate < a.dim) return "a row stride is smaller than dim";
    if (!std::isfinite(a.residual_scale)) return "residual_scale must be finite";
    if (!(a.eps >= 0.f) || !std::isfinite(a.eps)) return "eps must not be negative";
    unsigned drop;
    if (!share_of(a.p, drop)) return "p must be at least 0 and round to less than 1 in units of 2^-16";
    if (!aligned(a.dev_offset, 8)) return "a pointer is not aligned to its element";
    return nullptr;
}

JoinParams params_of(const pb_join_args& a, int lanes) {
    JoinParams p{};
    p.rows = a.rows; p.dim = (int)a.dim; p.lanes = lanes;
    p.u = a.u; p.ld_u = a.ld_u;
    p.gate = a.gate; p.ld_gate = a.ld_gate;
    p.by_gate = Quotient(a.gate ? a.rows_per_gate : std::max<int64_t>(a.rows, 1));
    p.post = a.post_weight; p.pre = a.pre_weight;
    p.weights_f32 = a.weight_dtype == PB_F32;
    p.rstd_post = a.rstd_post; p.rstd_pre = a.rstd_pre;
    p.rs = a.residual_scale; p.eps = a.eps; p.inv_dim = (float)(1.0 / (double)a.dim);
    unsigned drop = 0;
    share_of(a.p, drop);
    p.keep = keep_of(drop, a.seed, a.offset, a.dev_offset);
    p.wait_ns = kTcWaitNs;
    return p;
}

struct Span {
    const void* p;
    size_t n;
    int64_t ld;
    int type;
};
bool same(const Span& a, const Span& b) { return a.p == b.p && a.ld == b.ld && a.type == b.type; }
bool meet(const Span& a, const Span& b) { return a.p && b.p && overlap(a.p, a.n, b.p, b.n); }

// Pieces of eight columns, each in one access.
bool piece_ok(const void* p, int64_t ld, int64_t rows, int type) {
    return !p || (aligned(p, 8 * dtype_bytes(type)) && (ld % 8 == 0 || rows <= 1));
}

}  // namespace

extern "C" {

int pb_dropout(const void* dev_x, int dtype, int64_t rows, int64_t dim, int64_t ld_x, double p, uint64_t seed, int64_t offset, const int64_t* dev_offset,
               void* dev_out, int64_t ld_out, void* stream) {
    const char* who = "pb_dropout";
    if (!dtype_ok(dtype)) return refuse(who, "unknown element type");
    if (rows < 0 || rows > kMaxCount || dim < 0 || dim > kMaxCount) return refuse(who, "sizes out of range");
    if (ld_x < dim || ld_out < dim) return refuse(who, "a row stride is smaller than dim");
    unsigned drop;
    if (!share_of(p, drop)) return refuse(who, "p must be at least 0 and round to less than 1 in units of 2^-16");
    if (rows == 0 || dim == 0) return PB_OK;
    if (!dev_x || !dev_out) return refuse(who, "NULL pointer");
    const size_t es = dtype_bytes(dtype);
    if (!aligned(dev_x, es) || !aligned(dev_out, es) || !aligned(dev_offset, 8)) return refuse(who, "a pointer is not aligned to its element");
    const Span x{dev_x, extent(rows, dim, ld_x, es), ld_x, dtype}, out{dev_out, extent(rows, dim, ld_out, es), ld_out, dtype};
    if (meet(x, out) && !same(x, out)) return refuse(who, "out overlaps x (the very same buffer and stride is allowed)");
    if (dev_offset && overlap(dev_out, out.n, dev_offset, 8)) return refuse(who, "out overlaps the offset");
    const bool dense = rows == 1 || (ld_x == dim && ld_out == dim);
    const int64_t n = rows * dim;
    const bool pieces = aligned(dev_x, 8 * es) && aligned(dev_out, 8 * es) && (dense || (dim % 8 == 0 && ld_x % 8 == 0 && ld_out % 8 == 0));
    const int64_t items = pieces ? std::max<int64_t>(n / 8, 1) : (n + 3) / 4;
    const dim3 grid((unsigned)std::min<int64_t>((items + kDropThreads - 1) / kDropThreads, kSms * 32));
    const Keep k = keep_of(drop, seed, offset, dev_offset);
    auto go = [&](auto t) {
        using T = decltype(t);
        return launch(pieces ? dropout_kernel<T, true> : dropout_kernel<T, false>, grid, kDropThreads, (cudaStream_t)stream, (const T*)dev_x, (T*)dev_out, n, dim,
                      ld_x, ld_out, dense, k);
    };
    return launched(who, dtype == PB_F32 ? go(float()) : dtype == PB_BF16 ? go(__nv_bfloat16()) : go(__half()));
}

size_t pb_join_scratch_bytes(int64_t rows, int64_t dim, int64_t rows_per_gate) {
    if (rows < 0 || rows > kMaxJoinRows || dim < 1 || dim > kMaxJoinDim || rows_per_gate < 0) return 0;
    return join_bytes(std::max<int64_t>(rows, 1), dim, rows_per_gate);
}

int pb_join_forward(const pb_join_args* args, void* stream) {
    const char* who = "pb_join_forward";
    if (!args) return refuse(who, "NULL pointer");
    const pb_join_args& a = *args;
    if (const char* bad = bad_join(a)) return refuse(who, bad);
    if (a.ld_x < a.dim || a.ld_u < a.dim || a.ld_y < a.dim || (a.h && a.ld_h < a.dim)) return refuse(who, "a row stride is smaller than dim");
    if (a.rows == 0) return PB_OK;
    if (!a.x || !a.u || !a.y) return refuse(who, "NULL pointer");
    if ((a.h != nullptr) != (a.pre_weight != nullptr)) return refuse(who, "h and pre_weight go together");
    const size_t es = dtype_bytes(a.dtype), ss = dtype_bytes(a.stream_dtype), ws = dtype_bytes(a.weight_dtype);
    if (!aligned(a.x, ss) || !aligned(a.u, es) || !aligned(a.y, ss) || !aligned(a.h, es) || !aligned(a.gate, es) || !aligned(a.post_weight, ws) ||
        !aligned(a.pre_weight, ws) || !aligned(a.rstd_post, 4) || !aligned(a.rstd_pre, 4)) return refuse(who, "a pointer is not aligned to its element");
    const int64_t gates = a.gate ? (a.rows + a.rows_per_gate - 1) / a.rows_per_gate : 0;
    const size_t nr = (size_t)a.rows * 4;
    const Span x{a.x, extent(a.rows, a.dim, a.ld_x, ss), a.ld_x, a.stream_dtype}, u{a.u, extent(a.rows, a.dim, a.ld_u, es), a.ld_u, a.dtype};
    const Span in[] = {x, u, {a.gate, extent(gates, a.dim, a.ld_gate, es), 0, 0}, {a.post_weight, (size_t)a.dim * ws, 0, 0},
                       {a.pre_weight, (size_t)a.dim * ws, 0, 0}, {a.dev_offset, 8, 0, 0}};
    const Span out[] = {{a.y, extent(a.rows, a.dim, a.ld_y, ss), a.ld_y, a.stream_dtype}, {a.h, extent(a.rows, a.dim, a.ld_h, es), a.ld_h, a.dtype},
                        {a.rstd_post, nr, 0, -1}, {a.rstd_pre, nr, 0, -1}};
    for (int k = 0; k < 4; ++k) {
        for (int l = 0; l < 6; ++l)
            if (meet(out[k], in[l]) && !(k == l && k < 2 && same(out[k], in[l]))) return refuse(who, "an output overlaps an input (y may be x, h may be u)");
        for (int l = 0; l < k; ++l)
            if (meet(out[k], out[l])) return refuse(who, "two outputs overlap");
    }
    int units;
    // 16 columns per thread where that leaves every SM as many threads as it holds: half the instructions that a row's sums take.
    const int lanes = join_lanes(a.dim, a.rows * a.dim >= (int64_t)kSms * 1024 * 16 && a.dim >= 512 ? 511 : 8192, units);
    const int threads = join_threads(lanes);
    JoinParams p = params_of(a, lanes);
    p.x = a.x; p.ld_x = a.ld_x;
    p.y = a.y; p.ld_y = a.ld_y;
    p.h = a.h; p.ld_h = a.ld_h;
    const bool pieces = a.dim % 8 == 0 && piece_ok(a.x, a.ld_x, a.rows, a.stream_dtype) && piece_ok(a.u, a.ld_u, a.rows, a.dtype) &&
                        piece_ok(a.y, a.ld_y, a.rows, a.stream_dtype) && piece_ok(a.h, a.ld_h, a.rows, a.dtype) && piece_ok(a.gate, a.ld_gate, gates, a.dtype) &&
                        piece_ok(a.post_weight, 0, 1, a.weight_dtype) && piece_ok(a.pre_weight, 0, 1, a.weight_dtype);
    const int64_t slots = threads / lanes;
    bool ring = false;
    if (pieces && units == 2 && slots == 1) {
        p.row_bytes = (int)((a.dim * (ss + (a.gate ? 2 : 1) * es) + 127) / 128 * 128);
        p.depth = ring_depth(p.row_bytes, std::max(1, 512 / threads));
        // A plain sum with one norm is as fast as memory without (16384 x 4096: 84 us, 99 in the ring; with a norm behind the block 95 and 86, with
        // a gate and dropout too 120 and 116).
        ring = p.depth > 1 && a.rows >= 4 * kSms && (a.post_weight || a.gate);
    }
    const dim3 grid((unsigned)((a.rows + slots - 1) / slots));
    return launched(who, by_types(a.dtype, a.stream_dtype, [&](auto t, auto st) {
        using T = decltype(t);
        using S = decltype(st);
        if (ring) {
            auto in_ring = [&](auto l) {
                constexpr int L = decltype(l)::value;
                return threads <= 256 ? join_forward_ring_kernel<T, S, L, 256> : threads <= 512 ? join_forward_ring_kernel<T, S, L, 512> : join_forward_ring_kernel<T, S, L, 1024>;
            };
            auto kernel = a.dim == 16 * lanes ? in_ring(Layout<kFull>()) : in_ring(Layout<kEven>());
            const int64_t blocks = std::min(a.rows, kSms * std::max<int64_t>(1, 512 / threads));
            return launch_ring(kernel, (int)blocks, threads, p.depth * p.row_bytes, (cudaStream_t)stream, p);
        }
        auto by_layout = [&](auto l) {
            constexpr int L = decltype(l)::value;
            return units == 1 ? join_forward_kernel<T, S, L, 1> : join_forward_kernel<T, S, L, 2>;
        };
        return launch(pieces ? by_layout(Layout<kEven>()) : by_layout(Layout<kOdd>()), grid, threads, (cudaStream_t)stream, p);
    }));
}

int pb_join_backward(const pb_join_args* args, const pb_join_grads* grads, void* dev_scratch, size_t scratch_bytes, void* stream) {
    const char* who = "pb_join_backward";
    if (!args || !grads) return refuse(who, "NULL pointer");
    const pb_join_args& a = *args;
    const pb_join_grads& d = *grads;
    if (const char* bad = bad_join(a)) return refuse(who, bad);
    if (!dtype_ok(d.dweight_dtype) || (d.dweight_dtype != PB_F32 && d.dweight_dtype != a.dtype) || !dtype_ok(d.dgate_dtype) ||
        (d.dgate_dtype != PB_F32 && d.dgate_dtype != a.dtype)) return refuse(who, "gradients of weights and gates are float32 or of the block's type");
    if (a.ld_u < a.dim || d.ld_du < a.dim || (d.dx && d.ld_dx < a.dim) || (d.dy && d.ld_dy < a.dim) || (d.dh && (d.ld_dh < a.dim || a.ld_y < a.dim)) ||
        (d.dgate && d.ld_dgate < a.dim)) return refuse(who, "a row stride is smaller than dim");
    if (a.rows > 0) {                           // no rows may have no addresses
        if ((d.dgate && !a.gate) || (d.dpost_weight && !a.post_weight) || (d.dpre_weight && !d.dh))
            return refuse(who, "a gradient is asked for of what the join does not have");
        if (!a.u || !d.du || !dev_scratch) return refuse(who, "NULL pointer");
        if (!d.dy && !d.dh) return refuse(who, "neither dy nor dh is given");
        if (d.dh && (!a.y || !a.pre_weight || !a.rstd_pre)) return refuse(who, "dh needs y, pre_weight and rstd_pre");
        if (a.post_weight && !a.rstd_post) return refuse(who, "a post-norm needs rstd_post");
    }
    const size_t es = dtype_bytes(a.dtype), ss = dtype_bytes(a.stream_dtype), ws = dtype_bytes(a.weight_dtype), gw = dtype_bytes(d.dweight_dtype),
                 gg = dtype_bytes(d.dgate_dtype);
    if (!aligned(a.y, ss) || !aligned(a.u, es) || !aligned(a.gate, es) || !aligned(a.post_weight, ws) || !aligned(a.pre_weight, ws) ||
        !aligned(a.rstd_post, 4) || !aligned(a.rstd_pre, 4) || !aligned(d.dy, ss) || !aligned(d.dh, es) || !aligned(d.dx, ss) || !aligned(d.du, es) ||
        !aligned(d.dgate, gg) || !aligned(d.dpost_weight, gw) || !aligned(d.dpre_weight, gw)) return refuse(who, "a pointer is not aligned to its element");
    const cudaStream_t s = (cudaStream_t)stream;
    if (a.rows == 0) {                          // sums over no rows
        cudaError_t err = d.dpre_weight ? cudaMemsetAsync(d.dpre_weight, 0, (size_t)a.dim * gw, s) : cudaSuccess;
        if (d.dpost_weight && err == cudaSuccess) err = cudaMemsetAsync(d.dpost_weight, 0, (size_t)a.dim * gw, s);
        return launched(who, err);
    }
    if (!aligned(dev_scratch, 256)) return refuse(who, "scratch must be 256-byte aligned");
    const JoinPlan e = join_plan(a.rows, a.dim, a.gate ? a.rows_per_gate : 0, (char*)dev_scratch);
    if (scratch_bytes < std::max(e.bytes, join_bytes(a.rows, a.dim, a.gate ? a.rows_per_gate : 0))) return refuse(who, "scratch is smaller than pb_join_scratch_bytes");
    const int64_t gates = a.gate ? (a.rows + a.rows_per_gate - 1) / a.rows_per_gate : 0;
    const size_t nr = (size_t)a.rows * 4, nw = (size_t)a.dim * ws;
    const Span in[] = {{d.dy, extent(a.rows, a.dim, d.ld_dy, ss), d.ld_dy, a.stream_dtype}, {d.dh, extent(a.rows, a.dim, d.ld_dh, es), d.ld_dh, a.dtype},
                       {d.dh ? a.y : nullptr, extent(a.rows, a.dim, a.ld_y, ss), 0, 0}, {a.u, extent(a.rows, a.dim, a.ld_u, es), 0, 0},
                       {a.gate, extent(gates, a.dim, a.ld_gate, es), 0, 0}, {a.post_weight, nw, 0, 0}, {a.pre_weight, nw, 0, 0}, {a.rstd_post, nr, 0, 0},
                       {a.rstd_pre, nr, 0, 0}, {a.dev_offset, 8, 0, 0}};
    const Span out[] = {{d.dx, extent(a.rows, a.dim, d.ld_dx, ss), d.ld_dx, a.stream_dtype}, {d.du, extent(a.rows, a.dim, d.ld_du, es), d.ld_du, a.dtype},
                        {d.dgate, extent(gates, a.dim, d.ld_dgate, gg), 0, -1}, {d.dpost_weight, (size_t)a.dim * gw, 0, -1},
                        {d.dpre_weight, (size_t)a.dim * gw, 0, -1}, {dev_scratch, scratch_bytes, 0, -1}};
    for (int k = 0; k < 6; ++k) {
        for (int l = 0; l < 10; ++l)
            if (meet(out[k], in[l]) && !(k == l && k < 2 && same(out[k], in[l]))) return refuse(who, "an output overlaps an input (dx may be dy, du may be dh)");
        for (int l = 0; l < k; ++l)
            if (meet(out[k], out[l])) return refuse(who, "two outputs overlap");
    }
    JoinParams p = params_of(a, e.lanes);
    p.yin = a.y; p.ld_y = a.ld_y;
    p.dy = d.dy; p.ld_dy = d.ld_dy;
    p.dh = d.dh; p.ld_dh = d.ld_dh;
    p.dx = d.dx; p.ld_dx = d.ld_dx;
    p.du = d.du; p.ld_du = d.ld_du;
    p.rows_per_gate = (int)e.rows_per_gate;
    p.chunk_rows = (int)e.chunk_rows; p.chunks_per_gate = (int)e.chunks_per_gate; p.chunks = (int)e.chunks;
    p.by_chunks = Quotient(e.chunks_per_gate);
    p.dgate = d.dgate; p.ld_dgate = d.ld_dgate;
    p.dgate_f32 = d.dgate_dtype == PB_F32;
    p.gate_part = e.gate;
    p.part_pre = d.dpre_weight ? e.pre : nullptr;
    p.part_post = d.dpost_weight ? e.post : nullptr;
    const bool pieces = a.dim % 8 == 0 && piece_ok(d.dh ? a.y : nullptr, a.ld_y, a.rows, a.stream_dtype) && piece_ok(a.u, a.ld_u, a.rows, a.dtype) &&
                        piece_ok(d.dy, d.ld_dy, a.rows, a.stream_dtype) && piece_ok(d.dh, d.ld_dh, a.rows, a.dtype) &&
                        piece_ok(d.dx, d.ld_dx, a.rows, a.stream_dtype) && piece_ok(d.du, d.ld_du, a.rows, a.dtype) &&
                        piece_ok(a.gate, a.ld_gate, gates, a.dtype) && piece_ok(d.dgate, d.ld_dgate, gates, d.dgate_dtype) &&
                        piece_ok(a.post_weight, 0, 1, a.weight_dtype) && piece_ok(a.pre_weight, 0, 1, a.weight_dtype);
    size_t shared = e.slots > 1 ? (size_t)e.threads * 8 * e.units * 4 : 0;
    bool ring = false;
    if (pieces && e.slots == 1) {
        p.row_bytes = (int)((a.dim * (2 * ss + 3 * es) + 127) / 128 * 128);
        p.depth = ring_depth(p.row_bytes, std::max(1, 512 / e.threads));
        ring = p.depth > 1;
        if (ring) shared = (size_t)p.depth * p.row_bytes;
    }
    return launched(who, by_types(a.dtype, a.stream_dtype, [&](auto t, auto st) {
        using T = decltype(t);
        using S = decltype(st);
        auto by_layout = [&](auto l) {
            constexpr int L = decltype(l)::value;
            if (e.threads <= 256) return join_backward_kernel<T, S, L, 1, 256>;
            if (e.threads <= 512) return join_backward_kernel<T, S, L, 1, 512>;
            return e.units == 1 ? join_backward_kernel<T, S, L, 1, 1024> : join_backward_kernel<T, S, L, 2, 1024>;
        };
        auto in_ring = [&](auto l) {
            constexpr int L = decltype(l)::value;
            if (e.threads <= 256) return join_backward_ring_kernel<T, S, L, 1, 256>;
            if (e.threads <= 512) return join_backward_ring_kernel<T, S, L, 1, 512>;
            return e.units == 1 ? join_backward_ring_kernel<T, S, L, 1, 1024> : join_backward_ring_kernel<T, S, L, 2, 1024>;
        };
        auto kernel = ring ? (a.dim == 8 * e.units * e.lanes ? in_ring(Layout<kFull>()) : in_ring(Layout<kEven>())) : pieces ? by_layout(Layout<kEven>())
                                                                                                                       : by_layout(Layout<kOdd>());
        const int blocks = ring ? std::min(e.blocks, kSms * std::max(1, 512 / e.threads)) : e.blocks;      // what is resident
        cudaError_t err = launch_ring(kernel, blocks, e.threads, shared, s, p);
        const int first = p.part_pre || p.part_post ? 0 : 2;
        const int64_t jobs = 2 - first + (d.dgate && e.gate ? gates : 0);
        if (jobs > 0 && err == cudaSuccess)
            err = launch_after(join_sum_kernel<T>, dim3((unsigned)jobs, (unsigned)((a.dim + kJoinSumColumns - 1) / kJoinSumColumns)),
                               kJoinSumColumns * kJoinSumShares, s, p.part_pre, p.part_post, blocks, e.gate, e.chunks_per_gate, e.chunks, (int)a.dim,
                               d.dpre_weight, d.dpost_weight, d.dweight_dtype == PB_F32, d.dgate, d.ld_dgate, d.dgate_dtype == PB_F32, first);
        return err;
    }));
}

}  // extern "C"
