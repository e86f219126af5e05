// The join of a block to the residual stream, with the norms around it, and dropout.
//
//   b = u rstd_post post          rstd_post = (mean u^2 + eps)^-1/2      (b = u without a post-norm)
//   y = residual_scale x + keep gate b                                   keep: 0, or 1 / (1 - p)
//   h = y rstd_pre pre            rstd_pre  = (mean y^2 + eps)^-1/2
//
// and its gradient, with yn = y rstd_pre, un = u rstd_post:
//   dy' = dy + rstd_pre (dh pre - yn mean(dh pre yn))        dx = residual_scale dy'     dpre = sum_t dh yn
//   db  = keep dy'          dgate = sum over its rows of db un post                      dpost = sum_t db gate un
//   du  = rstd_post (db gate post - un mean(db gate post un))
//
// Everything is bound by the rows' bytes.  A row is held in registers by a group of threads (a power of two, kUnits pieces
// of eight columns each), so that it is read and written once; its two sums are the only thing that the threads of a
// group exchange.  In the backward a thread keeps the same columns in every row, so that the sums over rows
// stay in its registers; they end in one partial sum per block, and in one per chunk of rows that share a gate.
#pragma once
#include "tok_common.cuh"

namespace pb {

// ------------------------------------------------------------------ which elements are kept
// Element i of a call's [rows, dim] values (i = row * dim + column) has bits 16 (i mod 4) .. + 15 of the hash of counter i / 4 on the
// stream that (seed, offset) name; it is kept where they are at least `drop`.
struct Keep {
    unsigned long long seed;
    long long offset;
    const long long* dev_offset;
    unsigned drop;               // of 65536
    float scale;                 // 65536 / (65536 - drop)
};
__device__ __forceinline__ unsigned long long keep_base(const Keep& k) {
    return splitmix64(k.seed, (unsigned long long)(k.dev_offset ? *k.dev_offset : k.offset));
}
__device__ __forceinline__ void keep4(float (&f)[4], unsigned long long base, unsigned long long quad, const Keep& k) {
    const unsigned long long z = splitmix64(base, quad);
    const unsigned lo = (unsigned)z, hi = (unsigned)(z >> 32);
    f[0] = (lo & 0xffffu) >= k.drop ? k.scale : 0.f;
    f[1] = (lo >> 16) >= k.drop ? k.scale : 0.f;
    f[2] = (hi & 0xffffu) >= k.drop ? k.scale : 0.f;
    f[3] = (hi >> 16) >= k.drop ? k.scale : 0.f;
}

__device__ __forceinline__ void load_piece(float (&x)[8], const float* p) { load8_wide(x, p); }
template <typename T> __device__ __forceinline__ void load_piece(float (&x)[8], const T* p) { load8(x, p); }
__device__ __forceinline__ void store_piece(float* p, const float (&x)[8]) { store8_wide(p, x); }
template <typename T> __device__ __forceinline__ void store_piece(T* p, const float (&x)[8]) { store8(p, x); }

// What is dropped is zero, whatever it was.
__device__ __forceinline__ float kept(float f, float x) { return f != 0.f ? f * x : 0.f; }

constexpr int kDropThreads = 256;

// kDense: the rows follow each other without a gap, the whole is one row.  kPieces: eight elements at a time.
template <typename T, bool kPieces>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(const T* x, T* out, long long n, long long cols, long long ld_x, long long ld_out, bool dense, Keep k) {
    const unsigned long long base = keep_base(k);
    const long long step = (long long)gridDim.x * kDropThreads;
    if (kPieces) {
        for (long long i = blockIdx.x * (long long)kDropThreads + threadIdx.x; i < n / 8; i += step) {
            const long long r = dense ? 0 : i * 8 / cols, c = i * 8 - r * cols;
            float v[8], f[4], g[4];
            load_piece(v, x + r * ld_x + c);
            keep4(f, base, 2 * i, k);
            keep4(g, base, 2 * i + 1, k);
#pragma unroll
            for (int u = 0; u < 4; ++u) { v[u] = kept(f[u], v[u]); v[u + 4] = kept(g[u], v[u + 4]); }
            store_piece(out + r * ld_out + c, v);
        }
        if (blockIdx.x == 0 && threadIdx.x < n % 8) {         // dense only
            const long long i = n / 8 * 8 + threadIdx.x;
            float f[4];
            keep4(f, base, i / 4, k);
            out[i] = from_f32<T>(kept(i % 4 == 0 ? f[0] : i % 4 == 1 ? f[1] : i % 4 == 2 ? f[2] : f[3], to_f32(x[i])));
        }
        return;
    }
    for (long long q = blockIdx.x * (long long)kDropThreads + threadIdx.x; q < (n + 3) / 4; q += step) {
        float f[4];
        keep4(f, base, q, k);
        long long r = dense ? 0 : q * 4 / cols, c = q * 4 - r * cols;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (q * 4 + u < n) out[r * ld_out + c] = from_f32<T>(kept(f[u], to_f32(x[r * ld_x + c])));
            if (!dense && ++c == cols) { c = 0; ++r; }
            else if (dense) ++c;
        }
    }
}

// ------------------------------------------------------------------ join
struct JoinParams {
    long long rows;
    int dim, lanes;              // threads of a row: a power of two
    const void *x, *u, *gate, *post, *pre, *yin, *dy, *dh;
    void *y, *h, *dx, *du;
    long long ld_x, ld_u, ld_y, ld_h, ld_gate, ld_dy, ld_dh, ld_dx, ld_du, ld_dgate;
    float *rstd_post, *rstd_pre;
    bool weights_f32;            // else of u's type
    long long rows_per_gate;
    float rs, eps, inv_dim;
    Keep keep;                   // drop == 0: everything is kept
    // backward: chunks of rows that share a gate
    long long chunk_rows, chunks_per_gate, chunks;
    float* gate_part;            // [chunks][dim], or NULL: a chunk is all rows of its gate, and written to dgate
    void* dgate;
    bool dgate_f32;
    float *part_pre, *part_post; // [blocks][dim], or NULL
};

constexpr int kJoinThreads = 256;             // of a block, or the threads of a row if those are more
constexpr int kJoinMaxLanes = 1024;

// Sum over the threads of a row.  Rows of more than a warp meet in shared memory: all threads of the block call this.
__device__ __forceinline__ float row_sum(float v, int lanes, float* sm) {
    for (int k = min(lanes, 32) / 2; k; k /= 2) v += __shfl_xor_sync(0xffffffffu, v, k);
    if (lanes <= 32) return v;
    const int warp = threadIdx.x / 32, n = lanes / 32, first = warp / n * n;
    if (threadIdx.x % 32 == 0) sm[warp] = v;
    __syncthreads();
    const int l = threadIdx.x % 32;
    v = l < n ? sm[first + l] : 0.f;
#pragma unroll
    for (int k = 16; k; k /= 2) v += __shfl_xor_sync(0xffffffffu, v, k);
    return v;
}

// Eight columns of a row: in pieces consecutive ones, else `lanes` apart, so that neighbours read neighbours.
template <bool kPieces>
struct Columns {
    int first, step, n;          // n: how many exist
    __device__ __forceinline__ Columns(int lane, int unit, int lanes, int dim) {
        first = kPieces ? (unit * lanes + lane) * 8 : unit * 8 * lanes + lane;
        step = kPieces ? 1 : lanes;
        n = first >= dim ? 0 : min(8, (dim - first + step - 1) / step);
    }
    template <typename T> __device__ __forceinline__ void load(float (&v)[8], const T* row) const {
        if (kPieces) {
            if (n) load_piece(v, row + first);
            else
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = 0.f;
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = k < n ? to_f32(row[first + k * step]) : 0.f;
        }
    }
    template <typename T> __device__ __forceinline__ void store(T* row, const float (&v)[8]) const {
        if (kPieces) {
            if (n) store_piece(row + first, v);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < n) row[first + k * step] = from_f32<T>(v[k]);
        }
    }
    __device__ __forceinline__ void keep(float (&f)[8], unsigned long long base, long long row, int dim, const Keep& k) const {
        if (kPieces) {                                       // dim is a multiple of 8
            const unsigned long long q = ((unsigned long long)row * dim + first) / 4;
            float a[4], b[4];
            keep4(a, base, q, k);
            keep4(b, base, q + 1, k);
#pragma unroll
            for (int u = 0; u < 4; ++u) { f[u] = a[u]; f[u + 4] = b[u]; }
        } else {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const unsigned long long i = (unsigned long long)row * dim + first + u * step;
                const unsigned long long z = splitmix64(base, i / 4);
                f[u] = (unsigned)(z >> (16 * (i % 4)) & 0xffffu) >= k.drop ? k.scale : 0.f;
            }
        }
    }
};

template <bool kPieces, typename T>
__device__ __forceinline__ void load_weight(float (&v)[8], const Columns<kPieces>& c, const void* w, bool f32) {
    if (f32) c.load(v, (const float*)w); else c.load(v, (const T*)w);
}

template <typename T, typename S, bool kPieces, int kUnits>
__global__ void __launch_bounds__(kJoinMaxLanes) join_forward_kernel(const JoinParams p) {
    __shared__ float sm[2][32];
    const int lane = threadIdx.x % p.lanes, slot = threadIdx.x / p.lanes, slots = blockDim.x / p.lanes;
    const unsigned long long base = p.keep.drop ? keep_base(p.keep) : 0;
    const long long r = (long long)blockIdx.x * slots + slot;
    const bool live = r < p.rows;
    float y[kUnits][8], b[kUnits][8];
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        Columns<kPieces> c(lane, k, p.lanes, p.dim);
        if (!live) c.n = 0;
        c.load(y[k], (const S*)p.x + r * p.ld_x);
        c.load(b[k], (const T*)p.u + r * p.ld_u);
#pragma unroll
        for (int u = 0; u < 8; ++u) sum = fmaf(b[k][u], b[k][u], sum);
    }
    float rstd = 1.f;
    if (p.post) {
        rstd = 1.f / sqrtf(fmaf(row_sum(sum, p.lanes, sm[0]), p.inv_dim, p.eps));
        if (live && lane == 0 && p.rstd_post) p.rstd_post[r] = rstd;
    }
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        Columns<kPieces> c(lane, k, p.lanes, p.dim);
        if (!live) c.n = 0;
        float v[8];
        if (p.post) {
            load_weight<kPieces, T>(v, c, p.post, p.weights_f32);
#pragma unroll
            for (int u = 0; u < 8; ++u) b[k][u] = b[k][u] * rstd * v[u];
        }
        if (p.gate) {
            c.load(v, (const T*)p.gate + (live ? r / p.rows_per_gate : 0) * p.ld_gate);
#pragma unroll
            for (int u = 0; u < 8; ++u) b[k][u] *= v[u];
        }
        if (p.keep.drop) {
            c.keep(v, base, r, p.dim, p.keep);
#pragma unroll
            for (int u = 0; u < 8; ++u) b[k][u] = kept(v[u], b[k][u]);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            y[k][u] = fmaf(p.rs, y[k][u], b[k][u]);
            sum = fmaf(y[k][u], y[k][u], sum);               // columns that do not exist are zero
        }
        c.store((S*)p.y + r * p.ld_y, y[k]);
    }
    if (!p.h) return;
    rstd = 1.f / sqrtf(fmaf(row_sum(sum, p.lanes, sm[1]), p.inv_dim, p.eps));
    if (!live) return;
    if (lane == 0 && p.rstd_pre) p.rstd_pre[r] = rstd;
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        const Columns<kPieces> c(lane, k, p.lanes, p.dim);
        float v[8];
        load_weight<kPieces, T>(v, c, p.pre, p.weights_f32);
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] *= y[k][u] * rstd;
        c.store((T*)p.h + r * p.ld_h, v);
    }
}

template <typename T, typename S, bool kPieces, int kUnits, int kThreads>
__global__ void __launch_bounds__(kThreads) join_backward_kernel(const JoinParams p) {
    extern __shared__ float cross[];             // [slots][lanes * 8 * kUnits]
    __shared__ float sm[2][2][32];
    const int lane = threadIdx.x % p.lanes, slot = threadIdx.x / p.lanes, slots = blockDim.x / p.lanes;
    const unsigned long long base = p.keep.drop ? keep_base(p.keep) : 0;
    const long long workers = (long long)gridDim.x * slots;
    float dpre[kUnits][8] = {}, dpost[kUnits][8] = {}, dgate[kUnits][8] = {};
    int turn = 0;
    // every worker takes as many turns, so that the threads of a block meet in row_sum
    for (long long k0 = 0; k0 < p.chunks; k0 += workers) {
        const long long chunk = k0 + (long long)blockIdx.x * slots + slot;
        const long long group = chunk / p.chunks_per_gate;
        const long long first = group * p.rows_per_gate + (chunk - group * p.chunks_per_gate) * p.chunk_rows;
        const long long last = chunk < p.chunks ? min(min(first + p.chunk_rows, (group + 1) * p.rows_per_gate), p.rows) : first;
        for (long long q = 0; q < p.chunk_rows; ++q, turn ^= 1) {
            const long long r = first + q;
            const bool live = r < last;
            const float rp = live && p.post ? p.rstd_post[r] : 1.f, rr = live && p.dh ? p.rstd_pre[r] : 0.f;
            float g[kUnits][8], un[kUnits][8], yn[kUnits][8], w[kUnits][8];
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                Columns<kPieces> c(lane, k, p.lanes, p.dim);
                if (!live) c.n = 0;
                c.load(un[k], (const T*)p.u + r * p.ld_u);
                if (p.dy) c.load(g[k], (const S*)p.dy + r * p.ld_dy);
                else
#pragma unroll
                    for (int u = 0; u < 8; ++u) g[k][u] = 0.f;
                if (p.dh) {
                    float v[8];
                    c.load(yn[k], (const S*)p.yin + r * p.ld_y);
                    c.load(w[k], (const T*)p.dh + r * p.ld_dh);
                    load_weight<kPieces, T>(v, c, p.pre, p.weights_f32);
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        yn[k][u] *= rr;
                        dpre[k][u] = fmaf(w[k][u], yn[k][u], dpre[k][u]);
                        w[k][u] *= v[u];
                        sum = fmaf(w[k][u], yn[k][u], sum);
                    }
                }
            }
            if (p.dh) {
                const float m = row_sum(sum, p.lanes, sm[turn][0]) * p.inv_dim;
#pragma unroll
                for (int k = 0; k < kUnits; ++k)
#pragma unroll
                    for (int u = 0; u < 8; ++u) g[k][u] = fmaf(rr, fmaf(-m, yn[k][u], w[k][u]), g[k][u]);
            }
            sum = 0.f;
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                Columns<kPieces> c(lane, k, p.lanes, p.dim);
                if (!live) c.n = 0;
                float v[8];
                if (p.dx) {
#pragma unroll
                    for (int u = 0; u < 8; ++u) v[u] = p.rs * g[k][u];
                    c.store((S*)p.dx + r * p.ld_dx, v);
                }
                if (p.keep.drop) {
                    c.keep(v, base, r, p.dim, p.keep);
#pragma unroll
                    for (int u = 0; u < 8; ++u) g[k][u] = kept(v[u], g[k][u]);
                }
                float post[8];
                if (p.post) {
                    load_weight<kPieces, T>(post, c, p.post, p.weights_f32);
#pragma unroll
                    for (int u = 0; u < 8; ++u) un[k][u] *= rp;
                }
                if (p.gate) {
                    c.load(v, (const T*)p.gate + (live ? group : 0) * p.ld_gate);
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        dgate[k][u] = fmaf(g[k][u], p.post ? un[k][u] * post[u] : un[k][u], dgate[k][u]);
                        g[k][u] *= v[u];
                    }
                }
                if (p.post) {
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        dpost[k][u] = fmaf(g[k][u], un[k][u], dpost[k][u]);
                        g[k][u] *= post[u];
                        sum = fmaf(g[k][u], un[k][u], sum);
                    }
                }
            }
            float m = 0.f;
            if (p.post) m = row_sum(sum, p.lanes, sm[turn][1]) * p.inv_dim;
            if (live) {
#pragma unroll
                for (int k = 0; k < kUnits; ++k) {
                    const Columns<kPieces> c(lane, k, p.lanes, p.dim);
                    if (p.post) {
#pragma unroll
                        for (int u = 0; u < 8; ++u) g[k][u] = rp * fmaf(-m, un[k][u], g[k][u]);
                    }
                    c.store((T*)p.du + r * p.ld_du, g[k]);
                }
            }
        }
        if (p.dgate && chunk < p.chunks) {
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                const Columns<kPieces> c(lane, k, p.lanes, p.dim);
                if (p.gate_part) c.store(p.gate_part + chunk * p.dim, dgate[k]);
                else if (p.dgate_f32) c.store((float*)p.dgate + group * p.ld_dgate, dgate[k]);
                else c.store((T*)p.dgate + group * p.ld_dgate, dgate[k]);
#pragma unroll
                for (int u = 0; u < 8; ++u) dgate[k][u] = 0.f;
            }
        }
    }
    // the block's sums over its rows: its slots, in their order
    for (int which = 0; which < 2; ++which) {
        float* part = which ? p.part_post : p.part_pre;
        if (!part) continue;
        part += (long long)blockIdx.x * p.dim;
        const int width = p.lanes * 8 * kUnits;
        if (slots > 1) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kUnits; ++k)
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int column = kPieces ? (k * p.lanes + lane) * 8 + u : (k * 8 + u) * p.lanes + lane;
                    cross[slot * width + column] = which ? dpost[k][u] : dpre[k][u];
                }
            __syncthreads();
            for (int c = threadIdx.x; c < p.dim; c += blockDim.x) {
                float s = 0.f;
                for (int k = 0; k < slots; ++k) s += cross[k * width + c];
                part[c] = s;
            }
        } else {
#pragma unroll
            for (int k = 0; k < kUnits; ++k) Columns<kPieces>(lane, k, p.lanes, p.dim).store(part, which ? dpost[k] : dpre[k]);
        }
    }
}

// Sums of partial sums: job 0 and 1 the weights' gradients over blocks, job 2 + g the gate row g over its chunks.
constexpr int kJoinSumColumns = 32, kJoinSumShares = 32;
template <typename T>
__global__ void __launch_bounds__(kJoinSumColumns * kJoinSumShares) join_sum_kernel(const float* pre, const float* post, int blocks, const float* gate_part,
                                                                                    long long chunks_per_gate, long long chunks, int dim, void* dpre,
                                                                                    void* dpost, bool weights_f32, void* dgate, long long ld_dgate,
                                                                                    bool dgate_f32, int first_job) {
    __shared__ float sm[kJoinSumShares][kJoinSumColumns + 1];
    cudaGridDependencySynchronize();
    const int x = threadIdx.x % kJoinSumColumns, share = threadIdx.x / kJoinSumColumns, c = blockIdx.y * kJoinSumColumns + x;
    const long long job = (long long)blockIdx.x + first_job;
    const float* from = job == 0 ? pre : job == 1 ? post : gate_part + (job - 2) * chunks_per_gate * dim;
    if (!from) return;
    const long long n = job < 2 ? blocks : min(chunks_per_gate, chunks - (job - 2) * chunks_per_gate);
    float s = 0.f;
    if (c < dim)
        for (long long k = share; k < n; k += kJoinSumShares) s += from[k * dim + c];
    sm[share][x] = s;
    __syncthreads();
    for (int k = kJoinSumShares / 2; k; k /= 2) {
        if (share < k) sm[share][x] += sm[share + k][x];
        __syncthreads();
    }
    if (share || c >= dim) return;
    void* out = job == 0 ? dpre : job == 1 ? dpost : dgate;
    const long long at = (job < 2 ? 0 : (job - 2) * ld_dgate) + c;
    if (job < 2 ? weights_f32 : dgate_f32) ((float*)out)[at] = sm[0][x];
    else ((T*)out)[at] = from_f32<T>(sm[0][x]);
}

}  // namespace pb
