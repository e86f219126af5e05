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

// ------------------------------------------------------------------ eight columns
// Eight numbers of a thread as four pairs, on which one instruction works at a time: these kernels run out of instructions before they run out of
// memory bandwidth (16384 x 4096 with a gate and dropout: 242 us one by one).
struct Eight {
    Pair p[4];
    __device__ __forceinline__ void fill(float a) {
#pragma unroll
        for (int k = 0; k < 4; ++k) p[k] = Pair(a);
    }
    __device__ __forceinline__ void from(const float (&v)[8]) {
#pragma unroll
        for (int k = 0; k < 4; ++k) p[k] = Pair(v[2 * k], v[2 * k + 1]);
    }
    __device__ __forceinline__ void to(float (&v)[8]) const {
#pragma unroll
        for (int k = 0; k < 4; ++k) p[k].split(v[2 * k], v[2 * k + 1]);
    }
};
__device__ __forceinline__ Eight operator*(const Eight& a, const Eight& b) {
    Eight r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r.p[k] = a.p[k] * b.p[k];
    return r;
}
__device__ __forceinline__ Eight operator*(const Eight& a, float s) {
    const Pair f(s);
    Eight r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r.p[k] = a.p[k] * f;
    return r;
}
__device__ __forceinline__ Eight fma8(const Eight& a, const Eight& b, const Eight& c) {
    Eight r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r.p[k] = fma2(a.p[k], b.p[k], c.p[k]);
    return r;
}
__device__ __forceinline__ Eight fma8(float s, const Eight& b, const Eight& c) {
    const Pair f(s);
    Eight r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r.p[k] = fma2(f, b.p[k], c.p[k]);
    return r;
}
__device__ __forceinline__ float dot8(const Eight& a, const Eight& b) {
    Pair s = a.p[0] * b.p[0], t = a.p[1] * b.p[1];
    s = fma2(a.p[2], b.p[2], s);
    t = fma2(a.p[3], b.p[3], t);
    float x, y;
    (s + t).split(x, y);
    return x + y;
}

// ------------------------------------------------------------------ which elements are kept
// Element i of a call's [rows, dim] values (i = row * dim + column) has bits 16 (i mod 4) .. + 15 of the hash of counter i / 4 on the
// stream that (seed, offset) name; it is kept where they are at least `drop`.
struct Keep {
    unsigned long long seed;
    long long offset;
    const long long* dev_offset;
    unsigned drop;               // of 65536, in the upper half of the word
    float scale;                 // 65536 / (65536 - drop)
};
__device__ __forceinline__ unsigned long long keep_base(const Keep& k) {
    return splitmix64(k.seed, (unsigned long long)(k.dev_offset ? *k.dev_offset : k.offset));
}
// Zero where the half word is below `drop`, whatever was there; the low half is moved up, the upper one is compared with what is below it.
__device__ __forceinline__ Pair keep2(Pair v, unsigned bits, unsigned drop) {
    float a, b;
    v.split(a, b);
    return Pair((bits << 16) >= drop ? a : 0.f, bits >= drop ? b : 0.f);
}
// Elements 4 quad .. + 7, not scaled yet.
__device__ __forceinline__ Eight keep8(const Eight& v, unsigned long long base, unsigned long long quad, unsigned drop) {
    const unsigned long long y = splitmix64(base, quad), z = splitmix64(base, quad + 1);
    Eight r;
    r.p[0] = keep2(v.p[0], (unsigned)y, drop);
    r.p[1] = keep2(v.p[1], (unsigned)(y >> 32), drop);
    r.p[2] = keep2(v.p[2], (unsigned)z, drop);
    r.p[3] = keep2(v.p[3], (unsigned)(z >> 32), drop);
    return r;
}
__device__ __forceinline__ bool kept(unsigned long long base, unsigned long long i, unsigned drop) {
    return ((unsigned)(splitmix64(base, i / 4) >> (16 * (i % 4))) << 16) >= drop;
}

// Eight consecutive elements as they lie in memory.
template <typename T> struct RawEight {
    uint4 q;
    __device__ __forceinline__ void load(const T* p) { q = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void zero() { q = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ Eight get() const {
        float v[8];
        unpack8(v, q, T());
        Eight r;
        r.from(v);
        return r;
    }
};
template <> struct RawEight<float> {
    float v[8];
    __device__ __forceinline__ void load(const float* p) { load8_wide(v, p); }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = 0.f;
    }
    __device__ __forceinline__ Eight get() const {
        Eight r;
        r.from(v);
        return r;
    }
};
__device__ __forceinline__ void store_eight(float* p, const Eight& x) {
    float v[8];
    x.to(v);
    store8_wide(p, v);
}
template <typename T> __device__ __forceinline__ void store_eight(T* p, const Eight& x) {
    float v[8];
    x.to(v);
    store8(p, v);
}

constexpr int kDropThreads = 256;

// kPieces: eight elements at a time; dense: the rows follow each other without a gap, the whole is one row.
template <typename T, bool kPieces>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(const T* x, T* out, long long n, long long cols, long long ld_x, long long ld_out, bool dense, Keep k) {
    const unsigned long long base = keep_base(k);
    const long long step = (long long)gridDim.x * kDropThreads, first = blockIdx.x * (long long)kDropThreads + threadIdx.x;
    if constexpr (kPieces) {
        for (long long i = first; i < n / 8; i += step) {
            const long long r = dense ? 0 : i * 8 / cols, c = i * 8 - r * cols;
            RawEight<T> v;
            v.load(x + r * ld_x + c);
            store_eight(out + r * ld_out + c, keep8(v.get() * k.scale, base, 2 * i, k.drop));
        }
        if (blockIdx.x == 0 && threadIdx.x < n % 8) {         // dense only
            const long long i = n / 8 * 8 + threadIdx.x;
            out[i] = from_f32<T>(kept(base, i, k.drop) ? to_f32(x[i]) * k.scale : 0.f);
        }
    } else {
        for (long long q = first; q < (n + 3) / 4; q += step) {
            const unsigned long long z = splitmix64(base, q);
            long long r = dense ? 0 : q * 4 / cols, c = q * 4 - r * cols;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (q * 4 + u < n) out[r * ld_out + c] = from_f32<T>(((unsigned)(z >> (16 * u)) << 16) >= k.drop ? to_f32(x[r * ld_x + c]) * k.scale : 0.f);
                if (++c == cols && !dense) { c = 0; ++r; }
            }
        }
    }
}

// ------------------------------------------------------------------ join
struct JoinParams {
    long long rows;
    int dim, lanes;              // threads of a row: up to a warp a power of two, else the whole block
    const void *x, *u, *gate, *post, *pre, *yin, *dy, *dh;
    void *y, *h, *dx, *du;
    long long ld_x, ld_u, ld_y, ld_h, ld_gate, ld_dy, ld_dh, ld_dx, ld_du, ld_dgate;
    float *rstd_post, *rstd_pre;
    bool weights_f32;            // else of u's type
    Quotient by_gate;            // rows that share a row of the gate
    float rs, eps, inv_dim;
    Keep keep;                   // drop == 0: everything is kept
    // backward: chunks of rows that share a gate
    int rows_per_gate, chunk_rows, chunks_per_gate, chunks;
    Quotient by_chunks;
    float* gate_part;            // [chunks][dim], or NULL: a chunk is all rows of its gate, and written to dgate
    void* dgate;
    bool dgate_f32;
    float *part_pre, *part_post; // [blocks][dim], or NULL
};

constexpr int kJoinThreads = 256;             // of a block, or the threads of a row if those are more
constexpr int kJoinMaxLanes = 1024;

// Sum over the threads of a row.  Rows of more than a warp meet in shared memory: all threads of the block call this.
__device__ __forceinline__ float row_sum(float v, int lanes, float* sm) {
    if (lanes < 32) {
        for (int k = lanes / 2; k; k /= 2) v += __shfl_xor_sync(0xffffffffu, v, k);
        return v;
    }
#pragma unroll
    for (int k = 16; k; k /= 2) v += __shfl_xor_sync(0xffffffffu, v, k);
    if (lanes == 32) return v;
    const int l = threadIdx.x % 32;
    if (l == 0) sm[threadIdx.x / 32] = v;
    __syncthreads();
    v = l * 32 < lanes ? sm[l] : 0.f;
#pragma unroll
    for (int k = 16; k; k /= 2) v += __shfl_xor_sync(0xffffffffu, v, k);
    return v;
}

// 1 / sqrt(x) to 2^-23: the approximation, and one step of Newton's method where that is finite.
__device__ __forceinline__ float root_of(float x) {
    const float r = rsqrtf(x);
    return r > 0.f && r < INFINITY ? r * fmaf(-0.5f * x * r, r, 1.5f) : r;
}

// How a thread's eight columns lie: kOdd: `lanes` apart, so that neighbours read neighbours; kEven: consecutive; kFull: consecutive, and every
// thread has all of its own, in rows of a block each.
enum JoinLayout { kOdd = 0, kEven = 1, kFull = 2 };
template <typename T, bool kPieces> struct RawColumns : RawEight<T> {};
template <typename T> struct RawColumns<T, false> {
    T v[8];
    __device__ __forceinline__ Eight get() const {
        Eight r;
#pragma unroll
        for (int k = 0; k < 4; ++k) r.p[k] = Pair(to_f32(v[2 * k]), to_f32(v[2 * k + 1]));
        return r;
    }
};
template <int kLayout>
struct Columns {
    static constexpr bool kPieces = kLayout != kOdd;
    int first, step, n;          // n: how many exist
    __device__ __forceinline__ Columns(int lane, int unit, int lanes, int dim, bool live = true) {
        first = kPieces ? (unit * lanes + lane) * 8 : unit * 8 * lanes + lane;
        step = kPieces ? 1 : lanes;
        n = kLayout == kFull ? 8 : first >= dim || !live ? 0 : kPieces ? 8 : min(8, (dim - first + step - 1) / step);
    }
    template <typename T> __device__ __forceinline__ void load(RawColumns<T, kPieces>& v, const T* row) const {
        if constexpr (kLayout == kFull) {
            v.load(row + first);
        } else if constexpr (kPieces) {
            if (n) v.load(row + first); else v.zero();
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v.v[k] = k < n ? row[first + k * step] : from_f32<T>(0.f);
        }
    }
    template <typename T> __device__ __forceinline__ Eight get(const T* row) const {
        RawColumns<T, kPieces> v;
        load(v, row);
        return v.get();
    }
    template <typename T> __device__ __forceinline__ Eight weight(const void* w, bool f32) const {
        return f32 ? get((const float*)w) : get((const T*)w);
    }
    template <typename T> __device__ __forceinline__ void put(T* row, const Eight& x) const {
        if constexpr (kPieces) {
            if (kLayout == kFull || n) store_eight(row + first, x);
        } else {
            float v[8];
            x.to(v);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < n) row[first + k * step] = from_f32<T>(v[k]);
        }
    }
    // What dropout leaves of a row's columns.
    __device__ __forceinline__ Eight drop(const Eight& x, unsigned long long base, long long row, int dim, const Keep& k) const {
        const unsigned long long i = (unsigned long long)row * dim + first;
        if constexpr (kPieces) {
            return keep8(x * k.scale, base, i / 4, k.drop);  // dim is a multiple of 8
        } else {
            float v[8];
            (x * k.scale).to(v);
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = kept(base, i + u * step, k.drop) ? v[u] : 0.f;
            Eight r;
            r.from(v);
            return r;
        }
    }
};

template <typename T, typename S, int kLayout, int kUnits>
__global__ void __launch_bounds__(kJoinMaxLanes) join_forward_kernel(const JoinParams p) {
    __shared__ float sm[2][32];
    constexpr bool kAll = kLayout == kFull;
    const int lane = kAll || p.lanes > 32 ? threadIdx.x : threadIdx.x & (p.lanes - 1), slot = kAll || p.lanes > 32 ? 0 : threadIdx.x / p.lanes,
              slots = kAll || p.lanes > 32 ? 1 : blockDim.x / p.lanes;
    const unsigned long long base = p.keep.drop ? keep_base(p.keep) : 0;
    const long long r = (long long)blockIdx.x * slots + slot;
    const bool live = kAll || r < p.rows;
    Eight y[kUnits], b[kUnits];
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        const Columns<kLayout> c(lane, k, p.lanes, p.dim, live);
        b[k] = c.get((const T*)p.u + r * p.ld_u);
        y[k] = c.get((const S*)p.x + r * p.ld_x);
    }
    float rstd = 1.f;
    if (p.post) {
#pragma unroll
        for (int k = 0; k < kUnits; ++k) sum += dot8(b[k], b[k]);
        rstd = root_of(fmaf(row_sum(sum, p.lanes, sm[0]), p.inv_dim, p.eps));
        if (live && lane == 0 && p.rstd_post) p.rstd_post[r] = rstd;
    }
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        const Columns<kLayout> c(lane, k, p.lanes, p.dim, live);
        if (p.post) b[k] = b[k] * rstd * c.template weight<T>(p.post, p.weights_f32);
        if (p.gate) b[k] = b[k] * c.get((const T*)p.gate + (live ? p.by_gate((int)r) : 0) * p.ld_gate);
        if (p.keep.drop) b[k] = c.drop(b[k], base, r, p.dim, p.keep);
        y[k] = fma8(p.rs, y[k], b[k]);                       // columns that do not exist are zero
        c.put((S*)p.y + r * p.ld_y, y[k]);
        sum += dot8(y[k], y[k]);
    }
    if (!p.h) return;
    rstd = root_of(fmaf(row_sum(sum, p.lanes, sm[1]), p.inv_dim, p.eps));
    if (!live) return;
    if (lane == 0 && p.rstd_pre) p.rstd_pre[r] = rstd;
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        const Columns<kLayout> c(lane, k, p.lanes, p.dim);
        c.put((T*)p.h + r * p.ld_h, y[k] * rstd * c.template weight<T>(p.pre, p.weights_f32));
    }
}

// What the backward reads of a row.
template <typename T, typename S, bool kPieces>
struct JoinRow {
    RawColumns<T, kPieces> u, dh, gate;
    RawColumns<S, kPieces> y, dy;
    float rp, rr;
};

// kAhead: a row is read while the one before it is worked on, and the weights stay in registers.
template <typename T, typename S, int kLayout, int kUnits, int kThreads, bool kAhead>
__global__ void __launch_bounds__(kThreads, 512 / kThreads > 0 ? 512 / kThreads : 1) join_backward_kernel(const JoinParams p) {
    extern __shared__ float cross[];             // [slots][lanes * 8 * kUnits]
    __shared__ float sm[2][2][32];
    constexpr bool kAll = kLayout == kFull;
    const int lane = kAll || p.lanes > 32 ? threadIdx.x : threadIdx.x & (p.lanes - 1), slot = kAll || p.lanes > 32 ? 0 : threadIdx.x / p.lanes,
              slots = kAll || p.lanes > 32 ? 1 : blockDim.x / p.lanes;
    const unsigned long long base = p.keep.drop ? keep_base(p.keep) : 0;
    const int workers = (int)gridDim.x * slots;
    Eight dpre[kUnits], dpost[kUnits], dgate[kUnits], post[kUnits], pre[kUnits];
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        dpre[k].fill(0.f); dpost[k].fill(0.f); dgate[k].fill(0.f);
        if (kAhead) {
            const Columns<kLayout> c(lane, k, p.lanes, p.dim);
            if (p.post) post[k] = c.template weight<T>(p.post, p.weights_f32);
            if (p.dh) pre[k] = c.template weight<T>(p.pre, p.weights_f32);
        }
    }
    // The rows of a worker: chunk by chunk, every worker as many turns, since the workers of a warp move together; some are idle.
    struct Place {
        int chunk, q, group;
        long long r;
        bool live;
    };
    auto place = [&](int chunk, int q) {
        Place a;
        a.chunk = chunk; a.q = q;
        a.group = p.by_chunks(chunk);
        const int within = (chunk - a.group * p.chunks_per_gate) * p.chunk_rows + q;
        a.r = (long long)a.group * p.rows_per_gate + within;
        a.live = chunk < p.chunks && within < p.rows_per_gate && a.r < p.rows;
        return a;
    };
    auto read = [&](JoinRow<T, S, kLayout != kOdd> (&v)[kUnits], const Place& a) {
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const Columns<kLayout> c(lane, k, p.lanes, p.dim, a.live);
            if (kAll && !a.live) continue;                    // nothing of an idle turn is written
            c.load(v[k].u, (const T*)p.u + a.r * p.ld_u);
            if (p.dy) c.load(v[k].dy, (const S*)p.dy + a.r * p.ld_dy);
            if (p.dh) {
                c.load(v[k].y, (const S*)p.yin + a.r * p.ld_y);
                c.load(v[k].dh, (const T*)p.dh + a.r * p.ld_dh);
            }
            if (p.gate) c.load(v[k].gate, (const T*)p.gate + a.group * p.ld_gate);
        }
        v[0].rp = a.live && p.post ? p.rstd_post[a.r] : 1.f;
        v[0].rr = a.live && p.dh ? p.rstd_pre[a.r] : 0.f;
    };
    const int mine = (int)blockIdx.x * slots + slot, rounds = (p.chunks + workers - 1) / workers;
    JoinRow<T, S, kLayout != kOdd> row[kUnits];
    Place at = place(mine, 0);
    if (kAhead) read(row, at);
    for (int round = 0, q = 0, turn = 0; round < rounds; turn ^= 1) {
        if (!kAhead) read(row, at);
        Eight g[kUnits], un[kUnits], yn[kUnits], gate[kUnits];
        float sum = 0.f;
        const float rp = row[0].rp, rr = row[0].rr;
        const Place now = at;
        const bool idle = slots == 1 && !now.live;            // the whole block
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            if (idle) break;
            const Columns<kLayout> c(lane, k, p.lanes, p.dim);
            un[k] = row[k].u.get();
            if (p.gate) gate[k] = row[k].gate.get();
            if (p.dy) g[k] = row[k].dy.get(); else g[k].fill(0.f);
            if (p.dh) {
                const Eight w = kAhead ? pre[k] : c.template weight<T>(p.pre, p.weights_f32), dh = row[k].dh.get();
                yn[k] = row[k].y.get() * rr;
                dpre[k] = fma8(dh, yn[k], dpre[k]);
                const Eight wd = dh * w;
                sum += dot8(wd, yn[k]);
                g[k] = fma8(rr, wd, g[k]);
            }
        }
        const bool ends = ++q == p.chunk_rows;                // of the chunk
        if (ends) { q = 0; ++round; }
        at = place(mine + round * workers, q);
        if (kAhead && round < rounds) read(row, at);
        if (p.dh && !idle) {
            const float m = -rr * p.inv_dim * row_sum(sum, p.lanes, sm[turn][0]);
#pragma unroll
            for (int k = 0; k < kUnits; ++k) g[k] = fma8(m, yn[k], g[k]);
        }
        sum = 0.f;
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            if (idle) break;
            const Columns<kLayout> c(lane, k, p.lanes, p.dim, now.live);
            if (p.dx) c.put((S*)p.dx + now.r * p.ld_dx, g[k] * p.rs);
            if (p.keep.drop) g[k] = c.drop(g[k], base, now.r, p.dim, p.keep);
            if (!p.post) {
                if (p.gate) {
                    dgate[k] = fma8(g[k], un[k], dgate[k]);
                    g[k] = g[k] * gate[k];
                }
                c.put((T*)p.du + now.r * p.ld_du, g[k]);
            } else {
                const Eight w = kAhead ? post[k] : c.template weight<T>(p.post, p.weights_f32);
                un[k] = un[k] * rp;
                if (p.gate) {
                    dgate[k] = fma8(g[k], un[k] * w, dgate[k]);
                    g[k] = g[k] * gate[k];
                }
                dpost[k] = fma8(g[k], un[k], dpost[k]);
                g[k] = g[k] * w;
                sum += dot8(g[k], un[k]);
            }
        }
        if (p.post && !idle) {
            const float m = -rp * p.inv_dim * row_sum(sum, p.lanes, sm[turn][1]);
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                const Columns<kLayout> c(lane, k, p.lanes, p.dim, now.live);
                c.put((T*)p.du + now.r * p.ld_du, fma8(m, un[k], g[k] * rp));
            }
        }
        if (ends && p.dgate && now.chunk < p.chunks) {
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                const Columns<kLayout> c(lane, k, p.lanes, p.dim);
                if (p.gate_part) c.put(p.gate_part + (long long)now.chunk * p.dim, dgate[k]);
                else if (p.dgate_f32) c.put((float*)p.dgate + now.group * p.ld_dgate, dgate[k]);
                else c.put((T*)p.dgate + now.group * p.ld_dgate, dgate[k]);
                dgate[k].fill(0.f);
            }
        }
    }
    // the block's sums over its rows: its slots, in their order
    for (int which = 0; which < 2; ++which) {
        float* part = which ? p.part_post : p.part_pre;
        if (!part) continue;
        part += (long long)blockIdx.x * p.dim;
        const int width = 8 * kUnits * p.lanes;
        if (slots > 1) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                float v[8];
                (which ? dpost[k] : dpre[k]).to(v);
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int column = kLayout != kOdd ? (k * p.lanes + lane) * 8 + u : (k * 8 + u) * p.lanes + lane;
                    cross[slot * width + column] = v[u];
                }
            }
            __syncthreads();
            for (int c = threadIdx.x; c < p.dim; c += blockDim.x) {
                float s = 0.f;
                for (int k = 0; k < slots; ++k) s += cross[k * width + c];
                part[c] = s;
            }
        } else {
#pragma unroll
            for (int k = 0; k < kUnits; ++k) Columns<kLayout>(lane, k, p.lanes, p.dim).put(part, which ? dpost[k] : dpre[k]);
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
