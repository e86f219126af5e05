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
// In dy' = e - m1 yn, with e = dy + rstd_pre dh pre and m1 = rstd_pre mean(dh pre yn), the second mean is that of keep gate post un e less m1 times
// that of keep gate post un yn, so that the threads of a row meet once for three sums instead of twice for one.
//
// Everything is bound by the rows' bytes.  A row is held in registers by a group of threads (up to a warp a power of two, else whole warps; kUnits
// pieces of eight columns each), so that it is read and written once; its two sums are the only thing that the threads of a
// group exchange.  In the backward a thread keeps the same columns in every row, so that the sums over rows
// stay in its registers; they end in one partial sum per block, and in one per chunk of rows that share a gate.
#pragma once
#include "tc_common.cuh"
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
// Elements 4 quad .. + 7 of v, which is scaled already.
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
    __device__ __forceinline__ void load_shared(const T* p) { load(p); }
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
    __device__ __forceinline__ void load_shared(const float* p) {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
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
    int depth, row_bytes;        // rows of the ring, bytes of one: 128-byte aligned
    long long wait_ns;           // that a row's copies are waited for
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

// Three sums at once.
__device__ __forceinline__ void row_sums(float& a, float& b, float& c, int lanes, float (&sm)[3][32]) {
    if (lanes < 32) {
        for (int k = lanes / 2; k; k /= 2) {
            a += __shfl_xor_sync(0xffffffffu, a, k);
            b += __shfl_xor_sync(0xffffffffu, b, k);
            c += __shfl_xor_sync(0xffffffffu, c, k);
        }
        return;
    }
#pragma unroll
    for (int k = 16; k; k /= 2) {
        a += __shfl_xor_sync(0xffffffffu, a, k);
        b += __shfl_xor_sync(0xffffffffu, b, k);
        c += __shfl_xor_sync(0xffffffffu, c, k);
    }
    if (lanes == 32) return;
    const int l = threadIdx.x % 32, warp = threadIdx.x / 32;
    if (l < 3) sm[l][warp] = l == 0 ? a : l == 1 ? b : c;
    __syncthreads();
    const bool there = l * 32 < lanes;
    a = there ? sm[0][l] : 0.f; b = there ? sm[1][l] : 0.f; c = there ? sm[2][l] : 0.f;
#pragma unroll
    for (int k = 16; k; k /= 2) {
        a += __shfl_xor_sync(0xffffffffu, a, k);
        b += __shfl_xor_sync(0xffffffffu, b, k);
        c += __shfl_xor_sync(0xffffffffu, c, k);
    }
}

// 1 / sqrt(x) to 2^-23: the approximation, and one step of Newton's method where that is finite.
__device__ __forceinline__ float root_of(float x) {
    const float r = rsqrtf(x);
    return r > 0.f && r < INFINITY ? r * fmaf(-0.5f * x * r, r, 1.5f) : r;
}

// How a thread's eight columns lie: kOdd: `lanes` apart, so that neighbours read neighbours; kEven: consecutive; kFull: consecutive, and every thread has
// all of its own (what else asks at each access whether they exist: 7 % of the time of 8192 rows of 4096).
enum JoinLayout { kOdd = 0, kEven = 1, kFull = 2 };

// Rows that a block takes one after the other come by bulk copies into a ring in shared memory.  Should a row's copies not come in time, the block asks for
// no more of them, and what it would have written from that row on is NaN.
constexpr int kJoinRing = 4;                  // rows on their way at most
struct JoinRing {
    uint64_t full[kJoinRing];
    int fail[2];                              // a wait for this row has run out; rows take turns, so that all threads see the same after they have met
    int calm;                                 // always 0
};
__device__ __forceinline__ void bulk_row(unsigned char* dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// One thread sets the barriers up before the block meets for the first time.
__device__ __forceinline__ void ring_init(JoinRing& ring) {
    for (int k = 0; k < kJoinRing; ++k) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_u32(&ring.full[k])) : "memory");
    ring.fail[0] = ring.fail[1] = ring.calm = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
// The threads have met after a wait has run out.  The n rows that are under way, from place `at` on, land before the shared memory that they write goes back to
// the SM, or have had their time once more.
__device__ __forceinline__ void ring_lost(JoinRing& ring, int at, uint32_t phase, int depth, int n) {
    if (threadIdx.x == 0) {
        for (; n > 0; --n) {
            mbar_wait(smem_u32(&ring.full[at]), phase, &ring.calm);
            if (++at == depth) { at = 0; phase ^= 1; }
        }
    }
    __syncthreads();
}
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
        if constexpr (kPieces) {
            if (kLayout == kFull || n) v.load(row + first); else v.zero();
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
    template <typename T> __device__ __forceinline__ Eight get_shared(const void* row) const {
        RawEight<T> v;
        if (kLayout == kFull || n) v.load_shared((const T*)row + first); else v.zero();
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
    // What dropout leaves of a row's columns (x scaled already).
    __device__ __forceinline__ Eight drop(const Eight& x, unsigned long long base, long long row, int dim, const Keep& k) const {
        const unsigned long long i = (unsigned long long)row * dim + first;
        if constexpr (kPieces) {
            return keep8(x, base, i / 4, k.drop);            // dim is a multiple of 8
        } else {
            float v[8];
            x.to(v);
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
    const int lane = p.lanes > 32 ? threadIdx.x : threadIdx.x & (p.lanes - 1), slot = p.lanes > 32 ? 0 : threadIdx.x / p.lanes,
              slots = p.lanes > 32 ? 1 : blockDim.x / p.lanes;
    const unsigned long long base = p.keep.drop ? keep_base(p.keep) : 0;
    const long long r = (long long)blockIdx.x * slots + slot;
    const bool live = r < p.rows;
    Eight y[kUnits], b[kUnits], w[kUnits];
    RawColumns<T, kLayout != kOdd> gate[kUnits];
    float sum = 0.f;
    // what the sums are waited for with is on its way before they are formed
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        const Columns<kLayout> c(lane, k, p.lanes, p.dim, live);
        b[k] = c.get((const T*)p.u + r * p.ld_u);
        y[k] = c.get((const S*)p.x + r * p.ld_x);
        if (p.gate) c.load(gate[k], (const T*)p.gate + (live ? p.by_gate((int)r) : 0) * p.ld_gate);
        if (p.post) w[k] = c.template weight<T>(p.post, p.weights_f32);
    }
    float rstd = 1.f;
    if (p.post) {
#pragma unroll
        for (int k = 0; k < kUnits; ++k) sum += dot8(b[k], b[k]);
        rstd = root_of(fmaf(row_sum(sum, p.lanes, sm[0]), p.inv_dim, p.eps));
        if (live && lane == 0 && p.rstd_post) p.rstd_post[r] = rstd;
    }
    const float scale = p.keep.drop ? rstd * p.keep.scale : rstd;
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        const Columns<kLayout> c(lane, k, p.lanes, p.dim, live);
        b[k] = b[k] * scale;
        if (p.post) b[k] = b[k] * w[k];
        if (p.h) w[k] = c.template weight<T>(p.pre, p.weights_f32);
        if (p.gate) b[k] = b[k] * gate[k].get();
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
        c.put((T*)p.h + r * p.ld_h, y[k] * rstd * w[k]);
    }
}

// Rows that a block takes one after the other, 16 columns per thread: their parts come by bulk copies some rows ahead, and the weights stay in registers.
template <typename T, typename S, int kLayout, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads <= 256 ? 512 / kThreads : 1) join_forward_ring_kernel(const JoinParams p) {
    extern __shared__ __align__(128) unsigned char store[];
    __shared__ float sm[2][2][32];
    __shared__ JoinRing ring;
    constexpr int kUnits = 2;
    const int lane = threadIdx.x;
    const unsigned long long base = p.keep.drop ? keep_base(p.keep) : 0;
    if (lane == 0) ring_init(ring);
    __syncthreads();
    const uint32_t s_bytes = (uint32_t)(p.dim * sizeof(S)), t_bytes = (uint32_t)(p.dim * sizeof(T));
    auto ask = [&](long long r, int at) {
        const uint32_t bar = smem_u32(&ring.full[at]);
        unsigned char* to = store + at * p.row_bytes;
        mbar_arrive_tx(bar, s_bytes + (p.gate ? 2 : 1) * t_bytes);
        bulk_row(to, (const S*)p.x + r * p.ld_x, s_bytes, bar);
        bulk_row(to + s_bytes, (const T*)p.u + r * p.ld_u, t_bytes, bar);
        if (p.gate) bulk_row(to + s_bytes + t_bytes, (const T*)p.gate + (long long)p.by_gate((int)r) * p.ld_gate, t_bytes, bar);
    };
    if (lane == 0)
        for (int k = 0; k < p.depth; ++k)
            if (blockIdx.x + (long long)k * gridDim.x < p.rows) ask(blockIdx.x + (long long)k * gridDim.x, k);
    Eight post[kUnits], pre[kUnits];
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        const Columns<kLayout> c(lane, k, blockDim.x, p.dim);
        if (p.post) post[k] = c.template weight<T>(p.post, p.weights_f32);
        if (p.h) pre[k] = c.template weight<T>(p.pre, p.weights_f32);
    }
    int at = 0, turn = 0;
    uint32_t phase = 0;
    long long r = blockIdx.x;
    for (; r < p.rows; r += gridDim.x, turn ^= 1) {
        if (!mbar_wait(smem_u32(&ring.full[at]), phase, &ring.fail[turn], p.wait_ns)) ring.fail[turn] = 1;
        const unsigned char* from = store + at * p.row_bytes;
        Eight y[kUnits], b[kUnits], gate[kUnits];
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const Columns<kLayout> c(lane, k, blockDim.x, p.dim);
            y[k] = c.template get_shared<S>(from);
            b[k] = c.template get_shared<T>(from + s_bytes);
            if (p.gate) gate[k] = c.template get_shared<T>(from + s_bytes + t_bytes);
            if (p.post) sum += dot8(b[k], b[k]);
        }
        float rstd = 1.f;
        if (p.post) {
            rstd = root_of(fmaf(row_sum(sum, blockDim.x, sm[turn][0]), p.inv_dim, p.eps));
            if (lane == 0 && p.rstd_post) p.rstd_post[r] = rstd;
        } else {
            __syncthreads();
        }
        if (ring.fail[turn]) break;
        if (lane == 0 && r + (long long)p.depth * gridDim.x < p.rows) ask(r + (long long)p.depth * gridDim.x, at);     // all have read this row
        if (++at == p.depth) { at = 0; phase ^= 1; }
        const float scale = p.keep.drop ? rstd * p.keep.scale : rstd;
        sum = 0.f;
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const Columns<kLayout> c(lane, k, blockDim.x, p.dim);
            b[k] = b[k] * scale;
            if (p.post) b[k] = b[k] * post[k];
            if (p.gate) b[k] = b[k] * gate[k];
            if (p.keep.drop) b[k] = c.drop(b[k], base, r, p.dim, p.keep);
            y[k] = fma8(p.rs, y[k], b[k]);
            c.put((S*)p.y + r * p.ld_y, y[k]);
            sum += dot8(y[k], y[k]);
        }
        if (!p.h) continue;
        rstd = root_of(fmaf(row_sum(sum, blockDim.x, sm[turn][1]), p.inv_dim, p.eps));
        if (lane == 0 && p.rstd_pre) p.rstd_pre[r] = rstd;
#pragma unroll
        for (int k = 0; k < kUnits; ++k) Columns<kLayout>(lane, k, blockDim.x, p.dim).put((T*)p.h + r * p.ld_h, y[k] * rstd * pre[k]);
    }
    if (r >= p.rows) return;
    ring_lost(ring, at, phase, p.depth, (int)min((long long)p.depth, (p.rows - 1 - r) / gridDim.x + 1));
    Eight none;
    none.fill(__int_as_float(0x7fffffff));
    for (; r < p.rows; r += gridDim.x) {
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const Columns<kLayout> c(lane, k, blockDim.x, p.dim);
            c.put((S*)p.y + r * p.ld_y, none);
            if (p.h) c.put((T*)p.h + r * p.ld_h, none);
        }
        if (lane == 0 && p.post && p.rstd_post) p.rstd_post[r] = __int_as_float(0x7fffffff);
        if (lane == 0 && p.h && p.rstd_pre) p.rstd_pre[r] = __int_as_float(0x7fffffff);
    }
}

// Rows of any layout: a worker is the threads of a row, and goes through chunks of rows that share a gate.
template <typename T, typename S, int kLayout, int kUnits, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads <= 256 ? 3 : 1) join_backward_kernel(const JoinParams p) {
    extern __shared__ float cross[];             // [slots][lanes * 8 * kUnits]
    __shared__ float sm[2][2][32];
    const int lane = p.lanes > 32 ? threadIdx.x : threadIdx.x & (p.lanes - 1), slot = p.lanes > 32 ? 0 : threadIdx.x / p.lanes,
              slots = p.lanes > 32 ? 1 : blockDim.x / p.lanes;
    const unsigned long long base = p.keep.drop ? keep_base(p.keep) : 0;
    const int workers = (int)gridDim.x * slots, mine = (int)blockIdx.x * slots + slot;
    Eight dpre[kUnits], dpost[kUnits], dgate[kUnits];
#pragma unroll
    for (int k = 0; k < kUnits; ++k) { dpre[k].fill(0.f); dpost[k].fill(0.f); dgate[k].fill(0.f); }
    int turn = 0;
    // every worker takes as many turns, since those of a warp move together; some are idle, and read zeros
    for (int k0 = 0; k0 < p.chunks; k0 += workers) {
        const int chunk = k0 + mine, group = p.by_chunks(chunk), start = (chunk - group * p.chunks_per_gate) * p.chunk_rows;
        for (int q = 0; q < p.chunk_rows; ++q, turn ^= 1) {
            const long long r = (long long)group * p.rows_per_gate + start + q;
            const bool live = chunk < p.chunks && start + q < p.rows_per_gate && r < p.rows;
            const float rp = live && p.post ? p.rstd_post[r] : 1.f, rr = live && p.dh ? p.rstd_pre[r] : 0.f;
            Eight g[kUnits], un[kUnits], yn[kUnits];
            RawColumns<T, kLayout != kOdd> gate[kUnits];
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                const Columns<kLayout> c(lane, k, p.lanes, p.dim, live);
                un[k] = c.get((const T*)p.u + r * p.ld_u);
                if (p.gate) c.load(gate[k], (const T*)p.gate + group * p.ld_gate);
                if (p.dy) g[k] = c.get((const S*)p.dy + r * p.ld_dy); else g[k].fill(0.f);
                if (p.dh) {
                    const Eight dh = c.get((const T*)p.dh + r * p.ld_dh);
                    yn[k] = c.get((const S*)p.yin + r * p.ld_y) * rr;
                    dpre[k] = fma8(dh, yn[k], dpre[k]);
                    const Eight w = dh * c.template weight<T>(p.pre, p.weights_f32);
                    sum += dot8(w, yn[k]);
                    g[k] = fma8(rr, w, g[k]);
                }
            }
            if (p.dh) {
                const float m = -rr * p.inv_dim * row_sum(sum, p.lanes, sm[turn][0]);
#pragma unroll
                for (int k = 0; k < kUnits; ++k) g[k] = fma8(m, yn[k], g[k]);
            }
            sum = 0.f;
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                const Columns<kLayout> c(lane, k, p.lanes, p.dim, live);
                if (p.dx) c.put((S*)p.dx + r * p.ld_dx, g[k] * p.rs);
                if (p.keep.drop) g[k] = c.drop(g[k] * p.keep.scale, base, r, p.dim, p.keep);
                if (!p.post) {
                    if (p.gate) {
                        dgate[k] = fma8(g[k], un[k], dgate[k]);
                        g[k] = g[k] * gate[k].get();
                    }
                    c.put((T*)p.du + r * p.ld_du, g[k]);
                } else {
                    const Eight w = c.template weight<T>(p.post, p.weights_f32);
                    un[k] = un[k] * rp;
                    if (p.gate) {
                        dgate[k] = fma8(g[k], un[k] * w, dgate[k]);
                        g[k] = g[k] * gate[k].get();
                    }
                    dpost[k] = fma8(g[k], un[k], dpost[k]);
                    g[k] = g[k] * w;
                    sum += dot8(g[k], un[k]);
                }
            }
            if (p.post) {
                const float m = -rp * p.inv_dim * row_sum(sum, p.lanes, sm[turn][1]);
#pragma unroll
                for (int k = 0; k < kUnits; ++k) {
                    const Columns<kLayout> c(lane, k, p.lanes, p.dim, live);
                    c.put((T*)p.du + r * p.ld_du, fma8(m, un[k], g[k] * rp));
                }
            }
        }
        if (p.dgate && chunk < p.chunks) {
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                const Columns<kLayout> c(lane, k, p.lanes, p.dim);
                if (p.gate_part) c.put(p.gate_part + (long long)chunk * p.dim, dgate[k]);
                else if (p.dgate_f32) c.put((float*)p.dgate + group * p.ld_dgate, dgate[k]);
                else c.put((T*)p.dgate + group * p.ld_dgate, dgate[k]);
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

// Rows that a block takes one after the other, eight columns per thread (16 in rows of more than 8192): their parts come by bulk copies some rows
// ahead.
template <typename T, typename S, int kLayout, int kUnits, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads <= 256 ? 512 / kThreads : 1) join_backward_ring_kernel(const JoinParams p) {
    extern __shared__ __align__(128) unsigned char store[];
    __shared__ float sm[2][3][32];
    __shared__ JoinRing ring;
    const int lane = threadIdx.x, blocks = (int)gridDim.x;
    const unsigned long long base = p.keep.drop ? keep_base(p.keep) : 0;
    if (lane == 0) ring_init(ring);
    __syncthreads();
    const uint32_t s_bytes = (uint32_t)(p.dim * sizeof(S)), t_bytes = (uint32_t)(p.dim * sizeof(T));
    struct Chunk {
        int group, rows;
        long long first;
    };
    auto chunk_at = [&](int chunk) {
        Chunk c;
        c.group = p.by_chunks(chunk);
        const int start = (chunk - c.group * p.chunks_per_gate) * p.chunk_rows;
        c.first = (long long)c.group * p.rows_per_gate + start;
        c.rows = (int)min((long long)min(p.chunk_rows, p.rows_per_gate - start), p.rows - c.first);
        return c;
    };
    // the row that the next copies are for
    int ask_chunk = blockIdx.x, ask_q = 0, put = 0;
    Chunk asked = chunk_at(ask_chunk);
    auto ask = [&]() {
        if (ask_chunk >= p.chunks) return;
        const long long r = asked.first + ask_q;
        const uint32_t bar = smem_u32(&ring.full[put]);
        unsigned char* to = store + put * p.row_bytes;
        mbar_arrive_tx(bar, t_bytes * (1 + (p.dh != nullptr) + (p.gate != nullptr)) + s_bytes * ((p.dh != nullptr) + (p.dy != nullptr)));
        bulk_row(to, (const T*)p.u + r * p.ld_u, t_bytes, bar);
        if (p.gate) bulk_row(to + t_bytes, (const T*)p.gate + asked.group * p.ld_gate, t_bytes, bar);
        if (p.dh) {
            bulk_row(to + 2 * t_bytes, (const T*)p.dh + r * p.ld_dh, t_bytes, bar);
            bulk_row(to + 3 * t_bytes, (const S*)p.yin + r * p.ld_y, s_bytes, bar);
        }
        if (p.dy) bulk_row(to + 3 * t_bytes + s_bytes, (const S*)p.dy + r * p.ld_dy, s_bytes, bar);
        if (++put == p.depth) put = 0;
        if (++ask_q == asked.rows) {
            ask_q = 0;
            ask_chunk += blocks;
            if (ask_chunk < p.chunks) asked = chunk_at(ask_chunk);
        }
    };
    if (lane == 0)
        for (int k = 0; k < p.depth; ++k) ask();
    // What dpost and dgate have in common is the sum of db un over the rows of a gate: times post that is dgate, times the gate it goes to dpost.
    constexpr bool kKept = kUnits == 1;                       // the weights stay in registers
    Eight dpre[kUnits], dpost[kUnits], both[kUnits], post[kUnits], pre[kUnits];
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        dpre[k].fill(0.f); dpost[k].fill(0.f); both[k].fill(0.f);
        if (kKept) {
            const Columns<kLayout> c(lane, k, blockDim.x, p.dim);
            if (p.post) post[k] = c.template weight<T>(p.post, p.weights_f32);
            if (p.dh) pre[k] = c.template weight<T>(p.pre, p.weights_f32);
        }
    }
    int get = 0, turn = 0;
    uint32_t phase = 0;
    int chunk = blockIdx.x, q = 0;
    for (; chunk < p.chunks; chunk += blocks) {
        const Chunk now = chunk_at(chunk);
        for (q = 0; q < now.rows; ++q, turn ^= 1) {
            const long long r = now.first + q;
            const float rp = p.post ? p.rstd_post[r] : 1.f, rr = p.dh ? p.rstd_pre[r] : 0.f;
            if (!mbar_wait(smem_u32(&ring.full[get]), phase, &ring.fail[turn], p.wait_ns)) ring.fail[turn] = 1;
            const unsigned char* from = store + get * p.row_bytes;
            Eight g[kUnits], un[kUnits], yn[kUnits], gate[kUnits], keep[kUnits];
            float s1 = 0.f, s2 = 0.f, s3 = 0.f;
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                const Columns<kLayout> c(lane, k, blockDim.x, p.dim);
                un[k] = c.template get_shared<T>(from) * rp;
                if (p.gate) gate[k] = c.template get_shared<T>(from + t_bytes);
                if (p.dy) g[k] = c.template get_shared<S>(from + 3 * t_bytes + s_bytes); else g[k].fill(0.f);
                if (p.dh) {
                    const Eight dh = c.template get_shared<T>(from + 2 * t_bytes), w = dh * (kKept ? pre[k] : c.template weight<T>(p.pre, p.weights_f32));
                    yn[k] = c.template get_shared<S>(from + 3 * t_bytes) * rr;
                    dpre[k] = fma8(dh, yn[k], dpre[k]);
                    s1 += dot8(w, yn[k]);
                    g[k] = fma8(rr, w, g[k]);
                }
                keep[k].fill(p.keep.scale);
                if (p.keep.drop) keep[k] = c.drop(keep[k], base, r, p.dim, p.keep);
                if (p.post) {
                    Eight f = keep[k] * un[k] * (kKept ? post[k] : c.template weight<T>(p.post, p.weights_f32));
                    if (p.gate) f = f * gate[k];
                    s2 += dot8(f, g[k]);
                    if (p.dh) s3 += dot8(f, yn[k]);
                }
            }
            if (p.dh || p.post) row_sums(s1, s2, s3, blockDim.x, sm[turn]);
            const float m1 = -rr * p.inv_dim * s1, m2 = -rp * p.inv_dim * fmaf(m1, s3, s2);
            if (!(p.dh || p.post)) __syncthreads();               // (a row in the ring has more threads than a warp)
            if (ring.fail[turn]) break;
            if (lane == 0) ask();                             // all have read this row: another may have its place
            if (++get == p.depth) { get = 0; phase ^= 1; }
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                const Columns<kLayout> c(lane, k, blockDim.x, p.dim);
                if (p.dh) g[k] = fma8(m1, yn[k], g[k]);
                if (p.dx) c.put((S*)p.dx + r * p.ld_dx, g[k] * p.rs);
                if (p.keep.drop) g[k] = g[k] * keep[k];
                both[k] = fma8(g[k], un[k], both[k]);
                if (p.gate) g[k] = g[k] * gate[k];
                if (p.post) g[k] = fma8(m2, un[k], g[k] * (kKept ? post[k] : c.template weight<T>(p.post, p.weights_f32)) * rp);
                c.put((T*)p.du + r * p.ld_du, g[k]);
            }
        }
        if (q < now.rows) break;
        if (p.gate) {
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                const Columns<kLayout> c(lane, k, blockDim.x, p.dim);
                if (p.post) dpost[k] = fma8(c.get((const T*)p.gate + now.group * p.ld_gate), both[k], dpost[k]);
                if (p.dgate) {
                    const Eight d = p.post ? both[k] * (kKept ? post[k] : c.template weight<T>(p.post, p.weights_f32)) : both[k];
                    if (p.gate_part) c.put(p.gate_part + (long long)chunk * p.dim, d);
                    else if (p.dgate_f32) c.put((float*)p.dgate + now.group * p.ld_dgate, d);
                    else c.put((T*)p.dgate + now.group * p.ld_dgate, d);
                }
                both[k].fill(0.f);
            }
        }
    }
    if (chunk < p.chunks) {
        ring_lost(ring, get, phase, p.depth, (put - get + p.depth - 1) % p.depth + 1);       // of the first thread, which has asked: all places, but for the last rows
        Eight none;
        none.fill(__int_as_float(0x7fffffff));
        for (; chunk < p.chunks; chunk += blocks, q = 0) {
            const Chunk now = chunk_at(chunk);
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                const Columns<kLayout> c(lane, k, blockDim.x, p.dim);
                for (int i = q; i < now.rows; ++i) {
                    if (p.dx) c.put((S*)p.dx + (now.first + i) * p.ld_dx, none);
                    c.put((T*)p.du + (now.first + i) * p.ld_du, none);
                }
                if (p.gate && p.dgate) {
                    if (p.gate_part) c.put(p.gate_part + (long long)chunk * p.dim, none);
                    else if (p.dgate_f32) c.put((float*)p.dgate + now.group * p.ld_dgate, none);
                    else c.put((T*)p.dgate + now.group * p.ld_dgate, none);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kUnits; ++k) dpre[k] = dpost[k] = both[k] = none;
    }
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        const Columns<kLayout> c(lane, k, blockDim.x, p.dim);
        if (p.part_pre) c.put(p.part_pre + (long long)blockIdx.x * p.dim, dpre[k]);
        if (p.part_post) c.put(p.part_post + (long long)blockIdx.x * p.dim, p.gate ? dpost[k] : both[k]);
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
