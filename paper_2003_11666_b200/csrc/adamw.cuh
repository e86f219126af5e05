// One AdamW step over many tensors (decoupled weight decay, Loshchilov & Hutter 2019):
//   m <- b1 m + (1 - b1) g,   v <- b2 v + ((1 - b2) g) g,   r = sqrt(v),
//   u = (m / (1 - b1^t)) / (r / sqrt(1 - b2^t) + eps),   w <- w (1 - lr wd) - lr u,
// and, where asked for, the weights the next forward uses, w_forward = w - lr T u: the velocity
// form of linear weight prediction with this optimizer's step in the velocity's place (T = 0: a
// copy of w in the forward's type).
//
// The moments are float32 and every operation on them is rounded on its own (no contraction), so
// that an 8-bit state is the same whatever code computes it.  8-bit states hold, for every 256
// elements of a tensor, the moments over a float32 scale: m as a signed float of 4 exponent and 3
// mantissa bits (e4m3, nearest even, largest |m| at 448), r as an unsigned float of 4 exponent and
// 4 mantissa bits (code c > 0: 2^(c/16 - 15) (1 + (c%16)/16), largest r at 1.9375).  r is rounded
// up or down at random in proportion to the distance (16 bits of SplitMix64 per element): with
// b2 = 0.999 a step moves r by 0.05 % of itself, so rounding to the nearest of steps of 1/16 would
// leave it where it is.  A nonzero r never becomes zero, the update's denominator.
#pragma once
#include <cuda_fp8.h>

#include "tok_common.cuh"

namespace pb {

// The table of tensors is a kernel parameter: a call needs no copy and no memory of its own.  Launches
// of few tensors take the small table, whose parameters are quicker to hand over.
constexpr int kAdamFewTensors = 16, kAdamManyTensors = 330;
constexpr int kAdamNear = 256;
constexpr int kAdamBlock = 256;           // elements that share a scale: a warp, eight elements per lane
constexpr int kAdamThreads = 128;         // small blocks, so that few of an SM's warps load or compute at the same time
constexpr int kAdamRound = kAdamThreads * 8;   // elements of a thread block

struct AdamTensor {
    float* w;
    const void* g;
    void* m;
    void* v;
    float* m_scale;
    float* v_scale;
    void* fwd;
    long long n;
    unsigned long long rnd;      // start of the tensor's random stream, without seed and step
    float decay, horizon;
    unsigned first_round;
    int vec;                     // every pointer is aligned to eight elements
};

struct AdamScalars {
    double lr, beta1, beta2;
    float b1, o1, b2, o2, eps;
    float minus_zero;
    float c1, c2;                // 1 / (1 - beta1^step), 1 / sqrt(1 - beta2^step)
    long long step;
    unsigned long long seed;
    const float* grad_scale;
    const float* dev_lr;
    const long long* dev_step;
    int fwd_dtype;
    int subnormal;               // eps is so small that roots of numbers below 2^-126 count beside it
    int n;                       // tensors of this launch
    int near_shift;
    unsigned short near[kAdamNear];    // tensor that holds round k << near_shift
};

template <int MAXT>
struct AdamTable {
    AdamScalars s;
    AdamTensor t[MAXT];
};

constexpr float kMTop = 448.f, kRTop = 1.9375f;
constexpr int kRBias = 112 << 4;          // exponent and mantissa bits of 2^-15

__device__ __forceinline__ float decode_r(unsigned c) { return c ? __uint_as_float((c + kRBias) << 19) : 0.f; }

// Eight codes <-> eight values.
__device__ __forceinline__ void decode_m8(float (&x)[8], uint2 c) {
    const unsigned w[2] = {c.x, c.y};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[k >> 1] >> (16 * (k & 1))), __NV_E4M3);
        const float2 f = __half22float2(__half2(h));
        x[2 * k] = f.x;
        x[2 * k + 1] = f.y;
    }
}
__device__ __forceinline__ void decode_r8(float (&x)[8], uint2 c) {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = decode_r(((k < 4 ? c.x : c.y) >> (8 * (k & 3))) & 255u);
}
__device__ __forceinline__ uint2 encode_m8(const float (&x)[8]) {
    unsigned w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = __nv_cvt_float2_to_fp8x2(make_float2(x[2 * k], x[2 * k + 1]), __NV_SATFINITE, __NV_E4M3);
    return make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
}

// Eight elements of a lane: element k of lane l is base + 8 l + k in a whole block whose memory is aligned
// (VEC), else base + 32 k + l, with a test for the tensor's end.
template <bool VEC>
struct AdamLane {
    long long base, n;
    int lane;
    __device__ __forceinline__ long long at(int k) const { return VEC ? base + 8 * lane + k : base + 32 * k + lane; }
    __device__ __forceinline__ bool in(int k) const { return VEC || at(k) < n; }

    template <typename T>
    __device__ __forceinline__ void load(float (&x)[8], const T* p) const {
        if constexpr (VEC) {
            if constexpr (sizeof(T) == 4) load8_wide(x, p + at(0));
            else load8(x, p + at(0));
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = in(k) ? to_f32(p[at(k)]) : 0.f;
        }
    }
    // 16-bit elements as they are in memory: eight in four registers
    template <typename T>
    __device__ __forceinline__ uint4 load_raw(const T* p) const {
        if constexpr (VEC) {
            return *reinterpret_cast<const uint4*>(p + at(0));
        } else {
            unsigned h[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) h[k] = in(k) ? (unsigned)reinterpret_cast<const unsigned short*>(p)[at(k)] : 0u;
            return make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
        }
    }
    template <typename T>
    __device__ __forceinline__ void store(T* p, const float (&x)[8]) const {
        if constexpr (VEC) {
            if constexpr (sizeof(T) == 4) store8_wide(p + at(0), x);
            else store8(p + at(0), x);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (in(k)) p[at(k)] = from_f32<T>(x[k]);
        }
    }
    __device__ __forceinline__ uint2 load_codes(const unsigned char* p) const {
        if constexpr (VEC) {
            return *reinterpret_cast<const uint2*>(p + at(0));
        } else {
            unsigned c[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) c[k] = in(k) ? p[at(k)] : 0u;
            return make_uint2(c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24);
        }
    }
    __device__ __forceinline__ void store_codes(unsigned char* p, uint2 c) const {
        if constexpr (VEC) {
            *reinterpret_cast<uint2*>(p + at(0)) = c;
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (in(k)) p[at(k)] = (unsigned char)((k < 4 ? c.x : c.y) >> (8 * (k & 3)));
        }
    }
};

// The step uses pairs (tok_common.cuh) because with 8-bit states it is bound by the instructions it issues.
// x[k] <- s x[k] for eight elements
__device__ __forceinline__ void scale8(float (&x)[8], float s) {
#pragma unroll
    for (int k = 0; k < 8; k += 2) (Pair(x[k], x[k + 1]) * Pair(s)).split(x[k], x[k + 1]);
}

// Square root and reciprocal to 2^-23 or so of themselves; results, and arguments unless SUB, below 2^-126 count as
// zero.
template <bool SUB>
__device__ __forceinline__ float sqrt_near(float x) {
    float r;
    if (SUB) asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    else asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float rcp_near(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// Codes of eight second moments from their roots r (scaled by `ri`) and the random bits z of each four:
// the root's bits plus a random number below one step of the code, cut off.  The low byte of what
// is left is the code, since the exponent's bias there is a multiple of 256; the largest root, whose
// bits below the code are zero up to a rounding, cannot pass code 255.  Returns whether an element lies
// so near a border between two codes that r has to be the exactly rounded root.
template <bool VEC>
__device__ __forceinline__ bool encode_r8(uint2& code, const float (&v)[8], const float (&r)[8], float ri, const unsigned long long (&z)[VEC ? 2 : 8]) {
    unsigned near = 0xffffffffu, t[8];
    const float lowest = __uint_as_float((unsigned)(kRBias + 1) << 19);
    float s[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) s[k] = r[k];
    scale8(s, ri);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const unsigned noise = VEC ? (unsigned)(z[k >> 2] >> (16 * (k & 3))) & 0xffffu : (unsigned)z[k];
        const float x = v[k] > 0.f ? fmaxf(s[k], lowest) : 0.f;
        t[k] = __float_as_uint(x) + (noise << 3);
        near = min(near, (t[k] + 8u) & 0x7fff0u);
        t[k] >>= 19;
    }
    const unsigned a = __byte_perm(t[0], t[1], 0x0040), b = __byte_perm(t[2], t[3], 0x0040);
    const unsigned c = __byte_perm(t[4], t[5], 0x0040), d = __byte_perm(t[6], t[7], 0x0040);
    code = make_uint2(__byte_perm(a, b, 0x5410), __byte_perm(c, d, 0x5410));
    return near == 0;
}

struct AdamNow {                 // what a step's scalars come to
    float gs, c1, c2, lr, keep;   // keep: 1 - lr * weight decay
    unsigned long long key;
};

// What a block's update starts from, as it is in memory.
template <int BITS, typename GT, bool VEC>
struct AdamIn {
    float w[8], m[BITS == 32 ? 8 : 1], v[BITS == 32 ? 8 : 1], g[sizeof(GT) == 4 ? 8 : 1];
    uint4 g16;
    uint2 mc, vc;
    float ms, rs;
    __device__ __forceinline__ void load(const AdamTensor& t, long long block, const AdamLane<VEC>& q) {
        if constexpr (sizeof(GT) == 4) q.load(g, reinterpret_cast<const GT*>(t.g));
        else g16 = q.load_raw(reinterpret_cast<const GT*>(t.g));
        if constexpr (BITS == 8) {
            mc = q.load_codes(reinterpret_cast<const unsigned char*>(t.m));
            vc = q.load_codes(reinterpret_cast<const unsigned char*>(t.v));
            ms = t.m_scale[block];
            rs = t.v_scale[block];
        } else {
            q.load(m, reinterpret_cast<const float*>(t.m));
            q.load(v, reinterpret_cast<const float*>(t.v));
        }
        q.load(w, t.w);
    }
};

// One block of 256 elements by a warp.
template <int BITS, typename GT, bool VEC, bool SUB, typename Now>
__device__ __forceinline__ void adamw_block(const AdamScalars& a, const AdamTensor& t, long long block, int lane, Now scalars) {
    const AdamLane<VEC> q{block * kAdamBlock, t.n, lane};
    AdamIn<BITS, GT, VEC> in;
    in.load(t, block, q);
    AdamNow now;
    if (!scalars(now)) return;                       // read while the block is on its way
    float g[8], w[8], m[8], v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = in.w[k];
    if constexpr (sizeof(GT) == 4) {
#pragma unroll
        for (int k = 0; k < 8; ++k) g[k] = in.g[k];
    } else {
        unpack8(g, in.g16, GT());
    }
    if constexpr (BITS == 8) {
        decode_m8(m, in.mc);
        decode_r8(v, in.vc);
        scale8(m, in.ms);
        scale8(v, in.rs);
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
            const Pair x(v[k], v[k + 1]);
            (x * x).split(v[k], v[k + 1]);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) { m[k] = in.m[k]; v[k] = in.v[k]; }
    }
    const Pair ahead(-now.lr * t.horizon), down(-now.lr), keep(now.keep), b1(a.b1), o1(a.o1), b2(a.b2), o2(a.o2), c1(now.c1), c2(now.c2), eps(a.eps), none(a.minus_zero);
    float r[8], f[8];
    float mtop = 0.f;
    unsigned vmax = 0;                               // v is not negative: its values order like their bits, NaN on top
    scale8(g, now.gs);
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        const Pair gk(g[k], g[k + 1]);
        const Pair mk = fma2(b1, Pair(m[k], m[k + 1]), none) + fma2(o1, gk, none);
        const Pair vk = fma2(b2, Pair(v[k], v[k + 1]), none) + fma2(o2 * gk, gk, none);
        mk.split(m[k], m[k + 1]);
        vk.split(v[k], v[k + 1]);
        r[k] = sqrt_near<SUB>(v[k]);
        r[k + 1] = sqrt_near<SUB>(v[k + 1]);
        float d0, d1;                                // denominators, below 2^126
        fma2(Pair(r[k], r[k + 1]), c2, eps).split(d0, d1);
        const Pair u = (mk * c1) * Pair(rcp_near(d0), rcp_near(d1));
        const Pair wk = fma2(down, u, keep * Pair(w[k], w[k + 1]));
        wk.split(w[k], w[k + 1]);
        fma2(ahead, u, wk).split(f[k], f[k + 1]);
        mtop = max_nan(mtop, max_nan(fabsf(m[k]), fabsf(m[k + 1])));
        vmax = max(vmax, max(__float_as_uint(v[k]), __float_as_uint(v[k + 1])));
    }
    q.store(t.w, w);
    if (t.fwd) {
        if (a.fwd_dtype == 0) q.store(reinterpret_cast<float*>(t.fwd), f);
        else if (a.fwd_dtype == 1) q.store(reinterpret_cast<__nv_bfloat16*>(t.fwd), f);
        else q.store(reinterpret_cast<__half*>(t.fwd), f);
    }
    if constexpr (BITS == 32) {
        q.store(reinterpret_cast<float*>(t.m), m);
        q.store(reinterpret_cast<float*>(t.v), v);
    } else {
        const unsigned mmax = __reduce_max_sync(0xffffffffu, __float_as_uint(mtop));
        vmax = __reduce_max_sync(0xffffffffu, vmax);
        const float nan = __int_as_float(0x7fc00000);
        const float ma = __uint_as_float(mmax), ra = __fsqrt_rn(__uint_as_float(vmax));   // the root grows with v
        const bool m_live = ma >= 0x1p-100f, r_live = ra > 0.f;      // below: a zero block (1 / ma may overflow)
        const float mi = m_live ? __fdiv_rn(kMTop, ma) : 0.f, ri = r_live ? __fdiv_rn(kRTop, ra) : 0.f;
        if (lane == 0) {
            t.m_scale[block] = mmax >= 0x7f800000u ? nan : m_live ? __fmul_rn(ma, 1.f / kMTop) : 0.f;
            t.v_scale[block] = vmax >= 0x7f800000u ? nan : __fdiv_rn(ra, kRTop);
        }
        unsigned long long z[VEC ? 2 : 8];
        if constexpr (VEC) {
            z[0] = splitmix64(now.key, (unsigned long long)q.at(0) >> 2);
            z[1] = splitmix64(now.key, ((unsigned long long)q.at(0) >> 2) + 1);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) z[k] = (splitmix64(now.key, (unsigned long long)q.at(k) >> 2) >> (16 * (int)(q.at(k) & 3))) & 0xffffu;
        }
        scale8(m, mi);
        uint2 rc;
        // Exactly rounded roots: for one lane in some 8000, and for blocks so small that roots which count as
        // zero above are not far below the largest (2^-86: the smallest normal root is 2^-20 of its root).
        if (encode_r8<VEC>(rc, v, r, ri, z) || (vmax != 0 && __uint_as_float(vmax) < 0x1p-86f)) {
#pragma unroll
            for (int k = 0; k < 8; ++k) r[k] = __fsqrt_rn(v[k]);
            encode_r8<VEC>(rc, v, r, ri, z);
        }
        q.store_codes(reinterpret_cast<unsigned char*>(t.m), encode_m8(m));
        q.store_codes(reinterpret_cast<unsigned char*>(t.v), rc);
    }
}

// A thread block takes one round of kAdamRound elements.  What is in flight at any time is then one
// contiguous stretch of every array, which the DRAM's open pages reward: blocks of four consecutive
// rounds move an 8-bit step's bytes at 4.6 TB/s, single rounds at 6.5 (151 M elements, no arithmetic).
// Measured: 32-bit states, float32 gradients and a bf16 copy, 63 M elements: 277 us, 6.8 TB/s, the copy
// rate.  8-bit states, bf16 gradients and copy, 151 M elements: 443 us, 5.5 TB/s; there some 70
// instructions per element (roundings that have to be exact, random numbers, two encodings) take
// nearly as long to issue as the bytes take to move.  Seven blocks of 128 threads, 72 registers and a few spilled
// ones, beat four of 256 and eight of 128 by 2 to 3 %.  Inputs copied ahead into shared memory by the warp that
// uses them did not help.
template <int BITS, typename GT, int MAXT>
__global__ void __launch_bounds__(kAdamThreads, 7)
adamw_kernel(const __grid_constant__ AdamTable<MAXT> a) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int at = a.s.near[blockIdx.x >> a.s.near_shift]; // the tensor that holds this round
    while (at + 1 < a.s.n && a.t[at + 1].first_round <= blockIdx.x) ++at;
    const AdamTensor& t = a.t[at];
    const long long block = (long long)(blockIdx.x - t.first_round) * (kAdamRound / kAdamBlock) + warp;
    if (block * kAdamBlock >= t.n) return;
    auto scalars = [&](AdamNow& now) {
        long long step = a.s.step;
        now.gs = a.s.grad_scale ? *a.s.grad_scale : 1.f;
        const double lr = a.s.dev_lr ? (double)*a.s.dev_lr : a.s.lr;
        now.lr = (float)lr;
        now.c1 = a.s.c1;
        now.c2 = a.s.c2;
        if (a.s.dev_step) {
            step = *a.s.dev_step;
            // one lane's work for the warp
            float c = 0.f;
            if (lane < 2) {
                const double left = 1.0 - pow(lane ? a.s.beta2 : a.s.beta1, (double)step);
                c = (float)(1.0 / (lane ? sqrt(left) : left));
            }
            now.c1 = __shfl_sync(0xffffffffu, c, 0);
            now.c2 = __shfl_sync(0xffffffffu, c, 1);
        }
        now.keep = (float)(1.0 - lr * (double)t.decay);
        now.key = t.rnd + (a.s.seed + (unsigned long long)step) * 0xD1342543DE82EF95ull;
        return (bool)isfinite(now.gs);               // else the step is left out
    };
    const bool whole = t.vec && (block + 1) * kAdamBlock <= t.n;
    if (a.s.subnormal) {
        if (whole) adamw_block<BITS, GT, true, true>(a.s, t, block, lane, scalars);
        else adamw_block<BITS, GT, false, true>(a.s, t, block, lane, scalars);
    } else {
        if (whole) adamw_block<BITS, GT, true, false>(a.s, t, block, lane, scalars);
        else adamw_block<BITS, GT, false, false>(a.s, t, block, lane, scalars);
    }
}

template <bool VEC>
__device__ __forceinline__ void moments_block(const unsigned char* m, const float* m_scale, const unsigned char* v, const float* v_scale,
                                              long long block, const AdamLane<VEC>& q, float* m_out, float* v_out) {
    float x[8];
    if (m_out) {
        const float s = m_scale[block];
        decode_m8(x, q.load_codes(m));
        scale8(x, s);
        q.store(m_out, x);
    }
    if (v_out) {
        const float s = v_scale[block];
        decode_r8(x, q.load_codes(v));
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float r = __fmul_rn(x[k], s);
            x[k] = __fmul_rn(r, r);
        }
        q.store(v_out, x);
    }
}

__global__ void __launch_bounds__(kAdamThreads)
adamw_moments_kernel(const unsigned char* __restrict__ m, const float* __restrict__ m_scale, const unsigned char* __restrict__ v,
                     const float* __restrict__ v_scale, long long n, float* __restrict__ m_out, float* __restrict__ v_out, int vec) {
    const long long block = (long long)blockIdx.x * (kAdamRound / kAdamBlock) + (threadIdx.x >> 5), base = block * kAdamBlock;
    const int lane = threadIdx.x & 31;
    if (base >= n) return;
    if (vec && base + kAdamBlock <= n) moments_block(m, m_scale, v, v_scale, block, AdamLane<true>{base, n, lane}, m_out, v_out);
    else moments_block(m, m_scale, v, v_scale, block, AdamLane<false>{base, n, lane}, m_out, v_out);
}

}  // namespace pb
