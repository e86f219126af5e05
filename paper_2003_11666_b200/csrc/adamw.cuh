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

constexpr int kAdamMaxTensors = 256;      // tensors of one launch: their table is a kernel parameter
constexpr int kAdamBlock = 256;           // elements that share a scale
constexpr int kAdamChunk = 2048;          // elements of one thread block: a warp per 256

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
    unsigned first_chunk;
};

struct AdamTable {
    AdamTensor t[kAdamMaxTensors];
    int n;
    double lr, beta1, beta2, eps;
    long long step;
    unsigned long long seed;
    const float* grad_scale;
    const float* dev_lr;
    const long long* dev_step;
    int grad_dtype, fwd_dtype, bits;
};

__device__ __forceinline__ float load_as(const void* p, int dtype, long long i) {
    if (dtype == 0) return reinterpret_cast<const float*>(p)[i];
    if (dtype == 1) return to_f32(reinterpret_cast<const __nv_bfloat16*>(p)[i]);
    return to_f32(reinterpret_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_as(void* p, int dtype, long long i, float x) {
    if (dtype == 0) reinterpret_cast<float*>(p)[i] = x;
    else if (dtype == 1) reinterpret_cast<__nv_bfloat16*>(p)[i] = from_f32<__nv_bfloat16>(x);
    else reinterpret_cast<__half*>(p)[i] = from_f32<__half>(x);
}

constexpr float kMTop = 448.f, kRTop = 1.9375f;
constexpr int kRBias = 112 << 4;          // exponent and mantissa bits of 2^-15

__device__ __forceinline__ float decode_m(unsigned char c) {
    __nv_fp8_e4m3 q;
    q.__x = c;
    return (float)q;
}
__device__ __forceinline__ float decode_r(unsigned char c) {
    return c ? __uint_as_float((unsigned)(c + kRBias) << 19) : 0.f;
}

__global__ void __launch_bounds__(256)
adamw_kernel(const __grid_constant__ AdamTable a) {
    __shared__ float sh[4];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int lo = 0, hi = a.n - 1;                        // the tensor whose chunks hold this block
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.t[mid].first_chunk <= blockIdx.x) lo = mid; else hi = mid - 1;
    }
    const AdamTensor& t = a.t[lo];
    const long long step = a.dev_step ? *a.dev_step : a.step;
    if (threadIdx.x == 0) {
        const double lr = a.dev_lr ? (double)*a.dev_lr : a.lr;
        sh[0] = (float)(1.0 / (1.0 - pow(a.beta1, (double)step)));
        sh[1] = (float)(1.0 / sqrt(1.0 - pow(a.beta2, (double)step)));
        sh[2] = (float)lr;
        sh[3] = (float)(1.0 - lr * (double)t.decay);
    }
    __syncthreads();
    const float c1 = sh[0], c2 = sh[1], lr = sh[2], keep = sh[3];
    const float b1 = (float)a.beta1, o1 = (float)(1.0 - a.beta1), b2 = (float)a.beta2, o2 = (float)(1.0 - a.beta2), eps = (float)a.eps;
    const float gs = a.grad_scale ? *a.grad_scale : 1.f;
    if (!isfinite(gs)) return;                       // the step is left out
    const long long block = (long long)(blockIdx.x - t.first_chunk) * (kAdamChunk / kAdamBlock) + warp;
    const long long base = block * kAdamBlock;
    if (base >= t.n) return;
    float m[8], r[8], ms = 0.f, rs = 0.f;
    unsigned mmax = 0, rmax = 0;
    if (a.bits == 8) { ms = t.m_scale[block]; rs = t.v_scale[block]; }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const long long i = base + k * 32 + lane;
        if (i >= t.n) { m[k] = r[k] = 0.f; continue; }
        const float g = __fmul_rn(load_as(t.g, a.grad_dtype, i), gs);
        float mk, vk;
        if (a.bits == 8) {
            mk = __fmul_rn(decode_m(reinterpret_cast<const unsigned char*>(t.m)[i]), ms);
            vk = __fmul_rn(decode_r(reinterpret_cast<const unsigned char*>(t.v)[i]), rs);
            vk = __fmul_rn(vk, vk);
        } else {
            mk = reinterpret_cast<const float*>(t.m)[i];
            vk = reinterpret_cast<const float*>(t.v)[i];
        }
        mk = __fadd_rn(__fmul_rn(b1, mk), __fmul_rn(o1, g));
        vk = __fadd_rn(__fmul_rn(b2, vk), __fmul_rn(__fmul_rn(o2, g), g));
        m[k] = mk;
        r[k] = __fsqrt_rn(vk);
        const float u = (mk * c1) / fmaf(r[k], c2, eps);
        const float w = fmaf(-lr, u, keep * t.w[i]);
        t.w[i] = w;
        if (t.fwd) store_as(t.fwd, a.fwd_dtype, i, fmaf(-lr * t.horizon, u, w));
        if (a.bits == 32) {
            reinterpret_cast<float*>(t.m)[i] = mk;
            reinterpret_cast<float*>(t.v)[i] = vk;
        }
        mmax = max(mmax, __float_as_uint(mk) & 0x7fffffffu);
        rmax = max(rmax, __float_as_uint(r[k]) & 0x7fffffffu);
    }
    if (a.bits == 32) return;
    mmax = __reduce_max_sync(0xffffffffu, mmax);     // magnitudes order like their bits, NaN on top
    rmax = __reduce_max_sync(0xffffffffu, rmax);
    const float nan = __int_as_float(0x7fc00000);
    const float ma = __uint_as_float(mmax), ra = __uint_as_float(rmax);
    const bool m_live = ma >= 0x1p-100f, r_live = ra > 0.f;      // below: a zero block (1 / ma may overflow)
    const float mi = m_live ? __fdiv_rn(kMTop, ma) : 0.f, ri = r_live ? __fdiv_rn(kRTop, ra) : 0.f;
    if (lane == 0) {
        t.m_scale[block] = mmax >= 0x7f800000u ? nan : m_live ? __fmul_rn(ma, 1.f / kMTop) : 0.f;
        t.v_scale[block] = rmax >= 0x7f800000u ? nan : __fdiv_rn(ra, kRTop);
    }
    const unsigned long long key = t.rnd + (a.seed + (unsigned long long)step) * 0xD1342543DE82EF95ull;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const long long i = base + k * 32 + lane;
        if (i >= t.n) continue;
        reinterpret_cast<unsigned char*>(t.m)[i] = __nv_fp8_e4m3(__fmul_rn(m[k], mi)).__x;
        const unsigned noise = (unsigned)(splitmix64(key, (unsigned long long)i >> 2) >> (16 * (i & 3))) & 0xffffu;
        int c = (int)((__float_as_uint(__fmul_rn(r[k], ri)) + (noise << 3)) >> 19) - kRBias;
        c = min(max(c, 1), 255);
        reinterpret_cast<unsigned char*>(t.v)[i] = (unsigned char)(r[k] > 0.f ? c : 0);
    }
}

// The moments that an 8-bit state stands for.
__global__ void __launch_bounds__(256)
adamw_moments_kernel(const unsigned char* __restrict__ m, const float* __restrict__ m_scale,
                     const unsigned char* __restrict__ v, const float* __restrict__ v_scale, long long n,
                     float* __restrict__ m_out, float* __restrict__ v_out) {
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    if (m_out) m_out[i] = __fmul_rn(decode_m(m[i]), m_scale[i / kAdamBlock]);
    if (v_out) {
        const float r = __fmul_rn(decode_r(v[i]), v_scale[i / kAdamBlock]);
        v_out[i] = __fmul_rn(r, r);
    }
}

}  // namespace pb
