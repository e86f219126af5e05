// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and the
// gradient of the three row values.
//
// With y = inv_temperature * x, M = max x, d_i = inv_temperature * (x_i - M), e_i = exp(d_i):
//   Z = sum e_i,  lse = inv_temperature * M + log Z,  logp = d_token - log Z,
//   H = log Z - (sum e_i d_i) / Z.
// The elements equal to the maximum are counted apart from the rest of the sum,
// Z = count + rest, so that a confident row's log Z = log1p(rest) keeps its digits.
#pragma once
#include "tok_common.cuh"

namespace pb {

constexpr int kMaxTop = 32;

// Order of the alternatives: larger logit first, lower index among equal ones.  NaN sorts above
// everything (such a row's results are NaN anyway).
__device__ __forceinline__ unsigned long long top_key(float x, long long i) {
    unsigned b = __float_as_uint(x + 0.f);                    // -0 counts as 0
    b = (b & 0x80000000u) ? ~b : (b | 0x80000000u);
    return ((unsigned long long)b << 32) | (0xffffffffu - (unsigned)i);
}
__device__ __forceinline__ float top_value(unsigned long long key) {
    unsigned b = (unsigned)(key >> 32);
    b = (b & 0x80000000u) ? (b & 0x7fffffffu) : ~b;
    return __uint_as_float(b);
}

template <typename T, typename I>
__global__ void __launch_bounds__(512)
logprob_fwd_kernel(const T* __restrict__ logits, long long vocab, long long ld, const I* __restrict__ tokens,
                   double inv_temp, float* __restrict__ logp, float* __restrict__ entropy, float* __restrict__ lse,
                   int top, float* __restrict__ top_logp, int* __restrict__ top_ids, int* status) {
    __shared__ float sh_f[16];
    __shared__ double sh_d[3][16];
    __shared__ unsigned long long sh_k[16];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const long long r = blockIdx.x;
    const T* x = logits + r * ld;
    const float it = (float)inv_temp;
    float mx = -INFINITY;
    bool bad = false;
    for (long long i = tid; i < vocab; i += 512) {
        const float v = to_f32(x[i]);
        bad |= v != v;
        mx = fmaxf(mx, v);
    }
    mx = warp_max_f(mx);
    if (lane == 0) sh_f[warp] = mx;
    bad = __syncthreads_or(bad);
    for (int w = 0; w < 16; ++w) mx = fmaxf(mx, sh_f[w]);
    bad |= mx == INFINITY;
    const bool empty = mx == -INFINITY && !bad;
    double count = 0, rest = 0, moment = 0;
    for (long long i = tid; i < vocab; i += 512) {
        const float d = it * (to_f32(x[i]) - mx);
        if (d == 0.f) { count += 1; continue; }
        const float e = expf(d);
        if (e > 0.f) { rest += e; moment += (double)e * d; }
    }
    for (int o = 16; o > 0; o >>= 1) {
        count += __shfl_xor_sync(0xffffffffu, count, o);
        rest += __shfl_xor_sync(0xffffffffu, rest, o);
        moment += __shfl_xor_sync(0xffffffffu, moment, o);
    }
    if (lane == 0) { sh_d[0][warp] = count; sh_d[1][warp] = rest; sh_d[2][warp] = moment; }
    __syncthreads();
    count = rest = moment = 0;
    for (int w = 0; w < 16; ++w) { count += sh_d[0][w]; rest += sh_d[1][w]; moment += sh_d[2][w]; }
    double log_z = count > 0 ? log(count) + log1p(rest / count) : 0.0;
    const double nan = __longlong_as_double(0x7ff8000000000000ll);
    if (bad) log_z = nan;
    if (tid == 0) {
        if (logp) {
            const long long id = token_id(tokens, r, vocab, status);
            logp[r] = id < 0 ? 0.f : empty ? -INFINITY : (float)(((double)to_f32(x[id]) - mx) * inv_temp - log_z);
        }
        if (entropy) entropy[r] = empty ? 0.f : (float)(log_z - moment / (count + rest));
        if (lse) lse[r] = empty ? -INFINITY : (float)((double)mx * inv_temp + log_z);
    }
    unsigned long long last = ~0ull;
    for (int k = 0; k < top; ++k) {
        unsigned long long best = 0;
        for (long long i = tid; i < vocab; i += 512) {
            const unsigned long long key = top_key(to_f32(x[i]), i);
            if (key < last && key > best) best = key;
        }
        for (int o = 16; o > 0; o >>= 1) {
            const unsigned long long other = __shfl_xor_sync(0xffffffffu, best, o);
            best = other > best ? other : best;
        }
        __syncthreads();
        if (lane == 0) sh_k[warp] = best;
        __syncthreads();
        for (int w = 0; w < 16; ++w) best = sh_k[w] > best ? sh_k[w] : best;
        last = best;
        if (tid == 0) {
            const float v = top_value(best);
            const bool none = best == 0 || v == -INFINITY || bad;
            top_ids[r * top + k] = none ? -1 : (int)(0xffffffffu - (unsigned)best);
            top_logp[r * top + k] = bad ? __int_as_float(0x7fc00000) : none ? -INFINITY : (float)(((double)v - mx) * inv_temp - log_z);
        }
    }
}

// d x_i = it * ( g_logp (1[i = token] - p_i) - g_entropy p_i (log p_i + H) + g_lse p_i )
// with log p_i = it * x_i - lse.  At the token 1 - p is -expm1(log p).  A row without any
// finite logit has no gradient.
template <typename T, typename I>
__global__ void __launch_bounds__(256)
logprob_bwd_kernel(const T* logits, long long vocab, long long ld, const I* __restrict__ tokens, double inv_temp,
                   const float* __restrict__ lse, const float* __restrict__ entropy, const float* __restrict__ g_logp,
                   const float* __restrict__ g_entropy, const float* __restrict__ g_lse, T* dlogits, long long ld_d,
                   int* status) {
    const long long r = blockIdx.y;
    const float z = lse[r], it = (float)inv_temp;
    long long id = -1;
    float gl = 0.f, gh = 0.f, gz = 0.f, h = 0.f;
    if (g_logp) { id = token_id(tokens, r, vocab, status); gl = id >= 0 ? g_logp[r] : 0.f; }
    if (g_entropy) { gh = g_entropy[r]; h = entropy[r]; }
    if (g_lse) gz = g_lse[r];
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < vocab; i += (long long)gridDim.x * 256) {
        const float x = to_f32(logits[r * ld + i]);
        float g = 0.f;
        if (z != -INFINITY) {
            const float lp = i == id ? (float)((double)x * inv_temp - z) : fmaf(x, it, -z);
            const float p = expf(lp);
            g = (gz - gl) * p;
            if (i == id) g = gz * p - gl * expm1f(lp);
            if (p > 0.f) g -= gh * p * (lp + h);
        }
        dlogits[r * ld_d + i] = from_f32<T>(it * g);
    }
}

}  // namespace pb
