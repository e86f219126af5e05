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
// finite logit has no gradient.  One read and one write per logit: bound by memory traffic.
constexpr int kBwdThreads = 128;
template <typename T> constexpr int kBwdVecs = 16 / (int)sizeof(T);          // pieces of eight per thread
template <typename T> constexpr int kBwdTile = kBwdThreads * kBwdVecs<T> * 8;

constexpr float kLog2e = 1.4426950408889634f;

struct BwdRow {
    float it, z, h, all, gh;        // with the factor it: all = g_lse - g_logp, gh = g_entropy
    bool entropy;
    __device__ __forceinline__ void gradient(float (&x)[8]) const {
        const Pair t(it), mz(-z), log2e(kLog2e), f(all), mh(-gh), hh(h);
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
            float a, b;
            Pair lp = fma2(Pair(x[k], x[k + 1]), t, mz), factor = f;
            if (entropy) {
                lp.split(a, b);     // NaN stays NaN; a logit of -inf has p = 0, and a finite factor through this
                lp = Pair(max_nan(a, -1e30f), max_nan(b, -1e30f));
                factor = fma2(mh, lp + hh, f);
            }
            (lp * log2e).split(a, b);
            (Pair(exp2_near(a), exp2_near(b)) * factor).split(x[k], x[k + 1]);
        }
    }
    __device__ __forceinline__ float gradient(float x) const {
        float e[8] = {x, x, x, x, x, x, x, x};
        gradient(e);
        return e[0];
    }
};

template <typename T, typename I>
__global__ void __launch_bounds__(kBwdThreads)
logprob_bwd_kernel(const T* logits, long long vocab, long long ld, const I* __restrict__ tokens, double inv_temp,
                   const float* __restrict__ lse, const float* __restrict__ entropy, const float* __restrict__ g_logp,
                   const float* __restrict__ g_entropy, const float* __restrict__ g_lse, T* dlogits, long long ld_d,
                   int* status) {
    const long long r = blockIdx.y;
    const T* x = logits + r * ld;
    T* d = dlogits + r * ld_d;
    const int tid = threadIdx.x;
    // Pieces of eight start where the logits' row reaches their alignment, if the gradient's row does there too.
    constexpr int ALIGN = 8 * (int)sizeof(T);
    const long long head = min(vocab, (long long)((-(long long)reinterpret_cast<uintptr_t>(x)) & (ALIGN - 1)) / (int)sizeof(T));
    const bool vec = ((reinterpret_cast<uintptr_t>(d + head)) & (ALIGN - 1)) == 0;
    const long long pieces = vec ? (vocab - head) / 8 : 0;
    const long long first = (long long)blockIdx.x * kBwdThreads * kBwdVecs<T> + tid;
    uint4 raw[kBwdVecs<T>][sizeof(T) / 2];
#pragma unroll
    for (int k = 0; k < kBwdVecs<T>; ++k)
        if (first + k * kBwdThreads < pieces)
#pragma unroll
            for (int j = 0; j < (int)sizeof(T) / 2; ++j)
                raw[k][j] = *reinterpret_cast<const uint4*>(x + head + (first + k * kBwdThreads) * 8 + j * 4);
    BwdRow q;
    q.z = lse[r];
    q.it = (float)inv_temp;
    long long id = -1;
    float gl = 0.f, gz = 0.f;
    q.h = 0.f;
    if (g_logp) { id = token_id(tokens, r, vocab, tid == 0 && blockIdx.x == 0 ? status : nullptr); gl = id >= 0 ? g_logp[r] : 0.f; }
    float gh = 0.f;
    if (g_entropy) { gh = g_entropy[r]; q.h = entropy[r]; }
    if (g_lse) gz = g_lse[r];
    q.all = q.it * (gz - gl);
    q.gh = q.it * gh;
    q.entropy = g_entropy != nullptr;
    const bool empty = q.z == -INFINITY;
    // the token's own gradient replaces what the row's formula gives there
    auto at_token = [&](float xv) {
        const float lp = (float)((double)xv * inv_temp - q.z);
        const float p = expf(lp);
        const float g = gz * p - gl * expm1f(lp) - (p > 0.f ? gh * p * (lp + q.h) : 0.f);
        return empty ? 0.f : q.it * g;
    };
#pragma unroll
    for (int k = 0; k < kBwdVecs<T>; ++k) {
        const long long piece = first + k * kBwdThreads;
        if (piece >= pieces) continue;
        float f[8];
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                f[4 * j] = __uint_as_float(raw[k][j].x); f[4 * j + 1] = __uint_as_float(raw[k][j].y);
                f[4 * j + 2] = __uint_as_float(raw[k][j].z); f[4 * j + 3] = __uint_as_float(raw[k][j].w);
            }
        } else {
            unpack8(f, raw[k][0], T());
        }
        const long long i = head + piece * 8;
        const bool mine = id >= i && id < i + 8;
        float xt = 0.f;
        if (mine)
#pragma unroll
            for (int j = 0; j < 8; ++j) xt = id == i + j ? f[j] : xt;
        q.gradient(f);
        if (empty)
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = 0.f;
        if (mine) {
            const float g = at_token(xt);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = id == i + j ? g : f[j];
        }
        if constexpr (sizeof(T) == 4) store8_wide(d + i, f);
        else store8(d + i, f);
    }
    // what the pieces leave: the row's ends, or the whole tile
    auto one = [&](long long i) {
        const float xv = to_f32(x[i]);
        d[i] = from_f32<T>(i == id ? at_token(xv) : empty ? 0.f : q.gradient(xv));
    };
    if (vec) {
        const long long tail = head + pieces * 8;
        if (blockIdx.x == 0 && tid < head) one(tid);
        if (blockIdx.x == 0 && tid >= 32 && tail + tid - 32 < vocab) one(tail + tid - 32);
    } else {
        const long long i0 = (long long)blockIdx.x * kBwdTile<T>, i1 = min(vocab, i0 + kBwdTile<T>);
        for (long long i = i0 + tid; i < i1; i += kBwdThreads) one(i);
    }
}

}  // namespace pb
