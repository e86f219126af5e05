// Element types, conversions and warp helpers shared by the token operators
// (embedding, log probabilities) and the AdamW step.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace pb {

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }

template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

// Eight consecutive 16-bit elements, 16-byte aligned.
__device__ __forceinline__ void unpack8(float (&x)[8], const uint4& q, __nv_bfloat16) {
    const unsigned w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        x[2 * k] = __uint_as_float(w[k] << 16);
        x[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack8(float (&x)[8], const uint4& q, __half) {
    const unsigned w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[k]));
        x[2 * k] = f.x;
        x[2 * k + 1] = f.y;
    }
}
template <typename T> __device__ __forceinline__ void load8(float (&x)[8], const T* p) {
    unpack8(x, *reinterpret_cast<const uint4*>(p), T());
}
__device__ __forceinline__ unsigned pack2(float a, float b, __nv_bfloat16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const unsigned*>(&h);
}
__device__ __forceinline__ unsigned pack2(float a, float b, __half) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const unsigned*>(&h);
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack2(x[0], x[1], T()), pack2(x[2], x[3], T()), pack2(x[4], x[5], T()), pack2(x[6], x[7], T()));
}

// Eight consecutive floats, 32-byte aligned, in one access.
__device__ __forceinline__ void load8_wide(float (&x)[8], const float* p) {
    asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]) : "l"(p));
}
__device__ __forceinline__ void store8_wide(float* p, const float (&x)[8]) {
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]) : "memory");
}

// Index of a token, or -1 where there is none.  A value outside [0, n) other than -1 is
// reported through the status word, if the caller gave one, and then treated like -1.
template <typename I>
__device__ __forceinline__ long long token_id(const I* ids, long long t, long long n, int* status) {
    const long long id = (long long)ids[t];
    if (id >= 0 && id < n) return id;
    if (id != -1 && status) *status = 1;      // every writer writes the same value
    return -1;
}

__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float exp2_near(float x) {      // to 2^-22 of itself
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Pairs of float32 in one instruction, each rounded like the single operation.  The assembler contracts a product and a sum of pairs; a product that
// must be rounded before it is added is therefore a fused multiply-add of a -0 that it cannot see.
struct Pair {
    unsigned long long x;
    __device__ __forceinline__ Pair() {}
    __device__ __forceinline__ Pair(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(a), "f"(b)); }
    __device__ __forceinline__ explicit Pair(float a) : Pair(a, a) {}
    __device__ __forceinline__ void split(float& a, float& b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
};
__device__ __forceinline__ Pair operator*(Pair a, Pair b) { Pair r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.x) : "l"(a.x), "l"(b.x)); return r; }
__device__ __forceinline__ Pair operator+(Pair a, Pair b) { Pair r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.x) : "l"(a.x), "l"(b.x)); return r; }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) { Pair r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.x) : "l"(a.x), "l"(b.x), "l"(c.x)); return r; }
// Quotient of a number below 2^31 by d >= 1: n m >> s with m = floor(2^s / d) + 1, s = 31 + ceil(log2 d).
struct Quotient {
    unsigned m;
    int s;
    Quotient() = default;
    __host__ explicit Quotient(long long d) : m(0), s(31) {
        while ((1ll << (s - 31)) < d) ++s;
        m = (unsigned)((1ull << s) / (unsigned long long)d + 1);
    }
    __device__ __forceinline__ int operator()(int n) const { return (int)((unsigned long long)(unsigned)n * m >> s); }
};

// SplitMix64 finaliser (Steele, Lea & Flood 2014) of a counter on a stream that starts at `base`.
__host__ __device__ __forceinline__ unsigned long long splitmix64(unsigned long long base, unsigned long long counter) {
    unsigned long long z = base + (counter + 1ull) * 0x9E3779B97F4A7C15ull;
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

}  // namespace pb
