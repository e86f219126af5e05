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

// Index of a token, or -1 where there is none.  A value outside [0, n) other than -1 is
// reported through the status word, if the caller gave one, and then treated like -1.
template <typename I>
__device__ __forceinline__ long long token_id(const I* ids, long long t, long long n, int* status) {
    const long long id = (long long)ids[t];
    if (id >= 0 && id < n) return id;
    if (id != -1 && status) *status = 1;      // every writer writes the same value
    return -1;
}

__device__ __forceinline__ float warp_max_f(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
}

// SplitMix64 finaliser (Steele, Lea & Flood 2014) of a counter on a stream that starts at `base`.
__host__ __device__ __forceinline__ unsigned long long splitmix64(unsigned long long base, unsigned long long counter) {
    unsigned long long z = base + (counter + 1ull) * 0x9E3779B97F4A7C15ull;
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

}  // namespace pb
