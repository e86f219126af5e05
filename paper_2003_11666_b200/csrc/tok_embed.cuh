// Embedding lookup with scaling, and its gradient.
//
//   out[t, :]  = scale * table[id_t, :]                   (no token: a zero row)
//   dtable[v,:] (+)= scale * sum over t with id_t = v of dout[t, :],  v != padding
//
// Both are bound by memory traffic: one multiplication per element moved.
#pragma once
#include "tok_common.cuh"

namespace pb {

template <typename T, typename I>
__global__ void __launch_bounds__(256)
embed_fwd_kernel(const T* __restrict__ table, long long vocab, long long dim, long long ld_table,
                 const I* __restrict__ ids, float scale, T* __restrict__ out, long long ld_out, int* status) {
    const long long t = blockIdx.x;
    const long long id = token_id(ids, t, vocab, status);
    for (long long c = threadIdx.x; c < dim; c += blockDim.x)
        out[t * ld_out + c] = from_f32<T>(id >= 0 ? scale * to_f32(table[id * ld_table + c]) : 0.f);
}

template <typename G>
__global__ void __launch_bounds__(256)
embed_zero_kernel(G* __restrict__ dtable, long long dim, long long ld) {
    for (long long c = threadIdx.x; c < dim; c += blockDim.x) dtable[blockIdx.x * ld + c] = from_f32<G>(0.f);
}

// One block per token: the first token of each id adds up the rows of all tokens with that id,
// in their order, so the sum does not depend on scheduling.
template <typename T, typename G, typename I>
__global__ void __launch_bounds__(256)
embed_bwd_kernel(const T* __restrict__ dout, long long ld_dout, const I* __restrict__ ids, long long n,
                 long long vocab, long long dim, float scale, long long padding, G* __restrict__ dtable,
                 long long ld, int accumulate, int* status) {
    const long long t = blockIdx.x;
    const long long id = token_id(ids, t, vocab, status);
    if (id < 0 || id == padding) return;
    int earlier = 0;
    for (long long q = threadIdx.x; q < t && !earlier; q += blockDim.x) earlier = (long long)ids[q] == id;
    if (__syncthreads_or(earlier)) return;
    for (long long c = threadIdx.x; c < dim; c += blockDim.x) {
        float s = 0.f;
        for (long long q = t; q < n; ++q)
            if ((long long)ids[q] == id) s += to_f32(dout[q * ld_dout + c]);
        G* p = dtable + id * ld + c;
        *p = from_f32<G>(accumulate ? to_f32(*p) + scale * s : scale * s);
    }
}

}  // namespace pb
