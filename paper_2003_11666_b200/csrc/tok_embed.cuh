// Embedding lookup with scaling, and its gradient by sorted tokens.
//
//   out[t, :]  = scale * table[id_t, :]                   (no token: a zero row)
//   dtable[v,:] (+)= scale * sum over t with id_t = v of dout[t, :],  v != padding
//
// Both are bound by memory traffic: one multiplication or addition per element moved.
//
// Gradient.  The tokens are sorted by id (stable, so equal ids stay in their order) with a radix
// sort of (id, position) pairs; then groups of threads walk stretches of the sorted list, add the
// rows of a run of equal ids in registers and write each table row once.  Runs that cross
// stretches leave partial rows, which the group that arrives last adds up in list order; so
// sums depend on the ids alone, no addition to memory is atomic, and a row shared by
// thousands of tokens is still the work of many groups.
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

// ---------------------------------------------------------------- sort
constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32;
constexpr int kSortSub = 2048;             // tokens a block ranks at a time: 128 consecutive ones per warp
constexpr int kSortMaxBits = 9;            // digit bits of a pass: one bin per thread
constexpr int kSortMaxTiles = 256;         // blocks; longer lists give each block several sub-tiles

struct SortPlan {
    int passes, bits, tiles;
    long long n, tile;                     // tokens, tokens per block (a multiple of kSortSub)
    unsigned *key[2], *pos[2];             // ping-pong
    int* hist;                             // [passes][tiles][1 << bits]
    unsigned* zero;                        // words to clear for the reduction's counters
    long long n_zero;
};

struct SortShared {
    int warp[kSortWarps][1 << kSortMaxBits];
    int base[1 << kSortMaxBits];
    int scan[kSortWarps];
};

static_assert((1 << kSortMaxBits) <= kSortThreads, "a bin per thread");

// base[b] <- sum of base[0..b-1]
__device__ __forceinline__ void scan_bins(SortShared& sh, int bins) {
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const int v = tid < bins ? sh.base[tid] : 0;
    int sum = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int q = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += q;
    }
    if (lane == 31) sh.scan[w] = sum;
    __syncthreads();
    int before = 0;
    for (int q = 0; q < w; ++q) before += sh.scan[q];
    if (tid < bins) sh.base[tid] = before + sum - v;
    __syncthreads();
}

template <typename I>
struct SortIds {
    const I* ids;
    long long vocab, padding;
    int* status;
    // tokens without a gradient sort behind the last row
    __device__ __forceinline__ unsigned key(long long t) const {
        const long long id = token_id(ids, t, vocab, status);
        return (unsigned)(id < 0 || id == padding ? vocab : id);
    }
};

// One stable pass over the tokens [lo, hi) of a block whose first free place of digit b is sh.base[b].
template <typename I>
__device__ __forceinline__ void sort_scatter(const SortPlan& a, const SortIds<I>& in, int p, long long lo, long long hi, SortShared& sh) {
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const int bins = 1 << a.bits, shift = p * a.bits;
    const unsigned* ik = a.key[(p + 1) & 1];
    const unsigned* ip = a.pos[(p + 1) & 1];
    unsigned* ok = a.key[p & 1];
    unsigned* op = a.pos[p & 1];
    int* next = p + 1 < a.passes && a.tiles > 1 ? a.hist + (size_t)(p + 1) * a.tiles * bins : nullptr;
    for (long long s0 = lo; s0 < hi; s0 += kSortSub) {
        for (int b = tid; b < bins * kSortWarps; b += kSortThreads) sh.warp[b >> a.bits][b & (bins - 1)] = 0;
        __syncthreads();
        unsigned key[4], pos[4];
        int digit[4], rank[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const long long t = s0 + w * 128 + q * 32 + lane;
            const bool live = t < hi;
            key[q] = !live ? 0u : p == 0 ? in.key(t) : ik[t];
            pos[q] = !live ? 0u : p == 0 ? (unsigned)t : ip[t];
            digit[q] = live ? (int)((key[q] >> shift) & (bins - 1)) : -1;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {                      // rank among the warp's earlier tokens of the digit
            const unsigned peers = __match_any_sync(0xffffffffu, digit[q]);
            const int before = __popc(peers & ((1u << lane) - 1));
            int had = 0;
            if (digit[q] >= 0) had = sh.warp[w][digit[q]];
            __syncwarp();
            rank[q] = had + before;
            if (digit[q] >= 0 && before == 0) sh.warp[w][digit[q]] = had + __popc(peers);
            __syncwarp();
        }
        __syncthreads();
        for (int b = tid; b < bins; b += kSortThreads) {   // counts of the warps -> first places
            int at = sh.base[b];
#pragma unroll
            for (int q = 0; q < kSortWarps; ++q) {
                const int c = sh.warp[q][b];
                sh.warp[q][b] = at;
                at += c;
            }
            sh.base[b] = at;
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            int bin = -1;
            if (digit[q] >= 0) {
                const long long d = sh.warp[w][digit[q]] + rank[q];
                ok[d] = key[q];
                op[d] = pos[q];
                if (next) bin = (int)(d / a.tile) * bins + (int)((key[q] >> (shift + a.bits)) & (bins - 1));
            }
            if (next) {                                    // the next pass's counts, one addition per warp and bin
                const unsigned peers = __match_any_sync(0xffffffffu, bin);
                if (bin >= 0 && lane == __ffs(peers) - 1) atomicAdd(next + bin, __popc(peers));
            }
        }
        __syncthreads();
    }
}

// Counts of the first pass; clears what later launches count in.  A list that fits one block is
// sorted here altogether.
template <typename I>
__global__ void __launch_bounds__(kSortThreads)
embed_sort_kernel(const __grid_constant__ SortPlan a, const SortIds<I> in) {
    __shared__ SortShared sh;
    const int tid = threadIdx.x, bins = 1 << a.bits;
    for (long long k = (long long)blockIdx.x * kSortThreads + tid; k < a.n_zero; k += (long long)gridDim.x * kSortThreads) a.zero[k] = 0;
    const long long lo = (long long)blockIdx.x * a.tile, hi = min(a.n, lo + a.tile);
    const int passes = a.tiles == 1 ? a.passes : 1;
    for (int p = 0; p < passes; ++p) {
        for (int b = tid; b < bins; b += kSortThreads) sh.base[b] = 0;
        __syncthreads();
        for (long long t = lo + tid; t < hi; t += kSortThreads) {
            const unsigned k = p == 0 ? in.key(t) : a.key[(p + 1) & 1][t];
            atomicAdd(&sh.base[(k >> (p * a.bits)) & (bins - 1)], 1);
        }
        __syncthreads();
        if (a.tiles == 1) {
            scan_bins(sh, bins);
            sort_scatter(a, in, p, lo, hi, sh);            // ends with a barrier: its stores are visible to the block
        } else {
            for (int b = tid; b < bins; b += kSortThreads) a.hist[(size_t)blockIdx.x * bins + b] = sh.base[b];
            for (int q = 1; q < a.passes; ++q)
                for (int b = tid; b < bins; b += kSortThreads) a.hist[((size_t)q * a.tiles + blockIdx.x) * bins + b] = 0;
        }
    }
}

template <typename I>
__global__ void __launch_bounds__(kSortThreads)
embed_scatter_kernel(const __grid_constant__ SortPlan a, const SortIds<I> in, int p) {
    __shared__ SortShared sh;
    const int tid = threadIdx.x, bins = 1 << a.bits;
    const int* hist = a.hist + (size_t)p * a.tiles * bins;
    int before = 0, total = 0;                               // earlier blocks' count of this thread's digit, and all blocks'
    if (tid < bins) {
#pragma unroll 8
        for (int t = 0; t < a.tiles; ++t) {
            const int c = hist[(size_t)t * bins + tid];
            if (t < (int)blockIdx.x) before += c;
            total += c;
        }
        sh.base[tid] = total;
    }
    __syncthreads();
    scan_bins(sh, bins);
    if (tid < bins) sh.base[tid] += before;
    __syncthreads();
    const long long lo = (long long)blockIdx.x * a.tile;
    sort_scatter(a, in, p, lo, min(a.n, lo + a.tile), sh);
}

// ---------------------------------------------------------------- reduction
constexpr int kRedThreads = 256;
constexpr int kRedCols = 8;                // columns of a thread
constexpr int kRedGroup = 32;              // stretches whose partial rows are joined first
constexpr int kZeroRows = 32;              // table rows of a clearing block

struct RedPlan {
    const unsigned *key, *pos;             // sorted
    long long n, vocab, dim, ld_dout, ld;
    float scale;
    int len;                               // entries of a stretch, a multiple of 4
    int stretches, lanes;                  // lanes: threads across a row's columns (a power of two)
    int red_blocks;                        // blocks [0, red_blocks) reduce, the rest clear rows
    float* part;                           // [stretches][2][dim]: runs that came in from before, runs that go on
    unsigned* arrived;                     // [slabs][stretches][3]
    int accumulate;
};

// Eight columns of a row: thread-contiguous where everything is aligned, else interleaved.
template <bool VEC>
struct Cols {
    long long c;
    int lanes;
    long long dim;
    __device__ __forceinline__ long long at(int k) const { return VEC ? c + k : c + (long long)k * lanes; }
    __device__ __forceinline__ bool in(int k) const { return at(k) < dim; }
};

template <bool VEC, typename T>
__device__ __forceinline__ void load_cols(float (&x)[kRedCols], const T* row, const Cols<VEC>& q) {
    if constexpr (VEC) {
        if (q.c < q.dim) load8(x, row + q.c);
        else
#pragma unroll
            for (int k = 0; k < kRedCols; ++k) x[k] = 0.f;
    } else {
#pragma unroll
        for (int k = 0; k < kRedCols; ++k) x[k] = q.in(k) ? to_f32(row[q.at(k)]) : 0.f;
    }
}
template <bool VEC, typename T>
__device__ __forceinline__ void store_cols(T* row, const float (&x)[kRedCols], const Cols<VEC>& q) {
    if constexpr (VEC) {
        if (q.c < q.dim) store8(row + q.c, x);
    } else {
#pragma unroll
        for (int k = 0; k < kRedCols; ++k)
            if (q.in(k)) row[q.at(k)] = from_f32<T>(x[k]);
    }
}

// First entry of the sorted list with a key of at least v.
__device__ __forceinline__ long long lower_bound(const unsigned* key, long long n, unsigned v) {
    long long lo = 0, hi = n;
    while (lo < hi) {
        const long long mid = (lo + hi) >> 1;
        if (key[mid] < v) lo = mid + 1; else hi = mid;
    }
    return lo;
}

template <bool VEC, typename G>
__device__ __forceinline__ void finish_row(G* dtable, const RedPlan& a, unsigned v, float (&s)[kRedCols], const Cols<VEC>& q) {
    G* row = dtable + (long long)v * a.ld;
    float old[kRedCols];
    if (a.accumulate) load_cols<VEC>(old, row, q);
#pragma unroll
    for (int k = 0; k < kRedCols; ++k) s[k] = a.accumulate ? old[k] + a.scale * s[k] : a.scale * s[k];
    store_cols<VEC>(row, s, q);
}

// Sum of the partial rows `kind[first]`, head[first + step], ... in order; `slot(first)` is the first.
template <bool VEC>
__device__ __forceinline__ void add_parts(float (&s)[kRedCols], const RedPlan& a, int first, int first_kind, int last, int step, const Cols<VEC>& q) {
#pragma unroll
    for (int k = 0; k < kRedCols; ++k) s[k] = 0.f;
#pragma unroll 4
    for (int t = first; t <= last; t += step) {
        float x[kRedCols];
        const float* row = a.part + ((size_t)t * 2 + (t == first ? first_kind : 0)) * a.dim;
        if constexpr (VEC) {
            const float4* r4 = reinterpret_cast<const float4*>(row + (q.c < q.dim ? q.c : 0));
            const float4 y = __ldcg(r4), z = __ldcg(r4 + 1);
            x[0] = y.x; x[1] = y.y; x[2] = y.z; x[3] = y.w; x[4] = z.x; x[5] = z.y; x[6] = z.z; x[7] = z.w;
        } else {
#pragma unroll
            for (int k = 0; k < kRedCols; ++k) x[k] = q.in(k) ? __ldcg(row + q.at(k)) : 0.f;
        }
#pragma unroll
        for (int k = 0; k < kRedCols; ++k) s[k] += x[k];
        if (step > 1 && t == first) t = t / step * step;     // the first group starts where the run does
    }
}

template <bool VEC, typename T, typename G>
__global__ void __launch_bounds__(kRedThreads)
embed_reduce_kernel(const __grid_constant__ RedPlan a, const T* __restrict__ dout, G* __restrict__ dtable) {
    __shared__ int sh_last[kRedThreads][2];
    __shared__ int sh_touched[kZeroRows];
    const int tid = threadIdx.x;
    if ((int)blockIdx.x >= a.red_blocks) {                   // clear the rows that no token points to
        if (blockIdx.y) return;
        const long long v0 = (long long)(blockIdx.x - a.red_blocks) * kZeroRows;
        if (tid < kZeroRows && v0 + tid < a.vocab) {
            const long long e = lower_bound(a.key, a.n, (unsigned)(v0 + tid));
            sh_touched[tid] = e < a.n && a.key[e] == (unsigned)(v0 + tid);
        }
        __syncthreads();
        const int warp = tid >> 5, lane = tid & 31;
        float z[kRedCols] = {};
        for (int r = warp; r < kZeroRows && v0 + r < a.vocab; r += kRedThreads / 32) {
            if (sh_touched[r]) continue;
            G* row = dtable + (v0 + r) * a.ld;
            for (long long c = 0; c < a.dim; c += 32 * kRedCols)
                store_cols<VEC>(row, z, Cols<VEC>{VEC ? c + lane * kRedCols : c + lane, 32, a.dim});
        }
        return;
    }
    const int group = tid / a.lanes, lane = tid % a.lanes, per_block = kRedThreads / a.lanes;
    const int st = blockIdx.x * per_block + group;           // this group's stretch
    const long long slab = (long long)blockIdx.y * a.lanes * kRedCols;
    const Cols<VEC> q{slab + (VEC ? lane * kRedCols : lane), a.lanes, min(a.dim, slab + (long long)a.lanes * kRedCols)};
    const long long e0 = (long long)st * a.len, e1 = min(a.n, e0 + a.len);
    bool head = false, tail = false;                         // partial rows that this stretch leaves
    unsigned head_key = 0, tail_key = 0;
    if (st < a.stretches) {
        const unsigned before = e0 > 0 ? a.key[e0 - 1] : 0xffffffffu;
        const unsigned after = e1 < a.n ? a.key[e1] : 0xffffffffu;
        float s[kRedCols];
#pragma unroll
        for (int k = 0; k < kRedCols; ++k) s[k] = 0.f;
        bool from_before = a.key[e0] == before;
        for (long long e = e0; e < e1; e += 4) {
            unsigned key[5];
            float x[4][kRedCols];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                key[u] = e + u < e1 ? a.key[e + u] : 0xffffffffu;
                if (key[u] < a.vocab) load_cols<VEC>(x[u], dout + (long long)a.pos[e + u] * a.ld_dout, q);
            }
            key[4] = e + 4 < e1 ? a.key[e + 4] : 0xffffffffu;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (key[u] >= a.vocab) continue;             // tokens without a gradient, or behind the end
#pragma unroll
                for (int k = 0; k < kRedCols; ++k) s[k] += x[u][k];
                const bool last = e + u + 1 == e1;
                if (!last && key[u + 1] == key[u]) continue;
                const bool on = last && after == key[u];
                if (from_before || on) {
                    // a run that came in from before keeps that place even if it goes on
                    float* row = a.part + ((size_t)st * 2 + (from_before ? 0 : 1)) * a.dim;
                    store_cols<VEC>(row, s, q);
                    if (from_before) { head = true; head_key = key[u]; } else { tail = true; tail_key = key[u]; }
                } else {
                    finish_row<VEC>(dtable, a, key[u], s, q);
                }
                from_before = false;
#pragma unroll
                for (int k = 0; k < kRedCols; ++k) s[k] = 0.f;
            }
        }
    }
    if (!__syncthreads_or(head || tail)) return;
    // Joining: the stretches of a run inside one aligned group of kRedGroup first, then the groups.
    unsigned* arrived = a.arrived + (size_t)blockIdx.y * a.stretches * 3;
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
        const bool have = kind ? tail : head;
        const unsigned v = kind ? tail_key : head_key;
        int run_first = 0, run_last = 0, first = 0, last = 0;
        if (have) {
            run_first = kind ? st : (int)(lower_bound(a.key, e0, v) / a.len);
            run_last = (int)((lower_bound(a.key, a.n, v + 1) - 1) / a.len);
            const int g0 = st / kRedGroup * kRedGroup;
            first = max(run_first, g0);
            last = min(run_last, g0 + kRedGroup - 1);
        }
        const int first_kind = first == run_first ? 1 : 0;
        __threadfence();
        __syncthreads();
        if (lane == 0) sh_last[group][0] = have && atomicAdd(arrived + (size_t)first * 3 + first_kind, 1u) == (unsigned)(last - first);
        __syncthreads();
        bool top = have && sh_last[group][0];
        float s[kRedCols];
        const int g_first = run_first / kRedGroup, g_last = run_last / kRedGroup;
        if (top) {
            __threadfence();
            add_parts<VEC>(s, a, first, first_kind, last, 1, q);
            if (g_first != g_last) store_cols<VEC>(a.part + ((size_t)first * 2 + first_kind) * a.dim, s, q);
            else { finish_row<VEC>(dtable, a, v, s, q); top = false; }
        }
        __threadfence();
        __syncthreads();
        if (lane == 0) sh_last[group][1] = top && atomicAdd(arrived + (size_t)run_first * 3 + 2, 1u) == (unsigned)(g_last - g_first);
        __syncthreads();
        if (top && sh_last[group][1]) {
            __threadfence();
            add_parts<VEC>(s, a, run_first, 1, run_last, kRedGroup, q);
            finish_row<VEC>(dtable, a, v, s, q);
        }
    }
}

}  // namespace pb
