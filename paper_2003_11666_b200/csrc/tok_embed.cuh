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
// sums depend on the ids alone, every table row has one writer, which adds to it once, and a row
// shared by thousands of tokens is still the work of many groups.
#pragma once
#include <type_traits>

#include "tok_common.cuh"

namespace pb {

// `lanes` threads walk a row in pieces (16 bytes where rows are aligned to them, else one element);
// a group of them takes `ROWS` tokens, whose pieces are all on their way before the first is scaled.
template <typename T, typename I, bool VEC, int ROWS>
__global__ void __launch_bounds__(256)
embed_fwd_kernel(const T* __restrict__ table, long long vocab, long long dim, long long ld_table,
                 const I* __restrict__ ids, long long n, float scale, T* __restrict__ out, long long ld_out, int lanes, int* status) {
    constexpr int PIECE = VEC ? 16 / (int)sizeof(T) : 1;
    const int group = threadIdx.x / lanes, lane = threadIdx.x % lanes;
    const long long t0 = ((long long)blockIdx.x * (256 / lanes) + group) * ROWS;
    if (t0 >= n) return;
    long long id[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) id[k] = t0 + k < n ? token_id(ids, t0 + k, vocab, lane == 0 && blockIdx.y == 0 ? status : nullptr) : -2;
    for (long long c = ((long long)blockIdx.y * lanes + lane) * PIECE; c < dim; c += (long long)gridDim.y * lanes * PIECE) {
        if constexpr (VEC) {
            uint4 x[ROWS];
#pragma unroll
            for (int k = 0; k < ROWS; ++k)
                x[k] = id[k] >= 0 ? *reinterpret_cast<const uint4*>(table + id[k] * ld_table + c) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                if (id[k] == -2) continue;
                uint4 y;
                if constexpr (sizeof(T) == 4) {
                    y = make_uint4(__float_as_uint(scale * __uint_as_float(x[k].x)), __float_as_uint(scale * __uint_as_float(x[k].y)),
                                   __float_as_uint(scale * __uint_as_float(x[k].z)), __float_as_uint(scale * __uint_as_float(x[k].w)));
                } else {
                    float f[8];
                    unpack8(f, x[k], T());
                    y = make_uint4(pack2(scale * f[0], scale * f[1], T()), pack2(scale * f[2], scale * f[3], T()),
                                   pack2(scale * f[4], scale * f[5], T()), pack2(scale * f[6], scale * f[7], T()));
                }
                if (id[k] < 0) y = make_uint4(0, 0, 0, 0);          // even if the scale is not finite
                *reinterpret_cast<uint4*>(out + (t0 + k) * ld_out + c) = y;
            }
        } else {
            float x[ROWS];
#pragma unroll
            for (int k = 0; k < ROWS; ++k) x[k] = id[k] >= 0 ? to_f32(table[id[k] * ld_table + c]) : 0.f;
#pragma unroll
            for (int k = 0; k < ROWS; ++k)
                if (id[k] != -2) out[(t0 + k) * ld_out + c] = from_f32<T>(id[k] < 0 ? 0.f : scale * x[k]);
        }
    }
}

// ---------------------------------------------------------------- sort
constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32;
constexpr int kSortSmall = 4 * kSortThreads;       // tokens that one block sorts altogether
constexpr int kSortSub = 2 * kSortThreads;         // tokens that a block of many places at a time
constexpr int kSortMaxBits = 9;            // digit bits of a pass: one bin per thread
constexpr int kSortMaxTiles = 256;         // blocks; longer lists give each block several sub-tiles

struct SortPlan {
    int passes, bits, tiles, n;
    int tile_shift;                        // tokens per block: kSortSub times a power of two
    uint2* list[2];                        // (key, position), ping-pong
    int* hist;                             // [passes][tiles][1 << bits]
    unsigned* zero;                        // words to clear for the reduction's counters
    int n_zero;
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

// Place of each of the N x 512 tokens among those of its digit.  Warp w holds 32 N consecutive
// tokens, 32 at a time; `digit` is -1 where there is none.  Leaves each warp's counts in sh.warp.
template <int N>
__device__ __forceinline__ void rank_digits(const int (&digit)[N], int (&rank)[N], int bins, SortShared& sh) {
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    for (int b = lane; b < bins; b += 32) sh.warp[w][b] = 0;
    __syncwarp();
#pragma unroll
    for (int q = 0; q < N; ++q) {
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
}

// Counts of the warps -> first places of each warp's tokens of a digit; returns the digit's total.
__device__ __forceinline__ int place_warps(int bin, int at, SortShared& sh) {
    const int first = at;
#pragma unroll
    for (int q = 0; q < kSortWarps; ++q) {
        const int c = sh.warp[q][bin];
        sh.warp[q][bin] = at;
        at += c;
    }
    return at - first;
}

// A list of at most kSortSmall tokens: all passes in one block, the list in shared memory.
template <typename I>
__device__ __forceinline__ void sort_small(const SortPlan& a, const SortIds<I>& in, SortShared& sh, unsigned* sh_key, unsigned short* sh_pos) {
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, bins = 1 << a.bits;
    unsigned key[4], pos[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int t = w * 128 + q * 32 + lane;
        key[q] = t < a.n ? in.key(t) : 0u;
        pos[q] = t;
    }
    for (int p = 0; p < a.passes; ++p) {
        int digit[4], rank[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int t = w * 128 + q * 32 + lane;
            if (p > 0 && t < a.n) { key[q] = sh_key[t]; pos[q] = sh_pos[t]; }
            digit[q] = t < a.n ? (int)((key[q] >> (p * a.bits)) & (bins - 1)) : -1;
        }
        rank_digits(digit, rank, bins, sh);
        if (tid < bins) sh.base[tid] = place_warps(tid, 0, sh);
        __syncthreads();
        scan_bins(sh, bins);
        const bool last = p + 1 == a.passes;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (digit[q] < 0) continue;
            const int d = sh.base[digit[q]] + sh.warp[w][digit[q]] + rank[q];
            if (last) a.list[p & 1][d] = make_uint2(key[q], pos[q]);
            else { sh_key[d] = key[q]; sh_pos[d] = (unsigned short)pos[q]; }
        }
        __syncthreads();
    }
}

// First launch: the digit counts of the first pass, and the memory that later launches count in.
// A list that fits one block is sorted here altogether.
template <typename I>
__global__ void __launch_bounds__(kSortThreads)
embed_sort_kernel(const __grid_constant__ SortPlan a, const SortIds<I> in) {
    __shared__ SortShared sh;
    __shared__ unsigned sh_key[kSortSmall];
    __shared__ unsigned short sh_pos[kSortSmall];
    cudaTriggerProgrammaticLaunchCompletion();
    const int tid = threadIdx.x, bins = 1 << a.bits;
    for (int k = blockIdx.x * kSortThreads + tid; k < a.n_zero; k += a.tiles * kSortThreads) a.zero[k] = 0;
    if (a.tiles == 1) {
        sort_small(a, in, sh, sh_key, sh_pos);
        return;
    }
    const long long lo = (long long)blockIdx.x << a.tile_shift, hi = min((long long)a.n, lo + (1ll << a.tile_shift));
    if (tid < bins) sh.base[tid] = 0;
    __syncthreads();
    for (long long t = lo + tid; t < hi; t += kSortThreads) atomicAdd(&sh.base[in.key(t) & (bins - 1)], 1);
    __syncthreads();
    if (tid < bins) {
        a.hist[(size_t)blockIdx.x * bins + tid] = sh.base[tid];
        for (int q = 1; q < a.passes; ++q) a.hist[((size_t)q * a.tiles + blockIdx.x) * bins + tid] = 0;
    }
}

// One stable pass: every block places its stretch of tokens by the digit of this pass and counts
// the next pass's digits where the tokens land.
template <typename I>
__global__ void __launch_bounds__(kSortThreads)
embed_scatter_kernel(const __grid_constant__ SortPlan a, const SortIds<I> in, int p) {
    __shared__ SortShared sh;
    cudaTriggerProgrammaticLaunchCompletion();
    cudaGridDependencySynchronize();
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const int bins = 1 << a.bits, shift = p * a.bits;
    const int* hist = a.hist + (size_t)p * a.tiles * bins;
    int before = 0, total = 0;                             // earlier blocks' count of this thread's digit, and all blocks'
    if (tid < bins) {
#pragma unroll 16
        for (int t = 0; t < a.tiles; ++t) {
            const int c = hist[(size_t)t * bins + tid];
            if (t < (int)blockIdx.x) before += c;
            total += c;
        }
        sh.base[tid] = total;
    }
    __syncthreads();
    scan_bins(sh, bins);
    int place = tid < bins ? sh.base[tid] + before : 0;    // first free place of this thread's digit
    const uint2* from = a.list[(p + 1) & 1];
    uint2* to = a.list[p & 1];
    constexpr int N = kSortSub / kSortThreads;
    int* next = p + 1 < a.passes ? a.hist + (size_t)(p + 1) * a.tiles * bins : nullptr;
    const long long lo = (long long)blockIdx.x << a.tile_shift, hi = min((long long)a.n, lo + (1ll << a.tile_shift));
    for (long long s0 = lo; s0 < hi; s0 += kSortSub) {
        uint2 token[N];
        int digit[N], rank[N];
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const long long t = s0 + w * (32 * N) + q * 32 + lane;
            const bool live = t < hi;
            token[q] = !live ? make_uint2(0, 0) : p == 0 ? make_uint2(in.key(t), (unsigned)t) : from[t];
            digit[q] = live ? (int)((token[q].x >> shift) & (bins - 1)) : -1;
        }
        rank_digits(digit, rank, bins, sh);
        if (tid < bins) place += place_warps(tid, place, sh);
        __syncthreads();
#pragma unroll
        for (int q = 0; q < N; ++q) {
            int bin = -1;
            if (digit[q] >= 0) {
                const int d = sh.warp[w][digit[q]] + rank[q];
                to[d] = token[q];
                if (next) bin = (d >> a.tile_shift) * bins + (int)((token[q].x >> (shift + a.bits)) & (bins - 1));
            }
            if (next) {                                    // one addition per warp and bin: frequent ids meet here
                const unsigned peers = __match_any_sync(0xffffffffu, bin);
                if (bin >= 0 && lane == __ffs(peers) - 1) atomicAdd(next + bin, __popc(peers));
            }
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- reduction
constexpr int kRedThreads = 256;
constexpr int kRedCols = 8;                // columns of a thread
constexpr int kRedEntries = 2048;          // entries of a block's stretches, held in shared memory
constexpr int kRedGroup = 32;              // stretches whose partial rows are joined first
constexpr int kZeroRows = 1024;            // most table rows of a clearing block

struct RedPlan {
    const uint2* list;                     // sorted (key, position)
    long long n, vocab, dim, ld_dout, ld;
    float scale;
    int len;                               // entries of a stretch, a multiple of 8
    int stretches, lanes;                  // lanes: threads across a row's columns (a power of two)
    int red_blocks;                        // blocks [0, red_blocks) reduce, the rest clear `clear_rows` rows each
    int clear_rows;
    // Short lists: the ids themselves.  Clearing blocks look through them for their rows' tokens and so need not
    // wait for the sort, which one block does meanwhile.
    const void* ids;
    int id_bytes;
    long long padding;
    float* part;                           // [stretches][2][dim]: runs that came in from before, runs that go on
    unsigned* arrived;                     // [slabs][stretches][3]
    int accumulate;
};

// Eight columns of a row, as two pieces of four that lie `lanes` pieces apart where rows are aligned to a
// piece: then every access of a warp covers memory without gaps (pieces of eight leave half of each
// 32-byte sector to a second access, which for additions in memory doubles the work of the L2).
// Otherwise single columns, `lanes` apart.
template <bool VEC>
struct Cols {
    long long c;
    int lanes;
    long long dim;
    __device__ __forceinline__ long long at(int k) const { return VEC ? c + (k >> 2) * 4ll * lanes + (k & 3) : c + (long long)k * lanes; }
    __device__ __forceinline__ bool in(int k) const { return at(k) < dim; }
};

// A thread's columns of a row as they were loaded, converted only when they are added.
template <bool VEC, typename T> struct Raw { T x[kRedCols]; };
template <> struct Raw<true, float> { float4 x[2]; };
template <> struct Raw<true, __nv_bfloat16> { uint2 x[2]; };
template <> struct Raw<true, __half> { uint2 x[2]; };

template <bool VEC, typename T>
__device__ __forceinline__ void load_raw(Raw<VEC, T>& r, const T* row, const Cols<VEC>& q) {
    if constexpr (VEC) {
        using P = std::remove_reference_t<decltype(r.x[0])>;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (q.in(4 * h)) r.x[h] = __ldcs(reinterpret_cast<const P*>(row + q.at(4 * h)));
    } else {
#pragma unroll
        for (int k = 0; k < kRedCols; ++k) r.x[k] = q.in(k) ? row[q.at(k)] : from_f32<T>(0.f);
    }
}
__device__ __forceinline__ void widen4(float* x, const float4& r) { x[0] = r.x; x[1] = r.y; x[2] = r.z; x[3] = r.w; }

template <bool VEC, typename T>
__device__ __forceinline__ void widen(float (&x)[kRedCols], const Raw<VEC, T>& r) {
    if constexpr (!VEC) {
#pragma unroll
        for (int k = 0; k < kRedCols; ++k) x[k] = to_f32(r.x[k]);
    } else if constexpr (sizeof(T) == 4) {
        widen4(x, r.x[0]);
        widen4(x + 4, r.x[1]);
    } else {
        unpack8(x, make_uint4(r.x[0].x, r.x[0].y, r.x[1].x, r.x[1].y), T());
    }
}

template <bool VEC, typename T>
__device__ __forceinline__ void load_cols(float (&x)[kRedCols], const T* row, const Cols<VEC>& q) {
    Raw<VEC, T> r{};
    load_raw(r, row, q);
    widen(x, r);
}
template <bool VEC, typename T>
__device__ __forceinline__ void store_cols(T* row, const float (&x)[kRedCols], const Cols<VEC>& q) {
    if constexpr (VEC) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (!q.in(4 * h)) continue;
            T* p = row + q.at(4 * h);
            if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(p) = make_float4(x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]);
            else *reinterpret_cast<uint2*>(p) = make_uint2(pack2(x[4 * h], x[4 * h + 1], T()), pack2(x[4 * h + 2], x[4 * h + 3], T()));
        }
    } else {
#pragma unroll
        for (int k = 0; k < kRedCols; ++k)
            if (q.in(k)) row[q.at(k)] = from_f32<T>(x[k]);
    }
}

// First and last stretch of the run of v that passes through stretch st.  Most runs reach one stretch
// further, so the distance is doubled before it is halved.
__device__ __forceinline__ int first_stretch(const RedPlan& a, int st, unsigned v) {
    auto reaches = [&](int t) { return t >= 0 && a.list[(long long)t * a.len + a.len - 1].x == v; };    // t is before st: a full stretch
    int in = st, step = 1;                                   // the run is known to be in `in`
    while (reaches(in - step)) { in -= step; step *= 2; }
    int out = max(in - step, -1);                            // and known not to be in `out`
    while (in - out > 1) {
        const int mid = (in + out) / 2;
        if (reaches(mid)) in = mid; else out = mid;
    }
    return in;
}
__device__ __forceinline__ int last_stretch(const RedPlan& a, int st, unsigned v) {
    auto reaches = [&](int t) { return t < a.stretches && a.list[(long long)t * a.len].x == v; };
    int in = st, step = 1;
    while (reaches(in + step)) { in += step; step *= 2; }
    int out = min(in + step, a.stretches);
    while (out - in > 1) {
        const int mid = (in + out) / 2;
        if (reaches(mid)) in = mid; else out = mid;
    }
    return in;
}

// A row's only writer: float32 rows that accumulate are added to in memory, which needs no wait for the old
// values (65536 tokens of 2048 columns: 191 us; reading them first 255).  Such an addition flushes what is below
// 2^-126 to zero, which changes nothing if the addend is kRedLeast at least: an old value that is flushed is less
// than half a step of the sum (2^-126 to a step of 2^-124; to 2^-125 below a power of two), and a sum that
// cancels is a multiple of 2^-125, the step of both numbers.  Smaller addends, and zeros, are added to the value
// read, like those of 16-bit rows, whose sum is rounded once.
constexpr float kRedLeast = 0x1p-100f;
template <bool VEC, typename G>
__device__ __forceinline__ void finish_row(G* dtable, const RedPlan& a, unsigned v, float (&s)[kRedCols], const Cols<VEC>& q) {
    G* row = dtable + (long long)v * a.ld;
#pragma unroll
    for (int k = 0; k < kRedCols; ++k) s[k] *= a.scale;
    if (a.accumulate) {
        if constexpr (sizeof(G) == 4) {
            if constexpr (VEC) {
#pragma unroll
                for (int h = 0; h < 8; h += 4) {
                    if (!q.in(h)) continue;
                    float* p = row + q.at(h);
                    if (fminf(fminf(fabsf(s[h]), fabsf(s[h + 1])), fminf(fabsf(s[h + 2]), fabsf(s[h + 3]))) >= kRedLeast) {
                        asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(p), "f"(s[h]), "f"(s[h + 1]), "f"(s[h + 2]),
                                     "f"(s[h + 3]) : "memory");
                    } else {
                        const float4 old = *reinterpret_cast<const float4*>(p);
                        *reinterpret_cast<float4*>(p) = make_float4(s[h] + old.x, s[h + 1] + old.y, s[h + 2] + old.z, s[h + 3] + old.w);
                    }
                }
            } else {
#pragma unroll
                for (int k = 0; k < kRedCols; ++k) {
                    if (!q.in(k)) continue;
                    float* p = row + q.at(k);
                    if (fabsf(s[k]) >= kRedLeast) asm volatile("red.relaxed.gpu.global.add.f32 [%0], %1;" ::"l"(p), "f"(s[k]) : "memory");
                    else *p += s[k];
                }
            }
            return;
        }
        float old[kRedCols];
        load_cols<VEC>(old, row, q);
#pragma unroll
        for (int k = 0; k < kRedCols; ++k) s[k] += old[k];
    }
    store_cols<VEC>(row, s, q);
}

// Sum, in order, of the partial rows of stretch `first` (the one that goes on, or the one that came in) and of the
// stretches up to `last` at distance `step` (those that came in).
template <bool VEC>
__device__ __forceinline__ void add_parts(float (&s)[kRedCols], const RedPlan& a, int first, int first_kind, int last, int step, const Cols<VEC>& q) {
#pragma unroll
    for (int k = 0; k < kRedCols; ++k) s[k] = 0.f;
#pragma unroll 4
    for (int t = first; t <= last; t += step) {
        float x[kRedCols];
        const float* row = a.part + ((size_t)t * 2 + (t == first ? first_kind : 0)) * a.dim;
        if constexpr (VEC) {
#pragma unroll
            for (int h = 0; h < 2; ++h) widen4(x + 4 * h, q.in(4 * h) ? __ldcg(reinterpret_cast<const float4*>(row + q.at(4 * h))) : make_float4(0, 0, 0, 0));
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
__global__ void __launch_bounds__(kRedThreads, !VEC ? 2 : sizeof(T) == 4 ? 3 : 4)
embed_reduce_kernel(const __grid_constant__ RedPlan a, const T* __restrict__ dout, G* __restrict__ dtable) {
    __shared__ unsigned sh_key[kRedEntries + 2], sh_pos[kRedEntries];
    __shared__ int sh_last[kRedThreads][2];
    __shared__ unsigned sh_touched[kZeroRows / 32];
    const int tid = threadIdx.x;
    if ((int)blockIdx.x >= a.red_blocks) {                   // clear the rows that no token points to
        if (blockIdx.y) return;
        const long long v0 = (long long)(blockIdx.x - a.red_blocks) * a.clear_rows, v1 = min(a.vocab, v0 + a.clear_rows);
        const int warp = tid >> 5, lane = tid & 31;
        for (int k = tid; k < kZeroRows / 32; k += kRedThreads) sh_touched[k] = 0;
        __syncthreads();
        auto touch = [&](long long v) {
            if (v >= v0 && v < v1) atomicOr(&sh_touched[(v - v0) >> 5], 1u << ((v - v0) & 31));
        };
        if (a.ids) {
            for (long long t = tid; t < a.n; t += kRedThreads) {
                const long long id = a.id_bytes == 4 ? (long long)reinterpret_cast<const int*>(a.ids)[t] : reinterpret_cast<const long long*>(a.ids)[t];
                if (id != a.padding) touch(id);
            }
        } else {
            cudaGridDependencySynchronize();
            // 32-way search for the first entry of these rows, then a walk over theirs
            long long lo = 0, hi = a.n;                      // the answer is in [lo, hi]
            while (hi - lo > 32) {
                const long long step = (hi - lo) / 32, at = lo + step * (lane + 1) - 1;
                const unsigned below = __ballot_sync(0xffffffffu, a.list[at].x < (unsigned)v0);
                const int c = __popc(below);                 // the keys are sorted: the first c probes are below
                if (c < 32) hi = lo + step * (c + 1) - 1;
                lo += step * c;
            }
            for (long long e = lo + warp * 32; e < a.n; e += kRedThreads) {
                const unsigned k = e + lane < a.n ? a.list[e + lane].x : 0xffffffffu;
                if (k < a.vocab) touch(k);
                if (__any_sync(0xffffffffu, (long long)k >= v1)) break;
            }
        }
        __syncthreads();
        float z[kRedCols] = {};
        for (long long v = v0 + warp; v < v1; v += kRedThreads / 32) {
            if (sh_touched[(v - v0) >> 5] >> ((v - v0) & 31) & 1) continue;
            G* row = dtable + v * a.ld;
            for (long long c = 0; c < a.dim; c += 32 * kRedCols)
                store_cols<VEC>(row, z, Cols<VEC>{c + lane * (VEC ? 4 : 1), 32, a.dim});
        }
        return;
    }
    cudaGridDependencySynchronize();
    const int group = tid / a.lanes, lane = tid % a.lanes, per_block = kRedThreads / a.lanes;
    const int st = blockIdx.x * per_block + group;           // this group's stretch
    const long long slab = (long long)blockIdx.y * a.lanes * kRedCols;
    const Cols<VEC> q{slab + lane * (VEC ? 4 : 1), a.lanes, min(a.dim, slab + (long long)a.lanes * kRedCols)};
    {                                                        // the block's entries, one more on each side
        const long long b0 = (long long)blockIdx.x * per_block * a.len;
        for (int k = tid; k < per_block * a.len + 2; k += kRedThreads) {
            const long long e = b0 + k - 1;
            const uint2 token = e >= 0 && e < a.n ? a.list[e] : make_uint2(0xffffffffu, 0);
            sh_key[k] = token.x;
            if (k > 0 && k <= per_block * a.len) sh_pos[k - 1] = token.y;
        }
    }
    __syncthreads();
    const unsigned* key = sh_key + 1 + group * a.len;        // key[-1 .. len]
    const unsigned* pos = sh_pos + group * a.len;
    bool head = false, tail = false;                         // partial rows that this stretch leaves
    unsigned head_key = 0, tail_key = 0;
    if (st < a.stretches) {
        constexpr int U = sizeof(T) == 4 ? 2 : 4;            // rows of a batch; the next batch is on its way meanwhile
        Raw<VEC, T> x[U], y[U];
        auto load = [&](Raw<VEC, T>(&z)[U], int e) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (e + u < a.len && key[e + u] < a.vocab) load_raw(z[u], dout + (long long)pos[e + u] * a.ld_dout, q);
        };
        float s[kRedCols];
#pragma unroll
        for (int k = 0; k < kRedCols; ++k) s[k] = 0.f;
        bool from_before = key[0] == key[-1];
        auto add = [&](Raw<VEC, T>(&z)[U], int e) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const unsigned v = key[e + u];
                if (v >= a.vocab) continue;                  // tokens without a gradient, or behind the end
                float w[kRedCols];
                widen(w, z[u]);
#pragma unroll
                for (int k = 0; k < kRedCols; ++k) s[k] += w[k];
                const bool same = key[e + u + 1] == v, last = e + u + 1 == a.len;
                if (same && !last) continue;
                if (from_before || same) {
                    // a run that came in from before keeps that place even if it goes on
                    float* row = a.part + ((size_t)st * 2 + (from_before ? 0 : 1)) * a.dim;
                    store_cols<VEC>(row, s, q);
                    if (from_before) { head = true; head_key = v; } else { tail = true; tail_key = v; }
                } else {
                    finish_row<VEC>(dtable, a, v, s, q);
                }
                from_before = false;
#pragma unroll
                for (int k = 0; k < kRedCols; ++k) s[k] = 0.f;
            }
        };
        load(x, 0);
        for (int e = 0; e < a.len; e += 2 * U) {
            load(y, e + U);
            add(x, e);
            load(x, e + 2 * U);
            add(y, e + U);
        }
    }
    if (!__syncthreads_or(head || tail)) return;
    // Joining: the stretches of a run inside one aligned group of kRedGroup first, then the groups.
    // Of those who left a partial row, the one that arrives last adds them up in list order.
    unsigned* arrived = a.arrived + (size_t)blockIdx.y * a.stretches * 3;
    int run_first[2], run_last[2], first[2], last[2];
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
        run_first[kind] = run_last[kind] = first[kind] = last[kind] = 0;
        if (kind ? !tail : !head) continue;
        const unsigned v = kind ? tail_key : head_key;
        run_first[kind] = kind ? st : first_stretch(a, st, v);
        run_last[kind] = last_stretch(a, st, v);
        const int g0 = st / kRedGroup * kRedGroup;
        first[kind] = max(run_first[kind], g0);
        last[kind] = min(run_last[kind], g0 + kRedGroup - 1);
    }
    __threadfence();
    __syncthreads();
    if (lane == 0) {
#pragma unroll
        for (int kind = 0; kind < 2; ++kind)
            sh_last[group][kind] = (kind ? tail : head) &&
                atomicAdd(arrived + (size_t)first[kind] * 3 + (first[kind] == run_first[kind]), 1u) == (unsigned)(last[kind] - first[kind]);
    }
    __syncthreads();
    bool top[2] = {false, false};                            // joined a group of a run over several groups
    __threadfence();
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
        if (!sh_last[group][kind]) continue;
        const int first_kind = first[kind] == run_first[kind];
        float s[kRedCols];
        add_parts<VEC>(s, a, first[kind], first_kind, last[kind], 1, q);
        top[kind] = run_first[kind] / kRedGroup != run_last[kind] / kRedGroup;
        if (top[kind]) store_cols<VEC>(a.part + ((size_t)first[kind] * 2 + first_kind) * a.dim, s, q);
        else finish_row<VEC>(dtable, a, kind ? tail_key : head_key, s, q);
    }
    if (!__syncthreads_or(top[0] || top[1])) return;
    __threadfence();
    __syncthreads();
    if (lane == 0) {
#pragma unroll
        for (int kind = 0; kind < 2; ++kind)
            sh_last[group][kind] = top[kind] &&
                atomicAdd(arrived + (size_t)run_first[kind] * 3 + 2, 1u) == (unsigned)(run_last[kind] / kRedGroup - run_first[kind] / kRedGroup);
    }
    __syncthreads();
    __threadfence();
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
        if (!sh_last[group][kind]) continue;
        float s[kRedCols];
        add_parts<VEC>(s, a, run_first[kind], 1, run_last[kind], kRedGroup, q);
        finish_row<VEC>(dtable, a, kind ? tail_key : head_key, s, q);
    }
}

}  // namespace pb
