// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and the
// gradient of the three row values.
//
// With y = inv_temperature * x, M = max x, d_i = inv_temperature * (x_i - M), e_i = exp(d_i):
//   Z = sum e_i,  lse = inv_temperature * M + log Z,  logp = d_token - log Z,
//   H = log Z - (sum e_i d_i) / Z.
// The elements equal to the maximum are counted apart from the rest of the sum,
// Z = count + rest, so that a confident row's log Z = log1p(rest) keeps its digits.
#pragma once
#include <cooperative_groups.h>

#include <type_traits>

#include "tok_common.cuh"

namespace pb {

namespace cg = cooperative_groups;

constexpr int kMaxTop = 32;

// ---------------------------------------------------------------- forward
// One pass over the row.  A warp takes pieces of 256 consecutive logits, finds a piece's maximum with one
// warp reduction, and moves its running maximum (the same for all lanes) only when a piece exceeds it; the
// sums e and e d stay in registers.  The maxima of the pieces (of runs of them, for very long rows)
// stay in shared memory, and give the alternatives without a second pass: the k best elements, by value and
// then by index, lie in the k best segments by the same order, for each better segment holds a better
// element.  So at most 32 segments are read again, from L2.
// A few rows are split over a cluster of blocks, joined through distributed shared memory.
constexpr int kFwdThreads = 256, kFwdWarps = kFwdThreads / 32;
constexpr int kPiece = 256;                 // logits of a warp's step: eight per lane
constexpr int kMaxSegments = 2048;          // segments of a row
constexpr int kPickRegs = 16;               // maxima per lane that the pick keeps in registers
constexpr int kMaxCluster = 16;
template <typename T> constexpr int kFwdUnroll = 8 / (int)sizeof(T);       // pieces on their way while as many are added

struct FwdStats {                           // of a warp, a block or a row, relative to the maximum `mx`
    double count, rest, moment;             // elements at the maximum; sum of the others' e; sum of e d
    float mx;
    int bad;
};

struct FwdShared {
    float seg[kMaxSegments];                // of the whole row; a block of a cluster fills its stretch and copies the others'
    unsigned long long keys[kFwdWarps * kMaxTop], gathered[kMaxCluster * kMaxTop], best[kMaxTop];
    FwdStats warp_stats[kFwdWarps], block, row;
    int picked[kMaxTop];
    float threshold;
    int n_picked, n_keys, n_gathered;
    double log_z;
};

template <typename T>
struct FwdRow {
    const T* x;
    int vocab, head;                        // head: logits before the first aligned one, a segment of their own
    __device__ __forceinline__ bool full(int piece) const { return head + (piece + 1) * kPiece <= vocab; }
    // Lane's eight logits of a piece; -inf beyond the end.  Piece -1: the head.
    __device__ __forceinline__ int first(int piece, int lane) const { return piece < 0 ? lane * 8 : head + piece * kPiece + lane * 8; }
    __device__ __forceinline__ void load_any(float (&f)[8], int piece, int lane) const {
        const int i = first(piece, lane), end = piece < 0 ? head : vocab;
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = i + k < end ? to_f32(x[i + k]) : -INFINITY;
    }
    // a full piece as it is in memory
    __device__ __forceinline__ void load_raw(uint4 (&q)[sizeof(T) / 2], int piece, int lane) const {
#pragma unroll
        for (int k = 0; k < (int)sizeof(T) / 2; ++k) q[k] = *reinterpret_cast<const uint4*>(x + first(piece, lane) + 4 * k);
    }
    __device__ __forceinline__ void widen(float (&f)[8], const uint4 (&q)[sizeof(T) / 2]) const {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                f[4 * k] = __uint_as_float(q[k].x); f[4 * k + 1] = __uint_as_float(q[k].y);
                f[4 * k + 2] = __uint_as_float(q[k].z); f[4 * k + 3] = __uint_as_float(q[k].w);
            }
        } else {
            unpack8(f, q[0], T());
        }
    }
    __device__ __forceinline__ void load(float (&f)[8], int piece, int lane) const {
        if (piece >= 0 && full(piece)) {
            if constexpr (sizeof(T) == 4) load8_wide(f, x + first(piece, lane));
            else load8(f, x + first(piece, lane));
        } else {
            load_any(f, piece, lane);
        }
    }
};

__device__ __forceinline__ float warp_max_nan(float x) {
    float r;
    asm("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float max8(const float (&f)[8]) {
    return max_nan(max3(max3(f[0], f[1], f[2]), f[3], f[4]), max3(f[5], f[6], f[7]));
}

// A warp's running sums.
struct FwdAcc {
    float mx = -INFINITY;
    int count = 0;
    Pair rest{0.f, 0.f}, moment{0.f, 0.f};
    // c: log2(e) times the inverse temperature
    __device__ __forceinline__ void add(const float (&f)[8], float top, float c) {
        if (top > mx) {                      // the same for the whole warp
            if (mx > -INFINITY) {
                const float shift = mx - top, s = exp2_near(shift * c);
                float r0, r1;
                rest.split(r0, r1);
                r0 += (float)count;
                moment = (moment + Pair(r0, r1) * Pair(shift)) * Pair(s);
                rest = Pair(r0, r1) * Pair(s);
                count = 0;
            }
            mx = top;
        }
        if (top == mx) {
            if (mx > -INFINITY) add_at_top(f, c);
        } else {
            add_below(f, c);
        }
    }
    // every logit is below the maximum (or NaN)
    __device__ __forceinline__ void add_below(const float (&f)[8], float c) {
        const Pair m(-mx), cc(c);
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
            float a, b;
            (Pair(f[k], f[k + 1]) + m).split(a, b);
            const Pair d(max_nan(a, -1e30f), max_nan(b, -1e30f));      // e d is 0, not 0 times infinity, where e is 0
            (d * cc).split(a, b);
            const Pair e(exp2_near(a), exp2_near(b));
            rest = rest + e;
            moment = fma2(e, d, moment);
        }
    }
    // the maximum itself is counted, not added
    __device__ __forceinline__ void add_at_top(const float (&f)[8], float c) {
        float g[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            count += f[k] == mx;
            g[k] = f[k] == mx ? -INFINITY : f[k];
        }
        add_below(g, c);
    }
};

__device__ __forceinline__ FwdStats join(const FwdStats* p, int n, float c) {
    FwdStats t{0, 0, 0, -INFINITY, 0};
    for (int k = 0; k < n; ++k) { t.mx = fmaxf(t.mx, p[k].mx); t.bad |= p[k].bad; }
    if (t.mx == -INFINITY) return t;
    for (int k = 0; k < n; ++k) {
        if (p[k].mx == -INFINITY) continue;
        if (p[k].mx == t.mx) {
            t.count += p[k].count;
            t.rest += p[k].rest;
            t.moment += p[k].moment;
        } else {
            const float shift = p[k].mx - t.mx;
            const double s = exp2_near(shift * c), all = p[k].rest + p[k].count;
            t.rest += s * all;
            t.moment += s * (p[k].moment + all * shift);
        }
    }
    return t;
}

// Floats in the order of their values as unsigned numbers, and back.
__device__ __forceinline__ unsigned ordered(float x) {
    const unsigned b = __float_as_uint(x + 0.f);              // -0 counts as 0
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(unsigned b) {
    return __uint_as_float((b & 0x80000000u) ? (b & 0x7fffffffu) : ~b);
}

// The value whose ordered bits, without GRAIN low bits that are zero in the value itself, are `k`.
template <int GRAIN>
__device__ __forceinline__ float from_grain(unsigned k) {
    const unsigned b = k << GRAIN;
    return from_ordered((b & 0x80000000u) ? b : b | ((1u << GRAIN) - 1));
}

// The k best of n segments (by maximum, then by index) into sh.picked, and a value that the k-th best
// maximum reaches into sh.threshold; one warp.  Maxima are values of T: GRAIN low bits of them are zero.
template <int GRAIN>
__device__ __forceinline__ void pick_segments(FwdShared& sh, int n, int k, int lane) {
    float t = -INFINITY;
    if (n > k) {
        // largest t with at least k maxima of at least t, by bisection of its bits
        float v[kPickRegs];
        const bool in_regs = n <= 32 * kPickRegs;
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < kPickRegs; ++j) {
            v[j] = in_regs && lane + 32 * j < n ? sh.seg[lane + 32 * j] : -INFINITY;
            top = fmaxf(top, v[j]);
        }
        unsigned lo = ordered(-INFINITY) >> GRAIN, hi = ordered(INFINITY) >> GRAIN;
        if (in_regs) {
            // the k-th largest of the lanes' maxima is reached k times: the answer is there or above
            int above = 0;
            for (int j = 0; j < 32; ++j) {
                const float o = __shfl_sync(0xffffffffu, top, j);
                above += o > top || (o == top && j < lane);
            }
            const unsigned who = __ballot_sync(0xffffffffu, above == min(k, 32) - 1);
            if (who) lo = max(lo, ordered(__shfl_sync(0xffffffffu, top, __ffs(who) - 1)) >> GRAIN);
            hi = max(lo, __reduce_max_sync(0xffffffffu, ordered(top) >> GRAIN));
        }
        while (lo < hi) {
            const unsigned mid = lo + (hi - lo + 1) / 2;
            const float at = from_grain<GRAIN>(mid);
            int c = 0;
            if (in_regs) {
#pragma unroll
                for (int j = 0; j < kPickRegs; ++j) c += v[j] >= at;
            } else {
                for (int j = lane; j < n; j += 32) c += sh.seg[j] >= at;
            }
            c = __reduce_add_sync(0xffffffffu, c);
            if (c >= k) lo = mid; else hi = mid - 1;
            if (c == k) break;
        }
        t = from_grain<GRAIN>(lo);
    }
    int above = 0;                           // segments above t; those equal to t fill up in order
    for (int j = lane; j < n; j += 32) above += sh.seg[j] > t;
    above = __reduce_add_sync(0xffffffffu, above);
    const int equal = min(k, n) - above;
    int at = 0, taken = 0;
    for (int j0 = 0; j0 < n; j0 += 32) {
        const float v = j0 + lane < n ? sh.seg[j0 + lane] : 0.f;
        const bool more = j0 + lane < n && v > t, same = j0 + lane < n && v == t;
        const unsigned below = (1u << lane) - 1, ms = __ballot_sync(0xffffffffu, same);
        const bool take = more || (same && taken + __popc(ms & below) < equal);
        const unsigned mt = __ballot_sync(0xffffffffu, take);
        if (take) sh.picked[at + __popc(mt & below)] = j0 + lane;
        at += __popc(mt);
        taken += __popc(ms);
    }
    if (lane == 0) { sh.n_picked = at; sh.threshold = t; }
}

// A warp's best k keys, the j-th in lane j.
struct BestList {
    unsigned long long mine = 0, least = 0;
    __device__ __forceinline__ void offer(unsigned long long key, int k, int lane) {
        unsigned who = __ballot_sync(0xffffffffu, key > least);
        while (who) {
            const unsigned long long x = __shfl_sync(0xffffffffu, key, __ffs(who) - 1);
            const int at = __popc(__ballot_sync(0xffffffffu, mine > x));
            const unsigned long long up = __shfl_up_sync(0xffffffffu, mine, 1);
            mine = lane < at ? mine : lane == at ? x : up;
            least = __shfl_sync(0xffffffffu, mine, k - 1);
            who &= who - 1;
            who &= __ballot_sync(0xffffffffu, key > least);
        }
    }
};

// best[0..k) <- the k largest of n keys, in order; zero where there are fewer.  By all threads.
__device__ __forceinline__ void rank_keys(unsigned long long* best, const unsigned long long* keys, int n, int k) {
    if ((int)threadIdx.x < k) best[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kFwdThreads) {
        const unsigned long long x = keys[i];
        int above = 0;
        for (int j = 0; j < n; ++j) above += keys[j] > x;     // keys differ: each holds its index; zeros are none
        if (x != 0 && above < k) best[above] = x;
    }
    __syncthreads();
}

template <typename T, typename I, bool CLUSTER>
__global__ void __launch_bounds__(kFwdThreads, 4)
logprob_fwd_kernel(const T* __restrict__ logits, int vocab, long long ld, const I* __restrict__ tokens, double inv_temp,
                   float* __restrict__ logp, float* __restrict__ entropy, float* __restrict__ lse, int top,
                   float* __restrict__ top_logp, int* __restrict__ top_ids, int per_segment, int* status) {
    __shared__ FwdShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int parts = CLUSTER ? (int)cg::this_cluster().num_blocks() : 1, part = CLUSTER ? (int)cg::this_cluster().block_rank() : 0;
    const long long r = blockIdx.x / parts;
    FwdRow<T> row;
    row.x = logits + r * ld;
    row.vocab = vocab;
    constexpr int ALIGN = 8 * (int)sizeof(T);
    row.head = min(vocab, (int)((-(long long)reinterpret_cast<uintptr_t>(row.x)) & (ALIGN - 1)) / (int)sizeof(T));
    const int pieces = (vocab - row.head + kPiece - 1) / kPiece;
    // segments: [the head if there is one,] then runs of `per_segment` pieces; blocks take equal stretches of them
    const int heads = row.head > 0, segments = heads + (pieces + per_segment - 1) / per_segment;
    const int each = (segments + parts - 1) / parts, s_lo = min(segments, part * each), s_hi = min(segments, s_lo + each);
    const float c = (float)(1.4426950408889634 * inv_temp);
    long long id = -1;
    float x_token = 0.f;
    if (part == 0 && tid == 32 && logp) {
        id = token_id(tokens, r, vocab, status);
        if (id >= 0) x_token = to_f32(row.x[id]);
    }
    if (tid == 0) sh.n_keys = sh.n_gathered = 0;

    FwdAcc acc;
    bool bad = false;
    if (per_segment == 1) {
        constexpr int U = kFwdUnroll<T>;
        uint4 x[U][sizeof(T) / 2], y[U][sizeof(T) / 2];
        const int full = heads + (vocab - row.head) / kPiece;            // segments [heads, full) are full pieces
        const int lo = max(s_lo, heads), hi = min(s_hi, full);
        auto load = [&](uint4(&q)[U][sizeof(T) / 2], int s0) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (s0 + u * kFwdWarps < hi) row.load_raw(q[u], s0 + u * kFwdWarps - heads, lane);
        };
        auto one = [&](const float (&f)[8], int s) {
            const float m = warp_max_nan(max8(f));
            bad |= m != m;
            if (lane == 0) sh.seg[s] = m;
            acc.add(f, m, c);
        };
        auto add = [&](uint4(&q)[U][sizeof(T) / 2], int s0) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int s = s0 + u * kFwdWarps;
                if (s >= hi) break;
                float f[8];
                row.widen(f, q[u]);
                one(f, s);
            }
        };
        load(x, lo + warp);
        for (int s0 = lo + warp; s0 < hi; s0 += 2 * U * kFwdWarps) {
            load(y, s0 + U * kFwdWarps);
            add(x, s0);
            load(x, s0 + 2 * U * kFwdWarps);
            add(y, s0 + U * kFwdWarps);
        }
        // the row's ends
        float f[8];
        if (warp == kFwdWarps - 1 && s_lo < heads && s_hi > 0) { row.load_any(f, -1, lane); one(f, 0); }
        if (warp == kFwdWarps - 2 && full < segments && s_lo <= full && full < s_hi) { row.load_any(f, full - heads, lane); one(f, full); }
    } else {
        for (int s = s_lo + warp; s < s_hi; s += kFwdWarps) {
            const int p0 = s < heads ? -1 : (s - heads) * per_segment, p1 = s < heads ? 0 : min(pieces, p0 + per_segment);
            float best = -INFINITY;
            for (int p = p0; p < p1; ++p) {
                float f[8];
                row.load(f, p, lane);
                const float m = warp_max_nan(max8(f));
                best = max_nan(best, m);
                acc.add(f, m, c);
            }
            bad |= best != best;
            if (lane == 0) sh.seg[s] = best;
        }
    }
    {
        float a, b, p, q;
        acc.rest.split(a, b);
        acc.moment.split(p, q);
        a += b;
        p += q;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, o);
            p += __shfl_xor_sync(0xffffffffu, p, o);
        }
        const int count = __reduce_add_sync(0xffffffffu, acc.count);
        if (lane == 0) sh.warp_stats[warp] = FwdStats{(double)count, (double)a, (double)p, acc.mx, bad || acc.mx == INFINITY};
    }
    __syncthreads();
    FwdShared* first = &sh;
    if constexpr (CLUSTER) {
        cg::cluster_group cluster = cg::this_cluster();
        if (tid == 0) sh.block = join(sh.warp_stats, kFwdWarps, c);
        cluster.sync();
        first = cluster.map_shared_rank(&sh, 0);
        if (top > 0) {                                        // every block picks from the whole row's segments
            for (int s = tid; s < segments; s += kFwdThreads) {
                const int owner = s / each;
                if (owner != part) sh.seg[s] = cluster.map_shared_rank(&sh, owner)->seg[s];
            }
            __syncthreads();
        }
    }
    if (part == 0 && tid == 32) {                             // the row's values, beside the pick
        FwdStats all;
        if constexpr (CLUSTER) {
            FwdStats of[kMaxCluster];
            for (int k = 0; k < parts; ++k) of[k] = cg::this_cluster().map_shared_rank(&sh, k)->block;
            all = join(of, parts, c);
        } else {
            all = join(sh.warp_stats, kFwdWarps, c);
        }
        const bool empty = all.mx == -INFINITY && !all.bad;
        const double log_z = all.bad ? __longlong_as_double(0x7ff8000000000000ll) : empty ? 0.0 : log(all.count) + log1p(all.rest / all.count);
        if (logp) logp[r] = id < 0 ? 0.f : empty ? -INFINITY : (float)(((double)x_token - all.mx) * inv_temp - log_z);
        if (entropy) entropy[r] = empty ? 0.f : (float)(log_z - inv_temp * all.moment / (all.count + all.rest));
        if (lse) lse[r] = empty ? -INFINITY : (float)((double)all.mx * inv_temp + log_z);
        sh.log_z = log_z;
        sh.row = all;
    }
    if (top > 0) {
        constexpr int GRAIN = sizeof(T) == 4 ? 0 : std::is_same_v<T, __half> ? 13 : 16;
        if (warp == 0) pick_segments<GRAIN>(sh, segments, top, lane);
        __syncthreads();
        const float t = sh.threshold;
        BestList list;
        const int picked = sh.n_picked;
        for (int j = warp; j < picked; j += kFwdWarps) {
            const int s = sh.picked[j];
            if (s < s_lo || s >= s_hi) continue;
            const int p0 = s < heads ? -1 : (s - heads) * per_segment, p1 = s < heads ? 0 : min(pieces, p0 + per_segment);
            for (int p = p0; p < p1; ++p) {
                float f[8];
                row.load(f, p, lane);
                const int i = row.first(p, lane);
                if (!__any_sync(0xffffffffu, max8(f) >= t)) continue;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    list.offer(f[k] >= t && f[k] > -INFINITY ? (unsigned long long)ordered(f[k]) << 32 | (0xffffffffu - (unsigned)(i + k)) : 0ull, top, lane);
            }
        }
        const unsigned have = __ballot_sync(0xffffffffu, lane < top && list.mine != 0);
        int at = 0;
        if (lane == 0 && have) at = atomicAdd(&sh.n_keys, __popc(have));
        at = __shfl_sync(0xffffffffu, at, 0);
        if ((have >> lane) & 1) sh.keys[at + lane] = list.mine;                // valid keys are the first lanes
        __syncthreads();
        int n = sh.n_keys;
        rank_keys(sh.best, sh.keys, n, top);
        if constexpr (CLUSTER) {
            n = min(n, top);
            if (warp == 0) {
                if (lane == 0 && n) at = atomicAdd(&first->n_gathered, n);
                at = __shfl_sync(0xffffffffu, at, 0);
                if (lane < n) first->gathered[at + lane] = sh.best[lane];
            }
            cg::this_cluster().sync();
            if (part != 0) return;
            rank_keys(sh.best, sh.gathered, sh.n_gathered, top);
        }
        if (tid < top) {
            const unsigned long long key = sh.best[tid];
            const bool broken = sh.row.bad, none = key == 0 || broken;
            top_ids[r * top + tid] = none ? -1 : (int)(0xffffffffu - (unsigned)key);
            top_logp[r * top + tid] = broken ? __int_as_float(0x7fc00000) : none ? -INFINITY
                : (float)(((double)from_ordered((unsigned)(key >> 32)) - sh.row.mx) * inv_temp - sh.log_z);
        }
    } else if constexpr (CLUSTER) {
        cg::this_cluster().sync();                            // the first block has read the others' sums
    }
}

// ---------------------------------------------------------------- gradient
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
