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
#include "tok_select.h"

namespace pb {

namespace cg = cooperative_groups;

constexpr int kMaxTop = 32;

// ---------------------------------------------------------------- forward
// One pass over the row.  A warp takes pieces of 2 KB of consecutive logits, finds a piece's maximum with one
// warp reduction, and moves its running maximum (the same for all lanes) only when a piece exceeds it; the
// sums e and e d stay in registers.  The maxima of the pieces (of runs of them, for very long rows)
// stay in shared memory, and give the alternatives without a second pass: the k best elements, by value and
// then by index, lie in the k best segments by the same order, for each better segment holds a better
// element.  So at most 32 segments are read again, from L2.
// A few rows are split over a cluster of blocks, joined through distributed shared memory.
//
// Bound by memory traffic for long rows: among 50 to 500 calls in a row, 4096 x 100003 bf16 take 143 to 149 us
// without alternatives (5.6 TB/s of 6.6) and 169 to 175 with 8; the first calls after an idle time take some 25 us
// more.  Per logit it issues some 9 instructions and one exponential, which four blocks per SM overlap with the
// copies (register double-buffering instead of copies to shared memory: 40 us more).  Short batches are bound by
// latency: one row of 131072 takes 4.4 us on the device, 8.5 with 20 alternatives.
constexpr int kFwdWarps = 8, kFwdFewWarps = 2;   // warps of a block; few for rows of a few pieces
constexpr int kEight = 256;                 // logits of a warp, eight per lane
constexpr int kQuads = 4;                   // 16-byte quads of a lane in a piece
template <typename T> constexpr int kEights = 8 / (int)sizeof(T);          // times eight logits of a lane in a piece
template <typename T> constexpr int kPiece = kEight * kEights<T>;          // logits of a warp's step
constexpr int kMaxSegments = 1024, kMaxFewSegments = 32;    // segments of a row
constexpr int kPickRegs = 16;               // maxima per lane that the pick keeps in registers
constexpr int kMaxCluster = 16;
constexpr int kFwdStages = 2;               // pieces of a warp on their way through shared memory

struct FwdStats {                           // of a warp, a block or a row, relative to the maximum `mx`
    double count, rest, moment;             // elements at the maximum; sum of the others' e; sum of e log2(e)
    float mx;
    int bad;
};

template <int WARPS>
struct FwdShared {
    unsigned seg[WARPS == kFwdWarps ? kMaxSegments : kMaxFewSegments];   // maxima in order as ordered(); a block of a cluster fills its stretch
    unsigned long long keys[WARPS * kMaxTop], gathered[WARPS == kFwdWarps ? kMaxCluster * kMaxTop : 1], best[kMaxTop];
    FwdStats warp_stats[WARPS], block, row;
    int picked[kMaxTop];
    unsigned lane_top[WARPS * 32];          // every thread's own largest logit
    unsigned threshold, lane_threshold;
    int n_picked, n_keys, n_gathered;
    double log_z;
};

__device__ __forceinline__ float warp_max_nan(float x) {
    float r;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
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

// A lane's logits of a piece, as they are in memory.
template <typename T>
struct FwdPiece {
    uint4 q[kQuads];
    __device__ __forceinline__ void widen(float (&f)[8], int e) const {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                f[4 * k] = __uint_as_float(q[2 * e + k].x); f[4 * k + 1] = __uint_as_float(q[2 * e + k].y);
                f[4 * k + 2] = __uint_as_float(q[2 * e + k].z); f[4 * k + 3] = __uint_as_float(q[2 * e + k].w);
            }
        } else {
            unpack8(f, q[e], T());
        }
    }
    // 16-bit logits raised to at least lowest(), two at a time
    __device__ __forceinline__ void widen_raised(float (&f)[8], int e) const {
        const T low = from_f32<T>(lowest());
        const unsigned l = (unsigned)*reinterpret_cast<const unsigned short*>(&low) * 0x10001u;
        unpack8(f, make_uint4(max2(q[e].x, l), max2(q[e].y, l), max2(q[e].z, l), max2(q[e].w, l)), T());
    }
    // far below any maximum for which it is used, and finite times c
    static __device__ __forceinline__ float lowest() { return std::is_same_v<T, __half> ? -65504.f : -0x1p100f; }
    static __device__ __forceinline__ unsigned max2(unsigned a, unsigned b) {
        unsigned r;
        if constexpr (std::is_same_v<T, __half>) asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        else asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    __device__ __forceinline__ float top() const {
        if constexpr (sizeof(T) == 4) {
            float f[8], g[8];
            widen(f, 0);
            widen(g, 1);
            return max_nan(max8(f), max8(g));
        } else {
            unsigned m[kQuads];
#pragma unroll
            for (int k = 0; k < kQuads; ++k) m[k] = max2(max2(q[k].x, q[k].y), max2(q[k].z, q[k].w));
            const unsigned t = max2(max2(m[0], m[1]), max2(m[2], m[3]));
            float f[8];
            unpack8(f, make_uint4(t, t, t, t), T());
            return max_nan(f[0], f[1]);
        }
    }
};

template <typename T>
struct FwdRow {
    const T* x;
    int head;                               // logits before the first aligned one
    // eight logits of a lane from logit `at` + 8 lane on; -inf from `end` on
    __device__ __forceinline__ void load(float (&f)[8], int at, int end, int lane) const {
        const int i = at + 8 * lane;
        if (at >= head && at + kEight <= end) {
            if constexpr (sizeof(T) == 4) load8_wide(f, x + i);
            else load8(f, x + i);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] = i + k < end ? to_f32(x[i + k]) : -INFINITY;
        }
    }
};

// A warp's running sums, in units of log2: with c = log2(e) inverse_temperature and the rounded R = c max,
// y = fma(x, c, -R) takes one instruction for two logits, and the rounding of R, known exactly as
// delta = c max - R, is put right when the sums are used.  Sums: rest of 2^y, moment of 2^y y, over the logits
// below the maximum; those equal to it are counted.  delta is half a step of R at most, and 2^delta a factor of
// the sums: beyond |R| = kFarRef (masks of -1e10, a very low temperature) y = (x - max) c takes its place, which
// has no delta and rounds twice.
constexpr float kFarRef = 0x1p20f;          // delta is 2^-5 at most below it; past 2^31 2^delta would overflow

struct FwdAcc {
    float mx = -INFINITY, ref = 0.f, delta = 0.f;
    bool wide = false;                      // c max beyond kFarRef: y = (x - max) c
    bool raise = false;                     // logits may be raised to FwdPiece::lowest: 2^y is zero there as well
    int count = 0;
    Pair rest{0.f, 0.f}, moment{0.f, 0.f};

    __device__ __forceinline__ void move(float top, float c, float lowest) {
        const bool w = !(fabsf(top) < 1e36f && fabsf(top * c) < kFarRef);
        const float r = w ? 0.f : top * c, d = w ? 0.f : fmaf(top, c, -r);
        if (mx > -INFINITY) {
            const float shift = fmaxf((mx - top) * c, -1e30f) - delta + d, s = exp2_near(shift), own = (float)count * exp2_near(delta);
            float r0, r1, m0, m1;
            rest.split(r0, r1);
            moment.split(m0, m1);
            r0 += own;
            m0 = fmaf(own, delta, m0);
            moment = Pair(fmaf(r0, shift, m0) * s, fmaf(r1, shift, m1) * s);
            rest = Pair(r0 * s, r1 * s);
            count = 0;
        }
        mx = top;
        ref = r;
        delta = d;
        wide = w;
        raise = !w && c < 1e8f && (top - lowest) * c > 200.f;
    }
    // LOW: -inf may be among the logits
    template <bool LOW, bool WIDE>
    __device__ __forceinline__ void add_below(const float (&f)[8], float c) {
        const Pair m(WIDE ? -mx : -ref), cc(c);
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
            const Pair x(f[k], f[k + 1]);
            Pair y = WIDE ? (x + m) * cc : fma2(x, cc, m);
            float a, b;
            y.split(a, b);
            if (LOW) {                       // 2^y y is 0, not 0 times infinity, where 2^y is 0
                a = max_nan(a, -1e30f);
                b = max_nan(b, -1e30f);
                y = Pair(a, b);
            }
            const Pair e(exp2_near(a), exp2_near(b));
            rest = rest + e;
            moment = fma2(e, y, moment);
        }
    }
    // counts the logits at the maximum and leaves `instead` in their place
    __device__ __forceinline__ void take_top(float (&f)[8], float instead) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            count += f[k] == mx;
            f[k] = f[k] == mx ? instead : f[k];
        }
    }
    // eight logits per lane whose warp-wide maximum is `top`
    __device__ __forceinline__ void add(float (&f)[8], float top, float c, float lowest) {
        if (top > mx) move(top, c, lowest);
        if (mx == -INFINITY) return;         // nothing finite so far
        take_top(f, -INFINITY);
        if (wide) add_below<true, true>(f, c); else add_below<true, false>(f, c);
    }
    // a full piece; `again` gives eight of its logits a second time
    template <typename T, typename Again>
    __device__ __forceinline__ void add(const FwdPiece<T>& p, float top, float c, Again again) {
        const float lowest = FwdPiece<T>::lowest();
        if (top > mx) move(top, c, lowest);
        if (sizeof(T) == 2 ? raise : !wide && mx > -INFINITY) {
            const bool at_top = top == mx;
#pragma unroll
            for (int e = 0; e < kEights<T>; ++e) {
                float f[8];
                if constexpr (sizeof(T) == 2) p.widen_raised(f, e); else p.widen(f, e);
                if (at_top) take_top(f, sizeof(T) == 2 ? lowest : -INFINITY);
                add_below<sizeof(T) == 4, false>(f, c);
            }
        } else {
#pragma unroll 1
            for (int e = 0; e < kEights<T>; ++e) {
                float f[8];
                again(f, e);
                add(f, top, c, lowest);
            }
        }
    }
    // sums relative to the maximum itself, in natural units over the inverse temperature's: c d = y - delta
    __device__ __forceinline__ void finish(float (&out)[2]) const {
        float r0, r1, m0, m1;
        rest.split(r0, r1);
        moment.split(m0, m1);
        const float s = exp2_near(-delta);
        out[0] = (r0 + r1) * s;
        out[1] = fmaf(-delta, r0 + r1, m0 + m1) * s;
    }
};

// Floats in the order of their values as unsigned numbers, and back.
__device__ __forceinline__ unsigned ordered(float x) {
    const unsigned b = __float_as_uint(x + 0.f);              // -0 counts as 0
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(unsigned b) {
    return __uint_as_float((b & 0x80000000u) ? (b & 0x7fffffffu) : ~b);
}

__device__ __forceinline__ double warp_total(double x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
// Sums of the lanes' parts, relative to the largest maximum; the same in every lane.
__device__ __forceinline__ FwdStats join(FwdStats p, float c) {
    FwdStats t;
    t.bad = __any_sync(0xffffffffu, p.bad);
    t.mx = from_ordered(__reduce_max_sync(0xffffffffu, ordered(p.mx)));
    if (p.mx != t.mx || p.mx == -INFINITY) {
        const float shift = fmaxf((p.mx - t.mx) * c, -1e30f);         // finite: times a sum that it makes zero
        const double s = p.mx == -INFINITY ? 0.0 : exp2_near(shift), all = p.rest + p.count;
        p.rest = s * all;
        p.moment = s == 0.0 ? 0.0 : s * (p.moment + all * shift);
        p.count = 0;
    }
    t.count = warp_total(p.count);
    t.rest = warp_total(p.rest);
    t.moment = warp_total(p.moment);
    return t;
}

// Largest t such that at least k of n > k keys, without their low GRAIN bits, reach it; one warp.  By bisection,
// from the k-th largest of the lanes' largest keys up, if every lane has REGS keys at most.
template <int GRAIN, int REGS>
__device__ __forceinline__ unsigned kth_largest(const unsigned* key, int n, int k, int lane) {
    unsigned v[REGS];
    const bool in_regs = n <= 32 * REGS;
    unsigned top = 0;
#pragma unroll
    for (int j = 0; j < REGS; ++j) {
        v[j] = in_regs && lane + 32 * j < n ? key[lane + 32 * j] : 0;
        top = max(top, v[j]);
    }
    unsigned lo = 0, hi = 0xffffffffu >> GRAIN;
    if (in_regs) {
        int above = 0;
#pragma unroll 8
        for (int j = 0; j < 32; ++j) {
            const unsigned o = __shfl_sync(0xffffffffu, top, j);
            above += o > top || (o == top && j < lane);
        }
        const unsigned who = __ballot_sync(0xffffffffu, above == k - 1);
        lo = __shfl_sync(0xffffffffu, top, __ffs(who) - 1) >> GRAIN;
        hi = max(lo, __reduce_max_sync(0xffffffffu, top) >> GRAIN);
    }
    return highest_reached(lo, hi, k, [&](unsigned t) {
        const unsigned at = t << GRAIN;
        int c = 0;
        if (in_regs) {
#pragma unroll
            for (int j = 0; j < REGS; ++j) c += v[j] >= at;
        } else {
            for (int j = lane; j < n; j += 32) c += key[j] >= at;
        }
        return (int)__reduce_add_sync(0xffffffffu, c);
    });
}

// The k best of n segments (by maximum, then by index) into sh.picked, and a key that the k-th best
// maximum reaches into sh.threshold; one warp.  Maxima are values of T, in whose ordered() bits
// the low GRAIN are all alike.
template <int GRAIN, int WARPS>
__device__ __forceinline__ void pick_segments(FwdShared<WARPS>& sh, int n, int k, int lane) {
    if (n <= k) {
        if (lane < n) sh.picked[lane] = lane;
        if (lane == 0) { sh.n_picked = n; sh.threshold = 0; }
        return;
    }
    const unsigned t = n <= 128 ? kth_largest<GRAIN, 4>(sh.seg, n, k, lane) : kth_largest<GRAIN, kPickRegs>(sh.seg, n, k, lane);
    // segments above t; those equal to t (without the low bits) fill up in order
    int above = 0;
    for (int j = lane; j < n; j += 32) above += (sh.seg[j] >> GRAIN) > t;
    above = __reduce_add_sync(0xffffffffu, above);
    const int equal = min(k, n) - above;
    int at = 0, taken = 0;
    for (int j0 = 0; j0 < n; j0 += 32) {
        const unsigned v = j0 + lane < n ? sh.seg[j0 + lane] >> GRAIN : 0;
        const bool more = j0 + lane < n && v > t, same = j0 + lane < n && v == t;
        const unsigned below = (1u << lane) - 1, ms = __ballot_sync(0xffffffffu, same);
        const bool take = more || (same && taken + __popc(ms & below) < equal);
        const unsigned mt = __ballot_sync(0xffffffffu, take);
        if (take) sh.picked[at + __popc(mt & below)] = j0 + lane;
        at += __popc(mt);
        taken += __popc(ms);
    }
    if (lane == 0) { sh.n_picked = at; sh.threshold = t << GRAIN; }
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
template <int WARPS>
__device__ __forceinline__ void rank_keys(unsigned long long* best, const unsigned long long* keys, int n, int k) {
    if ((int)threadIdx.x < k) best[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += WARPS * 32) {
        const unsigned long long x = keys[i];
        int above = 0;
        for (int j = 0; j < n; ++j) above += keys[j] > x;     // keys differ: each holds its index; zeros are none
        if (x != 0 && above < k) best[above] = x;
    }
    __syncthreads();
}

template <typename T, typename I, int WARPS, bool CLUSTER>
__global__ void __launch_bounds__(WARPS * 32, WARPS == kFwdWarps ? 4 : 16)
logprob_fwd_kernel(const T* __restrict__ logits, int vocab, long long ld, const I* __restrict__ tokens, double inv_temp,
                   float* __restrict__ logp, float* __restrict__ entropy, float* __restrict__ lse, int top,
                   float* __restrict__ top_logp, int* __restrict__ top_ids, int per_segment, int* status) {
    __shared__ FwdShared<WARPS> sh;
    __shared__ uint4 sh_ring[WARPS * kFwdStages * kQuads * 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int parts = CLUSTER ? (int)cg::this_cluster().num_blocks() : 1, part = CLUSTER ? (int)cg::this_cluster().block_rank() : 0;
    const long long r = blockIdx.x / parts;
    FwdRow<T> row;
    row.x = logits + r * ld;
    constexpr int ALIGN = 8 * (int)sizeof(T);
    row.head = min(vocab, (int)((-(long long)reinterpret_cast<uintptr_t>(row.x)) & (ALIGN - 1)) / (int)sizeof(T));
    // Segments: the pieces, `per_segment` at a time, the logits before the first and behind the last full piece
    // included in the first and last segment; blocks take equal stretches of them.
    const int full = (vocab - row.head) / kPiece<T>;                      // full pieces
    const int shift = __ffs(per_segment) - 1, segments = max(1, (full + per_segment - 1) >> shift);
    const int each = (segments + parts - 1) / parts, s_lo = min(segments, part * each), s_hi = min(segments, s_lo + each);
    const float c = (float)(1.4426950408889634 * inv_temp);
    if (tid == 0) sh.n_keys = sh.n_gathered = 0;

    FwdAcc acc;
    float lane_top = -INFINITY;
    bool bad = false;
    for (int s = s_lo + tid; s < s_hi; s += WARPS * 32) sh.seg[s] = 0;
    __syncthreads();
    {
        // This warp's full pieces, WARPS apart: it copies each to shared memory, kFwdStages ahead, and a lane
        // copies what it reads itself, so nothing but the copy is waited for.
        uint4* ring = sh_ring + warp * kFwdStages * kQuads * 32 + lane;
        const unsigned ring_at = (unsigned)__cvta_generic_to_shared(ring);
        const int p_lo = (s_lo << shift) + warp, p_hi = min(full, s_hi << shift), count = max(0, (p_hi - p_lo + WARPS - 1) / WARPS);
        constexpr int STEP = WARPS * kPiece<T>;
        constexpr int QUAD = 16 / (int)sizeof(T);             // a warp's quads lie side by side
        const T* from = row.x + row.head + (long long)p_lo * kPiece<T> + QUAD * lane;
        auto ahead = [&](int j) {
            if (j < count) {
                const unsigned to = ring_at + (j & (kFwdStages - 1)) * (kQuads * 512);
#pragma unroll
                for (int k = 0; k < kQuads; ++k)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
                                 ::"r"(to + k * 512), "l"(from + k * 32 * QUAD) : "memory");
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            from += STEP;
        };
#pragma unroll
        for (int j = 0; j < kFwdStages; ++j) ahead(j);
        // The row's ends, 256 logits per warp, while the first pieces are on their way: before the first full piece (first
        // block) and behind the last (last block).
        const int behind = row.head + full * kPiece<T>, ends = 1 + (vocab - behind + kEight - 1) / kEight;
#pragma unroll 1
        for (int e = warp; e < ends; e += WARPS) {
            const int s = e == 0 ? 0 : segments - 1;
            if (s < s_lo || s >= s_hi || (e == 0 && row.head == 0)) continue;
            float f[8];
            row.load(f, e == 0 ? 0 : behind + (e - 1) * kEight, e == 0 ? row.head : vocab, lane);
            const float own = max8(f), m = warp_max_nan(own);
            lane_top = max_nan(lane_top, own);
            bad |= m != m;
            if (lane == 0) atomicMax(&sh.seg[s], ordered(m));
            acc.add(f, m, c, FwdPiece<T>::lowest());
        }
#pragma unroll 1
        for (int j = 0; j < count; ++j) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kFwdStages - 1) : "memory");
            FwdPiece<T> p;
#pragma unroll
            for (int k = 0; k < kQuads; ++k) p.q[k] = ring[(j & (kFwdStages - 1)) * kQuads * 32 + k * 32];
            const float own = p.top(), m = warp_max_nan(own);
            lane_top = max_nan(lane_top, own);
            ahead(j + kFwdStages);                            // the quads are in registers: their place is free
            bad |= m != m;
            const int piece = p_lo + j * WARPS;
            if (lane == 0) atomicMax(&sh.seg[piece >> shift], ordered(m));
            acc.add(p, m, c, [&](float(&f)[8], int e) { row.load(f, row.head + piece * kPiece<T> + e * kEight, vocab, lane); });
        }
    }
    sh.lane_top[tid] = ordered(lane_top);
    {
        float sums[2];
        acc.finish(sums);
        float a = sums[0], p = sums[1];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, o);
            p += __shfl_xor_sync(0xffffffffu, p, o);
        }
        const int count = __reduce_add_sync(0xffffffffu, acc.count);
        if (lane == 0) sh.warp_stats[warp] = FwdStats{(double)count, (double)a, (double)p, acc.mx, bad || acc.mx == INFINITY};
    }
    __syncthreads();
    FwdShared<WARPS>* first = &sh;
    if constexpr (CLUSTER) {
        cg::cluster_group cluster = cg::this_cluster();
        if (warp == 0) {
            const FwdStats all = join(lane < WARPS ? sh.warp_stats[lane] : FwdStats{0, 0, 0, -INFINITY, 0}, c);
            if (lane == 0) sh.block = all;
        }
        cluster.sync();
        first = cluster.map_shared_rank(&sh, 0);
        if (top > 0) {                                        // every block picks from the whole row's segments
            for (int s = tid; s < segments; s += WARPS * 32) {
                const int owner = s / each;
                if (owner != part) sh.seg[s] = cluster.map_shared_rank(&sh, owner)->seg[s];
            }
            __syncthreads();
        }
    }
    if (part == 0 && warp == 1) {                             // the row's values, beside the pick
        FwdStats mine{0, 0, 0, -INFINITY, 0};
        if constexpr (CLUSTER) {
            if (lane < parts) mine = cg::this_cluster().map_shared_rank(&sh, lane)->block;
        } else {
            if (lane < WARPS) mine = sh.warp_stats[lane];
        }
        const FwdStats all = join(mine, c);
        const bool empty = all.mx == -INFINITY && !all.bad;
        const double log_z = all.bad ? __longlong_as_double(0x7ff8000000000000ll) : empty ? 0.0 : log(all.count) + log1p(all.rest / all.count);
        if (lane == 0) {
            // the token's logit, in L2 by now
            const long long id = logp ? token_id(tokens, r, vocab, status) : -1;
            const float x_token = id >= 0 ? to_f32(row.x[id]) : 0.f;
            if (logp) logp[r] = id < 0 ? 0.f : empty ? -INFINITY : (float)(((double)x_token - all.mx) * inv_temp - log_z);
            if (entropy) entropy[r] = empty ? 0.f : (float)(log_z - 0.6931471805599453 * all.moment / (all.count + all.rest));
            if (lse) lse[r] = empty ? -INFINITY : (float)((double)all.mx * inv_temp + log_z);
            sh.log_z = log_z;
            sh.row = all;
        }
    }
    if (top > 0) {
        constexpr int GRAIN = sizeof(T) == 4 ? 0 : std::is_same_v<T, __half> ? 13 : 16;
        if (warp == 0) pick_segments<GRAIN, WARPS>(sh, segments, top, lane);
        if (warp == (WARPS > 2 ? WARPS - 1 : 0)) {            // k threads of this block have seen a logit of at least this
            const unsigned t = kth_largest<GRAIN, WARPS>(sh.lane_top, WARPS * 32, top, lane) << GRAIN;
            if (lane == 0) sh.lane_threshold = t;
        }
        __syncthreads();
        const unsigned t = max(max(sh.threshold, sh.lane_threshold), ordered(-INFINITY) + 1);
        const int picked = sh.n_picked;
        // The candidates of the picked segments, a piece (or one of the row's ends) per warp at a time.
        auto visit = [&](auto see) {
            for (int u = warp; u < picked * (per_segment + 2); u += WARPS) {
                const int s = sh.picked[u / (per_segment + 2)], j = u % (per_segment + 2), piece = (s << shift) + j;
                if (s < s_lo || s >= s_hi) continue;
                int from = row.head + piece * kPiece<T>, end = from + kPiece<T>;
                if (j < per_segment) {
                    if (piece >= full) continue;
                } else if (j == per_segment) {
                    if (s != segments - 1) continue;
                    from = row.head + full * kPiece<T>;
                    end = vocab;
                } else {
                    if (s != 0) continue;
                    from = 0;
                    end = row.head;
                }
                // loads that do not wait for each other find where there are candidates at all ...
                unsigned hits = 0;
                float f[kEights<T>][8];
#pragma unroll
                for (int e = 0; e < kEights<T>; ++e) row.load(f[e], from + e * kEight, end, lane);
#pragma unroll
                for (int e = 0; e < kEights<T>; ++e) hits |= (unsigned)__any_sync(0xffffffffu, ordered(max8(f[e])) >= t) << e;
                // ... and those, by now near, are read once more
                while (hits) {
                    const int at = from + (__ffs(hits) - 1) * kEight;
                    hits &= hits - 1;
                    float g[8];
                    row.load(g, at, end, lane);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const unsigned key = ordered(g[k]);
                        see(key >= t ? (unsigned long long)key << 32 | (0xffffffffu - (unsigned)(at + 8 * lane + k)) : 0ull);
                    }
                }
            }
        };
        constexpr int ROOM = WARPS * kMaxTop;
        visit([&](unsigned long long key) {
            if (key == 0) return;
            const int at = atomicAdd(&sh.n_keys, 1);
            if (at < ROOM) sh.keys[at] = key;
        });
        __syncthreads();
        int n = sh.n_keys, at = 0;
        if (n > ROOM) {                                       // many equal logits: each warp keeps its best only
            __syncthreads();
            if (tid == 0) sh.n_keys = 0;
            __syncthreads();
            BestList list;
            visit([&](unsigned long long key) { list.offer(key, top, lane); });
            const unsigned have = __ballot_sync(0xffffffffu, lane < top && list.mine != 0);
            if (lane == 0 && have) at = atomicAdd(&sh.n_keys, __popc(have));
            at = __shfl_sync(0xffffffffu, at, 0);
            if ((have >> lane) & 1) sh.keys[at + lane] = list.mine;            // valid keys are the first lanes
            __syncthreads();
            n = sh.n_keys;
        }
        rank_keys<WARPS>(sh.best, sh.keys, n, top);
        if constexpr (CLUSTER) {
            n = min(n, top);
            if (warp == 0) {
                if (lane == 0 && n) at = atomicAdd(&first->n_gathered, n);
                at = __shfl_sync(0xffffffffu, at, 0);
                if (lane < n) first->gathered[at + lane] = sh.best[lane];
            }
            cg::this_cluster().sync();
            if (part != 0) return;
            rank_keys<WARPS>(sh.best, sh.gathered, sh.n_gathered, top);
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

// log p = it x - lse carries the roundings of lse (float32) and of the product, |lse| 2^-23 at most.  Beyond kFarLse
// (a row of nothing but a finite mask of -1e10) that is more than 1, and p would be anything up to infinity.
// Such a row's lse is raised by twice that much: p stays between 0 and 1, and 0 times p is 0.  With a power of two
// for `it` the product is exact and lse no less than the largest one, so nothing is raised.
// (Holding log p at 0 instead, in the loop over the logits, takes 180 us for 4096 x 65536 bf16; this takes 169.)
constexpr float kFarLse = 0x1p23f;
__device__ __forceinline__ float safe_lse(float z, double inv_temp) {
    const float it = (float)inv_temp;
    const bool exact = !(__float_as_uint(it) & 0x7fffffu) && (double)it == inv_temp;
    return fmaf(!exact && fabsf(z) > kFarLse && z > -INFINITY ? fabsf(z) : 0.f, 0x1p-22f, z);
}

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
                // NaN stays NaN.  2^-288 is zero, so a masked logit has p = 0; the clamp keeps the factor beside it finite.
                lp.split(a, b);
                lp = Pair(max_nan(a, -200.f), max_nan(b, -200.f));
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
    q.z = safe_lse(q.z, inv_temp);
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
