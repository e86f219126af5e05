// Log probabilities straight from hidden states and the output head, and their gradients, without a
// matrix of logits in memory.
//
// With z[t, v] = it * hidden[t, :] . weight[v, :] and p = softmax over v:
//   forward   lse[t] = log sum_v exp z, logp[t] = z[t, token] - lse, entropy[t] = -sum p log p
//   backward  d[t, v] = it (g_logp (1[v = token] - p) - g_entropy p (log p + entropy) + g_lse p)
//             dhidden = d weight,  dweight (+)= d^T hidden
// so one product of T x V x D for the forward, and three for the backward: the logits again, and the
// two gradients.  The backward goes through the vocabulary in pieces; of each it holds d alone, in the
// operands' type, and both products of a piece read it from L2 or memory once.
//
// All four products are tiles of one kernel: 256 x 256 of D per pair of blocks (cta_group::2, each
// block holds 128 rows of A, 128 rows of B and 128 x 256 of D), K in chunks of 64 through a ring of
// stages filled by bulk tensor copies, two accumulators of 256 columns in tensor memory, so that eight
// warps work on the last tile while the next one is multiplied.  Up to 128 rows of hidden states run in
// single blocks of 128 x 128, since a pair would leave half of its rows empty: these calls are bound by
// reading the weights, and the fewer rows there are, the more stages fit (A's rows that do not exist are not
// copied; what the tensor core finds in their place goes to rows of D that nobody reads).
//   logits   A = hidden (K-major)        B = weight (K-major)      the row statistics, or d, are computed from the tile
//   hidden   A = d (K-major)             B = weight (MN-major)     float32 partial sums, one plane per split of K
//   weight   A = d, read transposed (MN-major)  B = hidden (MN-major)
// float32 operands are held in planes of 16 bits, and a product is a sum of products of planes.  Where the absolute size of an error
// counts (the logits; dhidden, a sum over tokens), two float16 planes do: x = 2^k (x0 + x1) to 2^-24 of x or 2^-39 of the largest number
// that shares k (a row of hidden states, 32 rows of the weights, a row of d), and x0 y0 + x0 y1 + x1 y0 leaves out 2^-24.  A row of
// dweight is a token's own, however improbable, so its product keeps float32's range: three bfloat16 planes (x0 + x1 + x2 to 2^-25)
// and the six terms x_i y_j with i + j <= 2.  (Six terms everywhere took the forward of 509 x 50021 x 1001 1.6 times as long.)
// The tensor core adds to its float32 accumulator without rounding to nearest, so a long K drifts:
// float32 products, and long rows' logits in the forward, leave the tensor core every few chunks and are
// added up in registers.
// What bounds it: 16-bit products wait for L2 (a pair reads 64 KB for 512 cycles of its tensor cores; 42 to 46 bytes per cycle reach an SM,
// the tensor cores are 68 to 75 % busy: 1340 TFLOP/s in the forward of 4096 x 131072 x 4096, and the power limit in long runs), float32 ones
// for the tensor cores (82 to 94 % busy, since a chunk's planes are read once for all terms) and their sums' way out of them.  One or two rows (four of float32) have a kernel without them.
// Every wait is bounded (see mbar_wait); a block whose wait runs out reports it and gives NaN for its tiles.
#pragma once
#include "tc_common.cuh"
#include "tok_common.cuh"

namespace pb {

constexpr int kHeadChunk = 64;                // K elements per stage: one 128-byte swizzled row
constexpr int kHeadOperand = 128 * 128;       // bytes of an operand's 128 x 64 tile
constexpr int kHeadMaxStages = 11;
constexpr int kHeadBuf = 32 * 128;            // bytes of an epilogue warp's buffer: 128 of each of its rows
constexpr int kHeadEpi = 8;                   // epilogue warps: quarter w % 4 of the tensor-memory lanes, half w / 4 of the columns
constexpr int kHeadThreads = 32 * (kHeadEpi + 2);
constexpr int kHeadRing = 196608;             // bytes for the stages: six of 32 KB; three with two planes of each operand, two with three; eleven with A
                                              // tiles of up to eight rows
constexpr int kHeadSmem = 1024 + kHeadRing + kHeadEpi * kHeadBuf;
constexpr int kHeadWide = 3, kHeadNear = 2;  // bfloat16 and float16 planes of a float32 operand
constexpr int kHeadGroup = 32;                // rows of the weights that share a power of two

enum HeadKind { kHeadStats = 0, kHeadGrad = 1, kHeadHidden = 2, kHeadWeight = 3 };

// One product: tiles_m x tiles_n tiles, K split `splits` ways.
struct alignas(64) HeadJob {
    CUtensorMap a, b;            // K-major: (k, row, plane); MN-major: (row, k, plane)
    CUtensorMap out;             // (column, row, plane) of what is stored by bulk copies: boxes of 128 bytes by 32 rows
    int kind;
    int a_mn, b_mn;              // operand is MN-major
    int half, planes;            // operands are float16; planes of each: 1, 2 or 3, of which 1, 3 or 6 products are taken
    int promote;                 // chunks of K that the tensor core adds up by itself
    int tiles_m, tiles_n, splits;
    int group_m;                 // row tiles that are walked through together, for one column tile after the other
    int chunks, chunks_per_split;
    int rows, cols;              // of D
    int tiles;                   // tiles_m * tiles_n * splits
    Quotient by_split, by_group, by_height, by_last;      // tiles of a split, of a group; row tiles of a group, of the last one
    int groups;
    int a_bytes;                 // bytes of A that a stage receives per block
};

// What a row of hidden states needs for d, scaled so that it fits the operands' type.
struct HeadRow {
    float a;                     // of the token's (1 - p)
    float c0, c1;                // of p and p log2 p
    float lse2;                  // lse in units of log 2
};

struct alignas(64) HeadArgs {
    HeadJob job[2];
    int jobs;
    int extra, late, rounds;     // see head_tile
    int stages, stage_bytes, a_slot;     // of the ring: a stage has the B tiles of a chunk's planes, then its A tiles, a_slot bytes each
    float c;                     // inv_temperature * log2(e)
    int col0;                    // first column (token) of this piece of the vocabulary
    int* status;
    // row statistics
    float* part;                 // [3][parts][rows]: HeadStat's
    int part0, parts, entropy;   // entropy: its sum is wanted, or its gradient given
    float* ztok;                 // the token's logit of each row
    const void* tokens;
    int token_bytes;
    long long vocab;
    // float32: the powers of two of the float16 planes (NULL: none), of hidden rows, of groups of the weights' rows, the largest of those; of d's rows
    const float *row_scale, *col_scale, *col_most, *d_scale;
    int store_near, store_wide;  // planes of d that are wanted: for dhidden (map job[1].out), for dweight (map job[0].out)
    // d
    const HeadRow* coef;
    const int* row_token;        // index of the token, or -1
    // products
    int add;                     // partial sums of dhidden: those of an earlier piece are there
    void* out;                   // of this piece of dweight
    long long ldo;
    int out_type, accumulate, bulk;      // pb_dtype; bulk: rows that bulk copies can store
    const float* unscale;
};

// ------------------------------------------------------------------ clusters
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_id() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%clusterid.x;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_count() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%nclusterid.x;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ uint32_t of_leader(uint32_t addr) {        // the same place in the pair's first block
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}
__device__ __forceinline__ void arrive_cluster(uint32_t addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}
// mbar_wait that also sees what the other block of the pair has done.
__device__ __forceinline__ bool mbar_wait_pair(uint32_t bar, uint32_t parity, const volatile int* fail) {
    uint32_t done = 0;
    long long t0 = 0;
    for (int it = 0; !done; ++it) {
        asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                     : "=r"(done) : "r"(bar), "r"(parity) : "memory");
        if (!done && (it & 63) == 63) {
            if (*fail) return false;
            const long long now = global_ns();
            if (t0 == 0) t0 = now;
            else if (now - t0 > kTcWaitNs) return false;
        }
    }
    return true;
}
// Bulk tensor copy of one block of a pair; the bytes count at the leader's barrier.
__device__ __forceinline__ void tma_3d_pair(uint32_t dst, const CUtensorMap* tm, int c0, int c1, int c2, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(tm), "r"(c0), "r"(c1), "r"(c2), "r"(bar) : "memory");
}

struct HeadShared {
    uint64_t full[kHeadMaxStages];   // a stage's operands have landed (at the leader: both blocks')
    uint64_t empty[kHeadMaxStages];  // the products that read a stage are done
    uint64_t acc_full[2], acc_empty[2];
    uint32_t tmem_base;
    int fail;
};

struct HeadTile {
    int m, n, split, chunk0, chunk1;
};

// The i-th tile of this block (or pair): its job, and its place there; false behind the last.  The first job's tiles go round the blocks, `late` of
// which get rounds + 1 and the others `rounds`.  The second job's are shorter: those others take `extra` of them before all take
// turns, so that all end together (4096 rows, 2048 columns, 25088 tokens: 128 long tiles for 74 pairs).
__device__ __forceinline__ bool head_tile(const HeadArgs& g, int i, int& j, HeadTile& x) {
    const int n = (int)cluster_count(), id = (int)cluster_id();
    int t = id + i * n;
    j = 0;
    if (t >= g.job[0].tiles) {
        if (g.jobs == 1) return false;
        j = 1;
        const bool is_late = id < g.late;
        const int early = n - g.late, ahead = early * g.extra;
        i -= g.rounds + is_late;                              // tiles of the second job that this block has had
        if (is_late) t = ahead + id + i * n;
        else if (i < g.extra) t = id - g.late + i * early;
        else t = ahead + id + (i - g.extra) * n;
        if (t >= g.job[1].tiles) return false;
    }
    const HeadJob& q = g.job[j];
    x.split = q.by_split(t);
    t -= x.split * q.tiles_m * q.tiles_n;
    const int group = q.by_group(t), m0 = group * q.group_m;
    t -= group * q.group_m * q.tiles_n;
    const bool last = group == q.groups - 1;
    x.n = last ? q.by_last(t) : q.by_height(t);
    x.m = m0 + t - x.n * (last ? q.tiles_m - m0 : q.group_m);
    x.chunk0 = x.split * q.chunks_per_split;
    x.chunk1 = min(q.chunks, x.chunk0 + q.chunks_per_split);
    return true;
}

// ------------------------------------------------------------------ copies (one thread of each block)
template <int CG>
__device__ void head_copies(const HeadArgs& g, unsigned char* smem, HeadShared& sh, int rank) {
    constexpr int kRows = 128 * CG;
    const uint32_t ring = smem_u32(smem), full0 = smem_u32(&sh.full[0]), empty0 = smem_u32(&sh.empty[0]), lead0 = CG == 2 ? of_leader(full0) : full0;
    const int stages = g.stages, stage = g.stage_bytes, slot = g.a_slot;
    int stg = 0, j;
    uint32_t phase = 1, off = 0;                              // every stage is free at first
    HeadTile x;
    for (int i = 0; head_tile(g, i, j, x); ++i) {
        const HeadJob& q = g.job[j];
        const int m0 = x.m * kRows + rank * 128, n0 = x.n * kRows + rank * 128, planes = q.planes;
        const bool a_mn = q.a_mn, b_mn = q.b_mn;
        const uint32_t bytes = (uint32_t)(planes * (q.a_bytes + kHeadOperand)) * CG;
        for (int c = x.chunk0; c < x.chunk1; ++c) {
            const uint32_t empty = empty0 + stg * 8, full = lead0 + stg * 8;
            if (!(CG == 2 ? mbar_wait_pair(empty, phase, &sh.fail) : mbar_wait(empty, phase, &sh.fail))) { sh.fail = 1; return; }
            if (rank == 0) mbar_arrive_tx(full0 + stg * 8, bytes);
            uint32_t sb = ring + off, sa = sb + planes * kHeadOperand;
            auto copy = [&](uint32_t dst, const CUtensorMap* tm, int u, int v, int w) {
                if (CG == 2) tma_3d_pair(dst, tm, u, v, w, full); else tma_3d(dst, tm, u, v, w, full);
            };
            const int k = c * kHeadChunk;
            for (int plane = 0; plane < planes; ++plane, sa += slot, sb += kHeadOperand) {
                if (a_mn) {
                    copy(sa, &q.a, m0, k, plane);
                    copy(sa + kHeadOperand / 2, &q.a, m0 + 64, k, plane);
                } else {
                    copy(sa, &q.a, k, m0, plane);
                }
                if (b_mn) {
                    copy(sb, &q.b, n0, k, plane);
                    copy(sb + kHeadOperand / 2, &q.b, n0 + 64, k, plane);
                } else {
                    copy(sb, &q.b, k, n0, plane);
                }
            }
            off += stage;
            if (++stg == stages) { stg = 0; off = 0; phase ^= 1; }
        }
    }
}

// ------------------------------------------------------------------ products (one thread of a block or pair)
// One product of 16 columns of K; the low words of the operands' descriptors, of which the high word is the same.
template <int CG>
__device__ __forceinline__ void head_mma(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
    constexpr uint64_t kHigh = (uint64_t)((1024 >> 4) | (1u << 14) | (2u << 29)) << 32;      // tc_desc's: 8 rows are 1024 bytes, version 1, 128-byte swizzle
    if (CG == 2)
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
                     ::"r"(d), "l"(kHigh | a), "l"(kHigh | b), "r"(idesc), "r"(acc) : "memory");
    else
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                     ::"r"(d), "l"(kHigh | a), "l"(kHigh | b), "r"(idesc), "r"(acc) : "memory");
}

// One thread issues everything, and a chunk of a pair's tile takes the tensor cores 512 cycles: what it does per chunk has to be short (with the descriptors
// put together for each product, and loops over the planes, 4096 x 131072 x 4096 took 3.29 ms where 2.94 are possible).
template <int CG>
__device__ void head_products(const HeadArgs& g, unsigned char* smem, HeadShared& sh) {
    constexpr int kCols = 128 * CG;
    const uint32_t ring = smem_u32(smem) >> 4, stage = (uint32_t)g.stage_bytes >> 4, slot = (uint32_t)g.a_slot >> 4, tmem = sh.tmem_base;
    const uint32_t full0 = smem_u32(&sh.full[0]), empty0 = smem_u32(&sh.empty[0]);
    const int stages = g.stages;
    int stg = 0, at = 0, j;
    uint32_t phase = 0, off = 0;
    HeadTile x;
    auto wait = [&](uint32_t bar, uint32_t parity) { return CG == 2 ? mbar_wait_pair(bar, parity, &sh.fail) : mbar_wait(bar, parity, &sh.fail); };
    auto commit = [&](uint32_t bar) {
        if (CG == 2)
            asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                         ::"r"(bar), "h"((unsigned short)3) : "memory");
        else
            asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    };
    for (int i = 0; head_tile(g, i, j, x); ++i) {
        const HeadJob& q = g.job[j];
        const uint32_t type = q.half ? 0u : (1u << 7) | (1u << 10);
        const uint32_t idesc = (1u << 4) | type | ((uint32_t)q.a_mn << 15) | ((uint32_t)q.b_mn << 16) | ((uint32_t)(kCols >> 3) << 17) |
                               ((uint32_t)(128 * CG >> 4) << 24);
        // in units of 16 bytes: 16 columns of K further; the distance of an MN-major tile's halves, in the upper half of the word
        const uint32_t step_a = q.a_mn ? 128 : 2, step_b = q.b_mn ? 128 : 2;
        const uint32_t a0 = (ring + (uint32_t)q.planes * (kHeadOperand >> 4)) | (q.a_mn ? (uint32_t)kHeadOperand / 2 >> 4 : 1u) << 16;
        const uint32_t b0 = ring | (q.b_mn ? (uint32_t)kHeadOperand / 2 >> 4 : 1u) << 16;
        const int planes = q.planes, promote = q.promote;
        for (int c0 = x.chunk0; c0 < x.chunk1; c0 += promote, ++at) {
            const int n = min(x.chunk1 - c0, promote), buf = at & 1;
            if (at >= 2 && !wait(smem_u32(&sh.acc_empty[buf]), (uint32_t)(((at >> 1) & 1) ^ 1))) { sh.fail = 1; return; }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t dcol = tmem + (uint32_t)(buf * kCols);
            for (int k = 0; k < n; ++k) {
                if (!wait(full0 + stg * 8, phase)) { sh.fail = 1; return; }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t a = a0 + off, b = b0 + off;
                uint32_t acc = k > 0;
                auto term = [&](int pa, int pb) {
#pragma unroll
                    for (int u = 0; u < kHeadChunk / 16; ++u, acc = 1)
                        head_mma<CG>(dcol, a + pa * slot + u * step_a, b + pb * (kHeadOperand >> 4) + u * step_b, idesc, acc);
                };
                // the products of planes, the smallest first: what is added to a small sum loses less
                if (planes == 3) { term(2, 0); term(0, 2); term(1, 1); }
                if (planes > 1) { term(1, 0); term(0, 1); }
                term(0, 0);
                commit(empty0 + stg * 8);
                if (k == n - 1) commit(smem_u32(&sh.acc_full[buf]));
                off += stage;
                if (++stg == stages) { stg = 0; off = 0; phase ^= 1; }
            }
        }
    }
}

// ------------------------------------------------------------------ what becomes of a tile (the epilogue warps)
// A thread holds a row, 32 threads of a warp 32 rows: stored as they are, an instruction would send 32 sectors of 32 rows one by one (2 us for
// a tile of 128 x 128, whatever its K).  Instead 128 bytes of each row go to a buffer of the warp, 16-byte piece k of row r at k ^ (r mod 8) as the
// 128-byte swizzle of the bulk copy that stores them.
__device__ __forceinline__ void buf_free(int lane) {           // the copy before has read the buffer
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
}
__device__ __forceinline__ void buf_put(unsigned char* buf, int lane, int k, uint4 w) {
    *reinterpret_cast<uint4*>(buf + lane * 128 + ((k ^ (lane & 7)) << 4)) = w;
}
// 64 columns in a 16-bit type, eight at a time: nothing is held beside the columns themselves, which fill the registers where parts of K are added up.
template <typename T>
__device__ __forceinline__ void buf_halves(unsigned char* buf, int lane, const float (&z)[64]) {
#pragma unroll
    for (int k = 0; k < 8; ++k)
        buf_put(buf, lane, k, make_uint4(pack2(z[8 * k], z[8 * k + 1], T()), pack2(z[8 * k + 2], z[8 * k + 3], T()), pack2(z[8 * k + 4], z[8 * k + 5], T()),
                                         pack2(z[8 * k + 6], z[8 * k + 7], T())));
}
template <bool kAdd>
__device__ __forceinline__ void buf_store(unsigned char* buf, int lane, const CUtensorMap* map, int c, int r, int plane) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
        if (kAdd) asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2, %3}], [%4];"
                               ::"l"(map), "r"(c), "r"(r), "r"(plane), "r"(smem_u32(buf)) : "memory");
        else asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];"
                          ::"l"(map), "r"(c), "r"(r), "r"(plane), "r"(smem_u32(buf)) : "memory");
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
}
// 64 columns of float32 rows.
__device__ __forceinline__ void buf_floats(const HeadJob& q, unsigned char* buf, int lane, const float (&z)[64], int c0, int r, int plane, bool add) {
#pragma unroll
    for (int h = 0; h < 64; h += 32) {
        if (c0 + h >= q.cols) break;
        buf_free(lane);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            buf_put(buf, lane, k, make_uint4(__float_as_uint(z[h + 4 * k]), __float_as_uint(z[h + 4 * k + 1]), __float_as_uint(z[h + 4 * k + 2]),
                                             __float_as_uint(z[h + 4 * k + 3])));
        if (add) buf_store<true>(buf, lane, &q.out, c0 + h, r, plane); else buf_store<false>(buf, lane, &q.out, c0 + h, r, plane);
    }
}

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// Exponents from here down give zero; a finite one, so that zero times it is zero too.  A NaN stays.
__device__ __forceinline__ float head_floor(float t) { return max_nan(t, -1000.f); }

// Statistics of one row's logits z: the largest, top; the sum of e = 2^(c (z - top)) less 1, over, so that where one token is all but sure what is left for the others
// keeps its digits; and the sum of e log2 e.  Without a logit above -inf over is -1.
struct HeadStat {
    float top, over, elog;
    __device__ __forceinline__ void start() { top = -INFINITY; over = -1.f; elog = 0.f; }
    template <bool kEntropy> __device__ __forceinline__ void add(const float (&z)[64], float c) {
        float m0 = fmaxf(z[0], z[1]), m1 = fmaxf(z[2], z[3]);
#pragma unroll
        for (int u = 4; u < 64; u += 4) {
            m0 = fmaxf(m0, fmaxf(z[u], z[u + 1]));
            m1 = fmaxf(m1, fmaxf(z[u + 2], z[u + 3]));
        }
        const float now = fmaxf(top, fmaxf(m0, m1)), base = now == -INFINITY ? 0.f : now;
        const Pair scale(c), from(-base);
        Pair s[2] = {Pair(0.f), Pair(0.f)}, l[2] = {Pair(0.f), Pair(0.f)};
#pragma unroll
        for (int u = 0; u < 64; u += 2) {
            float a, b;
            ((Pair(z[u], z[u + 1]) + from) * scale).split(a, b);
            if (kEntropy) { a = head_floor(a); b = head_floor(b); }
            const Pair e(exp2_near(a), exp2_near(b));
            s[u / 2 & 1] = s[u / 2 & 1] + e;
            if (kEntropy) l[u / 2 & 1] = fma2(e, Pair(a, b), l[u / 2 & 1]);
        }
        float a, b, sum, log = 0.f;
        (s[0] + s[1]).split(a, b);
        sum = a + b;
        if (kEntropy) {
            (l[0] + l[1]).split(a, b);                        // the largest has no part in it: its log2 e is 0
            log = a + b;
        }
        if (now > top) {
            if (sum < 1.0625f) {                             // the others by themselves: the largest is alone
                s[0] = s[1] = Pair(0.f);
#pragma unroll
                for (int u = 0; u < 64; u += 2) {
                    ((Pair(z[u], z[u + 1]) + from) * scale).split(a, b);
                    s[u / 2 & 1] = s[u / 2 & 1] + Pair(a == 0.f ? 0.f : exp2_near(a), b == 0.f ? 0.f : exp2_near(b));
                }
                (s[0] + s[1]).split(a, b);
                sum = a + b;
            } else {
                sum -= 1.f;
            }
            const float d = fmaxf((top - now) * c, -1000.f), f = exp2_near(d), all = 1.f + over;
            over = fmaf(f, all, sum);
            if (kEntropy) elog = fmaf(f, fmaf(d, all, elog), log);
            top = now;
        } else {
            over += sum;
            elog += log;
        }
    }
    // Joins another's.
    __device__ __forceinline__ void join(float m, float x, float l, float c) {
        const bool first = top >= m;
        const float d = fmaxf((first ? m - top : top - m) * c, -1000.f), f = exp2_near(d), all = 1.f + (first ? x : over);
        elog = fmaf(f, fmaf(d, all, first ? l : elog), first ? elog : l);
        over = fmaf(f, all, first ? over : x);
        top = fmaxf(top, m);
    }
};

// A tile as one thread sees it: a row, and what is read for that row before the tile is ready.
struct HeadView {
    HeadTile x;
    int j, row;
    bool live;
    HeadRow hr;
    int tok;                      // column of the row's token in the piece, or out of it
    float row_scale, d_scale;
};

template <int CG, int KIND>
__device__ __forceinline__ HeadView head_view(const HeadArgs& g, int i, int rank, int warp, int lane) {
    HeadView v;
    v.live = head_tile(g, i, v.j, v.x);
    if (!v.live) return v;
    const HeadJob& q = g.job[v.j];
    v.row = v.x.m * 128 * CG + rank * 128 + (warp & 3) * 32 + lane;
    v.tok = -1;
    v.row_scale = v.d_scale = 1.f;
    if ((KIND == kHeadStats || KIND == kHeadGrad) && g.row_scale && v.row < q.rows) v.row_scale = g.row_scale[v.row];
    if (KIND == kHeadGrad && g.d_scale && v.row < q.rows) v.d_scale = g.d_scale[v.row];
    if (KIND == kHeadStats && v.row < q.rows && g.tokens) {
        const long long id = g.token_bytes == 8 ? ((const long long*)g.tokens)[v.row] : (long long)((const int*)g.tokens)[v.row];
        if (id >= g.col0 && id < (long long)g.col0 + q.cols) v.tok = (int)(id - g.col0);
    }
    if (KIND == kHeadGrad && v.row < q.rows) {
        const float4 c = *reinterpret_cast<const float4*>(g.coef + v.row);
        v.hr = HeadRow{c.x, c.y, c.z, c.w};
        v.tok = g.row_token[v.row] - g.col0;
    }
    return v;
}

// d of 64 columns, to its planes.
template <bool kEntropy, bool kF32>
__device__ __forceinline__ void head_gradient(const HeadArgs& g, const HeadJob& q, const HeadView& v, float (&z)[64], int c0, unsigned char* buf, int lane) {
    const bool token = v.tok >= c0 && v.tok < c0 + 64;
    float own = 0.f;
    if (token) {                                             // c0 has -a: the token's 1 - p without the cancellation
#pragma unroll
        for (int u = 0; u < 64; ++u) own = v.tok == c0 + u ? z[u] : own;
        const float t = head_floor(fmaf(own, g.c, -v.hr.lse2)), p = exp2_near(t);
        own = p * fmaf(v.hr.c1, t, v.hr.c0 + v.hr.a) - v.hr.a * expm1f(t * 0.69314718055994531f);
    }
    const Pair scale(g.c), from(-v.hr.lse2), k0(v.hr.c0), k1(v.hr.c1);
#pragma unroll
    for (int u = 0; u < 64; u += 2) {
        float a, b;
        fma2(Pair(z[u], z[u + 1]), scale, from).split(a, b);
        if (kEntropy) { a = head_floor(a); b = head_floor(b); }
        const Pair p(exp2_near(a), exp2_near(b));
        (p * (kEntropy ? fma2(k1, Pair(a, b), k0) : k0)).split(z[u], z[u + 1]);
    }
    if (token) {
#pragma unroll
        for (int u = 0; u < 64; ++u) z[u] = v.tok == c0 + u ? own : z[u];
    }
    if (kF32 && g.store_near) {
        // two float16 planes, each column times its weights' power of two over the largest: those weights are smaller by as much
        // (the scales' quotient first: it is at most 1, where d_scale over a small scale may be beyond float32)
        const float most = 1.f / *g.col_most, f0 = g.col_scale[c0 / kHeadGroup] * most * v.d_scale,
                    f1 = c0 + kHeadGroup < q.cols ? g.col_scale[c0 / kHeadGroup + 1] * most * v.d_scale : 0.f;
#pragma unroll
        for (int plane = 0; plane < kHeadNear; ++plane) {
            buf_free(lane);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const Pair f(k < 4 ? f0 : f1);
                unsigned w[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    float a, b;
                    (Pair(z[8 * k + 2 * u], z[8 * k + 2 * u + 1]) * f).split(a, b);
                    w[u] = pack2(a, b, __half());
                    if (plane) {
                        const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&w[u]));
                        w[u] = pack2(a - h.x, b - h.y, __half());
                    }
                }
                buf_put(buf, lane, k, make_uint4(w[0], w[1], w[2], w[3]));
            }
            buf_store<false>(buf, lane, &g.job[1].out, c0, v.row - lane, plane);
        }
    }
    if (kF32) {
        if (!g.store_wide) return;
#pragma unroll
        for (int plane = 0; plane < kHeadWide; ++plane) {
            buf_free(lane);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                unsigned w[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    float &a = z[8 * k + 2 * u], &b = z[8 * k + 2 * u + 1];
                    w[u] = pack2(a, b, __nv_bfloat16());
                    a -= __uint_as_float(w[u] << 16);        // what the plane has left over; exact
                    b -= __uint_as_float(w[u] & 0xffff0000u);
                }
                buf_put(buf, lane, k, make_uint4(w[0], w[1], w[2], w[3]));
            }
            buf_store<false>(buf, lane, &q.out, c0, v.row - lane, plane);
        }
    } else {
        buf_free(lane);
        if (q.half) buf_halves<__half>(buf, lane, z); else buf_halves<__nv_bfloat16>(buf, lane, z);
        buf_store<false>(buf, lane, &q.out, c0, v.row - lane, 0);
    }
}

// 64 columns of dweight.
template <typename T>
__device__ __forceinline__ void head_weight(const HeadArgs& g, const HeadJob& q, const HeadView& v, float (&z)[64], int c0, unsigned char* buf, int lane) {
    if (g.bulk) {
        if constexpr (sizeof(T) == 4) {
            buf_floats(q, buf, lane, z, c0, v.row - lane, 0, g.accumulate);
        } else {
            buf_free(lane);
            buf_halves<T>(buf, lane, z);
            buf_store<false>(buf, lane, &q.out, c0, v.row - lane, 0);
        }
        return;
    }
    // Rows at any alignment, and 16-bit ones that are added to before they are rounded: 32 columns at a time by way of the buffer, from which the warp
    // writes one row after the other.  Column u of row r lies at u ^ r of its row there, so that neither way meets a bank twice.
    const int rows = min(32, q.rows - (v.row - lane));
    T* to = (T*)g.out + (long long)(v.row - lane) * g.ldo + c0 + lane;
    float* f = (float*)buf;
#pragma unroll
    for (int h = 0; h < 64; h += 32) {
        buf_free(lane);
#pragma unroll
        for (int u = 0; u < 32; ++u) f[lane * 32 + (u ^ lane)] = z[h + u];
        __syncwarp();
        if (c0 + h + lane < q.cols) {
            T* p = to + h;
            for (int r = 0; r < rows; r += 8, p += 8 * g.ldo) {
                T old[8];                                    // all of them under way before the first is written
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (g.accumulate && r + k < rows) old[k] = p[k * g.ldo];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (r + k >= rows) break;
                    const float s = f[(r + k) * 32 + (lane ^ (r + k))];
                    p[k * g.ldo] = from_f32<T>(g.accumulate ? s + to_f32(old[k]) : s);
                }
            }
        }
    }
}

// 64 columns of a tile from c0 on; the whole warp calls this.  kF32: the operands are float32 (the statistics do not ask).
template <int KIND, bool kF32>
__device__ __forceinline__ void head_take(const HeadArgs& g, const HeadJob& q, const HeadView& v, HeadStat& st, float (&z)[64], int c0, float unscale,
                                          unsigned char* buf, int lane) {
    if (c0 >= q.cols || v.row - lane >= q.rows) return;       // the same for all
    if ((KIND == kHeadStats || KIND == kHeadGrad) && kF32 && g.row_scale) {
        const float f0 = v.row_scale * g.col_scale[c0 / kHeadGroup], f1 = c0 + kHeadGroup < q.cols ? v.row_scale * g.col_scale[c0 / kHeadGroup + 1] : 0.f;
#pragma unroll
        for (int k = 0; k < 64; ++k) z[k] *= k < kHeadGroup ? f0 : f1;
    }
    if (KIND == kHeadStats) {
        if (c0 + 64 > q.cols) {
#pragma unroll
            for (int k = 0; k < 64; ++k) z[k] = c0 + k < q.cols ? z[k] : -INFINITY;
        }
        if (v.tok >= c0 && v.tok < c0 + 64) {
            float own = 0.f;
#pragma unroll
            for (int k = 0; k < 64; ++k) own = v.tok == c0 + k ? z[k] : own;
            g.ztok[v.row] = own;
        }
        if (g.entropy) st.add<true>(z, g.c); else st.add<false>(z, g.c);
    } else if (KIND == kHeadGrad) {
        if (g.entropy) head_gradient<true, kF32>(g, q, v, z, c0, buf, lane); else head_gradient<false, kF32>(g, q, v, z, c0, buf, lane);
    } else if (q.kind == kHeadHidden) {
        if (kF32) {
            const float f = *g.col_most;
#pragma unroll
            for (int k = 0; k < 64; ++k) z[k] *= f;
        }
        buf_floats(q, buf, lane, z, c0, v.row - lane, v.x.split, g.add);
    } else {
#pragma unroll
        for (int k = 0; k < 64; ++k) z[k] *= unscale;
        if (kF32 || g.out_type == 0) head_weight<float>(g, q, v, z, c0, buf, lane);
        else if (g.out_type == 1) head_weight<__nv_bfloat16>(g, q, v, z, c0, buf, lane);
        else head_weight<__half>(g, q, v, z, c0, buf, lane);
    }
}

template <int CG, int KIND, bool PROMOTE>
__device__ void head_epilogue(const HeadArgs& g, HeadShared& sh, unsigned char* area, int rank, int warp, int lane) {
    constexpr int kParts = kHeadEpi / 4, kCols = 128 * CG / kParts, kTakes = kCols / 64;       // columns of a thread
    const int part = warp >> 2;
    const float unscale = KIND == kHeadHidden && g.unscale ? *g.unscale : 1.f;
    unsigned char* buf = area + warp * kHeadBuf;
    int at = 0;
    bool ok = true;
    HeadView v = head_view<CG, KIND>(g, 0, rank, warp, lane);
    for (int i = 1; v.live; ++i) {
        HeadView next;
        if (!PROMOTE) next = head_view<CG, KIND>(g, i, rank, warp, lane);         // its reads are under way meanwhile
        const HeadJob& q = g.job[v.j];
        const int col = v.x.n * 128 * CG + part * kCols;
        HeadStat st;
        st.start();
        float sum[PROMOTE ? kTakes : 1][64];                  // 64 columns of the tile each, where the parts of K are added up here
        if (PROMOTE) {
#pragma unroll
            for (int u = 0; u < kTakes; ++u)
#pragma unroll
                for (int k = 0; k < 64; ++k) sum[u][k] = 0.f;
        }
        for (int c0 = v.x.chunk0; c0 < v.x.chunk1; c0 += q.promote, ++at) {
            const int half = at & 1;
            const uint32_t bar = smem_u32(&sh.acc_full[half]), parity = (uint32_t)((at >> 1) & 1);
            if (ok) ok = __all_sync(0xffffffffu, CG == 2 ? mbar_wait_pair(bar, parity, &sh.fail) : mbar_wait(bar, parity, &sh.fail));
            if (!ok) sh.fail = 1;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t from = sh.tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(half * 128 * CG + part * kCols);
#pragma unroll
            for (int u = 0; u < kTakes; ++u) {
                float (&z)[64] = sum[PROMOTE ? u : 0];
                if (PROMOTE) {
#pragma unroll
                    for (int h = 0; h < 64; h += 16) {
                        uint32_t r[16];
                        tmem_ld16(from + u * 64 + h, r);
#pragma unroll
                        for (int k = 0; k < 16; ++k) z[h + k] += __uint_as_float(r[k]);
                    }
                } else {
#pragma unroll
                    for (int h = 0; h < 64; h += 32) {
                        uint32_t r[32];
                        tmem_ld32(from + u * 64 + h, r);
#pragma unroll
                        for (int k = 0; k < 32; ++k) z[h + k] = __uint_as_float(r[k]);
                    }
                }
                if (u + 1 == kTakes) {                            // all of it is in registers: the next product may have the accumulator
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        const uint32_t done = smem_u32(&sh.acc_empty[half]);
                        if (CG == 2) arrive_cluster(of_leader(done)); else mbar_arrive(done);
                    }
                }
                if (!ok) {
#pragma unroll
                    for (int k = 0; k < 64; ++k) z[k] = __int_as_float(0x7fffffff);
                }
                if (!PROMOTE) head_take<KIND, PROMOTE>(g, q, v, st, z, col + u * 64, unscale, buf, lane);
            }
        }
        if (PROMOTE) {
#pragma unroll
            for (int u = 0; u < kTakes; ++u) head_take<KIND, PROMOTE>(g, q, v, st, sum[u], col + u * 64, unscale, buf, lane);
        }
        if (KIND == kHeadStats) {
            // the parts of the columns meet in shared memory, in one of two places by turns
            float* meet = (float*)area + (i & 1) * (kParts - 1) * 384 + (warp & 3) * 32 + lane;
            if (part) {
                float* m = meet + (part - 1) * 384;
                m[0] = st.top; m[128] = st.over; m[256] = st.elog;
            }
            asm volatile("bar.sync 1, %0;" ::"n"(128 * kParts) : "memory");
            if (!part && v.row < q.rows) {
#pragma unroll
                for (int k = 0; k < kParts - 1; ++k) st.join(meet[k * 384], meet[k * 384 + 128], meet[k * 384 + 256], g.c);
                float* p = g.part + (long long)(g.part0 + v.x.n) * q.rows + v.row;
                const long long plane = (long long)g.parts * q.rows;
                p[0] = st.top;
                p[plane] = st.over;
                if (g.entropy) p[2 * plane] = st.elog;
            }
        }
        v = PROMOTE ? head_view<CG, KIND>(g, i, rank, warp, lane) : next;         // the sums leave no registers for it any earlier
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");       // what this warp has stored is there
}

// KIND: kHeadStats, kHeadGrad, or kHeadHidden for both products of d.
template <int CG, int KIND, bool PROMOTE>
__global__ void __launch_bounds__(kHeadThreads, 1) head_kernel(const __grid_constant__ HeadArgs g) {
    extern __shared__ unsigned char head_smem[];
    __shared__ HeadShared sh;
    unsigned char* smem = (unsigned char*)(((uintptr_t)head_smem + 1023) & ~(uintptr_t)1023);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = CG == 2 ? (int)cluster_rank() : 0;
    constexpr uint32_t kColumns = 256 * CG;                   // two accumulators
    if (warp == 0) {
        if (CG == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)), "r"(kColumns) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)), "r"(kColumns) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    if (tid == 32) {
        for (int k = 0; k < kHeadMaxStages; ++k) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_u32(&sh.full[k])) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_u32(&sh.empty[k])) : "memory");
        }
        for (int k = 0; k < 2; ++k) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_u32(&sh.acc_full[k])) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(&sh.acc_empty[k])), "r"(kHeadEpi * CG) : "memory");
        }
        sh.fail = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (CG == 2) cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    cudaGridDependencySynchronize();                          // all before this touches nothing that an earlier launch has
    if (warp < kHeadEpi) head_epilogue<CG, KIND, PROMOTE>(g, sh, smem + kHeadRing, rank, warp, lane);
    else if (tid == 32 * kHeadEpi) head_copies<CG>(g, smem, sh, rank);
    else if (tid == 32 * (kHeadEpi + 1) && rank == 0) head_products<CG>(g, smem, sh);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (sh.fail) {
        // a wait ran out: report it, and let copies in flight land before their shared memory goes back to the SM
        if (tid == 0 && g.status) *g.status = 2;
        for (int k = 0; k < 512; ++k) __nanosleep(200);
    }
    __syncthreads();
    if (CG == 2) cluster_sync();                              // nothing reaches a block that has left
    if (warp == 0) {
        if (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(sh.tmem_base), "r"(kColumns) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(sh.tmem_base), "r"(kColumns) : "memory");
    }
}

// ------------------------------------------------------------------ around the products
// A copy of 16-bit rows at a stride of 16 bytes, where bulk copies cannot start on them; or three bfloat16 planes of float32 rows.  Columns behind dim
// are zero.  A value that bfloat16 has no finite number for stays in plane 0.
template <typename T>
__global__ void __launch_bounds__(256) head_pack_kernel(const T* x, long long rows, int dim, long long ld, unsigned short* out, int ldp, long long plane) {
    const int pairs = ldp / 2;
    const long long n = rows * pairs;
    cudaGridDependencySynchronize();
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < n; i += gridDim.x * 256LL) {
        const long long r = i / pairs;
        const int c = (int)(i - r * pairs) * 2;
        const T* p = x + r * ld + c;
        unsigned* to = (unsigned*)(out + r * ldp + c);
        if constexpr (sizeof(T) == 2) {
            const unsigned short* q = (const unsigned short*)p;
            *to = (c < dim ? (unsigned)q[0] : 0u) | (c + 1 < dim ? (unsigned)q[1] << 16 : 0u);
        } else {
            float a = c < dim ? p[0] : 0.f, b = c + 1 < dim ? p[1] : 0.f;
#pragma unroll
            for (int k = 0; k < kHeadWide; ++k) {
                const unsigned w = pack2(a, b, __nv_bfloat16());
                to[k * (plane / 2)] = w;
                a -= __uint_as_float(w << 16);
                b -= __uint_as_float(w & 0xffff0000u);
                if (!isfinite(a)) a = 0.f;
                if (!isfinite(b)) b = 0.f;
            }
        }
    }
}

// Two float16 planes of float32 rows, kGroup of them (a block) times a power of two that brings their largest finite number to between 2^14 and 2^15;
// scale[block] takes that back, and the largest scale goes to *most.  A group of 32 rows has a warp for each, a row by itself all of them.  What the
// first look has read stays in registers as far as they go (1024 columns of 32 rows; with every row read twice by eight warps 50021 x 1001 took 130 us,
// since the blocks at work together held more than L2).
template <int kGroup> constexpr int kNearThreads = kGroup > 1 ? 32 * kGroup : 256;
template <int kGroup, bool kVector>
__global__ void __launch_bounds__(kNearThreads<kGroup>) head_near_kernel(const float* x, long long rows, int dim, long long ld, unsigned short* out, int ldp,
                                                                 long long plane, float* scale, int* most) {
    __shared__ float tops[32];
    constexpr int kHeld = 8, kWarps = kNearThreads<kGroup> / 32, kStep = kGroup > 1 ? 128 : 128 * kWarps;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, start = (kGroup > 1 ? lane : (int)threadIdx.x) * 4;
    const long long r = (long long)blockIdx.x * kGroup + (kGroup > 1 ? warp : 0);
    const bool live = r < rows;
    const float* row = x + r * ld;
    cudaGridDependencySynchronize();
    auto four = [&](int c) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (!live) return v;
        if (kVector) {
            if (c < dim) v = *reinterpret_cast<const float4*>(row + c);
        } else {
            if (c < dim) v.x = row[c];
            if (c + 1 < dim) v.y = row[c + 1];
            if (c + 2 < dim) v.z = row[c + 2];
            if (c + 3 < dim) v.w = row[c + 3];
        }
        return v;
    };
    float top = 0.f;
    auto see = [&](const float4& v) {
        if (fabsf(v.x) < INFINITY) top = fmaxf(top, fabsf(v.x));
        if (fabsf(v.y) < INFINITY) top = fmaxf(top, fabsf(v.y));
        if (fabsf(v.z) < INFINITY) top = fmaxf(top, fabsf(v.z));
        if (fabsf(v.w) < INFINITY) top = fmaxf(top, fabsf(v.w));
    };
    float4 held[kHeld];
#pragma unroll
    for (int k = 0; k < kHeld; ++k) held[k] = four(start + k * kStep);
#pragma unroll
    for (int k = 0; k < kHeld; ++k) see(held[k]);
#pragma unroll 8
    for (int c = start + kHeld * kStep; c < dim; c += kStep) see(four(c));
#pragma unroll
    for (int k = 16; k; k /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
    if (lane == 0) tops[warp] = top;
    __syncthreads();
    top = tops[lane % kWarps];
#pragma unroll
    for (int k = kWarps / 2; k; k /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
    // Weights of nothing but zeros (a padded vocabulary) take the smallest scale there is, so that the largest one, which d is formed for, is that of numbers
    // that count: with a scale of 1, 16 or more of d's binary digits went to a product with zero (32 rows of zeros behind 128224 x 1024: dhidden off by 2.2e-4
    // of itself instead of 2.6e-7).
    int e = kGroup > 1 ? 15 - 120 : 15;
    if (top > 0.f) frexpf(top, &e);
    e = min(max(15 - e, -120), 120);
    const float f = ldexpf(1.f, e);
    if (threadIdx.x == 0) {
        scale[blockIdx.x] = ldexpf(1.f, -e);
        if (most) atomicMax(most, __float_as_int(ldexpf(1.f, -e)));     // of positive numbers
    }
    if (!live) return;
    auto split = [&](int c, const float4& v) {
        if (c >= ldp) return;                                // ldp is a multiple of 8
        float a[4] = {v.x * f, v.y * f, v.z * f, v.w * f};
        const uint2 w = make_uint2(pack2(a[0], a[1], __half()), pack2(a[2], a[3], __half()));
        *reinterpret_cast<uint2*>(out + r * ldp + c) = w;
        const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&w.x)), i = __half22float2(*reinterpret_cast<const __half2*>(&w.y));
        a[0] -= h.x; a[1] -= h.y; a[2] -= i.x; a[3] -= i.y;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (!isfinite(a[k])) a[k] = 0.f;                 // what is not finite is in the first plane
        *reinterpret_cast<uint2*>(out + plane + r * ldp + c) = make_uint2(pack2(a[0], a[1], __half()), pack2(a[2], a[3], __half()));
    };
#pragma unroll
    for (int k = 0; k < kHeld; ++k) split(start + k * kStep, held[k]);
#pragma unroll 8
    for (int c = start + kHeld * kStep; c < ldp; c += kStep) split(c, four(c));
}

// ------------------------------------------------------------------ a few rows
// Statistics of kRows rows without the tensor cores, whose tiles of 128 rows would be all but empty: a warp reads kHeadFewCols rows of the weights at a
// time, 256 elements of each per step, and multiplies them in float32 with the hidden rows, which stay in L1.  Its groups of columns are
// `gridDim * kHeadFewWarps` apart, neighbours in neighbouring blocks, so that a short vocabulary reaches every SM.  Bound by the weights' one pass: a row on
// 131072 x 2048 bf16 takes 80 us, 6.7 TB/s; four columns of a warp's took 83.
constexpr int kHeadFewWarps = 8, kHeadFewBlocks = 4, kHeadFewCols = 2;
struct HeadEight { uint4 q[2]; };            // eight elements; 16-bit ones take the first half

template <typename T, bool kStream> __device__ __forceinline__ HeadEight eight_of(const T* p) {
    HeadEight e;
#pragma unroll
    for (int k = 0; k < (int)sizeof(T) / 2; ++k) {
        uint4& q = e.q[k];
        if (kStream) asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "l"((const uint4*)p + k));
        else q = __ldg((const uint4*)p + k);
    }
    return e;
}
template <typename T> __device__ __forceinline__ void floats_of(Pair (&f)[4], const HeadEight& e, T) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            f[2 * k] = Pair(__uint_as_float(e.q[k].x), __uint_as_float(e.q[k].y));
            f[2 * k + 1] = Pair(__uint_as_float(e.q[k].z), __uint_as_float(e.q[k].w));
        }
    } else {
        float x[8];
        unpack8(x, e.q[0], T());
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] = Pair(x[2 * k], x[2 * k + 1]);
    }
}

template <typename T, int kRows>
__global__ void __launch_bounds__(32 * kHeadFewWarps, kRows == 4 ? 2 : kHeadFewBlocks) head_few_kernel(const T* hidden, const T* weight, int rows, int vocab, int dim,
                                                                                      long long ldh, long long ldw, const void* tokens, int token_bytes, float c,
                                                                                      float* part, float* ztok) {
    __shared__ HeadStat all[kHeadFewWarps][kRows];
    constexpr int kCols = kHeadFewCols;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, mine = lane % kRows, whole = dim & ~7;
    cudaGridDependencySynchronize();
    long long token = -1;                                    // of the lane's row
    if (tokens && mine < rows) token = token_bytes == 8 ? ((const long long*)tokens)[mine] : (long long)((const int*)tokens)[mine];
    HeadStat st;
    st.start();
    for (int c0 = (warp * gridDim.x + blockIdx.x) * kCols; c0 < vocab; c0 += gridDim.x * kHeadFewWarps * kCols) {
        const T* w[kCols];
#pragma unroll
        for (int u = 0; u < kCols; ++u) w[u] = weight + min(c0 + u, vocab - 1) * ldw;       // behind the last column: the last one again
        Pair sum[kRows][kCols];
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int u = 0; u < kCols; ++u) sum[r][u] = Pair(0.f);
        auto step = [&](const HeadEight (&e)[kCols], int k) {
            Pair f[kCols][4];
#pragma unroll
            for (int u = 0; u < kCols; ++u) floats_of(f[u], e[u], T());
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                Pair h[4];
                floats_of(h, eight_of<T, false>(hidden + (r < rows ? r : 0) * ldh + k), T());
#pragma unroll
                for (int u = 0; u < kCols; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[r][u] = fma2(f[u][i], h[i], sum[r][u]);
            }
        };
        constexpr int kAhead = sizeof(T) == 4 ? 2 : 4;       // steps whose weights are under way, as registers go
        int k = lane * 8;
        for (; k + (kAhead - 1) * 256 < whole; k += kAhead * 256) {
            HeadEight e[kAhead][kCols];
#pragma unroll
            for (int a = 0; a < kAhead; ++a)
#pragma unroll
                for (int u = 0; u < kCols; ++u) e[a][u] = eight_of<T, true>(w[u] + k + a * 256);
#pragma unroll
            for (int a = 0; a < kAhead; ++a) step(e[a], k + a * 256);
        }
        for (; k < whole; k += 256) {
            HeadEight e[kCols];
#pragma unroll
            for (int u = 0; u < kCols; ++u) e[u] = eight_of<T, true>(w[u] + k);
            step(e, k);
        }
        float z[kCols];
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int u = 0; u < kCols; ++u) {
                float a, b;
                sum[r][u].split(a, b);
                a += b;
                if (whole + lane < dim) a = fmaf(to_f32(w[u][whole + lane]), to_f32(hidden[(r < rows ? r : 0) * ldh + whole + lane]), a);
#pragma unroll
                for (int n = 16; n; n /= 2) a += __shfl_xor_sync(0xffffffffu, a, n);
                if (r == mine) z[u] = a;
            }
#pragma unroll
        for (int u = 0; u < kCols; ++u) {
            if (c0 + u >= vocab) break;
            if (token == c0 + u && lane < rows) ztok[lane] = z[u];
            const float total = 1.f + st.over;
            if (z[u] > st.top) {
                const float d = fmaxf((st.top - z[u]) * c, -1000.f), f = exp2f(d);
                st.elog = f * fmaf(d, total, st.elog);
                st.over = f * total;
                st.top = z[u];
            } else {
                const float d = head_floor((z[u] - (st.top == -INFINITY ? 0.f : st.top)) * c), e = exp2f(d);
                st.over += e;
                st.elog = fmaf(e, d, st.elog);
            }
        }
    }
    if (lane < kRows) all[warp][lane] = st;
    __syncthreads();
    if (threadIdx.x < rows) {
        st = all[0][threadIdx.x];
        for (int k = 1; k < kHeadFewWarps; ++k) st.join(all[k][threadIdx.x].top, all[k][threadIdx.x].over, all[k][threadIdx.x].elog, c);
        const long long at = (long long)blockIdx.x * rows + threadIdx.x, plane = (long long)gridDim.x * rows;
        part[at] = st.top;
        part[plane + at] = st.over;
        part[2 * plane + at] = st.elog;
    }
}

// Row values from the parts' statistics (it: inv_temperature, c: over log 2): kHeadRowThreads threads for `width` rows, which share a row's parts.  The largest logit is
// found first, so that the terms of the sums do not wait for one another.
constexpr int kHeadRowThreads = 512;
__global__ void __launch_bounds__(kHeadRowThreads) head_rows_kernel(const float* part, int parts, int rows, int width, const float* ztok, const void* tokens,
                                                                    int token_bytes, long long vocab, float c, double it, int with_entropy, float* logp, float* entropy, float* lse,
                                                                    int* status) {
    __shared__ float sm[3][kHeadRowThreads];
    const int tid = threadIdx.x, lane = tid % width, share = tid / width, shares = kHeadRowThreads / width;
    const int r = blockIdx.x * width + lane;
    const long long plane = (long long)parts * rows;
    cudaGridDependencySynchronize();
    float top = -INFINITY;
    if (r < rows) {
#pragma unroll 8
        for (int k = share; k < parts; k += shares) top = fmaxf(top, part[(long long)k * rows + r]);
    }
    sm[0][tid] = top;
    for (int n = shares / 2; n; n /= 2) {
        __syncthreads();
        if (share < n) sm[0][tid] = fmaxf(sm[0][tid], sm[0][tid + n * width]);
    }
    __syncthreads();
    top = sm[0][lane];
    float at_top = 0.f, over = 0.f, elog = 0.f;              // parts that have the largest logit; the rest of their sums, and the others'
    if (r < rows) {
#pragma unroll 8
        for (int k = share; k < parts; k += shares) {
            const float* p = part + (long long)k * rows + r;
            const float m = p[0], x = p[plane], e = with_entropy ? p[2 * plane] : 0.f, d = fmaxf((m - top) * c, -1000.f), f = exp2f(d), all = 1.f + x;
            const bool has = m == top;
            at_top += has ? 1.f : 0.f;
            over += has ? x : f * all;
            elog += has ? e : f * fmaf(d, all, e);
        }
    }
    __syncthreads();
    sm[0][tid] = at_top; sm[1][tid] = over; sm[2][tid] = elog;
    for (int n = shares / 2; n; n /= 2) {
        __syncthreads();
        if (share < n) {
#pragma unroll
            for (int k = 0; k < 3; ++k) sm[k][tid] += sm[k][tid + n * width];
        }
    }
    if (share != 0 || r >= rows) return;
    over = top == INFINITY ? __int_as_float(0x7fffffff) : sm[1][tid];
    elog = sm[2][tid];
    const double rest = (double)sm[0][tid] - 1.0 + (double)over, ls = log1p(rest);
    const bool none = rest == -1.0;                          // no logit is above -inf
    if (lse) lse[r] = none ? -INFINITY : (float)((double)top * it + ls);
    if (entropy) entropy[r] = none ? 0.f : (float)(ls - 0.69314718055994530942 * (double)elog / (1.0 + rest));
    if (logp) {
        const long long id = token_bytes == 8 ? token_id((const long long*)tokens, r, vocab, status) : token_id((const int*)tokens, r, vocab, status);
        logp[r] = id < 0 ? (rest == rest ? 0.f : (float)rest) : none ? -INFINITY : (float)(((double)ztok[r] - (double)top) * it - ls);
    }
}

// Coefficients of d for every row, and the power of two that brings the largest to 2^top: one block.  Powers up to 149, what float32's smallest numbers ask for
// at a top of 0, whose inverse float32 still holds.
__global__ void __launch_bounds__(1024) head_coef_kernel(int rows, long long vocab, const void* tokens, int token_bytes, double it, float c, const float* lse,
                                                         const float* entropy, const float* g_logp, const float* g_entropy, const float* g_lse, int top,
                                                         HeadRow* coef, int* row_token, float* unscale, float* d_scale, int* col_most,
                                                         int pieces, int* status) {
    __shared__ float most[32];
    const int tid = threadIdx.x;
    cudaGridDependencySynchronize();
    auto row = [&](int r, HeadRow& h) {
        long long id = -1;
        if (tokens) id = token_bytes == 8 ? token_id((const long long*)tokens, r, vocab, status) : token_id((const int*)tokens, r, vocab, status);
        const float z = lse[r];
        const bool none = z == -INFINITY;                     // no logit is finite: no gradient
        const float a = id >= 0 && g_logp && !none ? (float)(it * g_logp[r]) : 0.f;
        const float ge = g_entropy && !none ? (float)(it * g_entropy[r]) : 0.f;
        const float gz = g_lse && !none ? (float)(it * g_lse[r]) : 0.f;
        h.a = a;
        // Logits are multiplied by a float32 c, so lse is by the same number over it: what c is off by then counts for their difference alone.  What lse2 leaves of
        // it goes into the factors of p and p log2 p (logits near 130: 5e-6 of p without).
        const double l = (double)z * ((double)c / it);
        h.lse2 = none ? INFINITY : (float)l;
        const float rest = fabsf(h.lse2) < 0x1p30f ? (float)((double)h.lse2 - l) : 0.f, f = exp2f(rest);      // (beyond that no difference is left)
        h.c1 = -ge * 0.69314718055994531f;
        h.c0 = f * fmaf(h.c1, rest, gz - a - (ge != 0.f ? ge * entropy[r] : 0.f));
        h.c1 *= f;
        return (int)id;
    };
    float m = 0.f;
    for (int r = tid; r < rows; r += 1024) {
        HeadRow h;
        row_token[r] = row(r, h);
        coef[r] = h;
        const float s = fabsf(h.a) + fabsf(h.c0) + fabsf(h.c1);      // bounds |d|, since p |log2 p| < 1
        if (isfinite(s)) m = fmaxf(m, s);
    }
#pragma unroll
    for (int k = 16; k; k >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
    if ((tid & 31) == 0) most[tid >> 5] = m;
    __syncthreads();
    m = most[tid & 31];
#pragma unroll
    for (int k = 16; k; k >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
    int e = top;
    if (m > 0.f) {
        const bool power = frexpf(m, &e) == 0.5f;             // m < 2^e, or 2^(e - 1)
        e = top - e + power;
    }
    e = min(max(e, -120), 149);
    for (int r = tid; r < rows; r += 1024) {
        HeadRow h = coef[r];
        h.a = ldexpf(h.a, e); h.c0 = ldexpf(h.c0, e); h.c1 = ldexpf(h.c1, e);
        coef[r] = h;
        if (d_scale) {                                        // brings the row's own largest to between 2^13 and 2^14
            const float s = fabsf(h.a) + fabsf(h.c0) + fabsf(h.c1);
            int own = 14;
            if (s > 0.f && isfinite(s)) frexpf(s, &own);
            d_scale[r] = ldexpf(1.f, min(max(14 - own, -100), 100));
        }
    }
    if (tid == 0) *unscale = ldexpf(1.f, -e);
    for (int k = tid; k < pieces; k += 1024) col_most[k] = 0;
}

// dhidden from the planes of partial sums, in the order of the planes.
template <typename T>
__global__ void __launch_bounds__(256) head_sum_kernel(const float* plane, long long plane_size, int planes, int ldp, int rows, int dim, const float* unscale,
                                                       const float* d_scale, T* out, long long ldo) {
    const int groups = ldp / 8;
    cudaGridDependencySynchronize();
    const float f = *unscale;
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < (long long)rows * groups; i += gridDim.x * 256LL) {
        const long long r = i / groups;
        const int c = (int)(i - r * groups) * 8;
        float s[8] = {};
        for (int k = 0; k < planes; ++k) {
            float v[8];
            load8_wide(v, plane + k * plane_size + r * ldp + c);
#pragma unroll
            for (int u = 0; u < 8; ++u) s[u] += v[u];
        }
        const float own = d_scale ? 1.f / d_scale[r] : 1.f;      // (its product with f may be below float32's numbers)
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (c + u < dim) out[r * ldo + c + u] = from_f32<T>(s[u] * own * f);
    }
}

}  // namespace pb
