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
// block holds 128 rows of A, 128 rows of B and 128 x 256 of D), K in chunks of 64 through a ring of six
// stages filled by bulk tensor copies, two accumulators of 256 columns in tensor memory, so that eight
// warps work on the last tile while the next one is multiplied.  Up to 128 rows of hidden states run in
// single blocks of 128 x 128, since a pair would leave half of its rows empty: these calls are bound by
// reading the weights.
//   logits   A = hidden (K-major)        B = weight (K-major)      the row statistics, or d, are computed from the tile
//   hidden   A = d (K-major)             B = weight (MN-major)     float32 partial sums, one plane per split of K
//   weight   A = d, read transposed (MN-major)  B = hidden (MN-major)
// float32 operands are held as three bfloat16 planes (x = x0 + x1 + x2 to 2^-25 of x), and a product is
// the six terms x_i y_j with i + j <= 2; what is left out is below 2^-25.
// The tensor core adds to its float32 accumulator without rounding to nearest, so a long K drifts:
// float32 products, and the logits of the forward, leave the tensor core every kHeadPromote chunks and are
// added up in registers.
// Every wait is bounded (see mbar_wait); a block whose wait runs out reports it and gives NaN for its tiles.
#pragma once
#include "tc_common.cuh"
#include "tok_common.cuh"

namespace pb {

constexpr int kHeadChunk = 64;                // K elements per stage: one 128-byte swizzled row
constexpr int kHeadOperand = 128 * 128;       // bytes of an operand's 128 x 64 tile
constexpr int kHeadStages = 6;
constexpr int kHeadSmem = kHeadStages * 2 * kHeadOperand + 1024;
constexpr int kHeadEpiWarps = 8;              // quarter w % 4 of the tensor-memory lanes, half w / 4 of the columns
constexpr int kHeadThreads = 32 * (kHeadEpiWarps + 2);
constexpr int kHeadPlanes = 3;                // bfloat16 planes of a float32 operand

enum HeadKind { kHeadStats = 0, kHeadGrad = 1, kHeadHidden = 2, kHeadWeight = 3 };

// One product: tiles_m x tiles_n tiles, K split `splits` ways.
struct alignas(64) HeadJob {
    CUtensorMap a, b;            // K-major: (k, row, plane); MN-major: (row, k, plane)
    int kind;
    int a_mn, b_mn;              // operand is MN-major
    int tiles_m, tiles_n, splits;
    int group_m;                 // row tiles that are walked through together, for one column tile after the other
    int chunks, chunks_per_split;
    int rows, cols;              // of D
    int tiles;                   // tiles_m * tiles_n * splits
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
    int jobs, half;              // half: operands are float16
    int terms;                   // 1, or 6 products of planes
    int promote;                 // chunks of K that the tensor core adds up by itself
    float c;                     // inv_temperature * log2(e)
    int col0;                    // first column (token) of this piece of the vocabulary
    int* status;
    // row statistics
    float* part;                 // [3][parts][rows]: reference (log2), sum, sum of e log2 e
    int part0, parts;
    float* ztok;                 // the token's logit of each row
    const void* tokens;
    int token_bytes;
    long long vocab;
    // d
    const HeadRow* coef;
    const int* row_token;        // index of the token, or -1
    unsigned short* d;           // [planes][rows][ldd]
    long long d_plane;
    int ldd;
    // products
    float* plane;                // [splits][rows][ldp]
    long long plane_size;
    int ldp, add;                // add: an earlier piece is there
    void* out;                   // of this piece of dweight
    long long ldo;
    int out_type, accumulate, wide;      // pb_dtype; wide: rows start on 32 bytes
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
    uint64_t full[kHeadStages];   // a stage's operands have landed (at the leader: both blocks')
    uint64_t empty[kHeadStages];  // the products that read a stage are done
    uint64_t acc_full[2], acc_empty[2];
    uint32_t tmem_base;
    int fail;
};

struct HeadTile {
    int m, n, split, chunk0, chunk1;
};

// The job that tile `t` of the launch belongs to, and its place there; false behind the last.
__device__ __forceinline__ bool head_tile(const HeadArgs& g, int t, int& j, HeadTile& x) {
    j = 0;
    while (j < g.jobs && t >= g.job[j].tiles) t -= g.job[j++].tiles;
    if (j == g.jobs) return false;
    const HeadJob& q = g.job[j];
    const int per_split = q.tiles_m * q.tiles_n;
    x.split = t / per_split;
    t -= x.split * per_split;
    const int per_group = q.group_m * q.tiles_n, group = t / per_group;
    const int m0 = group * q.group_m, height = min(q.group_m, q.tiles_m - m0);
    t -= group * per_group;
    x.n = t / height;
    x.m = m0 + t - x.n * height;
    x.chunk0 = x.split * q.chunks_per_split;
    x.chunk1 = min(q.chunks, x.chunk0 + q.chunks_per_split);
    return true;
}

// Planes of the terms of a float32 product, the smallest first: what is added to a small sum loses less.
__device__ __forceinline__ void head_term(int terms, int k, int& pa, int& pb) {
    if (terms == 1) { pa = pb = 0; return; }
    pa = k == 0 ? 2 : k == 2 || k == 3 ? 1 : 0;              // (2,0) (0,2) (1,1) (1,0) (0,1) (0,0)
    pb = k == 1 ? 2 : k == 2 || k == 4 ? 1 : 0;
}

// ------------------------------------------------------------------ copies (one thread of each block)
template <int CG>
__device__ void head_copies(const HeadArgs& g, unsigned char* smem, HeadShared& sh, int rank) {
    int it = 0, j;
    HeadTile x;
    constexpr int kRows = 128 * CG;
    for (int t = cluster_id(); head_tile(g, t, j, x); t += cluster_count()) {
        const HeadJob& q = g.job[j];
        const int m0 = x.m * kRows + rank * 128, n0 = x.n * kRows + rank * 128;
        const uint32_t bytes = (uint32_t)(q.a_bytes + kHeadOperand) * CG;
        for (int c0 = x.chunk0; c0 < x.chunk1; c0 += g.promote) {
            const int c1 = min(x.chunk1, c0 + g.promote);
            for (int term = 0; term < g.terms; ++term) {
                int pa, pb;
                head_term(g.terms, term, pa, pb);
                for (int c = c0; c < c1; ++c, ++it) {
                    const int stg = it % kHeadStages;
                    const uint32_t empty = smem_u32(&sh.empty[stg]), parity = (uint32_t)(((it / kHeadStages) & 1) ^ 1);
                    if (it >= kHeadStages && !(CG == 2 ? mbar_wait_pair(empty, parity, &sh.fail) : mbar_wait(empty, parity, &sh.fail))) { sh.fail = 1; return; }
                    const uint32_t sa = smem_u32(smem + stg * 2 * kHeadOperand), sb = sa + kHeadOperand;
                    const uint32_t own = smem_u32(&sh.full[stg]), full = CG == 2 ? of_leader(own) : own;
                    if (rank == 0) mbar_arrive_tx(own, bytes);
                    auto copy = [&](uint32_t dst, const CUtensorMap* tm, int u, int v, int w) {
                        if (CG == 2) tma_3d_pair(dst, tm, u, v, w, full); else tma_3d(dst, tm, u, v, w, full);
                    };
                    const int k = c * kHeadChunk;
                    if (q.a_mn) {
                        copy(sa, &q.a, m0, k, pa);
                        copy(sa + kHeadOperand / 2, &q.a, m0 + 64, k, pa);
                    } else {
                        copy(sa, &q.a, k, m0, pa);
                    }
                    if (q.b_mn) {
                        copy(sb, &q.b, n0, k, pb);
                        copy(sb + kHeadOperand / 2, &q.b, n0 + 64, k, pb);
                    } else {
                        copy(sb, &q.b, k, n0, pb);
                    }
                }
            }
        }
    }
}

// ------------------------------------------------------------------ products (one thread of a block or pair)
template <int CG>
__device__ void head_products(const HeadArgs& g, unsigned char* smem, HeadShared& sh) {
    int it = 0, at = 0, j;
    HeadTile x;
    constexpr int kCols = 128 * CG;
    for (int t = cluster_id(); head_tile(g, t, j, x); t += cluster_count()) {
        const HeadJob& q = g.job[j];
        const uint32_t type = g.half ? 0u : (1u << 7) | (1u << 10);
        const uint32_t idesc = (1u << 4) | type | ((uint32_t)q.a_mn << 15) | ((uint32_t)q.b_mn << 16) | ((uint32_t)(kCols >> 3) << 17) |
                               ((uint32_t)(128 * CG >> 4) << 24);
        const uint32_t step_a = q.a_mn ? 2048 : 32, step_b = q.b_mn ? 2048 : 32;
        const uint32_t lead_a = q.a_mn ? kHeadOperand / 2 : 16, lead_b = q.b_mn ? kHeadOperand / 2 : 16;
        for (int c0 = x.chunk0; c0 < x.chunk1; c0 += g.promote, ++at) {
            const int n = (min(x.chunk1, c0 + g.promote) - c0) * g.terms, buf = at & 1;
            if (at >= 2) {
                const uint32_t bar = smem_u32(&sh.acc_empty[buf]), parity = (uint32_t)(((at >> 1) & 1) ^ 1);
                if (!(CG == 2 ? mbar_wait_pair(bar, parity, &sh.fail) : mbar_wait(bar, parity, &sh.fail))) { sh.fail = 1; return; }
            }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t dcol = sh.tmem_base + (uint32_t)(buf * kCols);
            for (int k = 0; k < n; ++k, ++it) {
                const int stg = it % kHeadStages;
                const uint32_t full = smem_u32(&sh.full[stg]), parity = (uint32_t)((it / kHeadStages) & 1);
                if (!(CG == 2 ? mbar_wait_pair(full, parity, &sh.fail) : mbar_wait(full, parity, &sh.fail))) { sh.fail = 1; return; }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t sa = smem_u32(smem + stg * 2 * kHeadOperand), sb = sa + kHeadOperand;
#pragma unroll
                for (int u = 0; u < kHeadChunk / 16; ++u) {
                    const uint64_t da = tc_desc(sa + u * step_a, lead_a, 1024), db = tc_desc(sb + u * step_b, lead_b, 1024);
                    const uint32_t acc = k > 0 || u > 0;
                    if (CG == 2)
                        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
                                     ::"r"(dcol), "l"(da), "l"(db), "r"(idesc), "r"(acc) : "memory");
                    else
                        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                                     ::"r"(dcol), "l"(da), "l"(db), "r"(idesc), "r"(acc) : "memory");
                }
                auto commit = [&](uint64_t* bar) {
                    if (CG == 2)
                        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                                     ::"r"(smem_u32(bar)), "h"((unsigned short)3) : "memory");
                    else
                        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
                };
                commit(&sh.empty[stg]);
                if (k == n - 1) commit(&sh.acc_full[buf]);
            }
        }
    }
}

// ------------------------------------------------------------------ what becomes of a tile (eight warps of each block)
// Running statistics of one row's logits, in units of log 2 around a reference.
struct HeadStat {
    float ref, sum, elog;
    __device__ __forceinline__ void start() { ref = -INFINITY; sum = elog = 0.f; }
    __device__ __forceinline__ void add(float (&z)[32], float c) {
        float top = z[0];
#pragma unroll
        for (int u = 1; u < 32; ++u) top = fmaxf(top, z[u]);
        const float now = fmaxf(ref, top * c);               // c > 0
        const float base = now == -INFINITY ? 0.f : now;
        if (now > ref && ref != -INFINITY) {
            const float shift = ref - now, f = exp2_near(shift);
            elog = f * fmaf(shift, sum, elog);
            sum *= f;
        }
        ref = now;
        float s0 = 0.f, s1 = 0.f, l0 = 0.f, l1 = 0.f;
#pragma unroll
        for (int u = 0; u < 32; u += 2) {
            const float t0 = fmaf(z[u], c, -base), t1 = fmaf(z[u + 1], c, -base);
            const float e0 = exp2_near(t0), e1 = exp2_near(t1);
            s0 += e0; s1 += e1;
            // what cannot occur has no entropy, though its logarithm is infinite
            l0 = e0 != 0.f ? fmaf(e0, t0, l0) : l0;
            l1 = e1 != 0.f ? fmaf(e1, t1, l1) : l1;
        }
        sum += s0 + s1;
        elog += l0 + l1;
    }
};

template <int CG, int KIND>
struct HeadEpilogue {
    const HeadArgs& g;
    const HeadJob& q;
    const HeadTile& x;
    int row, col;                 // this thread's row of D, first column of its half
    HeadStat st;
    HeadRow hr;
    int tok;                      // column of the row's token, in the piece
    float unscale;

    __device__ __forceinline__ HeadEpilogue(const HeadArgs& g_, const HeadJob& q_, const HeadTile& x_, int rank, int warp, int lane)
        : g(g_), q(q_), x(x_) {
        row = x.m * 128 * CG + rank * 128 + (warp & 3) * 32 + lane;
        col = x.n * 128 * CG + (warp >> 2) * 64 * CG;
        if (KIND == kHeadStats) {
            st.start();
            tok = -1;
            if (row < q.rows && g.tokens) {
                const long long id = g.token_bytes == 8 ? ((const long long*)g.tokens)[row] : (long long)((const int*)g.tokens)[row];
                if (id >= g.col0 && id < (long long)g.col0 + q.cols) tok = (int)(id - g.col0);
            }
        }
        if (KIND == kHeadGrad && row < q.rows) {
            hr = g.coef[row];
            tok = g.row_token[row] - g.col0;
        }
        if (KIND == kHeadHidden) unscale = g.unscale ? *g.unscale : 1.f;
    }

    // 32 columns from `c0` on.
    __device__ __forceinline__ void take(float (&z)[32], int c0) {
        if (KIND == kHeadStats) {
            if (c0 + 32 > q.cols) {
#pragma unroll
                for (int u = 0; u < 32; ++u) z[u] = c0 + u < q.cols ? z[u] : -INFINITY;
            }
            if (tok >= c0 && tok < c0 + 32) {
                float v = 0.f;
#pragma unroll
                for (int u = 0; u < 32; ++u) v = tok == c0 + u ? z[u] : v;
                g.ztok[row] = v;
            }
            st.add(z, g.c);
        } else if (KIND == kHeadGrad) {
            if (row < q.rows && c0 < g.ldd) gradient(z, c0);
        } else if (q.kind == kHeadHidden) {
            hidden(z, c0);
        } else {
            weight(z, c0);
        }
    }

    __device__ __forceinline__ void gradient(float (&z)[32], int c0) {
        const bool token = tok >= c0 && tok < c0 + 32;
        float own = 0.f;
        if (token) {                                         // c0 has -a: the token's 1 - p without the cancellation
#pragma unroll
            for (int u = 0; u < 32; ++u) own = tok == c0 + u ? z[u] : own;
            const float t = fmaf(own, g.c, -hr.lse2), p = exp2_near(t);
            own = (p == 0.f ? 0.f : p * fmaf(hr.c1, t, hr.c0 + hr.a)) - hr.a * expm1f(t * 0.69314718055994531f);
        }
#pragma unroll
        for (int u = 0; u < 32; ++u) {
            const float t = fmaf(z[u], g.c, -hr.lse2), p = exp2_near(t);
            z[u] = p == 0.f ? 0.f : p * fmaf(hr.c1, t, hr.c0);
        }
        if (token) {
#pragma unroll
            for (int u = 0; u < 32; ++u) z[u] = tok == c0 + u ? own : z[u];
        }
        unsigned short* to = g.d + (long long)row * g.ldd + c0;
        for (int plane = 0;; ++plane) {
            unsigned w[16];
#pragma unroll
            for (int u = 0; u < 16; ++u)
                w[u] = g.half ? pack2(z[2 * u], z[2 * u + 1], __half()) : pack2(z[2 * u], z[2 * u + 1], __nv_bfloat16());
#pragma unroll
            for (int u = 0; u < 2; ++u)
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to + 16 * u), "r"(w[8 * u]), "r"(w[8 * u + 1]), "r"(w[8 * u + 2]),
                             "r"(w[8 * u + 3]), "r"(w[8 * u + 4]), "r"(w[8 * u + 5]), "r"(w[8 * u + 6]), "r"(w[8 * u + 7]) : "memory");
            if (g.terms == 1 || plane == kHeadPlanes - 1) break;
#pragma unroll
            for (int u = 0; u < 16; ++u) {                   // what the plane has left over; exact
                z[2 * u] -= __uint_as_float(w[u] << 16);
                z[2 * u + 1] -= __uint_as_float(w[u] & 0xffff0000u);
            }
            to += g.d_plane;
        }
    }

    __device__ __forceinline__ void hidden(float (&z)[32], int c0) {
        if (row >= q.rows || c0 >= g.ldp) return;
        float* to = g.plane + x.split * g.plane_size + (long long)row * g.ldp + c0;
#pragma unroll
        for (int u = 0; u < 32; u += 8) {
            if (c0 + u >= g.ldp) break;                      // ldp is a multiple of 8
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = z[u + k];
            if (g.add) {
                float old[8];
                load8_wide(old, to + u);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] += old[k];
            }
            store8_wide(to + u, v);
        }
    }

    template <typename T>
    __device__ __forceinline__ void weight_as(float (&z)[32], int c0) {
        T* to = (T*)g.out + (long long)row * g.ldo + c0;
        constexpr int kEach = 32 / (int)sizeof(T);           // 32 bytes
        if (g.wide && c0 + 32 <= q.cols) {
#pragma unroll
            for (int u = 0; u < 32; u += kEach) {
                if constexpr (sizeof(T) == 4) {
                    float v[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = z[u + k] * unscale;
                    if (g.accumulate) {
                        float old[8];
                        load8_wide(old, (const float*)to + u);
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] += old[k];
                    }
                    store8_wide((float*)to + u, v);
                } else {
#pragma unroll
                    for (int h = 0; h < kEach; h += 8) {
                        float v[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] = z[u + h + k] * unscale;
                        if (g.accumulate) {
                            float old[8];
                            load8(old, to + u + h);
#pragma unroll
                            for (int k = 0; k < 8; ++k) v[k] += old[k];
                        }
                        store8(to + u + h, v);
                    }
                }
            }
            return;
        }
#pragma unroll
        for (int u = 0; u < 32; ++u)
            if (c0 + u < q.cols) to[u] = from_f32<T>(g.accumulate ? fmaf(z[u], unscale, to_f32(to[u])) : z[u] * unscale);
    }
    __device__ __forceinline__ void weight(float (&z)[32], int c0) {
        if (row >= q.rows || c0 >= q.cols) return;
        if (g.out_type == 0) weight_as<float>(z, c0);
        else if (g.out_type == 1) weight_as<__nv_bfloat16>(z, c0);
        else weight_as<__half>(z, c0);
    }

    __device__ __forceinline__ void finish(int half) {
        if (KIND == kHeadStats && row < q.rows) {
            float* p = g.part + (long long)(g.part0 + 2 * x.n + half) * q.rows + row;
            const long long plane = (long long)g.parts * q.rows;
            p[0] = st.ref;
            p[plane] = st.sum;
            p[2 * plane] = st.elog;
        }
    }
};

template <int CG, int KIND, bool PROMOTE>
__device__ void head_epilogue(const HeadArgs& g, HeadShared& sh, int rank, int warp, int lane) {
    constexpr int kHalf = 64 * CG;                            // columns of a thread
    int at = 0, j;
    bool ok = true;
    HeadTile x;
    for (int t = cluster_id(); head_tile(g, t, j, x); t += cluster_count()) {
        const HeadJob& q = g.job[j];
        HeadEpilogue<CG, KIND> e(g, q, x, rank, warp, lane);
        float sum[PROMOTE ? kHalf : 1];
        for (int c0 = x.chunk0; c0 < x.chunk1; c0 += g.promote, ++at) {
            const int buf = at & 1;
            const uint32_t bar = smem_u32(&sh.acc_full[buf]), parity = (uint32_t)((at >> 1) & 1);
            if (ok) ok = __all_sync(0xffffffffu, CG == 2 ? mbar_wait_pair(bar, parity, &sh.fail) : mbar_wait(bar, parity, &sh.fail));
            if (!ok) sh.fail = 1;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t from = sh.tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(buf * 128 * CG + (warp >> 2) * kHalf);
#pragma unroll
            for (int u = 0; u < kHalf; u += 32) {
                uint32_t r[32];
                tmem_ld32(from + u, r);
                if (!ok) {
#pragma unroll
                    for (int k = 0; k < 32; ++k) r[k] = 0x7fffffffu;
                }
                if (PROMOTE) {
                    if (c0 == x.chunk0) {
#pragma unroll
                        for (int k = 0; k < 32; ++k) sum[u + k] = __uint_as_float(r[k]);
                    } else {
#pragma unroll
                        for (int k = 0; k < 32; ++k) sum[u + k] += __uint_as_float(r[k]);
                    }
                } else {
                    float z[32];
#pragma unroll
                    for (int k = 0; k < 32; ++k) z[k] = __uint_as_float(r[k]);
                    e.take(z, e.col + u);
                }
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                const uint32_t done = smem_u32(&sh.acc_empty[buf]);
                if (CG == 2) arrive_cluster(of_leader(done)); else mbar_arrive(done);
            }
        }
        if (PROMOTE) {
#pragma unroll
            for (int u = 0; u < kHalf; u += 32) {
                float z[32];
#pragma unroll
                for (int k = 0; k < 32; ++k) z[k] = sum[u + k];
                e.take(z, e.col + u);
            }
        }
        e.finish(warp >> 2);
    }
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
        for (int k = 0; k < kHeadStages; ++k) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_u32(&sh.full[k])) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_u32(&sh.empty[k])) : "memory");
        }
        for (int k = 0; k < 2; ++k) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_u32(&sh.acc_full[k])) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(&sh.acc_empty[k])), "r"(kHeadEpiWarps * CG) : "memory");
        }
        sh.fail = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (CG == 2) cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp < kHeadEpiWarps) head_epilogue<CG, KIND, PROMOTE>(g, sh, rank, warp, lane);
    else if (tid == 32 * kHeadEpiWarps) head_copies<CG>(g, smem, sh, rank);
    else if (tid == 32 * (kHeadEpiWarps + 1) && rank == 0) head_products<CG>(g, smem, sh);
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
// Planes of a matrix whose rows the bulk copies cannot take as they are: three bfloat16 planes of float32, or a copy of 16-bit
// rows at a stride of 16 bytes.  Columns behind dim are zero.  A value that bfloat16 has no finite number for stays in plane 0.
template <typename T>
__global__ void __launch_bounds__(256) head_pack_kernel(const T* x, long long rows, int dim, long long ld, unsigned short* out, int ldp, long long plane) {
    const int pairs = ldp / 2;
    const long long n = rows * pairs;
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < n; i += gridDim.x * 256LL) {
        const long long r = i / pairs;
        const int c = (int)(i - r * pairs) * 2;
        const T* p = x + r * ld + c;
        unsigned* to = (unsigned*)(out + r * ldp + c);
        if constexpr (sizeof(T) == 2) {
            const unsigned short* q = (const unsigned short*)p;
            *to = (c < dim ? (unsigned)q[0] : 0u) | (c + 1 < dim ? (unsigned)q[1] << 16 : 0u);
        } else {
            float a = c < dim ? to_f32(p[0]) : 0.f, b = c + 1 < dim ? to_f32(p[1]) : 0.f;
#pragma unroll
            for (int k = 0; k < kHeadPlanes; ++k) {
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

// Row values from the parts' statistics: kHeadRowThreads threads for `width` rows, the others share a row's parts.
constexpr int kHeadRowThreads = 512;
__global__ void __launch_bounds__(kHeadRowThreads) head_rows_kernel(const float* part, int parts, int rows, int width, const float* ztok, const void* tokens,
                                                                    int token_bytes, long long vocab, float c, float* logp, float* entropy, float* lse,
                                                                    int* status) {
    __shared__ float sm[3][kHeadRowThreads];
    const int tid = threadIdx.x, lane = tid % width, share = tid / width, shares = kHeadRowThreads / width;
    const int r = blockIdx.x * width + lane;
    float ref = -INFINITY, sum = 0.f, elog = 0.f;
    auto join = [&](float m, float s, float e) {
        if (s == 0.f) return;                                 // nothing that can occur; a NaN goes on
        const float now = fmaxf(ref, m);
        const float f = ref == -INFINITY ? 0.f : exp2f(ref - now), h = exp2f(m - now);
        elog = (f > 0.f ? f * fmaf(ref - now, sum, elog) : 0.f) + h * fmaf(m - now, s, e);
        sum = f * sum + h * s;
        ref = now;
    };
    if (r < rows) {
        const long long plane = (long long)parts * rows;
#pragma unroll 4
        for (int k = share; k < parts; k += shares) {
            const float* p = part + (long long)k * rows + r;
            join(p[0], p[plane], p[2 * plane]);
        }
    }
    sm[0][tid] = ref; sm[1][tid] = sum; sm[2][tid] = elog;
    for (int n = shares / 2; n; n /= 2) {
        __syncthreads();
        if (share < n) {
            const int o = tid + n * width;
            join(sm[0][o], sm[1][o], sm[2][o]);
            sm[0][tid] = ref; sm[1][tid] = sum; sm[2][tid] = elog;
        }
    }
    if (share != 0 || r >= rows) return;
    const double ln2 = 0.69314718055994530942, ls = log((double)sum);
    if (lse) lse[r] = sum == 0.f ? -INFINITY : (float)((double)ref * ln2 + ls);
    if (entropy) entropy[r] = sum == 0.f ? 0.f : (float)(ls - ln2 * (double)elog / (double)sum);
    if (logp) {
        const long long id = token_bytes == 8 ? token_id((const long long*)tokens, r, vocab, status) : token_id((const int*)tokens, r, vocab, status);
        // the token's logit against the reference as the sum has it, so that a sure token's value keeps its digits
        logp[r] = id < 0 ? (sum == sum ? 0.f : sum) : sum == 0.f ? -INFINITY : (float)(ln2 * ((double)ztok[r] * (double)c - (double)ref) - ls);
    }
}

// Coefficients of d for every row, and the power of two that brings the largest to `top`: one block.
__global__ void __launch_bounds__(1024) head_coef_kernel(int rows, long long vocab, const void* tokens, int token_bytes, double it, const float* lse,
                                                         const float* entropy, const float* g_logp, const float* g_entropy, const float* g_lse, float top,
                                                         HeadRow* coef, int* row_token, float* unscale, int* status) {
    __shared__ float most[32];
    const int tid = threadIdx.x;
    auto row = [&](int r, HeadRow& h) {
        long long id = -1;
        if (tokens) id = token_bytes == 8 ? token_id((const long long*)tokens, r, vocab, status) : token_id((const int*)tokens, r, vocab, status);
        const float z = lse[r];
        const bool none = z == -INFINITY;                     // no logit is finite: no gradient
        const float a = id >= 0 && g_logp && !none ? (float)(it * g_logp[r]) : 0.f;
        const float ge = g_entropy && !none ? (float)(it * g_entropy[r]) : 0.f;
        const float gz = g_lse && !none ? (float)(it * g_lse[r]) : 0.f;
        h.a = a;
        h.c0 = gz - a - (ge != 0.f ? ge * entropy[r] : 0.f);
        h.c1 = -ge * 0.69314718055994531f;
        h.lse2 = none ? INFINITY : (float)((double)z * 1.4426950408889634074);
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
    int e = 0;
    if (m > 0.f) frexpf(top / m, &e);                         // 2^(e - 1) <= top / m
    e = min(max(e - 1, -120), 120);
    const float f = ldexpf(1.f, e);
    for (int r = tid; r < rows; r += 1024) {
        coef[r].a *= f; coef[r].c0 *= f; coef[r].c1 *= f;
    }
    if (tid == 0) *unscale = ldexpf(1.f, -e);
}

// dhidden from the planes of partial sums, in the order of the planes.
template <typename T>
__global__ void __launch_bounds__(256) head_sum_kernel(const float* plane, long long plane_size, int planes, int ldp, int rows, int dim, const float* unscale,
                                                       T* out, long long ldo) {
    const int groups = ldp / 8;
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
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (c + u < dim) out[r * ldo + c + u] = from_f32<T>(s[u] * f);
    }
}

}  // namespace pb
