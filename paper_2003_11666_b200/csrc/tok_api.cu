// C entry points of the token operators and the AdamW step: argument checks and launches.
// Nothing here allocates, and no state is kept between calls.
#include <cmath>
#include <type_traits>

#include "adamw.cuh"
#include "tok_embed.cuh"
#include "tok_host.h"
#include "tok_logprob.cuh"

using namespace pb;

namespace {

// Sizes and scratch layout of the embedding gradient.
constexpr int64_t kMaxEmbedDim = 1 << 26, kMaxLogprobVocab = 1 << 30;
// Blocks per SM that the reduction's stretches are cut for.  Four are resident for 16-bit rows in pieces of four columns,
// three for float32 ones, two for rows that move column by column.  More and shorter stretches even out the tail:
// 65536 tokens of 2048 columns take 230 us at 4, 192 at 8, 189 at 16.
constexpr int kRedWave = 16;

struct EmbedPlan {
    SortPlan sort;
    RedPlan red;
    int slabs;
    size_t bytes;
};

EmbedPlan embed_plan(int64_t n, int64_t vocab, int64_t dim, char* scratch) {
    EmbedPlan e{};
    int len = 1;
    while (vocab >> len) ++len;                              // bits of the largest key, vocab itself
    SortPlan& s = e.sort;
    s.n = (int)n;
    s.passes = (len + kSortMaxBits - 1) / kSortMaxBits;
    s.bits = (len + s.passes - 1) / s.passes;
    s.tile_shift = 10;                                       // kSortSub tokens a block; longer lists: several sub-tiles
    static_assert(kSortSub == 1 << 10, "tokens of a block");
    while (((n - 1) >> s.tile_shift) >= kSortMaxTiles) ++s.tile_shift;
    s.tiles = n <= kSortSmall ? n > 0 : (int)(((n - 1) >> s.tile_shift) + 1);
    RedPlan& r = e.red;
    r.n = n; r.vocab = vocab; r.dim = dim;
    r.lanes = 1;
    while (r.lanes < kRedThreads && (int64_t)r.lanes * kRedCols < dim) r.lanes *= 2;
    e.slabs = (int)((dim + (int64_t)r.lanes * kRedCols - 1) / ((int64_t)r.lanes * kRedCols));
    // Stretches of 8 to 128 entries: about kRedWave blocks per SM if the list is long enough.  Rows that move column by
    // column keep to 16 at least, since a stretch's end costs them more (17892 tokens of 754 columns: 57 us with 16, 67
    // with 8; 2047 of 1000 columns in pieces: 24 and 21).
    const int per_block = kRedThreads / r.lanes;
    const int64_t want = (n * e.slabs / ((int64_t)kSms * kRedWave * per_block) + 7) / 8 * 8;
    const int most = kRedEntries / per_block < 128 ? kRedEntries / per_block : 128;
    const int least = dim % 4 && most >= 16 ? 16 : 8;
    r.len = (int)(want < least ? least : want > most ? most : want);
    r.stretches = (int)((n + r.len - 1) / r.len);
    r.red_blocks = (r.stretches + per_block - 1) / per_block;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char* p = scratch ? scratch + at : nullptr;
        at += (bytes + 255) / 256 * 256;
        return p;
    };
    for (int k = 0; k < 2; ++k) s.list[k] = (uint2*)take((size_t)n * 8);
    s.hist = (int*)take(s.tiles > 1 ? ((size_t)s.passes * s.tiles << s.bits) * 4 : 0);
    s.n_zero = (int)((int64_t)e.slabs * r.stretches * 3);
    s.zero = r.arrived = (unsigned*)take((size_t)s.n_zero * 4);
    r.part = (float*)take((size_t)r.stretches * 2 * dim * 4);
    r.list = s.list[(s.passes - 1) & 1];
    e.bytes = at > 256 ? at : 256;
    return e;
}

// One launch over as many tensors from `k` on as the table takes; moves k behind them.
template <int MAXT>
int adamw_launch(const pb_adamw_tensor* tensors, const void* const* grads, int n_tensors, int& k, const AdamScalars& q,
                 const pb_adamw_args& args, cudaStream_t stream) {
    static_assert(sizeof(AdamTable<MAXT>) <= 32764, "kernel parameters");
    AdamTable<MAXT> a;
    a.s = q;
    a.s.n = 0;
    const size_t gb = dtype_bytes(args.grad_dtype), fb = dtype_bytes(args.forward_dtype), sb = args.state_bits == 8 ? 1 : 4;
    int64_t rounds = 0;
    for (; k < n_tensors && a.s.n < MAXT; ++k) {
        const pb_adamw_tensor& t = tensors[k];
        if (t.n == 0) continue;
        const int64_t c = (t.n + kAdamRound - 1) / kAdamRound;
        if (rounds + c > kMaxCount) break;
        AdamTensor& d = a.t[a.s.n++];
        d.w = t.w; d.g = grads[k]; d.m = t.m; d.v = t.v; d.m_scale = t.m_scale; d.v_scale = t.v_scale; d.fwd = t.w_forward;
        d.n = t.n; d.decay = t.weight_decay; d.horizon = t.horizon;
        d.rnd = (unsigned long long)k * 0xA0761D6478BD642Full;
        d.first_round = (unsigned)rounds;
        d.vec = aligned(t.w, 32) && aligned(grads[k], 8 * gb) && aligned(t.m, 8 * sb) && aligned(t.v, 8 * sb) && aligned(t.w_forward, 8 * fb);
        rounds += c;
    }
    if (a.s.n == 0) return PB_OK;
    while (((rounds - 1) >> a.s.near_shift) >= kAdamNear) ++a.s.near_shift;
    for (int64_t j = 0, at = 0; j <= (rounds - 1) >> a.s.near_shift; ++j) {
        while (at + 1 < a.s.n && (int64_t)a.t[at + 1].first_round <= j << a.s.near_shift) ++at;
        a.s.near[j] = (unsigned short)at;
    }
    auto go = [&](auto bits, auto g) {
        cudaLaunchConfig_t c{};
        c.gridDim = dim3((unsigned)rounds);
        c.blockDim = dim3(kAdamThreads);
        c.stream = stream;
        void* table[] = {&a};                                // as it is: a launch by values would copy it on the way
        return cudaLaunchKernelExC(&c, (const void*)adamw_kernel<decltype(bits)::value, decltype(g), MAXT>, table);
    };
    auto by_bits = [&](auto g) { return args.state_bits == 8 ? go(std::integral_constant<int, 8>(), g) : go(std::integral_constant<int, 32>(), g); };
    return launched("pb_adamw_step", args.grad_dtype == PB_F32 ? by_bits(float()) : args.grad_dtype == PB_BF16 ? by_bits(__nv_bfloat16()) : by_bits(__half()));
}

}  // namespace

extern "C" {

int pb_embed_forward(const void* dev_table, int dtype, int64_t vocab, int64_t dim, int64_t ld_table, const void* dev_ids,
                     int id_bytes, int64_t n_tokens, float scale, void* dev_out, int64_t ld_out, int32_t* dev_status,
                     void* stream) {
    PB_REFUSE(!dtype_ok(dtype), "pb_embed_forward: unknown element type");
    PB_REFUSE(id_bytes != 4 && id_bytes != 8, "pb_embed_forward: token ids have 4 or 8 bytes");
    PB_REFUSE(n_tokens < 0 || n_tokens > kMaxCount, "pb_embed_forward: n_tokens out of range");
    PB_REFUSE(vocab < 1 || vocab > kMaxCount || dim < 1 || dim > kMaxCount, "pb_embed_forward: vocab and dim must be between 1 and 2^31 - 1");
    PB_REFUSE(ld_table < dim || ld_out < dim, "pb_embed_forward: a row stride is smaller than dim");
    if (n_tokens == 0) return PB_OK;
    PB_REFUSE(!dev_table || !dev_ids || !dev_out, "pb_embed_forward: NULL pointer");
    const size_t es = dtype_bytes(dtype);
    PB_REFUSE(!aligned(dev_table, es) || !aligned(dev_out, es) || !aligned(dev_ids, id_bytes) || !aligned(dev_status, 4),
              "pb_embed_forward: a pointer is not aligned to its element");
    PB_REFUSE(overlap(dev_out, extent(n_tokens, dim, ld_out, es), dev_table, extent(vocab, dim, ld_table, es)),
              "pb_embed_forward: the output overlaps the table");
    PB_REFUSE(overlap(dev_out, extent(n_tokens, dim, ld_out, es), dev_ids, (size_t)n_tokens * id_bytes),
              "pb_embed_forward: the output overlaps the ids");
    const cudaStream_t s = (cudaStream_t)stream;
    const int64_t piece = 16 / (int64_t)es;
    const bool vec = dim % piece == 0 && ld_table % piece == 0 && ld_out % piece == 0 && aligned(dev_table, 16) && aligned(dev_out, 16);
    const int64_t pieces = vec ? dim / piece : dim;
    int lanes = 1;
    while (lanes < 256 && lanes < pieces) lanes *= 2;
    // Four tokens per group once that still gives every SM eight blocks; a few long rows are spread over blocks.
    const int64_t groups = 256 / lanes;
    const bool many = n_tokens >= (int64_t)kSms * 8 * 4 * groups;
    const int64_t blocks = (n_tokens + (many ? 4 : 1) * groups - 1) / ((many ? 4 : 1) * groups);
    const int64_t walks = (pieces + lanes - 1) / lanes;
    const int64_t spread = many ? 1 : walks < 16 ? walks : 16;
    auto go = [&](auto t, auto i) {
        using T = decltype(t);
        using I = decltype(i);
        auto kernel = vec ? (many ? embed_fwd_kernel<T, I, true, 4> : embed_fwd_kernel<T, I, true, 1>)
                          : (many ? embed_fwd_kernel<T, I, false, 4> : embed_fwd_kernel<T, I, false, 1>);
        return launch(kernel, dim3((unsigned)blocks, (unsigned)spread), 256, s, (const T*)dev_table, vocab, dim, ld_table, (const I*)dev_ids, n_tokens,
                      scale, (T*)dev_out, ld_out, lanes, dev_status);
    };
    auto by_id = [&](auto t) { return id_bytes == 4 ? go(t, int32_t()) : go(t, int64_t()); };
    return launched("pb_embed_forward", dtype == PB_F32 ? by_id(float()) : dtype == PB_BF16 ? by_id(__nv_bfloat16()) : by_id(__half()));
}

size_t pb_embed_scratch_bytes(int64_t n_tokens, int64_t vocab, int64_t dim) {
    if (n_tokens < 0 || n_tokens > kMaxCount || vocab < 1 || vocab > kMaxCount || dim < 1 || dim > kMaxEmbedDim) return 0;
    return embed_plan(n_tokens, vocab, dim, nullptr).bytes;
}

int pb_embed_backward(const void* dev_dout, int dtype, int64_t ld_dout, const void* dev_ids, int id_bytes, int64_t n_tokens,
                      int64_t vocab, int64_t dim, float scale, int64_t padding_idx, void* dev_dtable, int dtable_dtype,
                      int64_t ld_dtable, int accumulate, void* dev_scratch, size_t scratch_bytes, int32_t* dev_status,
                      void* stream) {
    PB_REFUSE(!dtype_ok(dtype) || !dtype_ok(dtable_dtype), "pb_embed_backward: unknown element type");
    PB_REFUSE(dtable_dtype != PB_F32 && dtable_dtype != dtype, "pb_embed_backward: the table's gradient is float32 or of dout's type");
    PB_REFUSE(id_bytes != 4 && id_bytes != 8, "pb_embed_backward: token ids have 4 or 8 bytes");
    PB_REFUSE(n_tokens < 0 || n_tokens > kMaxCount, "pb_embed_backward: n_tokens out of range");
    PB_REFUSE(vocab < 1 || vocab > kMaxCount, "pb_embed_backward: vocab must be between 1 and 2^31 - 1");
    PB_REFUSE(dim < 1 || dim > kMaxEmbedDim, "pb_embed_backward: dim must be between 1 and 2^26");
    PB_REFUSE(ld_dtable < dim || ld_dout < dim, "pb_embed_backward: a row stride is smaller than dim");
    PB_REFUSE(padding_idx < -1 || padding_idx >= vocab, "pb_embed_backward: padding_idx must be -1 or a row of the table");
    PB_REFUSE(accumulate != 0 && accumulate != 1, "pb_embed_backward: accumulate must be 0 or 1");
    if (n_tokens == 0 && accumulate) return PB_OK;
    PB_REFUSE(!dev_dtable, "pb_embed_backward: NULL pointer");
    PB_REFUSE(n_tokens > 0 && (!dev_dout || !dev_ids || !dev_scratch), "pb_embed_backward: NULL pointer");
    PB_REFUSE(n_tokens > 0 && scratch_bytes < pb_embed_scratch_bytes(n_tokens, vocab, dim), "pb_embed_backward: scratch is smaller than pb_embed_scratch_bytes");
    const size_t es = dtype_bytes(dtype), gs = dtype_bytes(dtable_dtype);
    PB_REFUSE(!aligned(dev_dtable, gs) || !aligned(dev_dout, es) || !aligned(dev_ids, id_bytes) || !aligned(dev_status, 4),
              "pb_embed_backward: a pointer is not aligned to its element");
    PB_REFUSE(n_tokens > 0 && !aligned(dev_scratch, 256), "pb_embed_backward: scratch must be 256-byte aligned");
    const size_t n_dt = extent(vocab, dim, ld_dtable, gs), n_do = extent(n_tokens, dim, ld_dout, es);
    // The ids are read several times and have to be the same each time: their places in the sorted list follow from them.
    const size_t n_id = (size_t)n_tokens * id_bytes, n_st = dev_status ? sizeof(int32_t) : 0;
    PB_REFUSE(overlap(dev_dtable, n_dt, dev_dout, n_do) || overlap(dev_scratch, scratch_bytes, dev_dtable, n_dt) ||
              overlap(dev_scratch, scratch_bytes, dev_dout, n_do) || overlap(dev_ids, n_id, dev_scratch, scratch_bytes) ||
              overlap(dev_ids, n_id, dev_dtable, n_dt) || overlap(dev_status, n_st, dev_scratch, scratch_bytes) ||
              overlap(dev_status, n_st, dev_ids, n_id), "pb_embed_backward: buffers overlap");
    const cudaStream_t s = (cudaStream_t)stream;
    EmbedPlan e = embed_plan(n_tokens, vocab, dim, (char*)dev_scratch);
    e.red.ld_dout = ld_dout; e.red.ld = ld_dtable; e.red.scale = scale; e.red.accumulate = accumulate;
    // columns move in pieces of four where every row starts on a piece
    const bool vec = dim % 4 == 0 && aligned(dev_dout, 4 * es) && aligned(dev_dtable, 4 * gs) && ld_dout % 4 == 0 && ld_dtable % 4 == 0;
    auto go = [&](auto t, auto g, auto i) {
        using T = decltype(t);
        using G = decltype(g);
        using I = decltype(i);
        const SortIds<I> in{(const I*)dev_ids, vocab, padding_idx, dev_status};
        cudaError_t err = cudaSuccess;
        if (n_tokens) {
            // One block up to 2048 tokens; else a launch for the first counts and one for each digit (65536 tokens: some
            // 28 us, with 64 blocks of 1024 tokens as with 32 of 2048; a single launch of a 16-block cluster took 40).
            err = launch(embed_sort_kernel<I>, dim3(e.sort.tiles), kSortThreads, s, e.sort, in);
            for (int p = 0; e.sort.tiles > 1 && p < e.sort.passes && err == cudaSuccess; ++p)
                err = launch_after(embed_scatter_kernel<I>, dim3(e.sort.tiles), kSortThreads, s, e.sort, in, p);
        }
        // A list that one block sorts leaves the GPU to the clearing, which goes by the ids then.
        if (e.sort.tiles == 1) {
            e.red.ids = dev_ids;
            e.red.id_bytes = id_bytes;
            e.red.padding = padding_idx < 0 ? -2 : padding_idx;
        }
        // Some 64 KB of the table per block: 2047 ids and 50021 rows of 4 KB take 39.7 us, 41.6 with 128 KB (a longer
        // tail), 45 with 32 KB (more looking through the ids).
        const int64_t rows = (int64_t)65536 / ((int64_t)gs * dim);
        e.red.clear_rows = (int)(rows < 4 ? 4 : rows > kZeroRows ? kZeroRows : rows);
        const int64_t blocks = e.red.red_blocks + (accumulate ? 0 : (vocab + e.red.clear_rows - 1) / e.red.clear_rows);
        const dim3 grid((unsigned)blocks, (unsigned)e.slabs);
        const T* x = (const T*)dev_dout;
        G* d = (G*)dev_dtable;
        if (err == cudaSuccess) err = vec ? launch_after(embed_reduce_kernel<true, T, G>, grid, kRedThreads, s, e.red, x, d)
                                          : launch_after(embed_reduce_kernel<false, T, G>, grid, kRedThreads, s, e.red, x, d);
        return err;
    };
    auto by_id = [&](auto t, auto g) { return id_bytes == 4 ? go(t, g, int32_t()) : go(t, g, int64_t()); };
    auto by_g = [&](auto t) { return dtable_dtype == PB_F32 ? by_id(t, float()) : by_id(t, t); };
    return launched("pb_embed_backward", dtype == PB_F32 ? by_id(float(), float()) : dtype == PB_BF16 ? by_g(__nv_bfloat16()) : by_g(__half()));
}

int pb_logprob_forward(const void* dev_logits, int dtype, int64_t rows, int64_t vocab, int64_t ld, const void* dev_tokens,
                       int token_bytes, double inv_temperature, float* dev_logp, float* dev_entropy, float* dev_lse, int top_k,
                       float* dev_top_logp, int32_t* dev_top_ids, int32_t* dev_status, void* stream) {
    PB_REFUSE(!dtype_ok(dtype), "pb_logprob_forward: unknown element type");
    PB_REFUSE(rows < 0 || rows > kMaxCount, "pb_logprob_forward: rows out of range");
    PB_REFUSE(vocab < 1 || vocab > kMaxLogprobVocab, "pb_logprob_forward: vocab must be between 1 and 2^30");
    PB_REFUSE(ld < vocab, "pb_logprob_forward: the row stride is smaller than vocab");
    PB_REFUSE(!(inv_temperature > 0.0) || !std::isfinite((float)inv_temperature) || (float)inv_temperature == 0.f, "pb_logprob_forward: inv_temperature must be positive and finite");
    PB_REFUSE(top_k < 0 || top_k > kMaxTop, "pb_logprob_forward: top_k must be between 0 and 32");
    PB_REFUSE(top_k > vocab, "pb_logprob_forward: top_k is larger than vocab");
    PB_REFUSE((dev_logp != nullptr) != (dev_tokens != nullptr) && rows > 0, "pb_logprob_forward: logp and tokens go together");
    PB_REFUSE(dev_tokens && token_bytes != 4 && token_bytes != 8, "pb_logprob_forward: tokens have 4 or 8 bytes");
    if (rows == 0) return PB_OK;
    PB_REFUSE(!dev_logits || (top_k > 0 && (!dev_top_logp || !dev_top_ids)), "pb_logprob_forward: NULL pointer");
    PB_REFUSE(!aligned(dev_logits, dtype_bytes(dtype)) || (dev_tokens && !aligned(dev_tokens, token_bytes)) || !aligned(dev_logp, 4) ||
              !aligned(dev_entropy, 4) || !aligned(dev_lse, 4) || !aligned(dev_top_logp, 4) || !aligned(dev_top_ids, 4) ||
              !aligned(dev_status, 4), "pb_logprob_forward: a pointer is not aligned to its element");
    const cudaStream_t s = (cudaStream_t)stream;
    // A few rows are split over clusters as long as all blocks are resident at once (four per SM) and every warp
    // of a block still has a piece.
    const int64_t pieces = vocab / (2048 / (int64_t)dtype_bytes(dtype));
    int parts = 1;
    while (parts < kMaxCluster && rows * parts * 2 <= kSms * 4 && pieces >= (int64_t)parts * kFwdWarps) parts *= 2;
    const bool few = parts == 1 && pieces < kMaxFewSegments && rows > kSms * 4;       // short rows: two warps each
    int per_segment = 1;
    while (pieces / per_segment + 1 > kMaxSegments) per_segment *= 2;
    auto go = [&](auto t, auto i) {
        using T = decltype(t);
        using I = decltype(i);
        const T* x = (const T*)dev_logits;
        const I* tok = (const I*)dev_tokens;
        if (parts > 1)
            return launch_cluster(logprob_fwd_kernel<T, I, kFwdWarps, true>, parts, rows * parts, kFwdWarps * 32, s, x, (int)vocab, (long long)ld, tok,
                                  inv_temperature, dev_logp, dev_entropy, dev_lse, top_k, dev_top_logp, dev_top_ids, per_segment, dev_status);
        auto kernel = few ? logprob_fwd_kernel<T, I, kFwdFewWarps, false> : logprob_fwd_kernel<T, I, kFwdWarps, false>;
        return launch(kernel, dim3((unsigned)rows), (few ? kFwdFewWarps : kFwdWarps) * 32, s, x, (int)vocab, (long long)ld, tok, inv_temperature, dev_logp,
                      dev_entropy, dev_lse, top_k, dev_top_logp, dev_top_ids, per_segment, dev_status);
    };
    auto by_id = [&](auto t) { return token_bytes == 8 ? go(t, int64_t()) : go(t, int32_t()); };
    return launched("pb_logprob_forward", dtype == PB_F32 ? by_id(float()) : dtype == PB_BF16 ? by_id(__nv_bfloat16()) : by_id(__half()));
}

int pb_logprob_backward(const void* dev_logits, int dtype, int64_t rows, int64_t vocab, int64_t ld, const void* dev_tokens,
                        int token_bytes, double inv_temperature, const float* dev_lse, const float* dev_entropy,
                        const float* dev_g_logp, const float* dev_g_entropy, const float* dev_g_lse, void* dev_dlogits,
                        int64_t ld_d, int32_t* dev_status, void* stream) {
    PB_REFUSE(!dtype_ok(dtype), "pb_logprob_backward: unknown element type");
    PB_REFUSE(rows < 0 || rows > kMaxCount, "pb_logprob_backward: rows out of range");
    PB_REFUSE(vocab < 1 || vocab > kMaxLogprobVocab, "pb_logprob_backward: vocab must be between 1 and 2^30");
    PB_REFUSE(ld < vocab || ld_d < vocab, "pb_logprob_backward: a row stride is smaller than vocab");
    PB_REFUSE(!(inv_temperature > 0.0) || !std::isfinite((float)inv_temperature) || (float)inv_temperature == 0.f, "pb_logprob_backward: inv_temperature must be positive and finite");
    if (rows == 0) return PB_OK;
    PB_REFUSE(!dev_logits || !dev_dlogits || !dev_lse, "pb_logprob_backward: NULL pointer");
    PB_REFUSE(dev_g_logp && !dev_tokens, "pb_logprob_backward: a gradient of logp needs the tokens");
    PB_REFUSE(dev_g_entropy && !dev_entropy, "pb_logprob_backward: a gradient of the entropy needs the entropy");
    PB_REFUSE(dev_tokens && token_bytes != 4 && token_bytes != 8, "pb_logprob_backward: tokens have 4 or 8 bytes");
    const size_t es = dtype_bytes(dtype);
    PB_REFUSE(!aligned(dev_logits, es) || !aligned(dev_dlogits, es) || (dev_tokens && !aligned(dev_tokens, token_bytes)) || !aligned(dev_lse, 4) ||
              !aligned(dev_entropy, 4) || !aligned(dev_g_logp, 4) || !aligned(dev_g_entropy, 4) || !aligned(dev_g_lse, 4) || !aligned(dev_status, 4),
              "pb_logprob_backward: a pointer is not aligned to its element");
    PB_REFUSE(!(dev_logits == dev_dlogits && ld == ld_d) &&
              overlap(dev_logits, extent(rows, vocab, ld, es), dev_dlogits, extent(rows, vocab, ld_d, es)),
              "pb_logprob_backward: dlogits overlaps logits (the very same buffer and stride is allowed)");
    const cudaStream_t s = (cudaStream_t)stream;
    const int64_t per_launch = 65535;                       // rows are the grid's second dimension
    for (int64_t r0 = 0; r0 < rows; r0 += per_launch) {
        const unsigned nr = (unsigned)(rows - r0 < per_launch ? rows - r0 : per_launch);
        auto go = [&](auto t, auto i) {
            using T = decltype(t);
            using I = decltype(i);
            auto at = [&](const float* p) { return p ? p + r0 : nullptr; };
            const unsigned gx = (unsigned)((vocab + kBwdTile<T> - 1) / kBwdTile<T>);
            return launch(logprob_bwd_kernel<T, I>, dim3(gx, nr), kBwdThreads, s, (const T*)dev_logits + r0 * ld, vocab, ld,
                          dev_tokens ? (const I*)dev_tokens + r0 : nullptr, inv_temperature, at(dev_lse), at(dev_entropy), at(dev_g_logp), at(dev_g_entropy),
                          at(dev_g_lse), (T*)dev_dlogits + r0 * ld_d, ld_d, dev_status);
        };
        auto by_id = [&](auto t) { return token_bytes == 8 ? go(t, int64_t()) : go(t, int32_t()); };
        const int rc = launched("pb_logprob_backward", dtype == PB_F32 ? by_id(float()) : dtype == PB_BF16 ? by_id(__nv_bfloat16()) : by_id(__half()));
        if (rc != PB_OK) return rc;
    }
    return PB_OK;
}

int pb_adamw_step(const pb_adamw_tensor* tensors, const void* const* dev_grads, int n_tensors, const pb_adamw_args* args, void* stream) {
    PB_REFUSE(n_tensors < 0, "pb_adamw_step: negative tensor count");
    PB_REFUSE(!args, "pb_adamw_step: NULL pointer");
    PB_REFUSE(args->state_bits != 32 && args->state_bits != 8, "pb_adamw_step: states have 32 or 8 bits");
    PB_REFUSE(!dtype_ok(args->grad_dtype) || !dtype_ok(args->forward_dtype), "pb_adamw_step: unknown element type");
    PB_REFUSE(!(args->beta1 >= 0.0 && args->beta1 < 1.0) || !(args->beta2 >= 0.0 && args->beta2 < 1.0), "pb_adamw_step: need 0 <= beta1, beta2 < 1");
    PB_REFUSE(!(args->lr >= 0.0) || !std::isfinite(args->lr) || !(args->eps >= 0.0) || !std::isfinite(args->eps), "pb_adamw_step: lr and eps must not be negative");
    PB_REFUSE(args->step < 1 && !args->dev_step, "pb_adamw_step: the first step has number 1");
    PB_REFUSE(!aligned(args->dev_grad_scale, 4) || !aligned(args->dev_lr, 4) || !aligned(args->dev_step, 8), "pb_adamw_step: a pointer is not aligned to its element");
    if (n_tensors == 0) return PB_OK;
    PB_REFUSE(!tensors || !dev_grads, "pb_adamw_step: NULL pointer");
    const size_t gb = dtype_bytes(args->grad_dtype), fb = dtype_bytes(args->forward_dtype), sb = args->state_bits == 8 ? 1 : 4;
    for (int k = 0; k < n_tensors; ++k) {
        const pb_adamw_tensor& t = tensors[k];
        PB_REFUSE(t.n < 0, "pb_adamw_step: negative tensor size");
        PB_REFUSE(t.n > (int64_t)kMaxCount * kAdamRound / 2, "pb_adamw_step: a tensor is too large");
        PB_REFUSE(!(t.weight_decay >= 0.f) || !std::isfinite(t.weight_decay) || !std::isfinite(t.horizon), "pb_adamw_step: weight_decay must not be negative, horizon must be finite");
        if (t.n == 0) continue;
        PB_REFUSE(!t.w || !t.m || !t.v || !dev_grads[k], "pb_adamw_step: NULL pointer");
        PB_REFUSE(args->state_bits == 8 && (!t.m_scale || !t.v_scale), "pb_adamw_step: an 8-bit state needs its scales");
        PB_REFUSE(!aligned(t.w, 4) || !aligned(dev_grads[k], gb) || !aligned(t.m, sb) || !aligned(t.v, sb) || !aligned(t.m_scale, 4) ||
                  !aligned(t.v_scale, 4) || !aligned(t.w_forward, fb), "pb_adamw_step: a pointer is not aligned to its element");
    }
    AdamScalars q{};
    q.lr = args->lr; q.beta1 = args->beta1; q.beta2 = args->beta2;
    q.b1 = (float)args->beta1; q.o1 = (float)(1.0 - args->beta1); q.b2 = (float)args->beta2; q.o2 = (float)(1.0 - args->beta2);
    q.eps = (float)args->eps;
    q.minus_zero = -0.f;
    q.c1 = (float)(1.0 / (1.0 - std::pow(args->beta1, (double)args->step)));
    q.c2 = (float)(1.0 / std::sqrt(1.0 - std::pow(args->beta2, (double)args->step)));
    q.step = args->step; q.seed = args->seed;
    q.grad_scale = args->dev_grad_scale; q.dev_lr = args->dev_lr; q.dev_step = (const long long*)args->dev_step;
    q.fwd_dtype = args->forward_dtype;
    // Roots below 2^-63, corrected by 1 / sqrt(1 - beta2) at most, are less than 2^-25 of an eps from here on.
    q.subnormal = args->eps < 0x1p-38 / std::sqrt(1.0 - args->beta2);
    auto by_size = [&](auto few) {
        for (int k = 0; k < n_tensors;) {
            const int rc = adamw_launch<decltype(few)::value>(tensors, dev_grads, n_tensors, k, q, *args, (cudaStream_t)stream);
            if (rc != PB_OK) return rc;
        }
        return (int)PB_OK;
    };
    return n_tensors <= kAdamFewTensors ? by_size(std::integral_constant<int, kAdamFewTensors>()) : by_size(std::integral_constant<int, kAdamManyTensors>());
}

int pb_adamw_moments(const void* dev_m, const float* dev_m_scale, const void* dev_v, const float* dev_v_scale, int64_t n,
                     float* dev_m_out, float* dev_v_out, void* stream) {
    PB_REFUSE(n < 0 || n > (int64_t)kMaxCount * 256, "pb_adamw_moments: size out of range");
    if (n == 0) return PB_OK;
    PB_REFUSE(!dev_m_out && !dev_v_out, "pb_adamw_moments: NULL pointer");
    PB_REFUSE((dev_m_out && (!dev_m || !dev_m_scale)) || (dev_v_out && (!dev_v || !dev_v_scale)), "pb_adamw_moments: NULL pointer");
    PB_REFUSE(!aligned(dev_m_scale, 4) || !aligned(dev_v_scale, 4) || !aligned(dev_m_out, 4) || !aligned(dev_v_out, 4),
              "pb_adamw_moments: a pointer is not aligned to its element");
    const bool vec = aligned(dev_m, 8) && aligned(dev_v, 8) && aligned(dev_m_out, 32) && aligned(dev_v_out, 32);
    return launched("pb_adamw_moments", launch(adamw_moments_kernel, dim3((unsigned)((n + kAdamRound - 1) / kAdamRound)), kAdamThreads, (cudaStream_t)stream,
                                               (const unsigned char*)dev_m, dev_m_scale, (const unsigned char*)dev_v, dev_v_scale, n, dev_m_out, dev_v_out, vec));
}

}  // extern "C"
