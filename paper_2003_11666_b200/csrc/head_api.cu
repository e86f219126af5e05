// C entry points of the log probabilities of hidden states under an output head: argument checks, plan, launches.
// Nothing here allocates, and no state is kept between calls.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "tok_head.cuh"
#include "tok_host.h"

namespace pb {
// pb_api.cu: map of a matrix of 16-bit (or float32) elements, innermost dimension first, strides in bytes.
bool tensor_map(CUtensorMap* map, const void* base, int rank, const unsigned long long* dims, const unsigned long long* strides, const unsigned* box,
                bool ahead, bool f32);
}

using namespace pb;

namespace {

constexpr int64_t kMaxHeadRows = 1 << 24, kMaxHeadVocab = 1 << 24, kMaxHeadDim = 1 << 20;
constexpr int64_t kHeadFewRows = 128;           // rows that one block's tile holds; more run in pairs of blocks
// Forwards that read the weights without the tensor cores, where their rows start on 16 bytes.  us among others, that way / by the tensor cores:
// bf16, 131072 tokens, 1 row: 23.8 / 18.9 (64 columns), 23.9 / 24.7 (256), 43.9 / 58.6 (1024), 80.2 / 95.5 (2048); 2 rows: 29.2 / 23.7 (256),
// 49.3 / 54.8 (1024), 86.7 / 96.6 (2048); 3 and 4 rows: 78 / 55 (1024).  f32, 131072 tokens, 1 row: 24 / 91 (64), 164 / 656 (2048); 4 rows: 40 / 93, 219 / 658;
// 1000 tokens, 1 row: 5.6 / 12.7 (64), 8.5 / 38.9 (2048).  Beside the time, these sums round to nearest (2e-8 of a logsumexp; 2e-6 there).
constexpr int64_t kHeadFewFloat = 4, kHeadFewHalf = 2, kHeadFewDim = 256;      // 16-bit rows: as many as dim has of kHeadFewDim
constexpr int64_t kHeadPieceBytes = 256 << 20;  // of d, or of packed weights, held at a time
constexpr int64_t kHeadPieceMin = 8192;         // tokens of a piece at least: dhidden's partial sums are read and written once for each
constexpr int64_t kHeadStatRows = 8192;         // rows whose statistics are held at a time
// Chunks of K that the tensor core adds up by itself.  It does not round to nearest, so its sums drift towards zero, with every step that it adds at full
// size (four of a chunk; of float32 operands twelve or 24): log probabilities of normal logits are off by 6e-8 of themselves after 16 steps, 2e-7 after 64, 8e-7
// after 256, 1.7e-6 after 512.
// float32 operands: 24 steps (three terms) for logits and dhidden, 48 (six terms) for dweight, whose errors are those of d.  With 24 or 12 for the logits the
// forward of 509 x 50021 x 1001 takes 9 or 34 % longer than with 48, and logits whose terms have one sign are off by 6e-7 or 3e-7 of themselves instead of 1.3e-6.  With 48 the
// gradients at low temperatures were several times as far off as those of float32 products; with 24 they are about as far.
constexpr int kHeadPromoteNear = 2, kHeadPromoteWide = 2;
constexpr int kHeadPromoteLong = 16;            // 16-bit ones of more than kHeadLong chunks in the forward: 4096 x 131072 x 4096 takes 3.50 ms, as it
constexpr int kHeadLong = 16;                   // does without
constexpr int kHeadNever = 1 << 28;
constexpr int kHeadTileCost = 2;                // what a tile costs beside its chunks, in chunks

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

struct HeadPlan {
    int cg;
    bool f32, packed;            // packed: 16-bit operands are copied
    bool few;                    // a forward without the tensor cores
    int64_t dp;                  // row stride of packed operands
    int64_t piece, pieces;       // tokens of a piece of the vocabulary
    int64_t stat_rows, parts;
    int64_t ldd, ldp;
    int splits;
    int64_t split_chunks;
    // scratch; `near` and `wide`: float16 and bfloat16 planes of float32 operands
    unsigned short *hidden, *hidden_wide, *weight, *d, *d_wide;
    float *part, *ztok, *plane, *unscale, *row_scale, *col_scale, *d_scale;
    int* col_most;               // of each piece
    HeadRow* coef;
    int* row_token;
    size_t bytes;
};

HeadPlan head_plan(int dtype, int64_t rows, int64_t vocab, int64_t dim, bool direct, bool backward, char* scratch) {
    HeadPlan e{};
    e.cg = rows <= kHeadFewRows ? 1 : 2;
    e.f32 = dtype == PB_F32;
    e.packed = !e.f32 && !direct;
    e.few = !backward && direct && rows <= (e.f32 ? kHeadFewFloat : std::min(kHeadFewHalf, dim / kHeadFewDim));
    e.dp = up(dim, 8);
    if (e.few) {
        const int64_t groups = (vocab + kHeadFewCols - 1) / kHeadFewCols;
        e.stat_rows = rows;
        e.parts = std::min<int64_t>(groups, kSms * kHeadFewBlocks);
        e.part = (float*)scratch;
        e.ztok = e.part + 3 * e.parts * rows;
        e.bytes = (size_t)((3 * e.parts + 1) * rows * 4);
        if (e.f32) e.bytes = std::max(e.bytes, head_plan(dtype, rows, vocab, dim, false, false, nullptr).bytes);      // a size for any rows
        return e;
    }
    const int64_t tile = 128 * e.cg, operand = e.f32 ? kHeadNear : 1, planes = e.f32 ? kHeadNear + kHeadWide : 1;
    int64_t most = vocab;
    if (e.f32 || e.packed) most = std::min(most, kHeadPieceBytes / (operand * e.dp * 2));
    if (backward) most = std::min(most, kHeadPieceBytes / (planes * rows * 2));
    e.piece = most >= vocab ? vocab : std::min(vocab, up(std::max(most, kHeadPieceMin), 256));
    e.pieces = (vocab + e.piece - 1) / e.piece;
    if (e.pieces > 1) e.piece = up((vocab + e.pieces - 1) / e.pieces, 256);    // of one size, but for the last
    e.pieces = (vocab + e.piece - 1) / e.piece;
    size_t at = 0;
    auto take = [&](int64_t bytes) {
        char* p = scratch ? scratch + at : nullptr;
        at += (size_t)up(bytes, 256);
        return p;
    };
    if (e.f32 || e.packed) {
        e.hidden = (unsigned short*)take(operand * rows * e.dp * 2);
        e.weight = (unsigned short*)take(operand * e.piece * e.dp * 2);
    }
    if (e.f32) {
        e.row_scale = (float*)take(rows * 4);
        e.col_scale = (float*)take((e.piece + kHeadGroup - 1) / kHeadGroup * 4);
    }
    if (!backward) {
        e.stat_rows = std::min(rows, kHeadStatRows);
        for (int64_t v = 0; v < vocab; v += e.piece) e.parts += (std::min(e.piece, vocab - v) + tile - 1) / tile;
        e.part = (float*)take(3 * e.parts * e.stat_rows * 4);
        e.ztok = (float*)take(e.stat_rows * 4);
    } else {
        e.ldd = up(e.piece, 64);
        e.ldp = up(dim, 8);
        e.d = (unsigned short*)take(operand * rows * e.ldd * 2);
        if (e.f32) {
            e.d_wide = (unsigned short*)take(kHeadWide * rows * e.ldd * 2);
            e.hidden_wide = (unsigned short*)take(kHeadWide * rows * e.dp * 2);
            e.d_scale = (float*)take(rows * 4);
            e.col_most = (int*)take(e.pieces * 4);
        }
        // Enough splits of K for every block where dhidden has few tiles, but no shorter than 16 chunks.
        const int64_t tiles = ((rows + tile - 1) / tile) * ((dim + tile - 1) / tile), chunks = (e.piece + kHeadChunk - 1) / kHeadChunk;
        const int64_t splits = std::max<int64_t>(1, std::min((kSms / e.cg) / tiles, chunks / 16));
        e.split_chunks = (chunks + splits - 1) / splits;
        e.splits = (int)((chunks + e.split_chunks - 1) / e.split_chunks);
        e.plane = (float*)take(e.splits * rows * e.ldp * 4);
        e.coef = (HeadRow*)take(rows * (int64_t)sizeof(HeadRow));
        e.row_token = (int*)take(rows * 4);
        e.unscale = (float*)take(4);
    }
    e.bytes = at;
    return e;
}

// Scratch for `rows` rows or fewer.  Fewer can need more: one or two rows have a kernel with parts of its own, up to 128 rows tiles of half the size and more splits,
// and the pieces of the vocabulary grow as the rows become fewer.
size_t head_bytes(int dtype, int64_t rows, int64_t vocab, int64_t dim, bool direct, bool backward) {
    const bool f32 = dtype == PB_F32;
    if (!backward) {
        size_t most = 0;
        for (int64_t r : {rows, std::min(rows, kHeadFewRows), std::min(rows, kHeadFewFloat), std::min(rows, kHeadFewHalf), int64_t(1)})
            for (bool d : {direct, true}) most = std::max(most, head_plan(dtype, r, vocab, dim, d, false, nullptr).bytes);     // a row alone may start on 16 bytes
        return most;
    }
    const HeadPlan one = head_plan(dtype, 1, vocab, dim, direct, true, nullptr);         // the longest piece
    const int64_t operand = f32 ? kHeadNear : 1, planes = f32 ? kHeadNear + kHeadWide : 1, held = kHeadPieceBytes / (planes * 2);
    // Numbers of d in a plane: of the whole vocabulary, or as many as the pieces are cut for (to a multiple of 256 tokens), or the shortest pieces of every row.
    const int64_t d = std::min(rows * up(vocab, 64), std::max(held + 256 * rows, kHeadPieceMin * rows));
    // Rows of partial sums: a plane for each split.
    int64_t sums = 0;
    for (int cg : {1, 2})
        for (int64_t tiles_m = 1;; ++tiles_m) {
            const int64_t tile = 128 * cg, tiles = tiles_m * ((dim + tile - 1) / tile);
            const int64_t splits = std::max<int64_t>(1, std::min((kSms / cg) / tiles, up(vocab, kHeadChunk) / kHeadChunk / 16));
            const bool last = (cg == 1 && tiles_m * tile >= kHeadFewRows) || tiles_m * tile >= rows || splits == 1;
            sums = std::max(sums, splits * (splits == 1 && cg == 2 ? rows : std::min(rows, tiles_m * tile)));
            if (last) break;
        }
    size_t at = 0;
    auto take = [&](int64_t bytes) { at += (size_t)up(bytes, 256); };
    if (f32 || !direct) {
        take(operand * rows * one.dp * 2);
        take(operand * one.piece * one.dp * 2);
    }
    take(operand * d * 2);
    take(sums * up(dim, 8) * 4);
    take(rows * (int64_t)sizeof(HeadRow));
    take(rows * 4);
    take(4);
    if (f32) {
        take(rows * 4);
        take((one.piece + kHeadGroup - 1) / kHeadGroup * 4);
        take(kHeadWide * d * 2);
        take(kHeadWide * rows * one.dp * 2);
        take(rows * 4);
        take((vocab + kHeadPieceMin - 1) / kHeadPieceMin * 4);
    }
    return at;
}

// A matrix that a product reads: 16-bit elements, planes of [rows, cols] with row stride ld.
struct HeadMatrix {
    const void* p;
    int64_t rows, cols, ld, plane;
    int planes;
};

bool map_of(CUtensorMap* map, const HeadMatrix& m, bool mn, int box_rows) {
    const unsigned long long dims[3] = {(unsigned long long)m.cols, (unsigned long long)m.rows, (unsigned long long)m.planes};
    const int64_t ld = m.rows > 1 ? m.ld : up(m.cols, 8);    // of a single row any will do
    const unsigned long long strides[2] = {(unsigned long long)ld * 2, (unsigned long long)std::max(m.plane, ld) * 2};
    const unsigned box[3] = {64u, mn ? 64u : (unsigned)box_rows, 1u};
    return tensor_map(map, m.p, 3, dims, strides, box, true, false);
}


// Map of what a product stores: planes of [rows, cols] with row stride ld, in boxes of 128 bytes by 32 rows.
bool map_of_out(CUtensorMap* map, const void* p, int64_t rows, int64_t cols, int64_t ld, int64_t plane, int planes, int elem) {
    if (rows == 1) ld = up(cols, 8);
    const unsigned long long dims[3] = {(unsigned long long)cols, (unsigned long long)rows, (unsigned long long)planes};
    const unsigned long long strides[2] = {(unsigned long long)(ld * elem), (unsigned long long)(std::max(plane, ld) * elem)};
    const unsigned box[3] = {128u / elem, 32u, 1u};
    return tensor_map(map, p, 3, dims, strides, box, false, elem == 4);
}

// D[m, n] = sum over k of a[m, k] b[n, k]; an MN-major operand lies as [k, m] or [k, n].
bool job_of(HeadJob& j, int kind, int cg, int dtype, const HeadMatrix& a, bool a_mn, const HeadMatrix& b, bool b_mn, int promote,
            int64_t chunks_per_split = 0) {
    const int64_t tile = 128 * cg, m = a_mn ? a.cols : a.rows, n = b_mn ? b.cols : b.rows, k = a_mn ? a.rows : a.cols;
    const int box = a_mn || m >= 128 ? 128 : (int)up(m, 8);
    if (!map_of(&j.a, a, a_mn, box) || !map_of(&j.b, b, b_mn, 128)) return false;
    j.kind = kind;
    j.a_mn = a_mn; j.b_mn = b_mn;
    j.half = dtype == PB_F16 || a.planes == kHeadNear;
    j.planes = a.planes;
    j.promote = promote;
    j.a_bytes = a_mn ? kHeadOperand : box * 128;
    j.tiles_m = (int)((m + tile - 1) / tile);
    j.tiles_n = (int)((n + tile - 1) / tile);
    // Row tiles of a group stay in L2 (4096 rows) while the columns go by.
    j.group_m = kind == kHeadWeight ? 1 : std::min(j.tiles_m, 16);
    j.chunks = (int)((k + kHeadChunk - 1) / kHeadChunk);
    j.chunks_per_split = chunks_per_split ? (int)chunks_per_split : j.chunks;
    j.splits = (j.chunks + j.chunks_per_split - 1) / j.chunks_per_split;
    j.rows = (int)m;
    j.cols = (int)n;
    j.tiles = j.tiles_m * j.tiles_n * j.splits;
    j.groups = (j.tiles_m + j.group_m - 1) / j.group_m;
    j.by_split = Quotient((int64_t)j.tiles_m * j.tiles_n);
    j.by_group = Quotient((int64_t)j.group_m * j.tiles_n);
    j.by_height = Quotient(j.group_m);
    j.by_last = Quotient(j.tiles_m - (j.groups - 1) * j.group_m);
    return true;
}

template <int CG, int KIND, bool PROMOTE>
cudaError_t head_launch(HeadArgs& g, cudaStream_t s) {
    auto kernel = head_kernel<CG, KIND, PROMOTE>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeadSmem);
    if (e != cudaSuccess) return e;
    int64_t tiles = 0;
    g.a_slot = 1024;
    int planes = 1;
    for (int j = 0; j < g.jobs; ++j) {
        tiles += g.job[j].tiles;
        planes = std::max(planes, g.job[j].planes);
        g.a_slot = std::max(g.a_slot, g.job[j].a_bytes);
    }
    const int clusters = (int)std::min<int64_t>(tiles, kSms / CG);
    g.late = g.job[0].tiles % clusters;
    g.rounds = g.job[0].tiles / clusters;
    g.extra = 0;
    if (g.jobs == 2) {
        const int64_t early = clusters - g.late;
        const int64_t ratio = (g.job[0].chunks_per_split + kHeadTileCost) / (g.job[1].chunks_per_split + kHeadTileCost);
        if (g.late) g.extra = (int)std::min(ratio, g.job[1].tiles / early);
    }
    // The tensor core reads whole A tiles: behind the last one's rows it finds the epilogue's buffers.
    g.stage_bytes = planes * (kHeadOperand + g.a_slot);
    g.stages = std::min(kHeadMaxStages, kHeadRing / g.stage_bytes);
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;      // barriers and tensor memory are set up while the launch before ends
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CG;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3((unsigned)(clusters * CG));
    c.blockDim = dim3(kHeadThreads);
    c.dynamicSmemBytes = kHeadSmem;
    c.stream = s;
    c.attrs = attr;
    c.numAttrs = 2;
    void* args[] = {&g};
    return cudaLaunchKernelExC(&c, (const void*)kernel, args);
}
template <int KIND>
cudaError_t head_launch(HeadArgs& g, int cg, bool promote, cudaStream_t s) {
    if (cg == 2) return promote ? head_launch<2, KIND, true>(g, s) : head_launch<2, KIND, false>(g, s);
    return promote ? head_launch<1, KIND, true>(g, s) : head_launch<1, KIND, false>(g, s);
}

// 16-bit rows copied, or the wide planes of float32 ones.
cudaError_t pack(int dtype, const void* x, int64_t rows, int64_t dim, int64_t ld, unsigned short* out, int64_t ldp, cudaStream_t s) {
    const int64_t pairs = rows * (ldp / 2);
    const dim3 grid((unsigned)std::min<int64_t>((pairs + 255) / 256, kSms * 16));
    if (dtype == PB_F32) return launch_after(head_pack_kernel<float>, grid, 256, s, (const float*)x, rows, (int)dim, ld, out, (int)ldp, rows * ldp);
    return launch_after(head_pack_kernel<__half>, grid, 256, s, (const __half*)x, rows, (int)dim, ld, out, (int)ldp, rows * ldp);
}
// The near planes of float32 rows.
template <int kGroup>
cudaError_t pack_near(const float* x, int64_t rows, int64_t dim, int64_t ld, unsigned short* out, int64_t ldp, float* scale, int* most, cudaStream_t s) {
    auto kernel = aligned(x, 16) && (ld % 4 == 0 || rows == 1) && dim % 4 == 0 ? head_near_kernel<kGroup, true> : head_near_kernel<kGroup, false>;
    return launch_after(kernel, dim3((unsigned)((rows + kGroup - 1) / kGroup)), kNearThreads<kGroup>, s, x, (long long)rows, (int)dim, (long long)ld, out, (int)ldp,
                        (long long)(rows * ldp), scale, most);
}
// What a call's products read of the hidden states and of a piece of the weights, packed where it has to be.
cudaError_t hidden_of(HeadMatrix& m, const HeadPlan& e, int dtype, const void* x, int64_t rows, int64_t dim, int64_t ld, cudaStream_t s) {
    m = HeadMatrix{x, rows, dim, ld, 0, 1};
    if (!e.f32 && !e.packed) return cudaSuccess;
    m = HeadMatrix{e.hidden, rows, dim, e.dp, rows * e.dp, e.f32 ? kHeadNear : 1};
    return e.f32 ? pack_near<1>((const float*)x, rows, dim, ld, e.hidden, e.dp, e.row_scale, nullptr, s) : pack(dtype, x, rows, dim, ld, e.hidden, e.dp, s);
}
cudaError_t weight_of(HeadMatrix& m, const HeadPlan& e, int dtype, const void* x, int64_t rows, int64_t dim, int64_t ld, int* most, cudaStream_t s) {
    m = HeadMatrix{x, rows, dim, ld, 0, 1};
    if (!e.f32 && !e.packed) return cudaSuccess;
    m = HeadMatrix{e.weight, rows, dim, e.dp, rows * e.dp, e.f32 ? kHeadNear : 1};
    return e.f32 ? pack_near<kHeadGroup>((const float*)x, rows, dim, ld, e.weight, e.dp, e.col_scale, most, s) : pack(dtype, x, rows, dim, ld, e.weight, e.dp, s);
}

// Statistics of a few rows.
template <typename T>
cudaError_t few_rows(const HeadPlan& e, const void* hidden, const void* weight, int64_t rows, int64_t vocab, int64_t dim, int64_t ldh, int64_t ldw,
                     const void* tokens, int token_bytes, float c, cudaStream_t s) {
    auto kernel = rows == 1 ? head_few_kernel<T, 1> : head_few_kernel<T, 2>;
    if constexpr (sizeof(T) == 4) {
        if (rows > 2) kernel = head_few_kernel<T, 4>;
    }
    return launch_after(kernel, dim3((unsigned)e.parts), 32 * kHeadFewWarps, s, (const T*)hidden, (const T*)weight, (int)rows, (int)vocab, (int)dim, (long long)ldh,
                        (long long)ldw, tokens, token_bytes, c, e.part, e.ztok);
}

// Rows that start on 16 bytes: a bulk copy can start on them, and a load of 16 bytes.
bool direct_rows(const void* p, int64_t rows, int64_t ld, size_t es) { return aligned(p, 16) && (ld * (int64_t)es % 16 == 0 || rows == 1); }

int no_map(const char* who) {
    char text[128];
    snprintf(text, sizeof text, "%s: no tensor map for an operand", who);
    return fail_text(PB_E_CUDA, text);
}

const char* bad_sizes(int dtype, int64_t rows, int64_t vocab, int64_t dim, int64_t ld_hidden, int64_t ld_weight) {
    if (!dtype_ok(dtype)) return "unknown element type";
    if (rows < 0 || rows > kMaxHeadRows) return "rows must be between 0 and 2^24";
    if (vocab < 1 || vocab > kMaxHeadVocab) return "vocab must be between 1 and 2^24";
    if (dim < 1 || dim > kMaxHeadDim) return "dim must be between 1 and 2^20";
    if (ld_hidden < dim || ld_weight < dim) return "a row stride is smaller than dim";
    if (ld_hidden > (int64_t(1) << 36) || ld_weight > (int64_t(1) << 36)) return "a row stride is above 2^36";
    return nullptr;
}
int refuse(const char* who, const char* what) {
    char text[256];
    snprintf(text, sizeof text, "%s: %s", who, what);
    return fail_text(PB_E_ARG, text);
}
bool bad_temperature(double it) { return !(it > 0.0) || !std::isfinite((float)(it * 1.5)) || (float)it == 0.f; }

}  // namespace

extern "C" {

size_t pb_head_scratch_bytes(int dtype, int64_t rows, int64_t vocab, int64_t dim, int aligned_rows, int backward) {
    if (bad_sizes(dtype, rows, vocab, dim, dim, dim)) return 0;
    return std::max<size_t>(256, head_bytes(dtype, std::max<int64_t>(rows, 1), vocab, dim, aligned_rows != 0, backward != 0));
}

int pb_head_logprob_forward(const void* dev_hidden, const void* dev_weight, int dtype, int64_t rows, int64_t vocab, int64_t dim, int64_t ld_hidden,
                            int64_t ld_weight, const void* dev_tokens, int token_bytes, double inv_temperature, float* dev_logp, float* dev_entropy,
                            float* dev_lse, void* dev_scratch, size_t scratch_bytes, int32_t* dev_status, void* stream) {
    const char* who = "pb_head_logprob_forward";
    if (const char* bad = bad_sizes(dtype, rows, vocab, dim, ld_hidden, ld_weight)) return refuse(who, bad);
    if (bad_temperature(inv_temperature)) return refuse(who, "inv_temperature must be positive and finite");
    if (rows == 0) return PB_OK;
    if ((dev_logp != nullptr) != (dev_tokens != nullptr)) return refuse(who, "logp and tokens go together");
    if (dev_tokens && token_bytes != 4 && token_bytes != 8) return refuse(who, "tokens have 4 or 8 bytes");
    if (!dev_hidden || !dev_weight || !dev_scratch) return refuse(who, "NULL pointer");
    const size_t es = dtype_bytes(dtype);
    if (!aligned(dev_hidden, es) || !aligned(dev_weight, es) || (dev_tokens && !aligned(dev_tokens, token_bytes)) || !aligned(dev_logp, 4) ||
        !aligned(dev_entropy, 4) || !aligned(dev_lse, 4) || !aligned(dev_status, 4)) return refuse(who, "a pointer is not aligned to its element");
    if (!aligned(dev_scratch, 256)) return refuse(who, "scratch must be 256-byte aligned");
    const bool direct = direct_rows(dev_hidden, rows, ld_hidden, es) && direct_rows(dev_weight, vocab, ld_weight, es);
    const HeadPlan e = head_plan(dtype, rows, vocab, dim, direct, false, (char*)dev_scratch);
    if (scratch_bytes < std::max(e.bytes, head_bytes(dtype, rows, vocab, dim, direct, false))) return refuse(who, "scratch is smaller than pb_head_scratch_bytes");
    const size_t n_h = extent(rows, dim, ld_hidden, es), n_w = extent(vocab, dim, ld_weight, es), n_t = dev_tokens ? (size_t)rows * token_bytes : 0,
                 n_st = dev_status ? 4 : 0;
    auto in_scratch = [&](const void* p, size_t n) { return overlap(p, p ? n : 0, dev_scratch, scratch_bytes); };
    if (in_scratch(dev_hidden, n_h) || in_scratch(dev_weight, n_w) || in_scratch(dev_tokens, n_t) || in_scratch(dev_status, n_st) ||
        in_scratch(dev_logp, rows * 4) || in_scratch(dev_entropy, rows * 4) || in_scratch(dev_lse, rows * 4)) return refuse(who, "buffers overlap");
    const cudaStream_t s = (cudaStream_t)stream;
    if (e.few) {
        const float c = (float)(inv_temperature * 1.4426950408889634074);
        auto few = dtype == PB_F32 ? few_rows<float> : dtype == PB_BF16 ? few_rows<__nv_bfloat16> : few_rows<__half>;
        cudaError_t err = few(e, dev_hidden, dev_weight, rows, vocab, dim, ld_hidden, ld_weight, dev_tokens, token_bytes, c, s);
        if (err == cudaSuccess)
            err = launch_after(head_rows_kernel, dim3((unsigned)rows), kHeadRowThreads, s, e.part, (int)e.parts, (int)rows, 1, e.ztok, dev_tokens, token_bytes,
                               (long long)vocab, c, inv_temperature, (int)(dev_entropy != nullptr), dev_logp, dev_entropy, dev_lse, dev_status);
        return launched(who, err);
    }
    HeadMatrix hidden, b;
    cudaError_t err = hidden_of(hidden, e, dtype, dev_hidden, rows, dim, ld_hidden, s);
    for (int64_t r0 = 0; r0 < rows && err == cudaSuccess; r0 += e.stat_rows) {
        const int64_t nr = std::min(e.stat_rows, rows - r0);
        HeadMatrix a = hidden;
        a.p = (const unsigned short*)hidden.p + r0 * hidden.ld;
        a.rows = nr;
        HeadArgs g{};
        g.jobs = 1;
        if (e.f32) { g.row_scale = e.row_scale + r0; g.col_scale = e.col_scale; }
        const bool promote = e.f32 || dim > kHeadLong * kHeadChunk;
        const int chunks = e.f32 ? kHeadPromoteNear : promote ? kHeadPromoteLong : kHeadNever;
        g.c = (float)(inv_temperature * 1.4426950408889634074);
        g.status = dev_status;
        g.part = e.part;
        g.parts = (int)e.parts;
        g.ztok = e.ztok;
        g.entropy = dev_entropy != nullptr;
        g.tokens = dev_tokens ? (const char*)dev_tokens + r0 * token_bytes : nullptr;
        g.token_bytes = token_bytes;
        g.vocab = vocab;
        for (int64_t v0 = 0; v0 < vocab && err == cudaSuccess; v0 += e.piece) {
            const int64_t nv = std::min(e.piece, vocab - v0);
            // a single piece stays packed for the next rows
            if (r0 == 0 || e.pieces > 1) err = weight_of(b, e, dtype, (const char*)dev_weight + v0 * ld_weight * (int64_t)es, nv, dim, ld_weight, nullptr, s);
            if (!job_of(g.job[0], kHeadStats, e.cg, dtype, a, false, b, false, chunks)) return no_map(who);
            g.col0 = (int)v0;
            if (err == cudaSuccess) err = head_launch<kHeadStats>(g, e.cg, promote, s);
            g.part0 += g.job[0].tiles_n;
        }
        int width = 1;
        while (width < 16 && width < nr) width *= 2;
        auto at = [&](float* p) { return p ? p + r0 : nullptr; };
        if (err == cudaSuccess)
            err = launch_after(head_rows_kernel, dim3((unsigned)((nr + width - 1) / width)), kHeadRowThreads, s, e.part, (int)e.parts, (int)nr, width, e.ztok, g.tokens,
                         token_bytes, (long long)vocab, g.c, inv_temperature, g.entropy, at(dev_logp), at(dev_entropy), at(dev_lse), dev_status);
    }
    return launched(who, err);
}

int pb_head_logprob_backward(const void* dev_hidden, const void* dev_weight, int dtype, int64_t rows, int64_t vocab, int64_t dim, int64_t ld_hidden,
                             int64_t ld_weight, const void* dev_tokens, int token_bytes, double inv_temperature, const float* dev_lse,
                             const float* dev_entropy, const float* dev_g_logp, const float* dev_g_entropy, const float* dev_g_lse, void* dev_dhidden,
                             int64_t ld_dhidden, void* dev_dweight, int dweight_dtype, int64_t ld_dweight, int accumulate, void* dev_scratch,
                             size_t scratch_bytes, int32_t* dev_status, void* stream) {
    const char* who = "pb_head_logprob_backward";
    if (const char* bad = bad_sizes(dtype, rows, vocab, dim, ld_hidden, ld_weight)) return refuse(who, bad);
    if (bad_temperature(inv_temperature)) return refuse(who, "inv_temperature must be positive and finite");
    if (accumulate != 0 && accumulate != 1) return refuse(who, "accumulate must be 0 or 1");
    if (dev_dhidden && ld_dhidden < dim) return refuse(who, "a row stride is smaller than dim");
    if (dev_dweight) {
        if (!dtype_ok(dweight_dtype) || (dweight_dtype != PB_F32 && dweight_dtype != dtype)) return refuse(who, "dweight is float32 or of the weight's type");
        if (ld_dweight < dim) return refuse(who, "a row stride is smaller than dim");
    }
    const size_t es = dtype_bytes(dtype), gs = dtype_bytes(dweight_dtype);
    const cudaStream_t s = (cudaStream_t)stream;
    if (!dev_dhidden && !dev_dweight) return rows == 0 ? PB_OK : refuse(who, "neither gradient is asked for");
    if (rows == 0) {
        if (!dev_dweight || accumulate) return PB_OK;
        if (!aligned(dev_dweight, gs)) return refuse(who, "a pointer is not aligned to its element");
        return launched(who, cudaMemset2DAsync(dev_dweight, (size_t)ld_dweight * gs, 0, (size_t)dim * gs, (size_t)vocab, s));
    }
    if (!dev_hidden || !dev_weight || !dev_lse || !dev_scratch) return refuse(who, "NULL pointer");
    if (dev_g_logp && !dev_tokens) return refuse(who, "a gradient of logp needs the tokens");
    if (dev_g_entropy && !dev_entropy) return refuse(who, "a gradient of the entropy needs the entropy");
    if (dev_tokens && token_bytes != 4 && token_bytes != 8) return refuse(who, "tokens have 4 or 8 bytes");
    if (!aligned(dev_hidden, es) || !aligned(dev_weight, es) || (dev_tokens && !aligned(dev_tokens, token_bytes)) || !aligned(dev_lse, 4) ||
        !aligned(dev_entropy, 4) || !aligned(dev_g_logp, 4) || !aligned(dev_g_entropy, 4) || !aligned(dev_g_lse, 4) || !aligned(dev_dhidden, es) ||
        !aligned(dev_dweight, gs) || !aligned(dev_status, 4)) return refuse(who, "a pointer is not aligned to its element");
    if (!aligned(dev_scratch, 256)) return refuse(who, "scratch must be 256-byte aligned");
    const bool direct = direct_rows(dev_hidden, rows, ld_hidden, es) && direct_rows(dev_weight, vocab, ld_weight, es);
    const HeadPlan e = head_plan(dtype, rows, vocab, dim, direct, true, (char*)dev_scratch);
    if (scratch_bytes < std::max(e.bytes, head_bytes(dtype, rows, vocab, dim, direct, true))) return refuse(who, "scratch is smaller than pb_head_scratch_bytes");
    struct Span { const void* p; size_t n; };
    const size_t nr4 = (size_t)rows * 4;
    const Span read[] = {{dev_hidden, extent(rows, dim, ld_hidden, es)}, {dev_weight, extent(vocab, dim, ld_weight, es)},
                         {dev_tokens, dev_tokens ? (size_t)rows * token_bytes : 0}, {dev_lse, nr4}, {dev_entropy, nr4}, {dev_g_logp, nr4},
                         {dev_g_entropy, nr4}, {dev_g_lse, nr4}};
    const Span written[] = {{dev_scratch, scratch_bytes}, {dev_dhidden, extent(rows, dim, ld_dhidden, es)},
                            {dev_dweight, extent(vocab, dim, ld_dweight, gs)}, {dev_status, 4}};
    for (int k = 0; k < 4; ++k) {
        if (!written[k].p) continue;
        for (const Span& r : read)
            if (r.p && overlap(written[k].p, written[k].n, r.p, r.n)) return refuse(who, "buffers overlap");
        for (int l = 0; l < k; ++l)
            if (written[l].p && overlap(written[k].p, written[k].n, written[l].p, written[l].n)) return refuse(who, "buffers overlap");
    }
    const float c2 = (float)(inv_temperature * 1.4426950408889634074);         // of logits, in units of log 2
    cudaError_t err = launch_after(head_coef_kernel, dim3(1), 1024, s, (int)rows, (long long)vocab, dev_tokens, token_bytes, inv_temperature, c2, dev_lse, dev_entropy,
                                   dev_g_logp, dev_g_entropy, dev_g_lse, dtype == PB_F16 ? 14 : 0, e.coef, e.row_token, e.unscale, e.d_scale, e.col_most,
                                   (int)(e.f32 ? e.pieces : 0), dev_status);
    HeadMatrix hidden, w;
    if (err == cudaSuccess) err = hidden_of(hidden, e, dtype, dev_hidden, rows, dim, ld_hidden, s);
    // dweight's own
    HeadMatrix hidden_wide = hidden;
    if (e.f32 && dev_dweight) {
        if (err == cudaSuccess) err = pack(dtype, dev_hidden, rows, dim, ld_hidden, e.hidden_wide, e.dp, s);
        hidden_wide = HeadMatrix{e.hidden_wide, rows, dim, e.dp, rows * e.dp, kHeadWide};
    }
    HeadArgs g{};
    const int near = e.f32 ? kHeadPromoteNear : kHeadNever, wide = e.f32 ? kHeadPromoteWide : kHeadNever;
    g.row_scale = e.row_scale;
    g.col_scale = e.col_scale;
    g.d_scale = e.d_scale;
    g.store_near = dev_dhidden != nullptr;
    g.store_wide = dev_dweight != nullptr;
    g.c = c2;
    g.status = dev_status;
    g.coef = e.coef;
    g.row_token = e.row_token;
    g.entropy = dev_g_entropy != nullptr;
    const int64_t d_plane = rows * e.ldd, plane_size = rows * e.ldp;
    g.unscale = e.unscale;
    g.out_type = dweight_dtype;
    g.ldo = ld_dweight;
    g.accumulate = accumulate;
    // Sums that are rounded to 16 bits once more are formed in registers.  A bulk store writes whole pieces of 16 bytes, so rows have to end on one.
    g.bulk = dev_dweight && aligned(dev_dweight, 16) && (ld_dweight * (int64_t)gs % 16 == 0 || vocab == 1) && dim * (int64_t)gs % 16 == 0 &&
             (dweight_dtype == PB_F32 || !accumulate);
    int planes = 0;
    for (int64_t v0 = 0; v0 < vocab && err == cudaSuccess; v0 += e.piece) {
        const int64_t nv = std::min(e.piece, vocab - v0);
        int* const most = e.f32 ? e.col_most + v0 / e.piece : nullptr;
        if (err == cudaSuccess) err = weight_of(w, e, dtype, (const char*)dev_weight + v0 * ld_weight * (int64_t)es, nv, dim, ld_weight, most, s);
        g.col_most = (const float*)most;
        const HeadMatrix d{e.d, rows, nv, e.ldd, d_plane, e.f32 ? kHeadNear : 1}, d_wide = e.f32 ? HeadMatrix{e.d_wide, rows, nv, e.ldd, d_plane, kHeadWide} : d;
        g.col0 = (int)v0;
        g.jobs = 1;
        if (!job_of(g.job[0], kHeadGrad, e.cg, dtype, hidden, false, w, false, near) ||
            !map_of_out(&g.job[0].out, d_wide.p, rows, nv, e.ldd, d_plane, d_wide.planes, 2) ||
            !map_of_out(&g.job[1].out, d.p, rows, nv, e.ldd, d_plane, d.planes, 2)) return no_map(who);
        if (err == cudaSuccess) err = head_launch<kHeadGrad>(g, e.cg, e.f32, s);
        g.jobs = 0;
        g.add = v0 > 0;
        if (dev_dhidden) {
            // as many chunks in each split of every piece, so that the first piece has the most splits
            HeadJob& j = g.job[g.jobs++];
            if (!job_of(j, kHeadHidden, e.cg, dtype, d, false, w, true, near, e.split_chunks) || !map_of_out(&j.out, e.plane, rows, dim, e.ldp, plane_size, e.splits, 4))
                return no_map(who);
            planes = std::max(planes, j.splits);
        }
        if (dev_dweight) {
            g.out = (char*)dev_dweight + v0 * ld_dweight * (int64_t)gs;
            HeadJob& j = g.job[g.jobs++];
            if (!job_of(j, kHeadWeight, e.cg, dtype, d_wide, true, hidden_wide, true, wide) || (g.bulk && !map_of_out(&j.out, g.out, nv, dim, ld_dweight, 0, 1, (int)gs))) return no_map(who);
        }
        if (e.f32 && g.jobs == 2) {              // stages of another size each: two launches
            g.jobs = 1;
            if (err == cudaSuccess) err = head_launch<kHeadHidden>(g, e.cg, e.f32, s);
            std::swap(g.job[0], g.job[1]);
        }
        // the longer product's tiles first
        if (g.jobs == 2 && g.job[1].chunks_per_split > g.job[0].chunks_per_split) std::swap(g.job[0], g.job[1]);
        if (err == cudaSuccess) err = head_launch<kHeadHidden>(g, e.cg, e.f32, s);
    }
    if (dev_dhidden && err == cudaSuccess) {
        const int64_t n = rows * (e.ldp / 8);
        const dim3 grid((unsigned)std::min<int64_t>((n + 255) / 256, kSms * 16));
        auto go = [&](auto t) {
            using T = decltype(t);
            return launch_after(head_sum_kernel<T>, grid, 256, s, e.plane, plane_size, planes, (int)e.ldp, (int)rows, (int)dim, e.unscale, e.d_scale, (T*)dev_dhidden, (long long)ld_dhidden);
        };
        err = dtype == PB_F32 ? go(float()) : dtype == PB_BF16 ? go(__nv_bfloat16()) : go(__half());
    }
    return launched(who, err);
}

}  // extern "C"
