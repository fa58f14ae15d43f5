// psops_xent.cu -- C ABI and host side of the linear cross entropy (kernels:
// psops_xent_kernels.cuh).

#include "psops.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <new>
#include <utility>

#include "psops_host.cuh"
#include "psops_xent_kernels.cuh"
#include "psops_xent_small.cuh"

using psops_host::Base;
using psops_host::OnDevice;
using psops_host::ceil_div;
using psops_host::round_up;

namespace {

// Bytes that the logits' gradients of one piece of the vocabulary may take, and
// those of its rows of w (and of dw) that pass through the workspace.
constexpr int64_t kPieceBytes = 512ll << 20;
constexpr int64_t kMinPiece = 2048;
// Pairs of CTAs that run at once on a B200 (148 SMs), where a layout must not ask the GPU.
constexpr int64_t kPairs = 74;
// From so many tokens on, dw of a small vocabulary is summed in shares.  Gradients
// in a CUDA graph, whole / in shares: 1,024 x 1,024 x 2,300: 41 / 46 us; 2,048 x 512
// x 300: 40 / 36; 4,000 x 1,000 x 500: 60 / 52; 8,192 x 2,048 x 177: 132 / 111.
constexpr int64_t kSplitTokens = 1536;
// Most blocks of the small kernels' launches (they have a partial result each).
constexpr int64_t kMostBlocks = 1024;
// Bytes that the fp32 sums of dh may take in more than one share.
constexpr int64_t kShareBytes = 256ll << 20;

bool config_ok(const psops_xent_config *c)
{
    return c != nullptr && c->max_tokens >= 1 && c->max_tokens <= (1 << 24) && c->dim >= 1 && c->dim <= (1 << 20) &&
           c->vocab >= 1 && c->vocab <= (1ll << 31) - (1 << 16) && (c->type == PSOPS_F16 || c->type == PSOPS_BF16) &&
           (c->flags & ~(PSOPS_XENT_GRADS | PSOPS_XENT_STAGED)) == 0;
}

struct Layout {
    int64_t rows;                               // compact rows, whole tiles
    int64_t padded;                             // dim in the workspace: a multiple of 64, so that rows are whole lines of 128 bytes
    int64_t piece;                              // vocabulary entries of a piece, a multiple of the tile
    bool staged;                                // w and dw may pass through the workspace
    int64_t parts;                              // softmax statistics per row
    int64_t sum_rows;                           // rows of the fp32 sums of dh, all shares together
    int64_t dw_most;                            // most shares of dw's sum over the tokens; 1: not split
    size_t control, row_of, compact_of, label, row_scale, row_lse, row_label, label_logit, partials, hidden, stats, w, dw, dlogits, sums, dw_sums, total;
};

Layout make_layout(const psops_xent_config *c)
{
    Layout L{};
    L.rows = (int64_t)round_up((size_t)c->max_tokens, kTileRows);
    L.padded = (int64_t)round_up((size_t)c->dim, 64);
    const int64_t whole = (int64_t)round_up((size_t)c->vocab, kTileCols);
    L.staged = c->dim % 8 != 0 || (c->flags & PSOPS_XENT_STAGED) != 0;
    const int64_t widest = L.staged ? std::max(L.rows, L.padded) : L.rows;
    L.piece = std::min(whole, std::max(kMinPiece, kPieceBytes / (2 * widest) / kTileCols * kTileCols));
    L.parts = whole / kHalf;
    L.sum_rows = L.rows * std::max<int64_t>(1, std::min<int64_t>(kMostShares, kShareBytes / (4 * L.rows * L.padded)));
    size_t at = 0;
    auto take = [&at](size_t bytes) {
        const size_t here = at;
        at += round_up(bytes, 1024);
        return here;
    };
    const size_t n = (size_t)L.rows;
    L.control = take(sizeof(XentControl));
    L.row_of = take(4 * n);
    L.compact_of = take(4 * n);
    L.label = take(4 * n);
    L.row_scale = take(4 * n);
    L.row_lse = take(4 * n);
    L.row_label = take(4 * n);
    L.label_logit = take(4 * n);
    L.partials = take(std::max<size_t>(8 * (n / kJoinRows), sizeof(double2) * kMostBlocks));
    L.hidden = take(2 * n * (size_t)L.padded);
    L.stats = take(std::max<size_t>(8 * n * (size_t)L.parts, 8 * kFewTokens * kMostBlocks));
    if (L.staged) L.w = take(2 * (size_t)L.piece * (size_t)L.padded);
    if (c->flags & PSOPS_XENT_GRADS) {
        if (L.staged) L.dw = take(2 * (size_t)L.piece * (size_t)L.padded);
        L.dlogits = take(2 * n * (size_t)L.piece);
        L.sums = take(4 * (size_t)L.sum_rows * (size_t)L.padded);
        // a small vocabulary gives dw few tiles: then its sum over the tokens is split
        const int64_t tiles = whole / kTile * ceil_div(L.padded, kTile);
        L.dw_most = c->max_tokens < kSplitTokens ? 1 : std::max<int64_t>(1, std::min<int64_t>(kMostShares, kPairs / tiles));
        if (L.dw_most > 1) L.dw_sums = take(4 * (size_t)(whole * L.dw_most) * (size_t)L.padded);
    }
    L.total = at;
    return L;
}

} // namespace

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

struct psops_xent : Base {
    psops_xent_config cfg;
    Layout lay;
    char *ws;
    EncodeTiled encode;
    template <class T> T *at(size_t offset) const { return (T *)(ws + offset); }
    XentControl *control() const { return at<XentControl>(lay.control); }
};

namespace {

template <typename... Params, typename... Args>
int launch(psops_xent *x, const char *name, void (*kernel)(Params...), dim3 grid, int threads, size_t shared, Args &&...args)
{
    return psops_host::launch(x, name, kernel, grid, threads, shared, 1, std::forward<Args>(args)...);
}
template <typename... Params, typename... Args>
int launch(psops_xent *x, const char *name, void (*kernel)(Params...), int64_t grid, int threads, size_t shared, Args &&...args)
{
    return launch(x, name, kernel, dim3((unsigned)std::max<int64_t>(1, grid)), threads, shared, std::forward<Args>(args)...);
}

// Blocks of a copy of so many 16-byte pieces, one or more a thread.
int64_t copy_grid(const psops_xent *x, int64_t pieces) { return std::min<int64_t>(ceil_div(pieces, kCopyThreads), (int64_t)x->sms * 8); }

#define PSOPS_DO(call)                       \
    do {                                     \
        const int rc_ = (call);              \
        if (rc_ != PSOPS_OK) return rc_;     \
    } while (0)

// Which products run with pairs of CTAs.
bool in_pairs(int job, int64_t tokens) { return job >= kDw || tokens > kSingleTokens; }

bool aligned16(const void *p, int64_t ld) { return ((uintptr_t)p & 15u) == 0 && ld % 8 == 0; }

int check_matrix(const void *p, int64_t ld, int64_t rows, int64_t dim)
{
    if (rows == 0) return PSOPS_OK;
    if (p == nullptr || ld < dim || ld > (1ll << 31)) return PSOPS_EINVAL;
    return ((uintptr_t)p & 1u) ? PSOPS_EALIGN : PSOPS_OK;
}

int check_call(const psops_xent *x, const void *h, int64_t h_ld, const void *w, int64_t w_ld, const int64_t *targets,
               int64_t tokens)
{
    if (tokens < 0 || tokens > x->cfg.max_tokens) return PSOPS_EINVAL;
    int rc = check_matrix(h, h_ld, tokens, x->cfg.dim);
    if (rc == PSOPS_OK) rc = check_matrix(w, w_ld, x->cfg.vocab, x->cfg.dim);
    if (rc != PSOPS_OK) return rc;
    if (tokens > 0 && targets == nullptr) return PSOPS_EINVAL;
    if ((uintptr_t)targets & 7u) return PSOPS_EALIGN;
    if (!x->lay.staged && !aligned16(w, w_ld)) return PSOPS_EALIGN;
    return PSOPS_OK;
}

// The tokens that count, and their hidden states.
int gather(psops_xent *x, IndexParams P, const void *h, int64_t h_ld)
{
    P.control = x->control();
    P.row_of = x->at<int>(x->lay.row_of);
    P.compact_of = x->at<int>(x->lay.compact_of);
    P.label = x->at<int>(x->lay.label);
    P.row_scale = x->at<float>(x->lay.row_scale);
    P.row_lse = x->at<float>(x->lay.row_lse);
    P.row_label = x->at<float>(x->lay.row_label);
    P.vocab = (int)x->cfg.vocab;
    P.headroom = x->cfg.type == PSOPS_F16 ? 32768.0f : 1.0f;
    // every piece of the vocabulary gives every share of dh something to add up, the shortest piece too
    const int64_t last = x->cfg.vocab - (x->cfg.vocab - 1) / x->lay.piece * x->lay.piece;
    P.steps = (int)ceil_div(last, kStepK);
    P.tiles_across = (int)ceil_div(x->lay.padded, kTile);
    P.sum_rows = (int)x->lay.sum_rows;
    P.pairs = in_pairs(kDh, P.tokens) ? x->sms / 2 : x->sms;
    P.dw_most = (int)x->lay.dw_most;
    P.dw_tiles = (int)(ceil_div(x->cfg.vocab, kTile) * P.tiles_across);
    P.dw_pairs = x->sms / 2;
    const GatherParams G{(const uint16_t *)h, h_ld, (int)x->cfg.dim, (int)x->lay.padded, aligned16(h, h_ld), x->at<uint16_t>(x->lay.hidden)};
    const int64_t pieces = (int64_t)round_up((size_t)std::max<int64_t>(1, P.tokens), kStepK) * x->lay.padded / 8;
    if (P.tokens <= kListTokens)
        return launch(x, "psops_xent_index_kernel", psops_xent_index_kernel<true>,
                      std::min<int64_t>(ceil_div(pieces, kIndexThreads), (int64_t)x->sms), kIndexThreads, 0, P, G);
    PSOPS_DO(launch(x, "psops_xent_index_kernel", psops_xent_index_kernel<false>, 1, kIndexThreads, 0, P, G));
    return launch(x, "psops_xent_gather_kernel", psops_xent_gather_kernel, copy_grid(x, pieces), kCopyThreads, 0, G, P.control, P.row_of);
}

// The rows of w of one piece as the products read them: in place, or packed into the workspace.
int piece_of_w(psops_xent *x, const void *w, int64_t w_ld, int64_t first, int64_t count, const void **out, int64_t *width, int64_t *out_ld)
{
    const uint16_t *from = (const uint16_t *)w + first * w_ld;
    if (x->cfg.dim % 8 == 0 && aligned16(w, w_ld)) {
        *out = from;
        *width = x->cfg.dim;
        *out_ld = w_ld;
        return PSOPS_OK;
    }
    uint16_t *to = x->at<uint16_t>(x->lay.w);
    *out = to;
    *width = *out_ld = x->lay.padded;
    return launch(x, "psops_xent_pack_kernel", psops_xent_pack_kernel, copy_grid(x, count * x->lay.padded / 8), kCopyThreads, 0, from,
                  w_ld, count, (int)x->cfg.dim, (int)x->lay.padded, aligned16(w, w_ld), to);
}

// A matrix of `height` rows of `width` consecutive elements as the tensor
// copies see it: boxes of 128 bytes by `box_rows` rows, swizzled; outside, reads give zeros.
int make_map(psops_xent *x, CUtensorMap *map, int type, const void *base, int64_t width, int64_t height, int64_t ld, int box_rows)
{
    const int bytes = type == PSOPS_F32 ? 4 : 2;
    const cuuint64_t size[2] = {(cuuint64_t)width, (cuuint64_t)height};
    const cuuint64_t stride[1] = {(cuuint64_t)(ld * bytes)};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / bytes), (cuuint32_t)box_rows}, step[2] = {1, 1};
    const CUtensorMapDataType kind = type == PSOPS_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                     : type == PSOPS_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    const CUresult r = x->encode(map, kind, 2, const_cast<void *>(base), size, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                 CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r == CUDA_SUCCESS) return PSOPS_OK;
    std::snprintf(x->err, sizeof(x->err), "cuTensorMapEncodeTiled: error %d", (int)r);
    return PSOPS_ECUDA;
}

using ProductKernel = void (*)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const ProductParams);
template <class T>
ProductKernel product_of(int job, bool pair)
{
    return job == kDw        ? psops_xent_product_kernel<T, kDw, true>
           : job == kDwLong  ? psops_xent_product_kernel<T, kDwLong, true>
           : job == kDwSums  ? psops_xent_product_kernel<T, kDwSums, true>
           : job == kLoss    ? (pair ? psops_xent_product_kernel<T, kLoss, true> : psops_xent_product_kernel<T, kLoss, false>)
           : job == kDlogits ? (pair ? psops_xent_product_kernel<T, kDlogits, true> : psops_xent_product_kernel<T, kDlogits, false>)
                             : (pair ? psops_xent_product_kernel<T, kDh, true> : psops_xent_product_kernel<T, kDh, false>);
}
ProductKernel product_of(const psops_xent *x, int job, bool pair)
{
    return x->cfg.type == PSOPS_F16 ? product_of<__half>(job, pair) : product_of<__nv_bfloat16>(job, pair);
}

// `tiles` (times shares): if every token counts.
int product(psops_xent *x, int job, int64_t tokens, int64_t tiles, const CUtensorMap &a, const CUtensorMap &b, const CUtensorMap &out,
            const ProductParams &P)
{
    const bool pair = in_pairs(job, tokens);
    const int64_t ctas = pair ? 2 : 1;
    const dim3 grid((unsigned)(ctas * std::max<int64_t>(1, std::min<int64_t>(tiles, x->sms / ctas))));
    return psops_host::launch(x, "psops_xent_product_kernel", product_of(x, job, pair), grid, kProductThreads,
                              pair ? ProductShape<true>::kShared : ProductShape<false>::kShared, (int)ctas, a, b, out, P);
}

ProductParams product_params(const psops_xent *x)
{
    ProductParams P{};
    P.control = x->control();
    P.label = x->at<int>(x->lay.label);
    P.row_lse = x->at<float>(x->lay.row_lse);
    P.row_scale = x->at<float>(x->lay.row_scale);
    P.row_label = x->at<float>(x->lay.row_label);
    P.stats = x->at<float2>(x->lay.stats);
    P.stats_ld = x->lay.rows;
    P.label_logit = x->at<float>(x->lay.label_logit);
    return P;
}

// What a call's products have in common.
struct Call {
    int64_t padded, rows, some_rows, tiles_m;   // rows: if every token counts, whole tiles; some_rows: whole steps
    CUtensorMap hidden;                         // rows by dim, summed over dim
};

int open_call(psops_xent *x, int64_t tokens, Call *c)
{
    c->padded = x->lay.padded;
    c->rows = (int64_t)round_up((size_t)std::max<int64_t>(1, tokens), kTileRows);
    c->some_rows = (int64_t)round_up((size_t)std::max<int64_t>(1, tokens), kStepK);
    c->tiles_m = c->rows / kTile;
    return make_map(x, &c->hidden, x->cfg.type, x->at<void>(x->lay.hidden), c->padded, c->some_rows, c->padded, kHalf);
}

HeadParams head_params(const psops_xent *x, const void *h, int64_t h_ld, const void *w, int64_t w_ld, const int64_t *targets,
                       int64_t tokens, int32_t reduction)
{
    HeadParams P{};
    P.h = h; P.h_ld = h_ld; P.w = w; P.w_ld = w_ld;
    P.targets = (const long long *)targets;
    P.tokens = (int)tokens; P.dim = (int)x->cfg.dim; P.vocab = (int)x->cfg.vocab; P.reduction = reduction;
    P.control = x->control();
    P.partials = x->at<double2>(x->lay.partials);
    return P;
}

// Passes of few classes, and the forward pass of few tokens.
template <class T>
int forward_head(psops_xent *x, HeadParams P)
{
    const int64_t grid = std::min<int64_t>(ceil_div(P.tokens, kSmallWarps), std::min<int64_t>(x->sms, kMostBlocks));
    return launch(x, "psops_xent_head_kernel", psops_xent_head_kernel<T, false>, grid, kSmallThreads, head_shared(P.vocab, P.dim), P);
}

template <class T>
int backward_head(psops_xent *x, HeadParams P, void *dw, int64_t dw_ld)
{
    const int64_t grid = std::min<int64_t>(ceil_div(P.tokens, kSmallWarps), std::min<int64_t>(x->sms, kMostBlocks));
    PSOPS_DO(launch(x, "psops_xent_head_kernel", psops_xent_head_kernel<T, true>, grid, kSmallThreads, head_shared(P.vocab, P.dim), P));
    if (dw == nullptr) return PSOPS_OK;
    return launch(x, "psops_xent_head_dw_kernel", psops_xent_head_dw_kernel<T>,
                  dim3((unsigned)ceil_div(P.dim, 32), (unsigned)ceil_div(P.vocab, kHeadDwClasses)), kHeadDwThreads, 0, (const T *)P.h, P.h_ld,
                  P.targets, (const float *)P.dlogits, P.tokens, P.dim, P.vocab, (T *)dw, dw_ld);
}

template <class T, bool ALIGNED>
void (*few_kernel(int few))(const FewParams)
{
    return few == 1 ? psops_xent_few_kernel<T, 1, ALIGNED> : few == 2 ? psops_xent_few_kernel<T, 2, ALIGNED>
           : psops_xent_few_kernel<T, 4, ALIGNED>;
}
template <class T>
void (*few_kernel(int few, bool aligned))(const FewParams)
{
    return aligned ? few_kernel<T, true>(few) : few_kernel<T, false>(few);
}

template <class T>
int forward_few(psops_xent *x, FewParams P)
{
    const auto kernel = few_kernel<T>(few_of(P.tokens), P.w_aligned && P.dim % 8 == 0);
    const int64_t grid = std::min<int64_t>(std::min<int64_t>((int64_t)x->sms * kFewBlocks, kMostBlocks), ceil_div(P.vocab, kSmallWarps));
    return launch(x, "psops_xent_few_kernel", kernel, grid, kSmallThreads, few_shared(P.tokens, P.dim), P);
}

template <class T, bool ALIGNED>
void (*few_grads_kernel(int few))(const FewGradParams)
{
    return few == 1 ? psops_xent_few_grads_kernel<T, 1, ALIGNED> : few == 2 ? psops_xent_few_grads_kernel<T, 2, ALIGNED>
           : psops_xent_few_grads_kernel<T, 4, ALIGNED>;
}

template <class T>
int backward_few(psops_xent *x, FewGradParams P, bool aligned, void *dh, int64_t dh_ld)
{
    const int few = few_of(P.tokens), teams_of_block = kSmallWarps / P.team;
    const int rows = few == 1 ? kFewGradRows<1> : few == 2 ? kFewGradRows<2> : kFewGradRows<4>;
    const int blocks = few == 1 ? kFewGradBlocks<1> : few == 2 ? kFewGradBlocks<2> : kFewGradBlocks<4>;
    // as many blocks as run at once, have rows to do and room for their parts of dh
    const int64_t grid = std::max<int64_t>(1, std::min({(int64_t)x->sms * blocks, ceil_div(ceil_div(P.vocab, rows), teams_of_block),
                                                        x->lay.sum_rows / (few * teams_of_block)}));
    PSOPS_DO(launch(x, "psops_xent_few_grads_kernel", aligned ? few_grads_kernel<T, true>(few) : few_grads_kernel<T, false>(few), grid,
                    kSmallThreads, 0, P));
    if (dh == nullptr) return PSOPS_OK;
    return launch(x, "psops_xent_few_dh_kernel", psops_xent_few_dh_kernel<T>, dim3((unsigned)ceil_div(P.dim, 32), (unsigned)P.tokens),
                  kSmallThreads, 0, (const float *)P.parts, (int)grid * teams_of_block, few, P.padded, P.targets, P.vocab, P.dim, (T *)dh, dh_ld);
}

int forward(psops_xent *x, const void *w, int64_t w_ld, int64_t tokens, JoinParams J)
{
    Call c;
    PSOPS_DO(open_call(x, tokens, &c));
    // w in place is one piece
    const bool in_place = x->cfg.dim % 8 == 0 && aligned16(w, w_ld);
    const int64_t piece = in_place ? x->cfg.vocab : x->lay.piece;
    for (int64_t first = 0; first < x->cfg.vocab; first += piece) {
        const int64_t count = std::min(piece, x->cfg.vocab - first);
        const void *rows_of_w;
        int64_t width, ld;
        CUtensorMap weights;
        PSOPS_DO(piece_of_w(x, w, w_ld, first, count, &rows_of_w, &width, &ld));
        PSOPS_DO(make_map(x, &weights, x->cfg.type, rows_of_w, width, count, ld, kHalf));
        ProductParams P = product_params(x);
        P.columns = (int)count;
        P.depth = (int)c.padded;
        P.first = (int)first;
        PSOPS_DO(product(x, kLoss, tokens, c.tiles_m * ceil_div(count, kTile), c.hidden, weights, weights, P));
    }
    J.stats = x->at<float2>(x->lay.stats);
    J.stats_ld = x->lay.rows;
    J.parts = (int)x->lay.parts;
    J.control = x->control();
    J.row_of = x->at<int>(x->lay.row_of);
    J.label_logit = x->at<float>(x->lay.label_logit);
    J.partials = x->at<double>(x->lay.partials);
    return launch(x, "psops_xent_join_kernel", psops_xent_join_kernel, ceil_div(tokens, kJoinRows), kJoinRows * kJoinParts, 0, J);
}

// dh (and a look at dw), or dw from its shares, from fp32 sums.
template <bool DW>
int results(psops_xent *x, const float *sums, int dw_share_rows, int rows, void *out, int64_t ld, void *dw = nullptr, int64_t dw_ld = 0)
{
    OutParams P{};
    P.dw = dw;
    P.dw_ld = dw_ld;
    P.dw_rows = x->cfg.vocab;
    P.sums = sums;
    P.sums_ld = x->lay.padded;
    P.control = x->control();
    P.compact_of = x->at<int>(x->lay.compact_of);
    P.rows = rows;
    P.dim = (int)x->cfg.dim;
    P.dw_share_rows = dw_share_rows;
    P.aligned = ((uintptr_t)out & 7u) == 0 && ld % 4 == 0;
    P.out = out;
    P.ld = ld;
    return launch(x, "psops_xent_out_kernel", x->cfg.type == PSOPS_F16 ? psops_xent_out_kernel<__half, DW> : psops_xent_out_kernel<__nv_bfloat16, DW>,
                  copy_grid(x, rows * ceil_div(x->cfg.dim, 4)), kCopyThreads, 0, P);
}

int backward(psops_xent *x, const void *w, int64_t w_ld, int64_t tokens, void *dh, int64_t dh_ld, void *dw, int64_t dw_ld)
{
    const int type = x->cfg.type;
    const bool direct = x->cfg.dim % 8 == 0 && aligned16(dw, dw_ld);
    Call c;
    PSOPS_DO(open_call(x, tokens, &c));
    const int64_t tiles_d = ceil_div(c.padded, kTile);
    CUtensorMap hidden_across, dlogits_out, dlogits_along, dlogits_across, sums;
    void *dlogits = x->at<void>(x->lay.dlogits);
    PSOPS_DO(make_map(x, &hidden_across, type, x->at<void>(x->lay.hidden), c.padded, c.some_rows, c.padded, kStepK));
    PSOPS_DO(make_map(x, &dlogits_out, type, dlogits, x->lay.piece, c.some_rows, x->lay.piece, 32));
    PSOPS_DO(make_map(x, &dlogits_along, type, dlogits, x->lay.piece, c.some_rows, x->lay.piece, kHalf));
    PSOPS_DO(make_map(x, &dlogits_across, type, dlogits, x->lay.piece, c.some_rows, x->lay.piece, kStepK));
    PSOPS_DO(make_map(x, &sums, PSOPS_F32, x->at<void>(x->lay.sums), c.padded, x->lay.sum_rows, c.padded, 32));
    for (int64_t first = 0; first < x->cfg.vocab; first += x->lay.piece) {
        const int64_t count = std::min(x->lay.piece, x->cfg.vocab - first);
        const void *rows_of_w;
        int64_t width, ld;
        CUtensorMap weights;
        PSOPS_DO(piece_of_w(x, w, w_ld, first, count, &rows_of_w, &width, &ld));
        PSOPS_DO(make_map(x, &weights, type, rows_of_w, width, count, ld, kHalf));
        ProductParams P = product_params(x);
        P.columns = (int)count;
        P.depth = (int)c.padded;
        P.first = (int)first;
        PSOPS_DO(product(x, kDlogits, tokens, c.tiles_m * ceil_div(count, kTile), c.hidden, weights, dlogits_out, P));
        if (dh != nullptr) {
            PSOPS_DO(make_map(x, &weights, type, rows_of_w, width, count, ld, kStepK));
            P.columns = (int)c.padded;
            P.depth = (int)count;
            P.add = first > 0;
            PSOPS_DO(product(x, kDh, tokens, c.tiles_m * tiles_d * kMostShares, dlogits_along, weights, sums, P));
        }
        if (dw != nullptr && x->lay.dw_most > 1 && tokens >= kSplitTokens) {
            CUtensorMap dw_sums;
            const int64_t share_rows = (int64_t)round_up((size_t)count, kTile);
            PSOPS_DO(make_map(x, &dw_sums, PSOPS_F32, x->at<void>(x->lay.dw_sums), c.padded, share_rows * x->lay.dw_most, c.padded, 32));
            P.columns = (int)c.padded;
            P.result_rows = (int)count;
            P.dw_share_rows = (int)share_rows;
            P.add = false;
            PSOPS_DO(product(x, kDwSums, tokens, ceil_div(count, kTile) * tiles_d * x->lay.dw_most, dlogits_across, hidden_across, dw_sums, P));
            PSOPS_DO(results<true>(x, x->at<float>(x->lay.dw_sums), (int)share_rows, (int)count, (uint16_t *)dw + first * dw_ld, dw_ld));
        } else if (dw != nullptr) {
            uint16_t *to = direct ? (uint16_t *)dw + first * dw_ld : x->at<uint16_t>(x->lay.dw);
            CUtensorMap dw_out;
            PSOPS_DO(make_map(x, &dw_out, type, to, direct ? x->cfg.dim : c.padded, count, direct ? dw_ld : c.padded, 32));
            P.columns = (int)c.padded;
            P.result_rows = (int)count;
            PSOPS_DO(product(x, tokens > kChainTokens ? kDwLong : kDw, tokens, ceil_div(count, kTile) * tiles_d, dlogits_across, hidden_across,
                             dw_out, P));
            if (!direct) {
                const int64_t grid = std::min<int64_t>(ceil_div(count, kCopyThreads / 32), (int64_t)x->sms * 8);
                PSOPS_DO(launch(x, "psops_xent_unpack_kernel", psops_xent_unpack_kernel, grid, kCopyThreads, 0, to, (int)c.padded, count,
                                (int)x->cfg.dim, (uint16_t *)dw + first * dw_ld, dw_ld));
            }
        }
    }
    if ((dh == nullptr || tokens == 0) && dw == nullptr) return PSOPS_OK;
    return results<false>(x, x->at<float>(x->lay.sums), 0, dh != nullptr ? (int)tokens : 0, dh, dh_ld, dw, dw_ld);
}

} // namespace

extern "C" {

size_t psops_xent_workspace_bytes(const psops_xent_config *cfg) { return config_ok(cfg) ? make_layout(cfg).total : 0; }

int psops_xent_create(psops_xent **out, const psops_xent_config *cfg, void *d_workspace, size_t workspace_bytes,
                      void *cuda_stream)
{
    if (out == nullptr) return PSOPS_EINVAL;
    *out = nullptr;
    if (!config_ok(cfg)) return PSOPS_EINVAL;
    const Layout lay = make_layout(cfg);
    if (d_workspace == nullptr || ((uintptr_t)d_workspace & 255u) || workspace_bytes < lay.total) return PSOPS_EWORKSPACE;
    psops_xent *x = new (std::nothrow) psops_xent();
    if (x == nullptr) return PSOPS_ENOMEM;
    x->cfg = *cfg;
    x->lay = lay;
    x->ws = (char *)d_workspace;
    x->stream = (cudaStream_t)cuda_stream;
    const int rc = psops_host::not_capturing(x);
    if (rc != PSOPS_OK) {
        delete x;
        return rc;
    }
    cudaError_t e = cudaGetDevice(&x->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&x->sms, cudaDevAttrMultiProcessorCount, x->device);
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    if (e == cudaSuccess)
        e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", (void **)&x->encode, 12000, cudaEnableDefault, &found);
    if (e == cudaSuccess && found != cudaDriverEntryPointSuccess) e = cudaErrorNotSupported;
    for (int job = kLoss; job <= kDwSums; ++job)
        for (int pair = 0; pair < 2 && e == cudaSuccess; ++pair)
            e = cudaFuncSetAttribute((const void *)product_of(x, job, pair != 0), cudaFuncAttributeMaxDynamicSharedMemorySize,
                                     job >= kDw || pair ? ProductShape<true>::kShared : ProductShape<false>::kShared);
    const bool half = cfg->type == PSOPS_F16;
    const void *heads[2] = {half ? (const void *)psops_xent_head_kernel<__half, false> : (const void *)psops_xent_head_kernel<__nv_bfloat16, false>,
                            half ? (const void *)psops_xent_head_kernel<__half, true> : (const void *)psops_xent_head_kernel<__nv_bfloat16, true>};
    for (const void *k : heads)
        if (e == cudaSuccess) e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeadShared);
    for (int few = 1; few <= kFewTokens; few *= 2)
        for (int aligned = 0; aligned < 2 && e == cudaSuccess; ++aligned)
            e = cudaFuncSetAttribute(half ? (const void *)few_kernel<__half>(few, aligned != 0) : (const void *)few_kernel<__nv_bfloat16>(few, aligned != 0),
                                     cudaFuncAttributeMaxDynamicSharedMemorySize, kFewShared);
    if (e == cudaSuccess) e = cudaMemsetAsync(x->control(), 0, sizeof(XentControl), x->stream);
    if (e != cudaSuccess) {
        delete x;
        return PSOPS_ECUDA;
    }
    *out = x;
    return PSOPS_OK;
}

int psops_xent_forward(psops_xent *x, const void *d_h, int64_t h_ld, const void *d_w, int64_t w_ld,
                       const int64_t *d_targets, int64_t tokens, int32_t reduction,
                       float *d_loss, float *d_rows, float *d_lse)
{
    if (x == nullptr || (reduction != PSOPS_MEAN && reduction != PSOPS_SUM)) return PSOPS_EINVAL;
    int rc = check_call(x, d_h, h_ld, d_w, w_ld, d_targets, tokens);
    if (rc != PSOPS_OK) return rc;
    if (((uintptr_t)d_loss | (uintptr_t)d_rows | (uintptr_t)d_lse) & 3u) return PSOPS_EALIGN;
    OnDevice guard(x);
    const bool half = x->cfg.type == PSOPS_F16;
    if (is_head(x->cfg.vocab, x->cfg.dim, tokens, false)) {
        HeadParams H = head_params(x, d_h, h_ld, d_w, w_ld, d_targets, tokens, reduction);
        H.loss = d_loss;
        H.rows = d_rows;
        H.lse_out = d_lse;
        return half ? forward_head<__half>(x, H) : forward_head<__nv_bfloat16>(x, H);
    }
    if (is_few(tokens, x->cfg.dim) && few_loss_pays(x->cfg.dim, x->cfg.vocab)) {
        FewParams F{};
        F.h = (const uint16_t *)d_h; F.h_ld = h_ld; F.h_aligned = aligned16(d_h, h_ld);
        F.w = (const uint16_t *)d_w; F.w_ld = w_ld; F.w_aligned = aligned16(d_w, w_ld);
        F.targets = (const long long *)d_targets;
        F.tokens = (int)tokens; F.dim = (int)x->cfg.dim; F.vocab = (int)x->cfg.vocab; F.reduction = reduction;
        F.control = x->control();
        F.stats = x->at<float2>(x->lay.stats);
        F.label_logit = x->at<float>(x->lay.label_logit);
        F.loss = d_loss; F.rows = d_rows; F.lse_out = d_lse;
        return half ? forward_few<__half>(x, F) : forward_few<__nv_bfloat16>(x, F);
    }
    IndexParams P{};
    P.targets = (const long long *)d_targets;
    P.rows_out = d_rows;
    P.lse_out = d_lse;
    P.tokens = (int)tokens;
    rc = gather(x, P, d_h, h_ld);
    if (rc != PSOPS_OK) return rc;
    JoinParams J{};
    J.rows_out = d_rows;
    J.lse_out = d_lse;
    J.loss = d_loss;
    J.reduction = reduction;
    return forward(x, d_w, w_ld, tokens, J);
}

int psops_xent_backward(psops_xent *x, const void *d_h, int64_t h_ld, const void *d_w, int64_t w_ld,
                        const int64_t *d_targets, int64_t tokens, const float *d_lse, const float *d_rows,
                        const float *d_grad, int32_t reduction, void *d_dh, int64_t dh_ld, void *d_dw, int64_t dw_ld)
{
    if (x == nullptr || reduction < PSOPS_MEAN || reduction > PSOPS_PER_TOKEN) return PSOPS_EINVAL;
    if (!(x->cfg.flags & PSOPS_XENT_GRADS)) return PSOPS_ESTATE;
    int rc = check_call(x, d_h, h_ld, d_w, w_ld, d_targets, tokens);
    if (rc == PSOPS_OK && d_dh != nullptr) rc = check_matrix(d_dh, dh_ld, tokens, x->cfg.dim);
    if (rc == PSOPS_OK && d_dw != nullptr) rc = check_matrix(d_dw, dw_ld, x->cfg.vocab, x->cfg.dim);
    if (rc != PSOPS_OK) return rc;
    if (d_grad == nullptr || (tokens > 0 && d_lse == nullptr)) return PSOPS_EINVAL;
    if (((uintptr_t)d_lse | (uintptr_t)d_rows | (uintptr_t)d_grad) & 3u) return PSOPS_EALIGN;
    if (d_dw != nullptr && !x->lay.staged && !aligned16(d_dw, dw_ld)) return PSOPS_EALIGN;
    OnDevice guard(x);
    if (is_head(x->cfg.vocab, x->cfg.dim, tokens, true)) {
        HeadParams H = head_params(x, d_h, h_ld, d_w, w_ld, d_targets, tokens, reduction);
        H.lse = d_lse;
        H.known_rows = d_rows;
        H.grad = d_grad;
        H.dlogits = x->at<float>(x->lay.dlogits);
        H.dh = d_dh;
        H.dh_ld = dh_ld;
        return x->cfg.type == PSOPS_F16 ? backward_head<__half>(x, H, d_dw, dw_ld) : backward_head<__nv_bfloat16>(x, H, d_dw, dw_ld);
    }
    const bool aligned = x->cfg.dim % 8 == 0 && aligned16(d_w, w_ld) && (d_dw == nullptr || aligned16(d_dw, dw_ld));
    if (is_few(tokens, x->cfg.dim) && x->cfg.dim <= kFewGradDim && few_grads_pay(tokens, x->cfg.dim, x->cfg.vocab, aligned)) {
        FewGradParams F{};
        F.h = (const uint16_t *)d_h; F.h_ld = h_ld; F.h_aligned = aligned16(d_h, h_ld);
        F.w = (const uint16_t *)d_w; F.w_ld = w_ld;
        F.targets = (const long long *)d_targets;
        F.tokens = (int)tokens; F.dim = (int)x->cfg.dim; F.vocab = (int)x->cfg.vocab; F.reduction = reduction;
        F.team = few_team(x->cfg.dim);
        F.lse = d_lse; F.known_rows = d_rows; F.grad = d_grad;
        F.parts = x->at<float>(x->lay.sums);
        F.padded = (int)x->lay.padded;
        F.want_dh = d_dh != nullptr;
        F.dw = (uint16_t *)d_dw; F.dw_ld = dw_ld;
        return x->cfg.type == PSOPS_F16 ? backward_few<__half>(x, F, aligned, d_dh, dh_ld) : backward_few<__nv_bfloat16>(x, F, aligned, d_dh, dh_ld);
    }
    IndexParams P{};
    P.targets = (const long long *)d_targets;
    P.grad = d_grad;
    P.lse = d_lse;
    P.rows = d_rows;
    P.tokens = (int)tokens;
    P.reduction = reduction;
    rc = gather(x, P, d_h, h_ld);
    if (rc != PSOPS_OK) return rc;
    return backward(x, d_w, w_ld, tokens, d_dh, dh_ld, d_dw, dw_ld);
}

int psops_xent_set_stream(psops_xent *x, void *cuda_stream) { return psops_host::set_stream(x, cuda_stream); }
int64_t psops_xent_launch_count(const psops_xent *x) { return x ? x->launches : 0; }
const char *psops_xent_last_error(const psops_xent *x) { return x ? x->err : ""; }

int psops_xent_destroy(psops_xent *x)
{
    if (x == nullptr) return PSOPS_EINVAL;
    OnDevice guard(x);
    const int rc = cudaStreamSynchronize(x->stream) == cudaSuccess ? PSOPS_OK : PSOPS_ECUDA;
    delete x;
    return rc;
}

} // extern "C"
