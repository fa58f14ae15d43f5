// psops_xent.cu -- C ABI and host side of the linear cross entropy (kernels:
// psops_xent_kernels.cuh).

#include "psops.h"

#include <cuda_runtime.h>

#include <algorithm>
#include <new>

#include "psops_host.cuh"
#include "psops_xent_kernels.cuh"

using psops_host::Base;
using psops_host::OnDevice;
using psops_host::ceil_div;
using psops_host::round_up;

namespace {

// Bytes that the logits' gradients of one piece of the vocabulary may take.
constexpr int64_t kPieceBytes = 512ll << 20;
constexpr int64_t kMinPiece = 2048;

bool config_ok(const psops_xent_config *c)
{
    return c != nullptr && c->max_tokens >= 1 && c->max_tokens <= (1 << 24) && c->dim >= 1 && c->dim <= (1 << 20) &&
           c->vocab >= 1 && c->vocab <= (1ll << 31) - (1 << 16) && (c->type == PSOPS_F16 || c->type == PSOPS_BF16) &&
           (c->flags & ~(PSOPS_XENT_GRADS | PSOPS_XENT_STAGED)) == 0;
}

struct Layout {
    int64_t rows;                               // compact rows, whole tiles
    int64_t padded;                             // dim, a multiple of 8
    int64_t piece;                              // vocabulary entries of a piece, a multiple of the tile
    bool staged;                                // w and dw may pass through the workspace
    int64_t parts;                              // softmax statistics per row
    size_t control, row_of, compact_of, label, row_scale, row_lse, label_logit, partials, hidden, stats, w, dw, dlogits, sums, total;
};

Layout make_layout(const psops_xent_config *c)
{
    Layout L{};
    L.rows = (int64_t)round_up((size_t)c->max_tokens, kTileRows);
    L.padded = (int64_t)round_up((size_t)c->dim, 8);
    const int64_t whole = (int64_t)round_up((size_t)c->vocab, kTileCols);
    L.piece = std::min(whole, std::max(kMinPiece, kPieceBytes / (2 * L.rows) / kTileCols * kTileCols));
    L.staged = c->dim % 8 != 0 || (c->flags & PSOPS_XENT_STAGED) != 0;
    L.parts = ceil_div(c->vocab, kSimple);
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
    L.label_logit = take(4 * n);
    L.partials = take(8 * (n / kJoinRows));
    L.hidden = take(2 * n * (size_t)L.padded);
    L.stats = take(8 * n * (size_t)L.parts);
    if (L.staged) L.w = take(2 * (size_t)L.piece * (size_t)L.padded);
    if (c->flags & PSOPS_XENT_GRADS) {
        if (L.staged) L.dw = take(2 * (size_t)L.piece * (size_t)L.padded);
        L.dlogits = take(2 * n * (size_t)L.piece);
        L.sums = take(4 * n * (size_t)L.padded);
    }
    L.total = at;
    return L;
}

} // namespace

struct psops_xent : Base {
    psops_xent_config cfg;
    Layout lay;
    char *ws;
    template <class T> T *at(size_t offset) const { return (T *)(ws + offset); }
    XentControl *control() const { return at<XentControl>(lay.control); }
};

namespace {

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
    P.vocab = (int)x->cfg.vocab;
    P.headroom = x->cfg.type == PSOPS_F16 ? 32768.0f : 1.0f;
    psops_xent_index_kernel<<<1, kIndexThreads, 0, x->stream>>>(P);
    int rc = x->launched("psops_xent_index_kernel");
    if (rc != PSOPS_OK) return rc;
    const int64_t rows = (int64_t)round_up((size_t)std::max<int64_t>(1, P.tokens), kTileRows);
    const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(rows, kCopyThreads / 32), (int64_t)x->sms * 8);
    psops_xent_gather_kernel<<<grid, kCopyThreads, 0, x->stream>>>((const uint16_t *)h, h_ld, (int)x->cfg.dim, (int)x->lay.padded,
                                                                  aligned16(h, h_ld), P.control, P.row_of,
                                                                  x->at<uint16_t>(x->lay.hidden));
    return x->launched("psops_xent_gather_kernel");
}

// The rows of w of one piece as the products read them: in place, or packed into the workspace.
int piece_of_w(psops_xent *x, const void *w, int64_t w_ld, int64_t first, int64_t count, const void **out, int64_t *out_ld)
{
    const uint16_t *from = (const uint16_t *)w + first * w_ld;
    if (x->cfg.dim % 8 == 0 && aligned16(w, w_ld)) {
        *out = from;
        *out_ld = w_ld;
        return PSOPS_OK;
    }
    uint16_t *to = x->at<uint16_t>(x->lay.w);
    const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(count, kCopyThreads / 32), (int64_t)x->sms * 8);
    psops_xent_pack_kernel<<<grid, kCopyThreads, 0, x->stream>>>(from, w_ld, count, (int)x->cfg.dim, (int)x->lay.padded, to);
    *out = to;
    *out_ld = x->lay.padded;
    return x->launched("psops_xent_pack_kernel");
}

LogitsParams logits_params(const psops_xent *x)
{
    LogitsParams P{};
    P.h = x->at<void>(x->lay.hidden);
    P.h_ld = (int)x->lay.padded;
    P.dim = (int)x->lay.padded;
    P.control = x->control();
    P.label = x->at<int>(x->lay.label);
    P.stats = x->at<float2>(x->lay.stats);
    P.stats_ld = x->lay.rows;
    P.label_logit = x->at<float>(x->lay.label_logit);
    P.row_lse = x->at<float>(x->lay.row_lse);
    P.row_scale = x->at<float>(x->lay.row_scale);
    P.dlogits = x->at<void>(x->lay.dlogits);
    P.dlogits_ld = x->lay.piece;
    return P;
}

template <class T>
int forward(psops_xent *x, const void *w, int64_t w_ld, int64_t tokens, JoinParams J)
{
    const unsigned tiles_m = (unsigned)(round_up((size_t)std::max<int64_t>(1, tokens), kTileRows) / kSimple);
    for (int64_t first = 0; first < x->cfg.vocab; first += x->lay.piece) {
        LogitsParams P = logits_params(x);
        const int64_t count = std::min(x->lay.piece, x->cfg.vocab - first);
        const int rc = piece_of_w(x, w, w_ld, first, count, &P.w, &P.w_ld);
        if (rc != PSOPS_OK) return rc;
        P.first = (int)first;
        P.count = (int)count;
        psops_xent_logits_kernel<T, false><<<dim3((unsigned)ceil_div(count, kSimple), tiles_m), kSimpleThreads, 0, x->stream>>>(P);
        if (x->launched("psops_xent_logits_kernel") != PSOPS_OK) return PSOPS_ECUDA;
    }
    J.stats = x->at<float2>(x->lay.stats);
    J.stats_ld = x->lay.rows;
    J.parts = (int)x->lay.parts;
    J.control = x->control();
    J.row_of = x->at<int>(x->lay.row_of);
    J.label_logit = x->at<float>(x->lay.label_logit);
    J.partials = x->at<double>(x->lay.partials);
    psops_xent_join_kernel<<<(unsigned)ceil_div(std::max<int64_t>(1, tokens), kJoinRows), kJoinRows * kJoinParts, 0, x->stream>>>(J);
    return x->launched("psops_xent_join_kernel");
}

template <class T>
int backward(psops_xent *x, const void *w, int64_t w_ld, int64_t tokens, void *dh, int64_t dh_ld, void *dw, int64_t dw_ld)
{
    const unsigned tiles_m = (unsigned)(round_up((size_t)std::max<int64_t>(1, tokens), kTileRows) / kSimple);
    const unsigned tiles_d = (unsigned)ceil_div(x->cfg.dim, kSimple);
    const bool direct = x->cfg.dim % 8 == 0 && aligned16(dw, dw_ld);
    int rc;
    for (int64_t first = 0; first < x->cfg.vocab; first += x->lay.piece) {
        LogitsParams P = logits_params(x);
        const int64_t count = std::min(x->lay.piece, x->cfg.vocab - first);
        rc = piece_of_w(x, w, w_ld, first, count, &P.w, &P.w_ld);
        if (rc != PSOPS_OK) return rc;
        P.first = (int)first;
        P.count = (int)count;
        psops_xent_logits_kernel<T, true><<<dim3((unsigned)ceil_div(count, kSimple), tiles_m), kSimpleThreads, 0, x->stream>>>(P);
        if (x->launched("psops_xent_logits_kernel") != PSOPS_OK) return PSOPS_ECUDA;
        if (dh != nullptr) {
            DhParams Q{};
            Q.dlogits = P.dlogits; Q.dlogits_ld = P.dlogits_ld; Q.w = P.w; Q.w_ld = P.w_ld;
            Q.dim = (int)x->lay.padded; Q.count = (int)count; Q.add = first > 0; Q.control = x->control();
            Q.sums = x->at<float>(x->lay.sums); Q.sums_ld = x->lay.padded;
            psops_xent_dh_kernel<T><<<dim3(tiles_d, tiles_m), kSimpleThreads, 0, x->stream>>>(Q);
            if (x->launched("psops_xent_dh_kernel") != PSOPS_OK) return PSOPS_ECUDA;
        }
        if (dw != nullptr) {
            DwParams Q{};
            Q.dlogits = P.dlogits; Q.dlogits_ld = P.dlogits_ld; Q.h = P.h; Q.h_ld = P.h_ld;
            Q.dim = (int)x->lay.padded; Q.count = (int)count; Q.control = x->control();
            Q.dw = direct ? (void *)((uint16_t *)dw + first * dw_ld) : x->at<void>(x->lay.dw);
            Q.dw_ld = direct ? dw_ld : x->lay.padded;
            psops_xent_dw_kernel<T><<<dim3(tiles_d, (unsigned)ceil_div(count, kSimple)), kSimpleThreads, 0, x->stream>>>(Q);
            if (x->launched("psops_xent_dw_kernel") != PSOPS_OK) return PSOPS_ECUDA;
            if (!direct) {
                const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(count, kCopyThreads / 32), (int64_t)x->sms * 8);
                psops_xent_unpack_kernel<<<grid, kCopyThreads, 0, x->stream>>>(x->at<uint16_t>(x->lay.dw), (int)x->lay.padded, count,
                                                                              (int)x->cfg.dim, (uint16_t *)dw + first * dw_ld, dw_ld);
                if (x->launched("psops_xent_unpack_kernel") != PSOPS_OK) return PSOPS_ECUDA;
            }
        }
    }
    if (dh != nullptr && tokens > 0) {
        const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(tokens, kCopyThreads / 32), (int64_t)x->sms * 8);
        psops_xent_dh_out_kernel<T><<<grid, kCopyThreads, 0, x->stream>>>(x->at<float>(x->lay.sums), x->lay.padded, x->control(),
                                                                         x->at<int>(x->lay.compact_of), (int)tokens,
                                                                         (int)x->cfg.dim, (T *)dh, dh_ld);
        rc = x->launched("psops_xent_dh_out_kernel");
        if (rc != PSOPS_OK) return rc;
    }
    return PSOPS_OK;
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
    cudaError_t e = cudaGetDevice(&x->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&x->sms, cudaDevAttrMultiProcessorCount, x->device);
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
    return x->cfg.type == PSOPS_F16 ? forward<__half>(x, d_w, w_ld, tokens, J) : forward<__nv_bfloat16>(x, d_w, w_ld, tokens, J);
}

int psops_xent_backward(psops_xent *x, const void *d_h, int64_t h_ld, const void *d_w, int64_t w_ld,
                        const int64_t *d_targets, int64_t tokens, const float *d_lse, const float *d_grad, int32_t reduction,
                        void *d_dh, int64_t dh_ld, void *d_dw, int64_t dw_ld)
{
    if (x == nullptr || reduction < PSOPS_MEAN || reduction > PSOPS_PER_TOKEN) return PSOPS_EINVAL;
    if (!(x->cfg.flags & PSOPS_XENT_GRADS)) return PSOPS_ESTATE;
    int rc = check_call(x, d_h, h_ld, d_w, w_ld, d_targets, tokens);
    if (rc == PSOPS_OK && d_dh != nullptr) rc = check_matrix(d_dh, dh_ld, tokens, x->cfg.dim);
    if (rc == PSOPS_OK && d_dw != nullptr) rc = check_matrix(d_dw, dw_ld, x->cfg.vocab, x->cfg.dim);
    if (rc != PSOPS_OK) return rc;
    if (d_grad == nullptr || (tokens > 0 && d_lse == nullptr)) return PSOPS_EINVAL;
    if (((uintptr_t)d_lse | (uintptr_t)d_grad) & 3u) return PSOPS_EALIGN;
    if (d_dw != nullptr && !x->lay.staged && !aligned16(d_dw, dw_ld)) return PSOPS_EALIGN;
    OnDevice guard(x);
    IndexParams P{};
    P.targets = (const long long *)d_targets;
    P.grad = d_grad;
    P.lse = d_lse;
    P.tokens = (int)tokens;
    P.reduction = reduction;
    rc = gather(x, P, d_h, h_ld);
    if (rc != PSOPS_OK) return rc;
    return x->cfg.type == PSOPS_F16 ? backward<__half>(x, d_w, w_ld, tokens, d_dh, dh_ld, d_dw, dw_ld)
                                    : backward<__nv_bfloat16>(x, d_w, w_ld, tokens, d_dh, dh_ld, d_dw, dw_ld);
}

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
