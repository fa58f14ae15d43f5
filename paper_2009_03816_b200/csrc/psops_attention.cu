// psops_attention.cu -- C entries of causal attention over packed sequences.
#include "psops.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstring>
#include <new>

#include "psops_attention_kernels.cuh"
#include "psops_host.cuh"

using namespace psops_attention_k;
using psops_host::ceil_div;
using psops_host::launch;
using psops_host::OnDevice;
using psops_host::round_up;

namespace {

constexpr int kMostFillBlocks = 592;             // blocks of the preparing kernel beside the list's

constexpr int kMostCtas = 320;                   // two for each SM forward; half as many, with twice the room, backward
constexpr int64_t kJoinWithin = 8192;            // so few sums of dbias are joined by the last CTA (26 a thread, some 2 us), more by a kernel
                                                 // of its own (a launch, 4 us)

struct Layout {
    int64_t capacity;                            // tiles of a call at most
    size_t count, ticket, items, fold, arrived, used, norms, delta, levels, beside, partials, total;
};

using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                            const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

} // namespace

struct psops_attention : psops_host::Base {
    psops_attention_config cfg{};
    Bias bias{};                                 // without the table's address
    Layout lay{};
    char *ws = nullptr;
    Encode encode = nullptr;

    template <class T>
    T *at(size_t offset) const { return (T *)(ws + offset); }
};

namespace {

#define PSOPS_DO(call)                     \
    do {                                   \
        const int rc_ = (call);            \
        if (rc_ != PSOPS_OK) return rc_;   \
    } while (0)

bool config_ok(const psops_attention_config *c)
{
    if (c == nullptr || c->max_tokens < 1 || c->max_tokens > ((int64_t)1 << 24) || c->max_sequences < 1 || c->max_sequences > (1 << 24) ||
        c->heads < 1 || c->heads > 1024 || c->kv_heads < 1 || c->heads % c->kv_heads != 0 || c->dim < 8 || c->dim > kMostDim || c->dim % 8 != 0 ||
        (c->type != PSOPS_F16 && c->type != PSOPS_BF16) || (c->flags & ~PSOPS_ATTENTION_GRADS) || !(c->scale > 0.0f) || !(c->scale < INFINITY) ||
        c->buckets < 0 || c->buckets > kMostBuckets)
        return false;
    if (((c->max_tokens / kTile) + c->max_sequences + 1) * c->heads > INT32_MAX) return false;
    if (c->buckets == 0) return true;
    if (c->first == nullptr || c->first[0] != 0) return false;
    for (int b = 1; b < c->buckets; ++b)
        if (c->first[b] <= c->first[b - 1] || c->first[b] > kMostDistance) return false;
    return true;
}

Layout make_layout(const psops_attention_config *c)
{
    Layout l{};
    l.capacity = c->max_tokens / kTile + c->max_sequences + 1;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += round_up(bytes, 256);
        return here;
    };
    l.count = take(sizeof(int));
    l.ticket = take(sizeof(int));
    l.items = take((size_t)l.capacity * sizeof(Item));
    if (c->buckets > 0) l.levels = take(sizeof(int));
    const bool grads = c->flags & PSOPS_ATTENTION_GRADS;
    const bool grouped = grads && c->heads > c->kv_heads;
    if (c->max_tokens * (grads ? c->heads / c->kv_heads : 1) > (int64_t)kChain * kTile)
        l.fold = take((size_t)kMostCtas * kFoldFloats * sizeof(float));
    else if (grouped)
        l.fold = take((size_t)std::min<int64_t>(kMostCtas, 2 * l.capacity * c->heads) * kFoldFloats * sizeof(float));
    if (grouped) l.arrived = take((size_t)kMostCtas * 2 * sizeof(int));
    if (grads) {
        l.used = take((size_t)l.capacity * sizeof(int));
        l.norms = take(kMostFillBlocks * sizeof(float2));
        l.delta = take((size_t)c->max_tokens * c->heads * sizeof(float));
        l.partials = take((size_t)l.capacity * c->heads * c->buckets * sizeof(float));
        if (c->buckets > 0) l.beside = take((size_t)c->max_tokens * c->heads * sizeof(float));
    }
    l.total = at;
    return l;
}

struct Call {
    int64_t tokens;
    int32_t sequences;
    const int32_t *offsets;
};

// A caller's tensor: strides in elements, all rows 16-byte aligned; in one that is written no two of them overlap.
int check_heads(const psops_attention *a, const psops_heads *h, int64_t tokens, int heads, bool written = false)
{
    if (h == nullptr || (tokens > 0 && h->p == nullptr)) return PSOPS_EINVAL;
    const int64_t dim = a->cfg.dim;
    if ((tokens > 1 && h->token_stride < dim) || (heads > 1 && h->head_stride < dim)) return PSOPS_EINVAL;
    const int64_t most = (int64_t)1 << 38;
    if (h->token_stride > most || h->head_stride > most) return PSOPS_EINVAL;
    if (written && tokens > 1 && heads > 1 && h->token_stride < (heads - 1) * h->head_stride + dim &&
        h->head_stride < (tokens - 1) * h->token_stride + dim)
        return PSOPS_EINVAL;
    if (((uintptr_t)h->p & 15u) || (tokens > 1 && h->token_stride % 8) || (heads > 1 && h->head_stride % 8)) return PSOPS_EALIGN;
    return PSOPS_OK;
}

// With strides that a tensor map takes also where there is only one token or head.
Heads heads_of(const psops_attention *a, const psops_heads *h, int64_t tokens, int heads)
{
    Heads r{h->p, h->token_stride, h->head_stride};
    if (heads == 1) r.head = a->cfg.dim;
    if (tokens <= 1) r.token = round_up((size_t)(heads * r.head), 8);
    return r;
}

int make_map(psops_attention *a, CUtensorMap *map, const Heads &h, int64_t tokens, int heads)
{
    const cuuint64_t size[3] = {(cuuint64_t)a->cfg.dim, (cuuint64_t)heads, (cuuint64_t)tokens};
    const cuuint64_t stride[2] = {(cuuint64_t)(h.head * 2), (cuuint64_t)(h.token * 2)};
    const cuuint32_t box[3] = {64, 1, kTile}, step[3] = {1, 1, 1};
    const CUtensorMapDataType kind = a->cfg.type == PSOPS_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    const CUresult r = a->encode(map, kind, 3, h.p, size, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                 CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r == CUDA_SUCCESS) return PSOPS_OK;
    std::snprintf(a->err, sizeof(a->err), "cuTensorMapEncodeTiled: error %d", (int)r);
    return PSOPS_ECUDA;
}

int check_call(const psops_attention *a, const psops_heads *q, const psops_heads *k, const psops_heads *v, const int32_t *offsets,
               int32_t sequences, int64_t tokens, const void *bias, int32_t bias_type)
{
    if (tokens < 0 || tokens > a->cfg.max_tokens || sequences < 0 || sequences > a->cfg.max_sequences) return PSOPS_EINVAL;
    if (offsets == nullptr && sequences > 0) return PSOPS_EINVAL;
    if ((a->cfg.buckets > 0) != (bias != nullptr)) return PSOPS_EINVAL;
    if (bias != nullptr && bias_type != PSOPS_F32 && bias_type != a->cfg.type) return PSOPS_EINVAL;
    if (((uintptr_t)offsets & 3u) || ((uintptr_t)bias & (bias_type == PSOPS_F32 ? 3u : 1u))) return PSOPS_EALIGN;
    PSOPS_DO(check_heads(a, q, tokens, a->cfg.heads));
    PSOPS_DO(check_heads(a, k, tokens, a->cfg.kv_heads));
    return check_heads(a, v, tokens, a->cfg.kv_heads);
}

PrepParams prepare_params(const psops_attention *a, const Call &c)
{
    PrepParams P{};
    P.offsets = c.offsets;
    P.sequences = c.sequences;
    P.tokens = (int)c.tokens;
    P.capacity = (int)(c.tokens / kTile + c.sequences + 1);
    P.items = a->at<Item>(a->lay.items);
    P.count = a->at<int>(a->lay.count);
    P.heads = a->cfg.heads;
    P.kv_heads = a->cfg.kv_heads;
    P.dim = a->cfg.dim;
    return P;
}

int prepare(psops_attention *a, PrepParams &P, int64_t blocks)
{
    P.blocks = (int)blocks;
    if (P.beside != nullptr) blocks += std::min<int64_t>(2 * a->sms, ceil_div((int64_t)P.tokens * P.heads, kPrepThreads / 16));
    else if (P.levels != nullptr) blocks += 1;
    return launch(a, "psops_attention_prepare_kernel",
                  a->cfg.type == PSOPS_F16 ? psops_attention_prepare_kernel<__half> : psops_attention_prepare_kernel<__nv_bfloat16>,
                  dim3((unsigned)(1 + blocks)), kPrepThreads, 0, 1, P);
}

using ForwardKernel = void (*)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const ForwardParams);
using BackwardKernel = void (*)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const BackwardParams);

template <class T>
ForwardKernel forward_kernel(bool wide, bool bias)
{
    return wide ? (bias ? psops_attention_forward_kernel<T, 2, true> : psops_attention_forward_kernel<T, 2, false>)
                : (bias ? psops_attention_forward_kernel<T, 1, true> : psops_attention_forward_kernel<T, 1, false>);
}
ForwardKernel forward_kernel(const psops_attention *a, size_t *shared)
{
    const bool wide = a->cfg.dim > 64, bias = a->cfg.buckets > 0;
    *shared = wide ? forward_shared<2>() : forward_shared<1>();
    return a->cfg.type == PSOPS_F16 ? forward_kernel<__half>(wide, bias) : forward_kernel<__nv_bfloat16>(wide, bias);
}
template <class T>
BackwardKernel backward_kernel(bool wide, bool bias)
{
    return wide ? (bias ? psops_attention_backward_kernel<T, 2, true> : psops_attention_backward_kernel<T, 2, false>)
                : (bias ? psops_attention_backward_kernel<T, 1, true> : psops_attention_backward_kernel<T, 1, false>);
}
BackwardKernel backward_kernel(const psops_attention *a, size_t *shared)
{
    const bool wide = a->cfg.dim > 64, bias = a->cfg.buckets > 0;
    *shared = wide ? (bias ? backward_shared<2, true>() : backward_shared<2, false>()) : (bias ? backward_shared<1, true>() : backward_shared<1, false>());
    return a->cfg.type == PSOPS_F16 ? backward_kernel<__half>(wide, bias) : backward_kernel<__nv_bfloat16>(wide, bias);
}

Divisor divisor(uint32_t by)
{
    uint32_t shift = 0;
    while (((uint32_t)1 << shift) < by) ++shift;
    return Divisor{by, (uint32_t)((((uint64_t)1 << (31 + shift)) + by - 1) / by), 31 + shift};
}

// As many CTAs as run at once, or as there can be works: tiles with all of `heads` heads.
dim3 works_grid(const psops_attention *a, const PrepParams &L, int heads, int to_an_sm)
{
    return dim3((unsigned)std::min<int64_t>((int64_t)(L.capacity - 1) * heads, std::min(a->sms * to_an_sm, kMostCtas / 2 * to_an_sm)));
}

Bias bias_of(const psops_attention *a, const void *bias, int32_t bias_type)
{
    Bias b = a->bias;
    b.p = bias;
    b.fp32 = bias_type == PSOPS_F32;
    return b;
}

} // namespace

extern "C" {

size_t psops_attention_workspace_bytes(const psops_attention_config *cfg) { return config_ok(cfg) ? make_layout(cfg).total : 0; }

int psops_attention_create(psops_attention **out, const psops_attention_config *cfg, void *d_workspace, size_t workspace_bytes,
                           void *cuda_stream)
{
    if (out == nullptr) return PSOPS_EINVAL;
    *out = nullptr;
    if (!config_ok(cfg)) return PSOPS_EINVAL;
    const Layout lay = make_layout(cfg);
    if (d_workspace == nullptr || ((uintptr_t)d_workspace & 255u) || workspace_bytes < lay.total) return PSOPS_EWORKSPACE;
    psops_attention *a = new (std::nothrow) psops_attention();
    if (a == nullptr) return PSOPS_ENOMEM;
    a->cfg = *cfg;
    a->cfg.first = nullptr;                      // copied:
    a->bias.buckets = cfg->buckets;
    for (int b = 0; b < cfg->buckets; ++b) a->bias.first[b] = cfg->first[b];
    a->bias.last = cfg->buckets > 0 ? cfg->first[cfg->buckets - 1] : 0;
    a->lay = lay;
    a->ws = (char *)d_workspace;
    a->stream = (cudaStream_t)cuda_stream;
    const int rc = psops_host::not_capturing(a);
    if (rc != PSOPS_OK) {
        delete a;
        return rc;
    }
    cudaError_t e = cudaGetDevice(&a->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&a->sms, cudaDevAttrMultiProcessorCount, a->device);
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    if (e == cudaSuccess)
        e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", (void **)&a->encode, 12000, cudaEnableDefault, &found);
    if (e == cudaSuccess && found != cudaDriverEntryPointSuccess) e = cudaErrorNotSupported;
    size_t shared = 0;
    const void *kernel = (const void *)forward_kernel(a, &shared);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shared);
    kernel = (const void *)backward_kernel(a, &shared);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shared);
    if (e != cudaSuccess) {
        delete a;
        return PSOPS_ECUDA;
    }
    *out = a;
    return PSOPS_OK;
}

int psops_attention_forward(psops_attention *a, const psops_heads *q, const psops_heads *k, const psops_heads *v, const int32_t *d_offsets,
                            int32_t sequences, int64_t tokens, const void *d_bias, int32_t bias_type, const psops_heads *out, float *d_lse,
                            int32_t zero_rest)
{
    if (a == nullptr) return PSOPS_EINVAL;
    PSOPS_DO(check_call(a, q, k, v, d_offsets, sequences, tokens, d_bias, bias_type));
    PSOPS_DO(check_heads(a, out, tokens, a->cfg.heads, true));
    if (tokens > 0 && d_lse == nullptr) return PSOPS_EINVAL;
    if ((uintptr_t)d_lse & 3u) return PSOPS_EALIGN;
    if (tokens == 0) return PSOPS_OK;
    OnDevice guard(a);
    const int H = a->cfg.heads, G = a->cfg.kv_heads;
    const Call c{tokens, sequences, d_offsets};
    PrepParams L = prepare_params(a, c);
    const Heads O = heads_of(a, out, tokens, H);
    if (zero_rest) {
        L.fill = 1;
        L.rest[0] = O;
        L.rest_heads[0] = H;
        L.rest_lse = d_lse;
    }
    if (a->cfg.buckets > 0) {
        L.levels = a->at<int>(a->lay.levels);
        L.bias = bias_of(a, d_bias, bias_type);
    }
    // no more tiles than CTAs run at once: they need no list (short batches, where a launch counts)
    const bool own = sequences > 0 && (L.capacity - 1) * H <= std::min(2 * a->sms, kMostCtas);
    if (!own) PSOPS_DO(prepare(a, L, zero_rest ? std::min<int64_t>(a->sms, ceil_div(tokens * H * (a->cfg.dim / 8), kPrepThreads)) : 0));
    if (sequences == 0) return PSOPS_OK;
    CUtensorMap mq, mk, mv;
    const Heads V = heads_of(a, v, tokens, G);
    PSOPS_DO(make_map(a, &mq, heads_of(a, q, tokens, H), tokens, H));
    PSOPS_DO(make_map(a, &mk, heads_of(a, k, tokens, G), tokens, G));
    PSOPS_DO(make_map(a, &mv, V, tokens, G));
    ForwardParams P{};
    P.items = L.items;
    P.count = L.count;
    P.tokens = (int)tokens;
    P.heads = H;
    P.by_heads = divisor(H);
    P.by_group = divisor(H / G);
    P.dim = a->cfg.dim;
    P.scale2 = a->cfg.scale * kLog2e;
    P.out = O;
    P.v = V;
    P.lse = d_lse;
    P.bias = bias_of(a, d_bias, bias_type);
    P.levels = L.levels;
    P.fold = a->at<float>(a->lay.fold);
    P.own = own;
    P.prep = L;
    size_t shared;
    ForwardKernel kernel = forward_kernel(a, &shared);
    return launch(a, "psops_attention_forward_kernel", kernel, works_grid(a, L, H, 2), kForwardThreads, shared, 1, mq, mk, mv, P);
}

int psops_attention_backward(psops_attention *a, const psops_heads *q, const psops_heads *k, const psops_heads *v, const int32_t *d_offsets,
                             int32_t sequences, int64_t tokens, const void *d_bias, int32_t bias_type, const psops_heads *out,
                             const float *d_lse, const psops_heads *grad, const psops_heads *dq, const psops_heads *dk, const psops_heads *dv,
                             void *d_dbias, int32_t zero_rest)
{
    if (a == nullptr) return PSOPS_EINVAL;
    if (!(a->cfg.flags & PSOPS_ATTENTION_GRADS)) return PSOPS_ESTATE;
    PSOPS_DO(check_call(a, q, k, v, d_offsets, sequences, tokens, d_bias, bias_type));
    const int H = a->cfg.heads, G = a->cfg.kv_heads;
    PSOPS_DO(check_heads(a, out, tokens, H));
    PSOPS_DO(check_heads(a, grad, tokens, H));
    if (dq != nullptr) PSOPS_DO(check_heads(a, dq, tokens, H, true));
    if (dk != nullptr) PSOPS_DO(check_heads(a, dk, tokens, G, true));
    if (dv != nullptr) PSOPS_DO(check_heads(a, dv, tokens, G, true));
    if ((tokens > 0 && d_lse == nullptr) || (d_dbias != nullptr && d_bias == nullptr)) return PSOPS_EINVAL;
    if (((uintptr_t)d_lse & 3u) || ((uintptr_t)d_dbias & (bias_type == PSOPS_F32 ? 3u : 1u))) return PSOPS_EALIGN;
    OnDevice guard(a);
    const Call c{tokens, sequences, d_offsets};
    PrepParams L = prepare_params(a, c);
    L.used = a->at<int>(a->lay.used);
    if (tokens > 0) {
        L.out = heads_of(a, out, tokens, H);
        L.grad = heads_of(a, grad, tokens, H);
        L.v = heads_of(a, v, tokens, G);
        L.delta = a->at<float>(a->lay.delta);
        if (a->cfg.type == PSOPS_F16) L.norms = a->at<float2>(a->lay.norms);
        if (a->cfg.buckets > 0) {
            L.levels = a->at<int>(a->lay.levels);
            L.bias = bias_of(a, d_bias, bias_type);
            L.beside = a->at<float>(a->lay.beside);
            L.lse = d_lse;
            L.q = heads_of(a, q, tokens, H);
            L.k = heads_of(a, k, tokens, G);
            L.scale2 = a->cfg.scale * kLog2e;
        }
        if (zero_rest) {
            const psops_heads *all[3] = {dq, dk, dv};
            for (int i = 0; i < 3; ++i)
                if (all[i] != nullptr) {
                    L.rest[L.fill] = heads_of(a, all[i], tokens, i == 0 ? H : G);
                    L.rest_heads[L.fill++] = i == 0 ? H : G;
                }
        }
    }
    const int64_t blocks = tokens > 0 ? std::min<int64_t>({(int64_t)a->sms * 4, kMostFillBlocks, ceil_div(tokens * H, kPrepThreads / 16)}) : 0;
    JoinParams J{};
    J.partials = a->at<float>(a->lay.partials);
    J.used = L.used;
    J.slots = tokens > 0 && sequences > 0 ? L.capacity : 0;
    J.heads = H;
    J.buckets = a->cfg.buckets;
    J.fp32 = bias_type == PSOPS_F32;
    J.out = d_dbias;
    const bool join_within = d_dbias != nullptr && J.slots > 0 && (int64_t)J.slots * H * a->cfg.buckets <= kJoinWithin;
    if (join_within) J.ticket = L.ticket = a->at<int>(a->lay.ticket);
    // few tiles: a CTA for each query head, and the last of those that share a key head adds them up (1,024 tokens, 8 heads
    // on 2, bias: 78 us a training pass with four heads a CTA, 66 to 73 so)
    const bool split = H > G && (L.capacity - 1) * H <= std::min(a->sms, kMostCtas / 2) && L.capacity * G <= kMostCtas;
    if (split) {
        L.zero = a->at<int>(a->lay.arrived);
        L.zeros = 2 * kMostCtas;
    }
    PSOPS_DO(prepare(a, L, blocks));
    if (tokens > 0 && sequences > 0) {
        CUtensorMap mq, mk, mv, mg;
        const Heads Q = heads_of(a, q, tokens, H), K = heads_of(a, k, tokens, G);
        PSOPS_DO(make_map(a, &mq, Q, tokens, H));
        PSOPS_DO(make_map(a, &mk, K, tokens, G));
        PSOPS_DO(make_map(a, &mv, L.v, tokens, G));
        PSOPS_DO(make_map(a, &mg, L.grad, tokens, H));
        BackwardParams P{};
        P.items = L.items;
        P.count = L.count;
        P.tokens = (int)tokens;
        P.heads = H;
        P.group = H / G;
        P.by_group = divisor(H / G);
        P.dim = a->cfg.dim;
        P.scale = a->cfg.scale;
        P.scale2 = a->cfg.scale * kLog2e;
        P.q = Q;
        P.k = K;
        P.grad = L.grad;
        P.lse = d_lse;
        P.levels = L.levels;
        P.beside = L.beside;
        P.delta = L.delta;
        P.norms = L.norms;
        P.blocks = (int)blocks;
        P.bias = bias_of(a, d_bias, bias_type);
        P.by_heads = divisor(H);
        P.by_kv_heads = divisor(G);
        if (dq != nullptr) P.dq = heads_of(a, dq, tokens, H);
        if (dk != nullptr) P.dk = heads_of(a, dk, tokens, G);
        if (dv != nullptr) P.dv = heads_of(a, dv, tokens, G);
        P.partials = d_dbias != nullptr ? a->at<float>(a->lay.partials) : nullptr;
        P.fold = a->at<float>(a->lay.fold);
        if (join_within) P.join = J;
        size_t shared;
        BackwardKernel kernel = backward_kernel(a, &shared);
        // dk and dbias need the delta that the queries' use leaves
        if (dq != nullptr || d_dbias != nullptr || dk != nullptr)
            PSOPS_DO(launch(a, "psops_attention_backward_kernel", kernel, works_grid(a, L, H, 1), kBackwardThreads, shared, 1, mq, mk, mv, mg, P));
        P.keys = 1;
        P.split = split;
        P.arrived = a->at<int>(a->lay.arrived);
        P.unclean = P.arrived + kMostCtas;
        if (split) P.by_kv_heads = divisor(H);
        if (dk != nullptr || dv != nullptr || d_dbias != nullptr)
            PSOPS_DO(launch(a, "psops_attention_backward_kernel", kernel, works_grid(a, L, split ? H : G, 1), kBackwardThreads, shared, 1, mq, mk, mv, mg, P));
    }
    if (d_dbias == nullptr || join_within) return PSOPS_OK;
    return launch(a, "psops_attention_join_kernel",
                  a->cfg.type == PSOPS_F16 ? psops_attention_join_kernel<__half> : psops_attention_join_kernel<__nv_bfloat16>,
                  dim3((unsigned)ceil_div(H * a->cfg.buckets, 32)), 32 * kJoinParts, 0, 1, J);
}

int psops_attention_set_stream(psops_attention *a, void *cuda_stream) { return psops_host::set_stream(a, cuda_stream); }
int64_t psops_attention_launch_count(const psops_attention *a) { return a ? a->launches : 0; }
const char *psops_attention_last_error(const psops_attention *a) { return a ? a->err : ""; }

int psops_attention_destroy(psops_attention *a)
{
    if (a == nullptr) return PSOPS_EINVAL;
    OnDevice guard(a);
    const int rc = cudaStreamSynchronize(a->stream) == cudaSuccess ? PSOPS_OK : PSOPS_ECUDA;
    delete a;
    return rc;
}

} // extern "C"
