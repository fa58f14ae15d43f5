// psops_optim.cu -- C ABI and host side of AdamW over many tensors and of the
// 2-norm of many gradients (kernels: psops_optim_kernels.cuh).

#include "psops.h"

#include <cuda_runtime.h>

#include <cmath>
#include <cstring>
#include <new>
#include <type_traits>
#include <vector>

#include "psops_host.cuh"
#include "psops_optim_kernels.cuh"

using psops_host::Base;
using psops_host::OnDevice;
using psops_host::Staging;
using psops_host::ceil_div;
using psops_host::round_up;

namespace {

constexpr int64_t kMaxElements = (int64_t)1 << 40;
constexpr int64_t kMaxChunks = (int64_t)1 << 30;

int type_bytes(int type) { return type == PSOPS_F32 ? 4 : type == PSOPS_F16 || type == PSOPS_BF16 ? 2 : 0; }

// Chunks of one tensor: enough for every alignment its arrays can have, so that
// new gradient addresses never change the list of chunks.
int64_t chunks_of(int64_t n, int64_t chunk, int64_t most_lo) { return n == 0 ? 0 : ceil_div(n + most_lo, chunk); }

bool adamw_config_ok(const psops_adamw_config *c)
{
    if (c == nullptr || c->n_tensors < 1 || c->steps_done < 0) return false;
    if (!(c->beta1 >= 0.0 && c->beta1 < 1.0 && c->beta2 >= 0.0 && c->beta2 < 1.0)) return false;
    if (!(c->eps >= 0.0) || !std::isfinite(c->eps)) return false;
    if (c->state_bits != 32 && c->state_bits != 8) return false;
    if (type_bytes(c->grad_type) == 0) return false;
    if (c->copy_type != PSOPS_NONE && type_bytes(c->copy_type) != 2) return false;
    return true;
}

// Total chunks, or -1 where a size is out of range.
int64_t adamw_chunks(const psops_adamw_config *c, const psops_adamw_tensor *t)
{
    int64_t total = 0;
    for (int32_t i = 0; i < c->n_tensors; ++i) {
        if (t[i].n < 0 || t[i].n > kMaxElements) return -1;
        total += chunks_of(t[i].n, kAdamwChunk, c->state_bits == 8 ? 0 : 7);
        if (total > kMaxChunks) return -1;
    }
    return total;
}

struct AdamwLayout { size_t entries, chunks, total; };
AdamwLayout adamw_layout(int32_t n_tensors, int64_t n_chunks)
{
    AdamwLayout L;
    L.entries = round_up(sizeof(AdamwState), 256);
    L.chunks = L.entries + round_up(sizeof(AdamwEntry) * (size_t)n_tensors, 256);
    L.total = L.chunks + round_up(sizeof(uint2) * (size_t)n_chunks, 256);
    return L;
}

void fill_chunks(std::vector<uint2> &list, int32_t tensor, int64_t count)
{
    for (int64_t k = 0; k < count; ++k) list.push_back(make_uint2((unsigned)tensor, (unsigned)k));
}

// Elements by which an array lies behind a group of eight, or -1 if it is not
// aligned to its elements.
int behind(const void *ptr, int element_bytes)
{
    const uintptr_t a = (uintptr_t)ptr;
    if (a % (uintptr_t)element_bytes) return -1;
    return (int)(a / (uintptr_t)element_bytes % 8u);
}

template <class T> T *moved_back(T *p, int64_t bytes) { return (T *)((uintptr_t)p - (uintptr_t)bytes); }

// The device's view of one tensor.
int adamw_entry(const psops_adamw_config *c, const psops_adamw_tensor *t, AdamwEntry *e)
{
    std::memset(e, 0, sizeof(*e));
    e->weight_decay = t->weight_decay;
    if (t->n == 0) return PSOPS_OK;
    const bool small = c->state_bits == 8;
    const bool copies = c->copy_type != PSOPS_NONE && t->copy != nullptr;
    if (t->p == nullptr || t->g == nullptr || t->m == nullptr || t->v == nullptr) return PSOPS_EINVAL;
    if (small && (t->m_scale == nullptr || t->v_scale == nullptr)) return PSOPS_EINVAL;
    if (c->copy_type == PSOPS_NONE && t->copy != nullptr) return PSOPS_EINVAL;
    const int gb = type_bytes(c->grad_type), sb = small ? 1 : 4;
    const int lo = behind(t->p, 4);
    const int at[4] = {behind(t->g, gb), behind(t->m, sb), behind(t->v, sb), copies ? behind(t->copy, 2) : lo};
    bool alike = true;
    if (lo < 0) return PSOPS_EALIGN;
    for (int a : at) {
        if (a < 0) return PSOPS_EALIGN;
        alike = alike && a == lo;
    }
    if (small && (((uintptr_t)t->m_scale | (uintptr_t)t->v_scale) & 3u)) return PSOPS_EALIGN;
    // an 8-bit moment's blocks of 256 start with the tensor, so there only lo == 0 will do
    e->vec = alike && (lo == 0 || !small) ? 1 : 0;
    const int64_t back = e->vec ? lo : 0;
    e->lo = back;
    e->hi = back + t->n;
    e->p = moved_back(t->p, back * 4);
    e->g = moved_back((const char *)t->g, back * gb);
    e->m = moved_back((char *)t->m, back * sb);
    e->v = moved_back((char *)t->v, back * sb);
    e->copy = copies ? moved_back((char *)t->copy, back * 2) : nullptr;
    e->m_scale = small ? t->m_scale : nullptr;
    e->v_scale = small ? t->v_scale : nullptr;
    return PSOPS_OK;
}

using AdamwKernel = void (*)(const AdamwParams);

template <int BITS, class G>
AdamwKernel pick_adamw_copy(int copy)
{
    return copy == PSOPS_NONE ? psops_adamw_kernel<BITS, G, void>
           : copy == PSOPS_F16 ? psops_adamw_kernel<BITS, G, __half> : psops_adamw_kernel<BITS, G, __nv_bfloat16>;
}
template <int BITS>
AdamwKernel pick_adamw_grad(int grad, int copy)
{
    return grad == PSOPS_F32 ? pick_adamw_copy<BITS, float>(copy)
           : grad == PSOPS_F16 ? pick_adamw_copy<BITS, __half>(copy) : pick_adamw_copy<BITS, __nv_bfloat16>(copy);
}
AdamwKernel pick_adamw(const psops_adamw_config *c)
{
    return c->state_bits == 8 ? pick_adamw_grad<8>(c->grad_type, c->copy_type)
                              : pick_adamw_grad<32>(c->grad_type, c->copy_type);
}

int open_base(Base *b, void *stream)
{
    b->stream = (cudaStream_t)stream;
    if (cudaGetDevice(&b->device) != cudaSuccess ||
        cudaDeviceGetAttribute(&b->sms, cudaDevAttrMultiProcessorCount, b->device) != cudaSuccess)
        return PSOPS_ECUDA;
    return psops_host::not_capturing(b);
}

// Blocks of a persistent launch: no more than run at once, and as many as have
// the same number of chunks to do (but for the last ones).
int grid_of(Base *b, const void *kernel, int64_t n_chunks, unsigned *grid)
{
    int per_sm = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kOptThreads, 0) != cudaSuccess) return PSOPS_ECUDA;
    const int64_t most = (int64_t)b->sms * (per_sm < 1 ? 1 : per_sm);
    const int64_t rounds = n_chunks < 1 ? 1 : ceil_div(n_chunks, most);
    *grid = (unsigned)(n_chunks < 1 ? 1 : ceil_div(n_chunks, rounds));
    return PSOPS_OK;
}

} // namespace

struct psops_adamw : Base {
    psops_adamw_config cfg;
    std::vector<psops_adamw_tensor> tensors;
    Staging staging;
    AdamwKernel kernel;
    AdamwState *state;
    AdamwEntry *entries;
    uint2 *chunks;
    int64_t n_chunks;
    unsigned grid;
};

struct psops_gradnorm : Base {
    int32_t grad_type;
    std::vector<int64_t> n;
    Staging staging;
    void (*kernel)(const NormParams);
    NormEntry *entries;
    uint2 *chunks;
    double *partials;
    unsigned *tickets;
    int64_t n_chunks;
    unsigned grid;
};

extern "C" {

size_t psops_adamw_workspace_bytes(const psops_adamw_config *cfg, const psops_adamw_tensor *tensors)
{
    if (!adamw_config_ok(cfg) || tensors == nullptr) return 0;
    const int64_t n = adamw_chunks(cfg, tensors);
    return n < 0 ? 0 : adamw_layout(cfg->n_tensors, n).total;
}

int psops_adamw_create(psops_adamw **out, const psops_adamw_config *cfg, const psops_adamw_tensor *tensors,
                       void *d_workspace, size_t workspace_bytes, void *cuda_stream)
{
    if (out == nullptr) return PSOPS_EINVAL;
    *out = nullptr;
    if (!adamw_config_ok(cfg) || tensors == nullptr) return PSOPS_EINVAL;
    const int64_t n_chunks = adamw_chunks(cfg, tensors);
    if (n_chunks < 0) return PSOPS_EINVAL;
    for (int32_t i = 0; i < cfg->n_tensors; ++i) {
        AdamwEntry e;
        if (!std::isfinite(tensors[i].weight_decay)) return PSOPS_EINVAL;
        const int rc = adamw_entry(cfg, &tensors[i], &e);
        if (rc != PSOPS_OK) return rc;
    }
    const AdamwLayout lay = adamw_layout(cfg->n_tensors, n_chunks);
    if (d_workspace == nullptr || ((uintptr_t)d_workspace & 255u) || workspace_bytes < lay.total) return PSOPS_EWORKSPACE;

    psops_adamw *a = new (std::nothrow) psops_adamw();
    if (a == nullptr) return PSOPS_ENOMEM;
    int rc = PSOPS_OK;
    try {
        a->cfg = *cfg;
        a->tensors.assign(tensors, tensors + cfg->n_tensors);
        a->state = (AdamwState *)d_workspace;
        a->entries = (AdamwEntry *)((char *)d_workspace + lay.entries);
        a->chunks = (uint2 *)((char *)d_workspace + lay.chunks);
        a->n_chunks = n_chunks;
        a->kernel = pick_adamw(cfg);
        std::vector<uint2> list;
        list.reserve((size_t)n_chunks);
        for (int32_t i = 0; i < cfg->n_tensors; ++i)
            fill_chunks(list, i, chunks_of(tensors[i].n, kAdamwChunk, cfg->state_bits == 8 ? 0 : 7));
        AdamwState s{};
        s.pow1 = std::pow(cfg->beta1, (double)(cfg->steps_done + 1));
        s.pow2 = std::pow(cfg->beta2, (double)(cfg->steps_done + 1));
        s.steps = cfg->steps_done;
        rc = open_base(a, cuda_stream);
        if (rc == PSOPS_OK) rc = grid_of(a, (const void *)a->kernel, n_chunks, &a->grid);
        const size_t bytes = sizeof(AdamwEntry) * (size_t)cfg->n_tensors;
        cudaError_t e = rc == PSOPS_OK ? a->staging.reserve(bytes) : cudaSuccess;
        if (rc == PSOPS_OK && e == cudaSuccess) {
            for (int32_t i = 0; i < cfg->n_tensors; ++i) adamw_entry(cfg, &tensors[i], (AdamwEntry *)a->staging.host() + i);
            e = a->staging.send(a->entries, bytes, a->stream);
            if (e == cudaSuccess)
                e = cudaMemcpyAsync(a->state, &s, sizeof(s), cudaMemcpyHostToDevice, a->stream);
            if (e == cudaSuccess && n_chunks > 0)
                e = cudaMemcpyAsync(a->chunks, list.data(), sizeof(uint2) * (size_t)n_chunks, cudaMemcpyHostToDevice, a->stream);
            if (e == cudaSuccess) e = cudaStreamSynchronize(a->stream);      // s and list are pageable
        }
        if (e != cudaSuccess) rc = PSOPS_ECUDA;
    } catch (const std::bad_alloc &) {
        rc = PSOPS_ENOMEM;
    }
    if (rc != PSOPS_OK) {
        delete a;
        return rc;
    }
    *out = a;
    return PSOPS_OK;
}

int psops_adamw_set_grads(psops_adamw *a, const void *const *grads)
{
    if (a == nullptr || grads == nullptr) return PSOPS_EINVAL;
    OnDevice guard(a);
    const int32_t n = a->cfg.n_tensors;
    for (int32_t i = 0; i < n; ++i) {
        psops_adamw_tensor t = a->tensors[(size_t)i];
        AdamwEntry e;
        t.g = grads[i];
        const int rc = adamw_entry(&a->cfg, &t, &e);
        if (rc != PSOPS_OK) return rc;
    }
    const int rc = psops_host::not_capturing(a);
    if (rc != PSOPS_OK) return rc;
    PSOPS_TRY(a, a->staging.wait());
    for (int32_t i = 0; i < n; ++i) {
        a->tensors[(size_t)i].g = grads[i];
        adamw_entry(&a->cfg, &a->tensors[(size_t)i], (AdamwEntry *)a->staging.host() + i);
    }
    PSOPS_TRY(a, a->staging.send(a->entries, sizeof(AdamwEntry) * (size_t)n, a->stream));
    return PSOPS_OK;
}

int psops_adamw_step(psops_adamw *a, double lr, const float *d_scale)
{
    if (a == nullptr || !std::isfinite(lr)) return PSOPS_EINVAL;
    if ((uintptr_t)d_scale & 3u) return PSOPS_EALIGN;
    OnDevice guard(a);
    AdamwParams P{};
    P.entries = a->entries;
    P.chunks = a->chunks;
    P.state = a->state;
    P.scale = d_scale;
    P.lr = lr;
    P.beta1 = a->cfg.beta1;
    P.beta2 = a->cfg.beta2;
    P.b1 = (float)a->cfg.beta1;
    P.b1c = (float)(1.0 - a->cfg.beta1);
    P.b2 = (float)a->cfg.beta2;
    P.b2c = (float)(1.0 - a->cfg.beta2);
    P.eps = (float)a->cfg.eps;
    P.n_chunks = (unsigned)a->n_chunks;
    return psops_host::launch(a, "psops_adamw_kernel", a->kernel, dim3(a->grid), kOptThreads, 0, 1, P);
}

int psops_adamw_steps(psops_adamw *a, int64_t *steps)
{
    if (a == nullptr || steps == nullptr) return PSOPS_EINVAL;
    OnDevice guard(a);
    const int rc = psops_host::not_capturing(a);
    if (rc != PSOPS_OK) return rc;
    AdamwState s;
    PSOPS_TRY(a, cudaMemcpyAsync(&s, a->state, sizeof(s), cudaMemcpyDeviceToHost, a->stream));
    PSOPS_TRY(a, cudaStreamSynchronize(a->stream));
    *steps = s.steps;
    return PSOPS_OK;
}

int psops_adamw_set_stream(psops_adamw *a, void *cuda_stream) { return psops_host::set_stream(a, cuda_stream); }
int64_t psops_adamw_launch_count(const psops_adamw *a) { return a ? a->launches : 0; }
const char *psops_adamw_last_error(const psops_adamw *a) { return a ? a->err : ""; }

int psops_adamw_destroy(psops_adamw *a)
{
    if (a == nullptr) return PSOPS_EINVAL;
    OnDevice guard(a);
    const int rc = cudaStreamSynchronize(a->stream) == cudaSuccess ? PSOPS_OK : PSOPS_ECUDA;
    delete a;
    return rc;
}

} // extern "C"

// ---------------------------------------------------------------------------
// 2-norm
// ---------------------------------------------------------------------------
namespace {

constexpr int kNormMaxBlocks = 4096;            // room for one partial sum each

int64_t norm_chunk(int type) { return type == PSOPS_F32 ? NormShape<float>::kChunk : NormShape<__half>::kChunk; }
int64_t norm_chunks(int32_t count, const int64_t *n, int type)
{
    int64_t total = 0;
    for (int32_t i = 0; i < count; ++i) {
        if (n[i] < 0 || n[i] > kMaxElements) return -1;
        total += chunks_of(n[i], norm_chunk(type), type == PSOPS_F32 ? 7 : 15);
        if (total > kMaxChunks) return -1;
    }
    return total;
}

struct NormLayout { size_t entries, chunks, total; };
NormLayout norm_layout(int32_t count, int64_t n_chunks)
{
    NormLayout L;
    L.entries = 256 + sizeof(double) * kNormMaxBlocks;
    L.chunks = L.entries + round_up(sizeof(NormEntry) * (size_t)count, 256);
    L.total = L.chunks + round_up(sizeof(uint2) * (size_t)n_chunks, 256);
    return L;
}

int norm_entry(const void *g, int64_t n, int type, NormEntry *e)
{
    e->g = nullptr;
    e->lo = e->hi = 0;
    if (n == 0) return PSOPS_OK;
    const uintptr_t a = (uintptr_t)g, es = (uintptr_t)type_bytes(type);
    if (g == nullptr) return PSOPS_EINVAL;
    if (a % es) return PSOPS_EALIGN;
    e->lo = (long long)(a % 32u / es);
    e->hi = e->lo + n;
    e->g = (const void *)(a / 32u * 32u);
    return PSOPS_OK;
}

} // namespace

extern "C" {

size_t psops_gradnorm_workspace_bytes(int32_t n_tensors, const int64_t *n)
{
    if (n_tensors < 1 || n == nullptr) return 0;
    const int64_t chunks = norm_chunks(n_tensors, n, PSOPS_F32);     // the shorter chunks: enough for every type
    return chunks < 0 ? 0 : norm_layout(n_tensors, chunks).total;
}

int psops_gradnorm_create(psops_gradnorm **out, int32_t n_tensors, const void *const *grads, const int64_t *n,
                          int32_t grad_type, void *d_workspace, size_t workspace_bytes, void *cuda_stream)
{
    if (out == nullptr) return PSOPS_EINVAL;
    *out = nullptr;
    const size_t need = psops_gradnorm_workspace_bytes(n_tensors, n);
    if (need == 0 || grads == nullptr || type_bytes(grad_type) == 0) return PSOPS_EINVAL;
    for (int32_t i = 0; i < n_tensors; ++i) {
        NormEntry e;
        const int rc = norm_entry(grads[i], n[i], grad_type, &e);
        if (rc != PSOPS_OK) return rc;
    }
    if (d_workspace == nullptr || ((uintptr_t)d_workspace & 255u) || workspace_bytes < need) return PSOPS_EWORKSPACE;

    psops_gradnorm *q = new (std::nothrow) psops_gradnorm();
    if (q == nullptr) return PSOPS_ENOMEM;
    int rc = PSOPS_OK;
    try {
        q->grad_type = grad_type;
        q->n.assign(n, n + n_tensors);
        q->n_chunks = norm_chunks(n_tensors, n, grad_type);
        const NormLayout lay = norm_layout(n_tensors, q->n_chunks);
        q->tickets = (unsigned *)d_workspace;
        q->partials = (double *)((char *)d_workspace + 256);
        q->entries = (NormEntry *)((char *)d_workspace + lay.entries);
        q->chunks = (uint2 *)((char *)d_workspace + lay.chunks);
        q->kernel = grad_type == PSOPS_F32 ? psops_gradnorm_kernel<float>
                    : grad_type == PSOPS_F16 ? psops_gradnorm_kernel<__half> : psops_gradnorm_kernel<__nv_bfloat16>;
        std::vector<uint2> list;
        list.reserve((size_t)q->n_chunks);
        for (int32_t i = 0; i < n_tensors; ++i)
            fill_chunks(list, i, chunks_of(n[i], norm_chunk(grad_type), grad_type == PSOPS_F32 ? 7 : 15));
        rc = open_base(q, cuda_stream);
        if (rc == PSOPS_OK) rc = grid_of(q, (const void *)q->kernel, q->n_chunks, &q->grid);
        if (q->grid > (unsigned)kNormMaxBlocks) q->grid = kNormMaxBlocks;
        const size_t bytes = sizeof(NormEntry) * (size_t)n_tensors;
        cudaError_t e = rc == PSOPS_OK ? q->staging.reserve(bytes) : cudaSuccess;
        if (rc == PSOPS_OK && e == cudaSuccess) {
            for (int32_t i = 0; i < n_tensors; ++i)
                norm_entry(grads[i], n[i], grad_type, (NormEntry *)q->staging.host() + i);
            e = q->staging.send(q->entries, bytes, q->stream);
            if (e == cudaSuccess) e = cudaMemsetAsync(q->tickets, 0, 256, q->stream);
            if (e == cudaSuccess && q->n_chunks > 0)
                e = cudaMemcpyAsync(q->chunks, list.data(), sizeof(uint2) * list.size(), cudaMemcpyHostToDevice, q->stream);
            if (e == cudaSuccess) e = cudaStreamSynchronize(q->stream);      // list is pageable
        }
        if (e != cudaSuccess) rc = PSOPS_ECUDA;
    } catch (const std::bad_alloc &) {
        rc = PSOPS_ENOMEM;
    }
    if (rc != PSOPS_OK) {
        delete q;
        return rc;
    }
    *out = q;
    return PSOPS_OK;
}

int psops_gradnorm_set_grads(psops_gradnorm *q, const void *const *grads)
{
    if (q == nullptr || grads == nullptr) return PSOPS_EINVAL;
    OnDevice guard(q);
    for (size_t i = 0; i < q->n.size(); ++i) {
        NormEntry e;
        const int rc = norm_entry(grads[i], q->n[i], q->grad_type, &e);
        if (rc != PSOPS_OK) return rc;
    }
    const int rc = psops_host::not_capturing(q);
    if (rc != PSOPS_OK) return rc;
    PSOPS_TRY(q, q->staging.wait());
    for (size_t i = 0; i < q->n.size(); ++i)
        norm_entry(grads[i], q->n[i], q->grad_type, (NormEntry *)q->staging.host() + i);
    PSOPS_TRY(q, q->staging.send(q->entries, sizeof(NormEntry) * q->n.size(), q->stream));
    return PSOPS_OK;
}

int psops_gradnorm_run(psops_gradnorm *q, float max_norm, float *d_out)
{
    if (q == nullptr || d_out == nullptr || !(max_norm >= 0.0f)) return PSOPS_EINVAL;
    if ((uintptr_t)d_out & 3u) return PSOPS_EALIGN;
    OnDevice guard(q);
    NormParams P{};
    P.entries = q->entries;
    P.chunks = q->chunks;
    P.partials = q->partials;
    P.tickets = q->tickets;
    P.out = d_out;
    P.max_norm = max_norm;
    P.n_chunks = (unsigned)q->n_chunks;
    return psops_host::launch(q, "psops_gradnorm_kernel", q->kernel, dim3(q->grid), kOptThreads, 0, 1, P);
}

int psops_gradnorm_set_stream(psops_gradnorm *q, void *cuda_stream) { return psops_host::set_stream(q, cuda_stream); }
int64_t psops_gradnorm_launch_count(const psops_gradnorm *q) { return q ? q->launches : 0; }
const char *psops_gradnorm_last_error(const psops_gradnorm *q) { return q ? q->err : ""; }

int psops_gradnorm_destroy(psops_gradnorm *q)
{
    if (q == nullptr) return PSOPS_EINVAL;
    OnDevice guard(q);
    const int rc = cudaStreamSynchronize(q->stream) == cudaSuccess ? PSOPS_OK : PSOPS_ECUDA;
    delete q;
    return rc;
}

} // extern "C"
