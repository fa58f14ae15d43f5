// psops_xent_small.cuh -- the linear cross entropy where tensor-core tiles do
// not pay: few classes (a classifier's head), and few tokens.
//
// Each form does a whole forward pass in one launch and the gradients in two;
// tokens that are left out are simply passed over, so nothing is listed or
// gathered first.  Products and sums are fp32, and gradients are rounded to 16
// bits only at the end.
#pragma once

#include "psops_xent_kernels.cuh"

namespace {

constexpr int kSmallThreads = 256, kSmallWarps = kSmallThreads / 32;

// ---- few classes ----------------------------------------------------------------
// Up to 64 classes whose weights fit into shared memory beside a hidden state
// per warp.  A warp takes a token: 32 / `wide` slices of the features by `wide`
// classes (the power of two above their number), then the softmax across lanes.
// Every block loads all weights, element by element, and a warp's tokens come one
// after the other; dw's few blocks walk through all tokens.  Measured in a CUDA
// graph, this form / the tensor cores, us, dim x classes:
//   tokens          256            1,024         2,048         4,096          8,192
//   loss   84 x 10  7.4 / 17       7.4 / 17      9.4 / 18      13 / 20        19 / 22
//          512 x 10 12 / 17        13 / 18       19 / 18       30 / 21        47 / 24
//          84 x 64  9.8 / 17       10 / 17       14 / 18       21 / 20        33 / 22
//          512 x 64 33 / 17        34 / 17       51 / 18       84 / 21        135 / 24
//   grads  84 x 10  13 / 28        26 / 32       50 / 32       95 / 35        177 / 39
//          512 x 10 20 / 27        37 / 32       64 / 34       123 / 38       234 / 47
//          84 x 64  16 / 29        32 / 33       55 / 33       106 / 35       200 / 40
//          512 x 64 42 / 28        60 / 32       102 / 34      186 / 39       337 / 48
// (16 tokens take what 256 do, but for the gradients of 84 x 10: 7.4 / 25.)  Loading
// grows with dim times `wide`, the tensor cores' time with dim alone: 64 tokens x
// 192 x 64 16 / 17, 16 x 1,200 x 10 23 / 22, 64 x 2,000 x 4 22 / 26.
constexpr int kHeadClasses = 64;
constexpr int64_t kHeadWeights = 12000;                                  // dim times `wide` beyond 5.5
constexpr int64_t kHeadLossTokens = 8192, kHeadLossWork = 1 << 24;       // work: tokens times dim times `wide`
constexpr int64_t kHeadGradTokens = 1024, kHeadGradWork = 1 << 22;
constexpr int kHeadShared = 200 * 1024;

__host__ __device__ inline int head_wide(int vocab) { return vocab <= 8 ? 8 : vocab <= 16 ? 16 : vocab <= 32 ? 32 : 64; }
inline size_t head_shared(int vocab, int dim) { return 4ull * (size_t)dim * (head_wide(vocab) + 1 + kSmallWarps) + 4ull * kSmallWarps * kHeadClasses; }
inline bool is_head(int64_t vocab, int64_t dim, int64_t tokens, bool grads)
{
    if (vocab > kHeadClasses) return false;
    const int64_t wide = head_wide((int)vocab), weights = dim * wide;
    return 2 * weights - 11 * dim <= 2 * kHeadWeights && tokens <= (grads ? kHeadGradTokens : kHeadLossTokens) &&
           tokens * weights <= (grads ? kHeadGradWork : kHeadLossWork) && head_shared((int)vocab, (int)dim) <= (size_t)kHeadShared;
}

struct HeadParams {
    const void *h, *w;
    long long h_ld, w_ld;
    const long long *targets;
    int tokens, dim, vocab, reduction;
    XentControl *control;
    double2 *partials;                           // (loss, tokens that count) of each block
    float *loss, *rows, *lse_out;                // forward
    const float *lse, *known_rows, *grad;        // backward; known_rows: the forward pass's, or NULL
    float *dlogits;                              // tokens x wide
    void *dh;
    long long dh_ld;
};

template <class T> __device__ __forceinline__ float wide16(T x);
template <> __device__ __forceinline__ float wide16(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float wide16(__nv_bfloat16 x) { return __bfloat162float(x); }
template <class T> __device__ __forceinline__ T narrow16(float x);
template <> __device__ __forceinline__ __half narrow16(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 narrow16(float x) { return __float2bfloat16_rn(x); }

template <class T, bool GRADS>
__global__ void __launch_bounds__(kSmallThreads) psops_xent_head_kernel(const HeadParams P)
{
    extern __shared__ float head_shared_memory[];
    __shared__ double block_loss[kSmallWarps];
    __shared__ int block_count[kSmallWarps];
    __shared__ bool last;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int wide = head_wide(P.vocab), pitch = wide + 1;
    float *w = head_shared_memory;                                   // dim x pitch
    float *hidden = w + (size_t)P.dim * pitch + (size_t)warp * P.dim;
    float *mine = w + (size_t)P.dim * (pitch + kSmallWarps) + warp * kHeadClasses;
    after_the_kernel_before();
    for (int i = threadIdx.x; i < P.vocab * P.dim; i += kSmallThreads) {
        const int v = i / P.dim, d = i - v * P.dim;
        w[d * pitch + v] = wide16(((const T *)P.w)[v * P.w_ld + d]);
    }
    for (int i = threadIdx.x; i < (wide - P.vocab) * P.dim; i += kSmallThreads) {
        const int v = i / P.dim;
        w[(i - v * P.dim) * pitch + P.vocab + v] = 0.0f;
    }
    float common = 0.0f;
    if (GRADS) {
        int count = 0;
        if (P.reduction == PSOPS_MEAN) {
            for (int t = threadIdx.x; t < P.tokens; t += kSmallThreads) {
                const long long y = P.targets[t];
                count += y >= 0 && y < P.vocab ? 1 : 0;
            }
            count = __reduce_add_sync(0xffffffffu, count);
            if (lane == 0) block_count[warp] = count;
        }
        __syncthreads();
        if (P.reduction == PSOPS_MEAN) {
            count = 0;
            for (int k = 0; k < kSmallWarps; ++k) count += block_count[k];
        }
        if (P.reduction != PSOPS_PER_TOKEN) common = P.reduction == PSOPS_MEAN ? __fdiv_rn(P.grad[0], (float)max(1, count)) : P.grad[0];
    } else {
        __syncthreads();
    }
    double loss = 0.0;
    int counted = 0;
    for (int t = blockIdx.x * kSmallWarps + warp; t < P.tokens; t += gridDim.x * kSmallWarps) {
        const long long label = P.targets[t];
        const bool in = label >= 0 && label < P.vocab;
        if (!in) {
            if (!GRADS) {
                if (lane == 0 && P.rows != nullptr) P.rows[t] = 0.0f;
                if (lane == 0 && P.lse_out != nullptr) P.lse_out[t] = 0.0f;
            } else if (P.dh != nullptr) {
                for (int d = lane; d < P.dim; d += 32) ((T *)P.dh)[t * P.dh_ld + d] = narrow16<T>(0.0f);
            }
            continue;
        }
        for (int d = lane; d < P.dim; d += 32) hidden[d] = wide16(((const T *)P.h)[t * P.h_ld + d]);
        __syncwarp();
        float x0 = 0.0f, x1 = 0.0f;                                  // classes lane % wide, and lane + 32 of 64
        if (wide == 64) {
#pragma unroll 4
            for (int d = 0; d < P.dim; ++d) {
                x0 = fmaf(hidden[d], w[d * pitch + lane], x0);
                x1 = fmaf(hidden[d], w[d * pitch + lane + 32], x1);
            }
        } else {
            const int slices = 32 / wide, v = lane & (wide - 1);
#pragma unroll 4
            for (int d = lane / wide; d < P.dim; d += slices) x0 = fmaf(hidden[d], w[d * pitch + v], x0);
            for (int off = wide; off < 32; off <<= 1) x0 += __shfl_xor_sync(0xffffffffu, x0, off);
        }
        const int v = wide == 64 ? lane : lane & (wide - 1);
        const bool there0 = v < P.vocab, there1 = wide == 64 && lane + 32 < P.vocab;
        const int y = (int)label;
        if (!GRADS) {
            float top = fmaxf(there0 ? x0 : -INFINITY, there1 ? x1 : -INFINITY);
            for (int off = min(wide, 32) / 2; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            const float ref = top > -INFINITY ? top : 0.0f;
            float sum = (there0 ? expf(x0 - ref) : 0.0f) + (there1 ? expf(x1 - ref) : 0.0f);
            for (int off = min(wide, 32) / 2; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
            const float lse = top + logf(sum);
            const float a = __shfl_sync(0xffffffffu, x0, y & 31), b = __shfl_sync(0xffffffffu, x1, y & 31);
            const float row = lse - (y < 32 ? a : b);
            if (lane == 0 && P.rows != nullptr) P.rows[t] = row;
            if (lane == 0 && P.lse_out != nullptr) P.lse_out[t] = lse;
            loss += row;
            ++counted;
        } else {
            const float lse = P.lse[t], g = P.reduction == PSOPS_PER_TOKEN ? P.grad[t] : common;
            const bool known = P.known_rows != nullptr;
            const float at_label = known ? expm1f(-P.known_rows[t]) : 0.0f;
            auto bracket = [&](float x, bool label) { return !label ? expf(x - lse) : known ? at_label : expm1f(x - lse); };
            const float d0 = there0 ? bracket(x0, v == y) * g : 0.0f;
            const float d1 = there1 ? bracket(x1, lane + 32 == y) * g : 0.0f;
            if (lane < wide) {
                mine[lane] = d0;
                P.dlogits[(long long)t * wide + lane] = d0;
            }
            if (wide == 64) {
                mine[lane + 32] = d1;
                P.dlogits[(long long)t * wide + lane + 32] = d1;
            }
            __syncwarp();
            if (P.dh != nullptr)
                for (int d = lane; d < P.dim; d += 32) {
                    float s = 0.0f;
#pragma unroll 4
                    for (int k = 0; k < P.vocab; ++k) s = fmaf(mine[k], w[d * pitch + k], s);
                    ((T *)P.dh)[t * P.dh_ld + d] = narrow16<T>(s);
                }
        }
        __syncwarp();
    }
    if (GRADS) return;
    if (lane == 0) {
        block_loss[warp] = loss;
        block_count[warp] = counted;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        counted = 0;
        loss = 0.0;
        for (int k = 0; k < kSmallWarps; ++k) {
            loss += block_loss[k];
            counted += block_count[k];
        }
        P.partials[blockIdx.x] = make_double2(loss, (double)counted);
        __threadfence();
        last = atomicAdd(&P.control->tickets, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last || threadIdx.x >= 32) return;
    __threadfence();
    double total = 0.0, n = 0.0;
    for (unsigned b = lane; b < gridDim.x; b += 32) {
        const double2 p = __ldcg(P.partials + b);
        total += p.x;
        n += p.y;
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        total += __shfl_xor_sync(0xffffffffu, total, off);
        n += __shfl_xor_sync(0xffffffffu, n, off);
    }
    if (lane == 0) {
        if (P.loss != nullptr) *P.loss = (float)(P.reduction == PSOPS_MEAN ? total / (n > 0.0 ? n : 1.0) : total);
        P.control->tickets = 0;
    }
}

// dw of a head: a block has 32 features of 8 classes, its warps share the
// tokens, and the warps' sums are added in order.
constexpr int kHeadDwThreads = 512, kHeadDwWarps = kHeadDwThreads / 32, kHeadDwClasses = 8;

template <class T>
__global__ void __launch_bounds__(kHeadDwThreads) psops_xent_head_dw_kernel(const T *h, long long h_ld, const long long *targets,
                                                                            const float *dlogits, int tokens, int dim, int vocab,
                                                                            T *dw, long long dw_ld)
{
    __shared__ float sums[kHeadDwWarps][kHeadDwClasses][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int d = blockIdx.x * 32 + lane, v0 = blockIdx.y * kHeadDwClasses, wide = head_wide(vocab);
    after_the_kernel_before();
    float acc[kHeadDwClasses] = {};
#pragma unroll 4
    for (int t = warp; t < tokens; t += kHeadDwWarps) {
        const long long y = targets[t];
        if (y < 0 || y >= vocab) continue;
        const float x = d < dim ? wide16(h[t * h_ld + d]) : 0.0f;
        const float4 a = *reinterpret_cast<const float4 *>(dlogits + (long long)t * wide + v0);
        const float4 b = *reinterpret_cast<const float4 *>(dlogits + (long long)t * wide + v0 + 4);
        const float g[kHeadDwClasses] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int k = 0; k < kHeadDwClasses; ++k) acc[k] = fmaf(g[k], x, acc[k]);
    }
#pragma unroll
    for (int k = 0; k < kHeadDwClasses; ++k) sums[warp][k][lane] = acc[k];
    __syncthreads();
    if (warp < kHeadDwClasses && v0 + warp < vocab && d < dim) {
        float s = 0.0f;
        for (int k = 0; k < kHeadDwWarps; ++k) s += sums[k][warp][lane];
        dw[(v0 + warp) * dw_ld + d] = narrow16<T>(s);
    }
}

// ---- few tokens -------------------------------------------------------------------
// Up to 4 tokens against the whole vocabulary: bound by reading w once.  The
// hidden states lie in shared memory as fp32; every warp has an equal share of
// w's rows and takes four at a time; lane t keeps the softmax of token t.
// Measured with 268 MB of w (32,768 x 4,096): 1 / 2 / 4 tokens 47 to 53 / 51 to 56
// / 59 to 62 us by the box (5.7 TB/s down to 4.3) where the tensor-core form takes
// 62 to 65 us whatever their number; 8 tokens took 91 us, so from 5 on the tensor
// cores do it.  With short rows a warp's turn is mostly its reductions: four tokens in
// a CUDA graph, this form / the tensor cores, us, by dim x entries:
//          8,192        32,768       65,536       131,072
//   64     9.0 / 15     17 / 16      25 / 20      42 / 28
//   61     10 / 17      21 / 18      33 / 23      58 / 34
//   192    9.4 / 16     17 / 17      25 / 21      42 / 32
//   320    9.8 / 17     18 / 18      25 / 24      43 / 37
//   512    9.8 / 18     18 / 21      26 / 27      43 / 45
constexpr int kFewTokens = 4, kFewRows = 4, kFewBlocks = 2;          // blocks of an SM
// Pieces of a row (512 bytes) on their way under the arithmetic: four where the registers are there.
template <int N> constexpr int kFewAhead = N == 1 ? 4 : 2;
constexpr int kFewShared = 96 * 1024;

inline int few_of(int64_t tokens) { return tokens <= 1 ? 1 : tokens <= 2 ? 2 : 4; }
inline size_t few_shared(int64_t tokens, int64_t dim) { return 4ull * (size_t)few_of(tokens) * (size_t)((dim + 255) / 256 * 256); }
inline bool is_few(int64_t tokens, int64_t dim) { return tokens >= 1 && tokens <= kFewTokens && dim <= kFewShared / 4 && few_shared(tokens, dim) <= (size_t)kFewShared; }
inline bool few_loss_pays(int64_t dim, int64_t vocab) { return dim > 320 || vocab <= 1 << 15; }

struct FewParams {
    const uint16_t *h, *w;
    long long h_ld, w_ld;
    bool h_aligned, w_aligned;
    const long long *targets;
    int tokens, dim, vocab, reduction;
    XentControl *control;
    float2 *stats;                               // block x token
    float *label_logit;
    float *loss, *rows, *lse_out;
};

template <class T> __device__ __forceinline__ void eight_numbers(const uint4 u, float (&x)[8])
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        T e[2];
        memcpy(e, &w[i], 4);
        x[2 * i] = wide16(e[0]);
        x[2 * i + 1] = wide16(e[1]);
    }
}

__device__ __forceinline__ uint4 load_once(const uint16_t *p)
{
    uint4 u;
    asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p));
    return u;
}

template <class T, int N, bool ALIGNED>
__global__ void __launch_bounds__(kSmallThreads, kFewBlocks) psops_xent_few_kernel(const FewParams P)
{
    extern __shared__ float4 few_hidden[];       // N x chunks of 256 x (first, second four of a lane's eight) x 32 lanes
    __shared__ float2 warp_stats[kSmallWarps][N];
    __shared__ float token_loss[N];
    __shared__ bool last;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int chunks = (P.dim + 255) / 256;
    after_the_kernel_before();
    for (int i = threadIdx.x; i < N * chunks * 32; i += kSmallThreads) {
        const int t = i / (chunks * 32), g = i - t * chunks * 32;    // group g of eight of token t
        uint4 u = make_uint4(0, 0, 0, 0);
        if (t < P.tokens && P.targets[t] >= 0 && P.targets[t] < P.vocab) u = eight_of_row(P.h + t * P.h_ld, g, P.dim, P.h_aligned);
        float x[8];
        eight_numbers<T>(u, x);
        float4 *to = few_hidden + ((t * chunks + (g >> 5)) * 2) * 32 + (g & 31);
        to[0] = make_float4(x[0], x[1], x[2], x[3]);
        to[32] = make_float4(x[4], x[5], x[6], x[7]);
    }
    __syncthreads();
    const long long label = lane < P.tokens ? P.targets[lane] : -1;
    float top = -INFINITY, sum = 0.0f;
    const long long warps = (long long)gridDim.x * kSmallWarps, at = (long long)blockIdx.x * kSmallWarps + warp;
    const int first = (int)(P.vocab * at / warps), end = (int)(P.vocab * (at + 1) / warps);
    for (int v = first; v < end; v += kFewRows) {
        const uint16_t *row[kFewRows];
#pragma unroll
        for (int j = 0; j < kFewRows; ++j) row[j] = P.w + (long long)min(v + j, end - 1) * P.w_ld;
        float acc[kFewRows][N] = {};
        uint4 next[kFewRows][kFewAhead<N>];             // rows' pieces on their way
        auto fetch = [&](int c, int slot) {
            const bool there = c * 256 + lane * 8 < P.dim;
#pragma unroll
            for (int j = 0; j < kFewRows; ++j) {
                next[j][slot] = make_uint4(0, 0, 0, 0);
                if (there) next[j][slot] = ALIGNED ? load_once(row[j] + c * 256 + lane * 8) : eight_of_row(row[j], c * 32 + lane, P.dim, false);
            }
        };
#pragma unroll
        for (int q = 0; q < kFewAhead<N>; ++q) fetch(q, q);
        for (int c0 = 0; c0 < chunks; c0 += kFewAhead<N>) {
#pragma unroll
            for (int q = 0; q < kFewAhead<N>; ++q) {
                const int c = min(c0 + q, chunks - 1);       // beyond the end: pieces of zeros
                float x[kFewRows][8];
#pragma unroll
                for (int j = 0; j < kFewRows; ++j) eight_numbers<T>(next[j][q], x[j]);
                fetch(c0 + q + kFewAhead<N>, q);
#pragma unroll
                for (int t = 0; t < N; ++t) {
                    const float4 a = few_hidden[((t * chunks + c) * 2) * 32 + lane], b = few_hidden[((t * chunks + c) * 2 + 1) * 32 + lane];
#pragma unroll
                    for (int j = 0; j < kFewRows; ++j) {
                        float s = acc[j][t];
                        s = fmaf(a.x, x[j][0], s); s = fmaf(a.y, x[j][1], s); s = fmaf(a.z, x[j][2], s); s = fmaf(a.w, x[j][3], s);
                        s = fmaf(b.x, x[j][4], s); s = fmaf(b.y, x[j][5], s); s = fmaf(b.z, x[j][6], s); s = fmaf(b.w, x[j][7], s);
                        acc[j][t] = s;
                    }
                }
            }
        }
#pragma unroll
        for (int j = 0; j < kFewRows; ++j) {
            float logit = 0.0f;
#pragma unroll
            for (int t = 0; t < N; ++t) {
                float s = acc[j][t];
#pragma unroll
                for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
                if (lane == t) logit = s;
            }
            if (v + j < end && lane < N) {
                if (v + j == label) P.label_logit[lane] = logit;
                const float x = logit * kLog2e, both = fmaxf(top, x), ref = both > -INFINITY ? both : 0.0f;
                sum = sum * exp2f(top - ref) + exp2f(x - ref);
                top = both;
            }
        }
    }
    if (lane < N) warp_stats[warp][lane] = make_float2(top, sum);
    __syncthreads();
    if (threadIdx.x < N) {
        for (int k = 1; k < kSmallWarps; ++k) join(top, sum, warp_stats[k][threadIdx.x].x, warp_stats[k][threadIdx.x].y);
        P.stats[blockIdx.x * N + threadIdx.x] = make_float2(top, sum);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicAdd(&P.control->tickets, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    if (warp < N) {                              // one warp per token joins the blocks
        const long long mine = warp < P.tokens ? P.targets[warp] : -1;
        const bool counts = mine >= 0 && mine < P.vocab;
        top = -INFINITY;
        sum = 0.0f;
        for (unsigned b = lane; b < gridDim.x; b += 32) {
            const float2 s = __ldcg(P.stats + b * N + warp);
            join(top, sum, s.x, s.y);
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            const float t2 = __shfl_xor_sync(0xffffffffu, top, off), s2 = __shfl_xor_sync(0xffffffffu, sum, off);
            join(top, sum, t2, s2);
        }
        if (lane == 0) {
            const float lse = counts ? (top + log2f(sum)) * kLn2 : 0.0f, one = counts ? lse - __ldcg(P.label_logit + warp) : 0.0f;
            if (warp < P.tokens) {
                if (P.rows != nullptr) P.rows[warp] = one;
                if (P.lse_out != nullptr) P.lse_out[warp] = lse;
            }
            token_loss[warp] = one;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        int n = 0;
        double total = 0.0;
        for (int t = 0; t < N && t < P.tokens; ++t) {
            n += P.targets[t] >= 0 && P.targets[t] < P.vocab ? 1 : 0;
            total += token_loss[t];
        }
        if (P.loss != nullptr) *P.loss = (float)(P.reduction == PSOPS_MEAN ? total / max(1, n) : total);
        P.control->tickets = 0;
    }
}

// ---- gradients of few tokens ------------------------------------------------------
// Up to 4 tokens: w is read once and dw written once, and that is all the
// traffic.  A team of warps (one for each 512 features, up to the whole block)
// takes a few rows of w at a time: the logits of the rows, then, with the rows still in registers, their part of dh and their rows
// of dw.  The teams' parts of dh are added up by a kernel behind.  fp32
// throughout, so nothing but the results is rounded to 16 bits.
// Rows at a time and blocks of an SM: what registers allow, the best of 1, 2 and 4
// rows with 1 to 4 blocks.
// Measured in a CUDA graph, this form / the tensor cores, us:
//   one token    32,768 x 4,096: 99 / 185 (537 MB: 82)    131,072 x 600: 89 / 157
//   two          32,768 x 4,096: 122 / 183   131,072 x 4,096: 454 / 659   131,072 x 64: 65 / 73
//   three, four  131,072 x 512: 98 / 126     32,768 x 1,024: 61 / 70      131,072 x 1,024: 193 / 200
//                16,384 x 4,096: 102 / 114   4,096 x 3,000: 31 / 58       32,768 x 768: 59 / 59
//                32,768 x 4,096: 190 / 185   131,072 x 2,048: 367 / 347   32,768 x 3,000: 187 / 158
//                32,768 x 1,536: 100 / 90    65,536 x 768: 104 / 96       65,536 x 128: 56 / 50
// From three tokens on the arithmetic bounds it, on whole warps of 512 features;
// the tensor cores cost some 15 us more in launches, then less per feature that
// is there and a little per row.  Where rows are not 16-byte aligned the element
// by element loads bound it from two tokens on: 4,096 x 2,100 with four tokens
// 61 / 70, 16,384 x 1,100 with two 90 / 90, 8,192 x 4,001 with two 177 / 159,
// 65,536 x 1,100 with two 387 / 299; with one 16,384 x 1,100 63 / 89.
constexpr int kFewGradDim = 4096;
template <int N> constexpr int kFewGradRows = N == 2 ? 4 : 2;
template <int N> constexpr int kFewGradBlocks = N == 1 ? 2 : 1;
inline int few_team(int64_t dim) { return dim <= 512 ? 1 : dim <= 1024 ? 2 : dim <= 2048 ? 4 : 8; }

inline bool few_grads_pay(int64_t tokens, int64_t dim, int64_t vocab, bool aligned)
{
    if (tokens == 1) return true;
    if (!aligned) return vocab * dim <= 1 << 24;
    return tokens == 2 || vocab * (9 * 512 * few_team(dim) - 8 * dim - 1024) < 3 << 25;
}

struct FewGradParams {
    const uint16_t *h, *w;
    long long h_ld, w_ld;
    bool h_aligned;
    const long long *targets;
    int tokens, dim, vocab, reduction, team;
    const float *lse, *known_rows, *grad;
    float *parts;                                // team x token x padded features
    int padded;
    bool want_dh;
    uint16_t *dw;                                // or NULL
    long long dw_ld;
};

__device__ __forceinline__ bool few_counts(const FewGradParams &P, int t)
{
    return t < P.tokens && P.targets[t] >= 0 && P.targets[t] < P.vocab;
}
__device__ __forceinline__ void team_sync(int team, int team_index)
{
    if (team == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(team_index + 1), "r"(team * 32) : "memory");
}

template <class T, int N, bool ALIGNED>
__global__ void __launch_bounds__(kSmallThreads, kFewGradBlocks<N>) psops_xent_few_grads_kernel(const FewGradParams P)
{
    constexpr int R = kFewGradRows<N>;
    __shared__ float sums[2][kSmallWarps][R * N];
    after_the_kernel_before();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int team_index = warp / P.team, in_team = warp - team_index * P.team;
    const int teams = gridDim.x * (kSmallWarps / P.team), me = blockIdx.x * (kSmallWarps / P.team) + team_index;
    const int group[2] = {(in_team * 2) * 32 + lane, (in_team * 2 + 1) * 32 + lane};     // this lane's groups of eight features
    const bool there[2] = {group[0] * 8 < P.dim, group[1] * 8 < P.dim};

    uint4 hidden[N][2];
    float dh[N][16];
    int n = 0;
#pragma unroll
    for (int t = 0; t < N; ++t) {
        const bool counts = few_counts(P, t);
        n += counts ? 1 : 0;
#pragma unroll
        for (int q = 0; q < 2; ++q)
            hidden[t][q] = counts && there[q] ? eight_of_row(P.h + t * P.h_ld, group[q], P.dim, P.h_aligned) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 16; ++e) dh[t][e] = 0.0f;
    }
    // lane (r * N + t) turns the logit of row r and token t into its gradient
    const int mt = lane % N, mr = lane / N;
    const bool mine = lane < R * N && few_counts(P, mt);
    const float lse = mine ? P.lse[mt] : 0.0f;
    const float at_label = mine && P.known_rows != nullptr ? expm1f(-P.known_rows[mt]) : 2.0f;
    const long long label = mine ? P.targets[mt] : -1;
    const float g = !mine ? 0.0f : P.reduction == PSOPS_PER_TOKEN ? P.grad[mt] : P.reduction == PSOPS_MEAN ? __fdiv_rn(P.grad[0], (float)max(1, n)) : P.grad[0];

    auto fetch = [&](long long v0, uint4 (&u)[R][2]) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                u[r][q] = make_uint4(0, 0, 0, 0);
                if (v0 + r < P.vocab && there[q]) {
                    const uint16_t *row = P.w + (v0 + r) * P.w_ld;
                    u[r][q] = ALIGNED ? load_once(row + group[q] * 8) : eight_of_row(row, group[q], P.dim, false);
                }
            }
    };
    auto sixteen = [](const uint4 (&u)[2], float (&x)[16]) {
        float a[8], b[8];
        eight_numbers<T>(u[0], a);
        eight_numbers<T>(u[1], b);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] = a[j];
            x[8 + j] = b[j];
        }
    };
    uint4 now[R][2], next[R][2];
    long long v0 = (long long)me * R;
    fetch(v0, next);
    for (int turn = 0; v0 < P.vocab; v0 += (long long)teams * R, turn ^= 1) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int q = 0; q < 2; ++q) now[r][q] = next[r][q];
        fetch(v0 + (long long)teams * R, next);
        // logits: this lane's features, the warp's, the team's
        float logit = 0.0f;                      // of row mr and token mt
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float x[16];
            sixteen(now[r], x);
#pragma unroll
            for (int t = 0; t < N; ++t) {
                float k[16], s = 0.0f;
                sixteen(hidden[t], k);
#pragma unroll
                for (int e = 0; e < 16; ++e) s = fmaf(x[e], k[e], s);
#pragma unroll
                for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
                if (lane == r * N + t) logit = s;
            }
        }
        if (P.team > 1) {
            if (lane < R * N) sums[turn][warp][lane] = logit;
            team_sync(P.team, team_index);
            if (lane < R * N) {
                logit = 0.0f;
                for (int k = 0; k < P.team; ++k) logit += sums[turn][team_index * P.team + k][lane];
            }
        }
        float d = 0.0f;
        if (mine && v0 + mr < P.vocab) {
            if (v0 + mr != label) d = expf(logit - lse) * g;
            else d = (at_label > 1.0f ? expm1f(logit - lse) : at_label) * g;
        }
        // dh and dw of these rows
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float row[16], x[16];
            sixteen(now[r], x);
#pragma unroll
            for (int e = 0; e < 16; ++e) row[e] = 0.0f;
#pragma unroll
            for (int t = 0; t < N; ++t) {
                const float dt = __shfl_sync(0xffffffffu, d, r * N + t);
                float k[16];
                sixteen(hidden[t], k);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    row[e] = fmaf(dt, k[e], row[e]);
                    dh[t][e] = fmaf(dt, x[e], dh[t][e]);
                }
            }
            if (P.dw != nullptr && v0 + r < P.vocab) {
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    if (there[q]) {
                        uint16_t *to = P.dw + (v0 + r) * P.dw_ld + group[q] * 8;
                        const uint4 u = make_uint4(pack2<T>(row[q * 8], row[q * 8 + 1]), pack2<T>(row[q * 8 + 2], row[q * 8 + 3]),
                                                   pack2<T>(row[q * 8 + 4], row[q * 8 + 5]), pack2<T>(row[q * 8 + 6], row[q * 8 + 7]));
                        if (ALIGNED) {
                            *reinterpret_cast<uint4 *>(to) = u;
                        } else {
                            uint16_t e[8];
                            memcpy(e, &u, 16);
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                if (group[q] * 8 + j < P.dim) to[j] = e[j];
                        }
                    }
            }
        }
    }
    if (!P.want_dh) return;
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
        for (int q = 0; q < 2; ++q)
            if (there[q]) {
                float4 *to = reinterpret_cast<float4 *>(P.parts + ((long long)me * N + t) * P.padded + group[q] * 8);
                to[0] = make_float4(dh[t][q * 8], dh[t][q * 8 + 1], dh[t][q * 8 + 2], dh[t][q * 8 + 3]);
                to[1] = make_float4(dh[t][q * 8 + 4], dh[t][q * 8 + 5], dh[t][q * 8 + 6], dh[t][q * 8 + 7]);
            }
}

// dh from the teams' parts: a block has 32 features of a token, its warps share the teams.
template <class T>
__global__ void __launch_bounds__(kSmallThreads) psops_xent_few_dh_kernel(const float *parts, int teams, int few, int padded,
                                                                          const long long *targets, int vocab, int dim, T *dh, long long ld)
{
    __shared__ float sums[kSmallWarps][33];
    after_the_kernel_before();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = blockIdx.y, d = blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (d < dim)
#pragma unroll 8
        for (int k = warp; k < teams; k += kSmallWarps) s += parts[((long long)k * few + t) * padded + d];
    sums[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && d < dim) {
        for (int k = 1; k < kSmallWarps; ++k) s += sums[k][lane];
        const long long y = targets[t];
        dh[t * ld + d] = narrow16<T>(y >= 0 && y < vocab ? s : 0.0f);
    }
}

} // namespace
