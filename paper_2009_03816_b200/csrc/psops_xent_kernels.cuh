// psops_xent_kernels.cuh -- softmax cross entropy of a linear head and its
// gradients (C entries: psops_xent.cu).
//
// A call first lists the tokens that count (psops_xent_index_kernel) and
// gathers their hidden states, padded with zeros to whole tiles
// (psops_xent_gather_kernel); everything after works on these "compact" rows,
// so that tokens without a loss cost nothing and their contents cannot reach a
// result.  The number of compact rows is known on the device only.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace {

constexpr int kTileRows = 256;                   // compact rows are padded to this
constexpr int kTileCols = 256;                   // vocabulary entries of a logits tile
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct XentControl {
    int rows;                                    // tokens that count
    unsigned tickets;
    float unscale;                               // power of two: gradient sums * unscale = gradients
    int error;
};

template <class T> __device__ __forceinline__ float widen16(T x);
template <> __device__ __forceinline__ float widen16(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float widen16(__nv_bfloat16 x) { return __bfloat162float(x); }
template <class T> __device__ __forceinline__ T narrow16(float x);
template <> __device__ __forceinline__ __half narrow16(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 narrow16(float x) { return __float2bfloat16_rn(x); }

struct IndexParams {
    const long long *targets;
    const float *grad;                           // NULL in the forward pass
    XentControl *control;
    int *row_of;                                 // compact row -> token
    int *compact_of;                             // token -> compact row, or -1
    int *label;                                  // compact row -> label
    float *row_scale;                            // compact row -> grad_t times a power of two (backward)
    float *rows_out, *lse_out;                   // zeroed where a token is left out (forward)
    const float *lse;                            // (backward) by token
    float *row_lse;                              // (backward) by compact row, times log2 e
    int tokens;
    int vocab;
    int reduction;
    float headroom;                              // largest |dlogits| that the 16-bit type should see
};

constexpr int kIndexThreads = 1024;

// One block lists the tokens that count, in order.
__global__ void __launch_bounds__(kIndexThreads) psops_xent_index_kernel(const IndexParams P)
{
    __shared__ int warp_sum[32];
    __shared__ float warp_top[32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (P.tokens + kIndexThreads - 1) / kIndexThreads;
    const int first = tid * per, last = min(P.tokens, first + per);
    int mine = 0;
    float top = 0.0f;
    for (int t = first; t < last; ++t) {
        const long long y = P.targets[t];
        if (y >= 0 && y < P.vocab) {
            ++mine;
            if (P.grad != nullptr && P.reduction == PSOPS_PER_TOKEN) top = fmaxf(top, fabsf(P.grad[t]));
        }
    }
    int upto = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, upto, off);
        if (lane >= off) upto += v;
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    if (lane == 31) warp_sum[warp] = upto;
    if (lane == 0) warp_top[warp] = top;
    __syncthreads();
    int before = 0, total = 0;
    top = 0.0f;
    for (int w = 0; w < 32; ++w) {
        if (w < warp) before += warp_sum[w];
        total += warp_sum[w];
        top = fmaxf(top, warp_top[w]);
    }
    float common = 0.0f, up = 1.0f;
    if (P.grad != nullptr) {
        if (P.reduction != PSOPS_PER_TOKEN) {
            common = P.reduction == PSOPS_MEAN ? __fdiv_rn(P.grad[0], (float)max(1, total)) : P.grad[0];
            top = fabsf(common);
        }
        // gradients are normalised by a power of two, so that the largest |grad_t| lies in (1/2, 1] * headroom
        int e = 0;
        if (top > 0.0f && top < INFINITY) e = min(120, max(-100, ilogbf(top) + 1));
        up = ldexpf(P.headroom, -e);
        if (tid == 0) P.control->unscale = 1.0f / up;
    }
    int at = before + upto - mine;
    for (int t = first; t < last; ++t) {
        const long long y = P.targets[t];
        if (y >= 0 && y < P.vocab) {
            P.row_of[at] = t;
            P.label[at] = (int)y;
            P.compact_of[t] = at;
            if (P.grad != nullptr) {
                P.row_scale[at] = (P.reduction == PSOPS_PER_TOKEN ? P.grad[t] : common) * up;
                P.row_lse[at] = P.lse[t] * kLog2e;
            }
            ++at;
        } else {
            P.compact_of[t] = -1;
            if (P.rows_out != nullptr) P.rows_out[t] = 0.0f;
            if (P.lse_out != nullptr) P.lse_out[t] = 0.0f;
        }
    }
    if (tid == 0) {
        P.control->rows = total;
        P.control->tickets = 0;
    }
}

// A row of 16-bit values, `n` of them, into a row of `padded` (a multiple of
// 8, 16-byte aligned) with zeros behind; src == nullptr: all zeros.
__device__ __forceinline__ void copy_row(uint16_t *dst, const uint16_t *src, int n, int padded, bool aligned, int lane, int lanes)
{
    for (int g = lane; g < padded / 8; g += lanes) {
        uint4 u = make_uint4(0, 0, 0, 0);
        if (src != nullptr) {
            if (aligned && g * 8 + 8 <= n) {
                u = *reinterpret_cast<const uint4 *>(src + g * 8);
            } else {
                uint16_t e[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) e[j] = g * 8 + j < n ? src[g * 8 + j] : (uint16_t)0;
                u = make_uint4(e[0] | (unsigned)e[1] << 16, e[2] | (unsigned)e[3] << 16, e[4] | (unsigned)e[5] << 16, e[6] | (unsigned)e[7] << 16);
            }
        }
        *reinterpret_cast<uint4 *>(dst + g * 8) = u;
    }
}

constexpr int kCopyThreads = 256;

// Hidden states of the tokens that count, one warp per row; zero rows up to a whole tile.
__global__ void __launch_bounds__(kCopyThreads) psops_xent_gather_kernel(const uint16_t *h, long long ld, int dim, int padded,
                                                                         bool aligned, const XentControl *control,
                                                                         const int *row_of, uint16_t *out)
{
    const int rows = control->rows;
    const int whole = max(1, (rows + kTileRows - 1) / kTileRows) * kTileRows;
    const int warps = gridDim.x * (kCopyThreads / 32);
    for (int r = blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5); r < whole; r += warps)
        copy_row(out + (long long)r * padded, r < rows ? h + row_of[r] * ld : nullptr, dim, padded, aligned, threadIdx.x & 31, 32);
}

// Rows of w that cannot be read in place.
__global__ void __launch_bounds__(kCopyThreads) psops_xent_pack_kernel(const uint16_t *w, long long ld, long long rows, int dim,
                                                                       int padded, uint16_t *out)
{
    const long long warps = (long long)gridDim.x * (kCopyThreads / 32);
    for (long long r = (long long)blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5); r < rows; r += warps)
        copy_row(out + r * padded, w + r * ld, dim, padded, false, threadIdx.x & 31, 32);
}

// Rows of dw that could not be written in place.
__global__ void __launch_bounds__(kCopyThreads) psops_xent_unpack_kernel(const uint16_t *in, int padded, long long rows, int dim,
                                                                         uint16_t *dw, long long ld)
{
    const long long warps = (long long)gridDim.x * (kCopyThreads / 32);
    for (long long r = (long long)blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5); r < rows; r += warps)
        for (int d = threadIdx.x & 31; d < dim; d += 32) dw[r * ld + d] = in[r * padded + d];
}

// ---------------------------------------------------------------------------
// Products: 64 x 64 tiles of fp32 sums, 256 threads with 4 x 4 sums each
// ---------------------------------------------------------------------------
constexpr int kSimple = 64, kSimpleK = 16, kSimpleThreads = 256;

template <class LoadA, class LoadB>
__device__ __forceinline__ void simple_tile(LoadA a, LoadB b, int depth, float (&acc)[4][4])
{
    __shared__ float sa[kSimpleK][kSimple + 1], sb[kSimpleK][kSimple + 1];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) acc[i][j] = 0.0f;
    for (int k0 = 0; k0 < depth; k0 += kSimpleK) {
        __syncthreads();
        for (int i = threadIdx.x; i < kSimple * kSimpleK; i += kSimpleThreads) {
            const int k = i % kSimpleK, m = i / kSimpleK;
            sa[k][m] = k0 + k < depth ? a(m, k0 + k) : 0.0f;
            sb[k][m] = k0 + k < depth ? b(m, k0 + k) : 0.0f;
        }
        __syncthreads();
        for (int k = 0; k < kSimpleK; ++k)
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sa[k][ty * 4 + i], sb[k][tx * 4 + j], acc[i][j]);
    }
}

struct LogitsParams {
    const void *h, *w;                           // compact hidden states; the piece's rows of w
    int64_t w_ld;
    int h_ld, dim;
    int first, count;                            // the piece: vocabulary entries [first, first + count)
    const XentControl *control;
    const int *label;
    float2 *stats;                               // (max, sum of exp2) by part of the vocabulary and compact row, base 2
    long long stats_ld;
    float *label_logit;
    const float *row_lse, *row_scale;
    void *dlogits;                               // compact rows x piece
    long long dlogits_ld;
};

template <class T, bool GRADS>
__global__ void __launch_bounds__(kSimpleThreads) psops_xent_logits_kernel(const LogitsParams P)
{
    const int rows = P.control->rows;
    const int whole = max(1, (rows + kTileRows - 1) / kTileRows) * kTileRows;
    const int m0 = blockIdx.y * kSimple, n0 = blockIdx.x * kSimple;
    if (m0 >= whole) return;
    const T *h = (const T *)P.h, *w = (const T *)P.w;
    float acc[4][4];
    simple_tile([&](int m, int k) { return widen16(h[(long long)(m0 + m) * P.h_ld + k]); },
                [&](int n, int k) { return n0 + n < P.count ? widen16(w[(n0 + n) * P.w_ld + k]) : 0.0f; }, P.dim, acc);
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (int i = 0; i < 4; ++i) {
        const int r = m0 + ty * 4 + i;
        const int y = r < rows ? P.label[r] - P.first : -1;
        float top = -INFINITY;
        for (int j = 0; j < 4; ++j) {
            const int c = n0 + tx * 4 + j;
            if (c == y && !GRADS) P.label_logit[r] = acc[i][j];
            acc[i][j] *= kLog2e;
            if (c >= P.count) acc[i][j] = -INFINITY;
            top = fmaxf(top, acc[i][j]);
        }
        if (!GRADS) {
            for (int off = 8; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            const float ref = top > -INFINITY ? top : 0.0f;
            float s = 0.0f;
            for (int j = 0; j < 4; ++j) s += exp2f(acc[i][j] - ref);
            for (int off = 8; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
            if (tx == 0) P.stats[(long long)((P.first + n0) / kSimple) * P.stats_ld + r] = make_float2(top, s);
        } else {
            const float lse = r < rows ? P.row_lse[r] : 0.0f, g = r < rows ? P.row_scale[r] : 0.0f;
            for (int j = 0; j < 4; ++j) {
                const int c = n0 + tx * 4 + j;
                float d = 0.0f;
                if (r < rows && c < P.count) d = (exp2f(acc[i][j] - lse) - (c == y ? 1.0f : 0.0f)) * g;
                if (c < P.dlogits_ld) ((T *)P.dlogits)[r * P.dlogits_ld + c] = narrow16<T>(d);
            }
        }
    }
}

struct DhParams {
    const void *dlogits, *w;
    long long dlogits_ld, w_ld;
    int dim, count;
    bool add;
    const XentControl *control;
    float *sums;
    long long sums_ld;
};

template <class T>
__global__ void __launch_bounds__(kSimpleThreads) psops_xent_dh_kernel(const DhParams P)
{
    const int rows = P.control->rows;
    const int m0 = blockIdx.y * kSimple, n0 = blockIdx.x * kSimple;
    if (m0 >= rows) return;
    const T *d = (const T *)P.dlogits, *w = (const T *)P.w;
    float acc[4][4];
    simple_tile([&](int m, int k) { return widen16(d[(m0 + m) * P.dlogits_ld + k]); },
                [&](int n, int k) { return n0 + n < P.dim ? widen16(w[k * P.w_ld + n0 + n]) : 0.0f; }, P.count, acc);
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int r = m0 + ty * 4 + i, c = n0 + tx * 4 + j;
            if (r < rows && c < P.dim) {
                float *at = P.sums + r * P.sums_ld + c;
                *at = P.add ? *at + acc[i][j] : acc[i][j];
            }
        }
}

struct DwParams {
    const void *dlogits, *h;
    long long dlogits_ld;
    int h_ld, dim, count;
    const XentControl *control;
    void *dw;
    long long dw_ld;
};

template <class T>
__global__ void __launch_bounds__(kSimpleThreads) psops_xent_dw_kernel(const DwParams P)
{
    const int rows = P.control->rows;
    const float unscale = P.control->unscale;
    const long long m0 = (long long)blockIdx.y * kSimple;
    const int n0 = blockIdx.x * kSimple;
    const T *d = (const T *)P.dlogits, *h = (const T *)P.h;
    float acc[4][4];
    simple_tile([&](int m, int k) { return m0 + m < P.count ? widen16(d[k * P.dlogits_ld + m0 + m]) : 0.0f; },
                [&](int n, int k) { return n0 + n < P.dim ? widen16(h[(long long)k * P.h_ld + n0 + n]) : 0.0f; }, rows, acc);
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const long long r = m0 + ty * 4 + i;
            const int c = n0 + tx * 4 + j;
            if (r < P.count && c < P.dim) ((T *)P.dw)[r * P.dw_ld + c] = narrow16<T>(acc[i][j] * unscale);
        }
}

// ---------------------------------------------------------------------------
// Joining the pieces
// ---------------------------------------------------------------------------
constexpr int kJoinRows = 32, kJoinParts = 8;    // a block: 32 compact rows, each joined by 8 threads

struct JoinParams {
    const float2 *stats;
    long long stats_ld;
    int parts;
    XentControl *control;
    const int *row_of;
    const float *label_logit;
    float *rows_out, *lse_out, *loss;
    double *partials;                            // one per block
    int reduction;
};

__device__ __forceinline__ void join(float &top, float &sum, float top2, float sum2)
{
    // maxima leave NaN out, sums carry it on
    const float both = fmaxf(top, top2), ref = both > -INFINITY ? both : 0.0f;
    sum = sum * exp2f(top - ref) + sum2 * exp2f(top2 - ref);
    top = both;
}

// lse and loss of every row from its parts' maxima and sums; the block that
// comes last adds up the loss, always in the same order.
__global__ void __launch_bounds__(kJoinRows * kJoinParts) psops_xent_join_kernel(const JoinParams P)
{
    __shared__ float tops[kJoinParts][kJoinRows], sums[kJoinParts][kJoinRows];
    __shared__ double row_loss[kJoinRows];
    __shared__ bool last;
    const int rows = P.control->rows;
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int r = blockIdx.x * kJoinRows + lane;
    float top = -INFINITY, sum = 0.0f;
    if (r < rows)
        for (int k = part; k < P.parts; k += kJoinParts) {
            const float2 s = P.stats[k * P.stats_ld + r];
            join(top, sum, s.x, s.y);
        }
    tops[part][lane] = top;
    sums[part][lane] = sum;
    __syncthreads();
    if (part == 0) {
        double loss = 0.0;
        if (r < rows) {
            for (int k = 1; k < kJoinParts; ++k) join(top, sum, tops[k][lane], sums[k][lane]);
            const float lse = (top + log2f(sum)) * kLn2, mine = lse - P.label_logit[r];
            const int t = P.row_of[r];
            if (P.rows_out != nullptr) P.rows_out[t] = mine;
            if (P.lse_out != nullptr) P.lse_out[t] = lse;
            loss = mine;
        }
        row_loss[lane] = loss;
        __syncwarp();
        if (lane == 0) {
            for (int k = 1; k < kJoinRows; ++k) loss += row_loss[k];
            P.partials[blockIdx.x] = loss;
            __threadfence();
            last = atomicAdd(&P.control->tickets, 1u) == gridDim.x - 1;
        }
    }
    __syncthreads();
    if (!last || threadIdx.x >= 32 || P.loss == nullptr) return;
    __threadfence();
    double total = 0.0;
    for (unsigned b = lane; b < gridDim.x; b += 32) total += __ldcg(P.partials + b);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) total += __shfl_xor_sync(0xffffffffu, total, off);
    if (lane == 0) *P.loss = P.reduction == PSOPS_MEAN ? (float)(total / (double)max(1, rows)) : (float)total;
}

// dh in the caller's rows from the compact sums, rounded once; zero where a token is left out.
template <class T>
__global__ void __launch_bounds__(kCopyThreads) psops_xent_dh_out_kernel(const float *sums, long long sums_ld, const XentControl *control,
                                                                         const int *compact_of, int tokens, int dim, T *dh, long long ld)
{
    const float unscale = control->unscale;
    const int warps = gridDim.x * (kCopyThreads / 32);
    for (int t = blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5); t < tokens; t += warps) {
        const int r = compact_of[t];
        for (int d = threadIdx.x & 31; d < dim; d += 32)
            dh[t * ld + d] = r < 0 ? narrow16<T>(0.0f) : narrow16<T>(sums[r * sums_ld + d] * unscale);
    }
}

} // namespace
