// psops_attention_kernels.cuh -- causal attention over packed sequences, with
// grouped heads and a learned bias by buckets of the distance, and its gradients.
//
//   x[i, j] = scale q_i . k_j + bias[bucket(i - j)],  j <= i of one sequence
//   p = exp(x - lse),  o_i = sum_j p[i, j] v_j
//   dv_j = sum_i p[i, j] do_i,  ds[i, j] = p[i, j] (do_i . v_j - do_i . o_i)
//   dq_i = scale sum_j ds[i, j] k_j,  dk_j = scale sum_i ds[i, j] q_i,  dbias[b] = sum of ds over pairs of bucket b
//
// Scores live in tensor memory only.  A sequence is cut into tiles of 128 tokens
// from its first one, so that only tiles on the diagonal have masked pairs.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>
#include <cstring>

#include "psops_umma.cuh"

namespace psops_attention_k {

constexpr int kTile = 128;
constexpr int kMostBuckets = 64, kMostDistance = 1024;
constexpr int kMostDim = 128;
constexpr int kHalfBytes = kTile * 128;          // 64 elements of each of 128 tokens
constexpr int kBefore = 128;                     // places of the distance table for pairs above the diagonal
constexpr int kTableFloats = kBefore + kMostDistance + 2 * kTile;
constexpr int kPrepThreads = 512, kBins = 1024;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// A tile of a sequence.
struct Item {
    int first, length;       // first token and tokens of its sequence
    int level;               // its number, counted so that its work grows with it
    int slot;                // the same for the same tile of the same batch in any call
};

struct Heads {               // tokens x heads x dim, elements of a head consecutive
    void *p;
    long long token, head;   // strides in elements
};

struct PrepParams {
    const int *offsets;
    int sequences, tokens, capacity;
    Item *items;
    int *count;
    int *used;               // NULL, or by slot whether a tile has it
    int heads, kv_heads, dim;
    int fill;                // how many of `rest` are to be zeroed where no sequence is
    Heads rest[3];
    int rest_heads[3];
    float *rest_lse;
    // backward
    Heads out, grad, v;
    float *delta;            // NULL in a forward pass
    float2 *norms;           // NULL, or for each block but the first the largest squared norms of grad's and v's rows
};

__device__ __forceinline__ int clamped(int x, int low, int high) { return min(max(x, low), high); }

template <class T> __device__ __forceinline__ float2 unpack2(uint32_t u);
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t u)
{
    __half2 h;
    memcpy(&h, &u, 4);
    return __half22float2(h);
}
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t u)
{
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}
template <class T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    uint32_t u;
    memcpy(&u, &h, 4);
    return u;
}
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    uint32_t u;
    memcpy(&u, &h, 4);
    return u;
}
// Off by some units of 2^-23 of the result, less than the rounding of a probability to 16 bits by far.
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Two fp32 numbers in one instruction, each as by itself.
__device__ __forceinline__ uint64_t pair_of(uint32_t low, uint32_t high)
{
    uint64_t x;
    asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "r"(low), "r"(high));
    return x;
}
__device__ __forceinline__ uint64_t both(float x) { return pair_of(__float_as_uint(x), __float_as_uint(x)); }
__device__ __forceinline__ float low_of(uint64_t x) { return __uint_as_float((uint32_t)x); }
__device__ __forceinline__ float high_of(uint64_t x) { return __uint_as_float((uint32_t)(x >> 32)); }
__device__ __forceinline__ uint64_t fma_both(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t x;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(x) : "l"(a), "l"(b), "l"(c));
    return x;
}
__device__ __forceinline__ uint64_t add_both(uint64_t a, uint64_t b)
{
    uint64_t x;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(x) : "l"(a), "l"(b));
    return x;
}
__device__ __forceinline__ uint64_t mul_both(uint64_t a, uint64_t b)
{
    uint64_t x;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(x) : "l"(a), "l"(b));
    return x;
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float x;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(x) : "f"(a), "f"(b), "f"(c));
    return x;
}

// ---------------------------------------------------------------------------
// The list of tiles, most work first; rows of no sequence; delta
// ---------------------------------------------------------------------------

// One block.  Tiles go into bins by level (several levels to a bin only beyond
// kBins of them); within a bin the order is left to chance, which changes when
// a tile is done and nothing else.
__device__ __forceinline__ void make_list(const PrepParams &P)
{
    __shared__ int sequences_at[kBins + 1], rest_at[kBins + 1], next[kBins];
    const int most = (P.tokens + kTile - 1) / kTile;
    int shift = 0;
    while ((most >> shift) >= kBins) ++shift;
    const int bins = (most >> shift) + 1;
    for (int i = threadIdx.x; i <= bins; i += kPrepThreads) sequences_at[i] = rest_at[i] = 0;
    if (P.used != nullptr)
        for (int i = threadIdx.x; i < P.capacity; i += kPrepThreads) P.used[i] = 0;
    __syncthreads();
    auto bounds = [&](int b, int &first, int &length) {
        first = clamped(P.offsets[b], 0, P.tokens);
        length = max(clamped(P.offsets[b + 1], 0, P.tokens) - first, 0);
    };
    for (int b = threadIdx.x; b < P.sequences; b += kPrepThreads) {
        int first, length;
        bounds(b, first, length);
        const int tiles = (length + kTile - 1) / kTile;
        atomicAdd(&sequences_at[tiles >> shift], 1);
        atomicAdd(&rest_at[tiles >> shift], tiles & ((1 << shift) - 1));
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        // lane 0 has the highest bins
        const int lane = threadIdx.x, each = (bins + 31) / 32;
        const int top = bins - lane * each, low = max(top - each, 0);
        int above = 0;
        for (int j = top - 1; j >= low; --j) above += sequences_at[j];
        const int mine = above;
        for (int d = 1; d < 32; d *= 2) {
            const int n = __shfl_up_sync(0xffffffffu, above, d);
            if (lane >= d) above += n;
        }
        above -= mine;                                       // sequences that go beyond this lane's bins
        int total = 0;
        for (int j = top - 1; j >= low; --j) {
            next[j] = total;
            total += (above << shift) + rest_at[j];
            above += sequences_at[j];
        }
        int before = total;
        for (int d = 1; d < 32; d *= 2) {
            const int n = __shfl_up_sync(0xffffffffu, before, d);
            if (lane >= d) before += n;
        }
        for (int j = top - 1; j >= low; --j) next[j] += before - total;
        if (lane == 31) *P.count = min(before, P.capacity);
    }
    __syncthreads();
    auto place = [&](int first, int length, int slot, int level) {
        const int at = atomicAdd(&next[level >> shift], 1);
        if (at < P.capacity && slot + level < P.capacity) {
            P.items[at] = Item{first, length, level, slot + level};
            if (P.used != nullptr) P.used[slot + level] = 1;
        } else if (at < P.capacity) {
            P.items[at] = Item{0, 0, 0, 0};                  // offsets that decrease
        }
    };
    const int lane = threadIdx.x & 31;
    for (int b0 = threadIdx.x & ~31; b0 < P.sequences; b0 += kPrepThreads) {
        const int b = b0 + lane;
        int first = 0, length = 0;
        if (b < P.sequences) bounds(b, first, length);
        const int tiles = (length + kTile - 1) / kTile, slot = first / kTile + b;
        if (tiles <= 2)
            for (int l = 0; l < tiles; ++l) place(first, length, slot, l);
        for (uint32_t left = __ballot_sync(0xffffffffu, tiles > 2); left != 0; left &= left - 1) {
            const int of = __ffs(left) - 1;
            const int f = __shfl_sync(0xffffffffu, first, of), n = __shfl_sync(0xffffffffu, length, of);
            const int s = __shfl_sync(0xffffffffu, slot, of), many = (n + kTile - 1) / kTile;
            for (int l = lane; l < many; l += 32) place(f, n, s, l);
        }
    }
}

// Zeroes what the call's own tensors hold where no sequence is.
__device__ __forceinline__ void fill_rest(const PrepParams &P, int block, int blocks)
{
    const int low = P.sequences > 0 ? clamped(P.offsets[0], 0, P.tokens) : 0;
    const int high = P.sequences > 0 ? max(clamped(P.offsets[P.sequences], 0, P.tokens), low) : 0;
    const int count = low + P.tokens - high, words = P.dim / 8;
    for (int t = 0; t < P.fill; ++t) {
        const int per_token = P.rest_heads[t] * words;
        for (long long i = (long long)block * kPrepThreads + threadIdx.x; i < (long long)count * per_token; i += (long long)blocks * kPrepThreads) {
            const int n = (int)(i / per_token), w = (int)(i % per_token), token = n < low ? n : high + n - low;
            uint16_t *row = (uint16_t *)P.rest[t].p + token * P.rest[t].token + (w / words) * P.rest[t].head;
            *(uint4 *)(row + (w % words) * 8) = make_uint4(0, 0, 0, 0);
        }
    }
    if (P.rest_lse != nullptr)
        for (long long i = (long long)block * kPrepThreads + threadIdx.x; i < (long long)count * P.heads; i += (long long)blocks * kPrepThreads) {
            const int n = (int)(i % count), token = n < low ? n : high + n - low;
            P.rest_lse[i / count * P.tokens + token] = 0.0f;
        }
}

template <class T>
__device__ __forceinline__ float dot8(uint4 a, uint4 b)
{
    float sum = 0.0f;
    const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 u = unpack2<T>(x[j]), v = unpack2<T>(y[j]);
        sum = __fmaf_rn(u.x, v.x, sum);
        sum = __fmaf_rn(u.y, v.y, sum);
    }
    return sum;
}

// delta[h, t] = do . o of each token and head: 16 lanes a row.  With norms, the
// largest squared norm of a row of do and of v (rows that are not finite left
// out): together they bound ds.
template <class T>
__device__ __forceinline__ void make_delta(const PrepParams &P, int block, int blocks)
{
    const int lane = threadIdx.x & 15, teams = kPrepThreads / 16;
    const bool on = lane * 8 < P.dim;
    const long long rows = (long long)P.tokens * P.heads, step = (long long)blocks * teams;
    float most_grad = 0.0f, most_v = 0.0f;
    constexpr int U = 4;
    for (long long r0 = (long long)block * teams + threadIdx.x / 16; r0 - threadIdx.x / 16 < rows; r0 += U * step) {
        uint4 g[U], o[U];
        long long to[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long r = r0 + u * step;
            g[u] = o[u] = make_uint4(0, 0, 0, 0);
            to[u] = -1;
            if (r < rows) {
                const int token = (int)(r / P.heads), head = (int)(r % P.heads);
                to[u] = (long long)head * P.tokens + token;
                if (on) {
                    g[u] = *(const uint4 *)((const uint16_t *)P.grad.p + token * P.grad.token + head * P.grad.head + lane * 8);
                    o[u] = *(const uint4 *)((const uint16_t *)P.out.p + token * P.out.token + head * P.out.head + lane * 8);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float sum = dot8<T>(g[u], o[u]), square = P.norms != nullptr ? dot8<T>(g[u], g[u]) : 0.0f;
#pragma unroll
            for (int d = 8; d > 0; d /= 2) {
                sum += __shfl_xor_sync(0xffffffffu, sum, d);
                square += __shfl_xor_sync(0xffffffffu, square, d);
            }
            if (lane == 0 && to[u] >= 0) P.delta[to[u]] = sum;
            if (square < INFINITY) most_grad = fmaxf(most_grad, square);
        }
    }
    if (P.norms == nullptr) return;
    const long long v_rows = (long long)P.tokens * P.kv_heads;
    for (long long r = (long long)block * teams + threadIdx.x / 16; r - threadIdx.x / 16 < v_rows; r += step) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (r < v_rows && on)
            v = *(const uint4 *)((const uint16_t *)P.v.p + r / P.kv_heads * P.v.token + r % P.kv_heads * P.v.head + lane * 8);
        float square = dot8<T>(v, v);
#pragma unroll
        for (int d = 8; d > 0; d /= 2) square += __shfl_xor_sync(0xffffffffu, square, d);
        if (square < INFINITY) most_v = fmaxf(most_v, square);
    }
    __shared__ float2 most[kPrepThreads / 32];
#pragma unroll
    for (int d = 16; d > 0; d /= 2) {
        most_grad = fmaxf(most_grad, __shfl_xor_sync(0xffffffffu, most_grad, d));
        most_v = fmaxf(most_v, __shfl_xor_sync(0xffffffffu, most_v, d));
    }
    if ((threadIdx.x & 31) == 0) most[threadIdx.x / 32] = make_float2(most_grad, most_v);
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kPrepThreads / 32; ++w) {
            most_grad = fmaxf(most_grad, most[w].x);
            most_v = fmaxf(most_v, most[w].y);
        }
        P.norms[block] = make_float2(most_grad, most_v);
    }
}

template <class T>
__global__ void __launch_bounds__(kPrepThreads) psops_attention_prepare_kernel(const PrepParams P)
{
    umma::after_the_kernel_before();
    if (blockIdx.x == 0) {
        make_list(P);
        return;
    }
    const int block = blockIdx.x - 1, blocks = gridDim.x - 1;
    if (P.fill > 0) fill_rest(P, block, blocks);
    if (P.delta != nullptr) make_delta<T>(P, block, blocks);
}

// ---------------------------------------------------------------------------
// What the two tensor-core kernels share
// ---------------------------------------------------------------------------

struct Bias {
    const void *p;                           // buckets x heads, NULL for none
    int fp32;                                // else of the call's 16-bit type
    int buckets, last;                       // last: the first distance of the last bucket
    int first[kMostBuckets];                 // the first distance of each bucket
};

// In base 2.  What lies below -1e30, such as the lowest number of a type, takes its
// pairs out as -inf does: no row's lse could hold it beside a logarithm.
template <class T>
__device__ __forceinline__ float bias_at(const Bias &B, int bucket, int heads, int head)
{
    const long long i = (long long)bucket * heads + head;
    const float b = B.fp32 ? ((const float *)B.p)[i] : (float)((const T *)B.p)[i];
    const float x = b * kLog2e;
    return x < -1e30f ? -INFINITY : x;
}
__device__ __forceinline__ void barrier_named(int id, int threads)
{
    asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// What the softmax threads of a CTA keep of the bias; distances up to a tile's
// reach beyond the last bucket's beginning.
struct Tables {
    float value[kMostBuckets];               // of the head at hand
    int first[kMostBuckets];
    uint8_t bucket[kMostDistance + 2 * kTile];
    float distance[kTableFloats];            // [kBefore + d]: the bias of distance d
};
// By THREADS threads that share barrier 1, after each has put its part of `value` in place.
template <int THREADS, bool BUCKETS>
__device__ __forceinline__ void make_tables(const Bias &B, Tables &t)
{
    const int many = B.last + 2 * kTile;
    if (BUCKETS && threadIdx.x < kMostBuckets) t.first[threadIdx.x] = threadIdx.x < B.buckets ? B.first[threadIdx.x] : INT32_MAX;
    barrier_named(1, THREADS);
    if (BUCKETS && threadIdx.x < kBefore) t.distance[threadIdx.x] = 0.0f;
    for (int d = threadIdx.x; d < many; d += THREADS) {
        int bucket;
        if (BUCKETS) {
            bucket = 0;
#pragma unroll
            for (int step = kMostBuckets / 2; step > 0; step /= 2)           // the last one that begins at d or before
                if (t.first[bucket + step] <= d) bucket += step;
            t.bucket[d] = (uint8_t)bucket;
        } else {
            bucket = t.bucket[d];
        }
        t.distance[kBefore + d] = t.value[bucket];
    }
    barrier_named(1, THREADS);
}

// Numbers that are not finite in a row of a tile (two boxes of 64 elements for
// dim > 64) become zeros, so that a probability of zero meets none.  True if
// there were any.  The row's eight 16-byte words are taken in the swizzle's order.
template <class T>
__device__ __forceinline__ bool clean_row(uint8_t *tile, int row, int halves)
{
    bool any = false;
    for (int h = 0; h < halves; ++h) {
        uint8_t *at = tile + h * kHalfBytes + row * 128;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            uint4 *word = (uint4 *)(at + ((c ^ (row & 7)) << 4));
            uint4 w = *word;
            uint32_t x[4] = {w.x, w.y, w.z, w.w};
            constexpr uint32_t kExponent = __is_same(T, __half) ? 0x7c00u : 0x7f80u;
            bool bad = false;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                bad |= (x[j] & kExponent) == kExponent || ((x[j] >> 16) & kExponent) == kExponent;
            if (bad) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if ((x[j] & kExponent) == kExponent) x[j] &= 0xffff0000u;
                    if (((x[j] >> 16) & kExponent) == kExponent) x[j] &= 0xffffu;
                }
                *word = make_uint4(x[0], x[1], x[2], x[3]);
                any = true;
            }
        }
    }
    return any;
}
// What clean_row took away and a sum over rows from..to-1 should have met.
template <class T>
__device__ __noinline__ float taken_away(const uint16_t *column, long long stride, int from, int to)
{
    float sum = 0.0f;
    for (int r = from; r < to; ++r) {
        const float x = unpack2<T>(column[r * stride]).x;
        if (!(fabsf(x) < INFINITY)) sum += x;
    }
    return sum;
}

__device__ __forceinline__ bool wait_all(const uint64_t *bar, uint32_t parity, volatile int *failed)
{
    return __all_sync(0xffffffffu, umma::barrier_wait(umma::shared_address(bar), parity, failed));
}

// Eight results of a row, rounded to the 16-bit type.
template <class T>
__device__ __forceinline__ void put8(uint16_t *to, const float *x)
{
    *(uint4 *)to = make_uint4(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]), pack2<T>(x[4], x[5]), pack2<T>(x[6], x[7]));
}

// ---------------------------------------------------------------------------
// Forward
// ---------------------------------------------------------------------------

struct None {};
template <bool BIAS> struct Choose { using Type = Tables; };
template <> struct Choose<false> { using Type = None; };

struct ForwardParams {
    const Item *items;
    const int *count;
    int tokens, heads, group, dim;
    float scale2;                            // scale, base 2
    Heads out, v;
    float *lse;
    Bias bias;
};

constexpr int kForwardThreads = 192;         // four warps of softmax, one of copies, one of products
constexpr float kLazy = 8.0f;                // a maximum moves only when it grows by more than this (base 2)

template <int HALVES>
constexpr int forward_shared() { return 1024 + (HALVES == 1 ? 5 : 3) * HALVES * kHalfBytes; }

// A CTA has 128 queries of one head; two CTAs share an SM, so that one's softmax
// runs under the other's products.  Per tile of 128 keys: S = Q K^T into tensor
// memory; each thread has one row of it, twice read (maximum; probabilities),
// which needs no word from another thread; P goes back into tensor memory as the
// left operand of O += P V.  For dim <= 64 the half of an SM's tensor memory that
// a CTA has holds P beside S: the next scores are computed as soon as S has been
// read, with two tiles of K and V under way.  For more, P takes the place of S.
template <class T, int HALVES, bool BIAS>
__global__ void __launch_bounds__(kForwardThreads, 2)
psops_attention_forward_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                               const __grid_constant__ CUtensorMap map_v, const __grid_constant__ ForwardParams P)
{
    constexpr bool kBf16 = __is_same(T, __nv_bfloat16);
    constexpr int kTileBytes = HALVES * kHalfBytes;
    constexpr bool kAhead = HALVES == 1;
    constexpr int kStages = kAhead ? 2 : 1;
    // fp16 has no numbers below 2^-24: probabilities, at most 2^kLazy, are kept higher up
    constexpr float kShift = kBf16 ? 0.0f : 7.0f;
    extern __shared__ uint8_t raw[];
    __shared__ alignas(8) uint64_t bar_q, bar_k_full[kStages], bar_k_empty[kStages], bar_v_full[kStages], bar_v_empty[kStages], bar_s,
        bar_read, bar_p, bar_o;
    __shared__ uint32_t tensor_base_slot;
    __shared__ int failed_slot, dirty;
    __shared__ typename Choose<BIAS>::Type tables;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int *failed = &failed_slot;
    umma::after_the_kernel_before();
    const int head = blockIdx.x % P.heads;
    const int index = blockIdx.x / P.heads;
    if (index >= *P.count) return;
    const Item item = P.items[index];
    if (item.length <= 0) return;
    const int tile = item.level, first = item.first + tile * kTile;
    uint8_t *tiles = raw + (((umma::shared_address(raw) + 1023u) & ~1023u) - umma::shared_address(raw));
    const uint32_t q_at = umma::shared_address(tiles), k_at = q_at + kTileBytes, v_at = k_at + kStages * kTileBytes;

    if (threadIdx.x == 0) {
        for (uint64_t *b : {&bar_q, &bar_s, &bar_o}) umma::barrier_init(umma::shared_address(b), 1);
        for (int i = 0; i < kStages; ++i)
            for (uint64_t *b : {&bar_k_full[i], &bar_k_empty[i], &bar_v_full[i], &bar_v_empty[i]}) umma::barrier_init(umma::shared_address(b), 1);
        umma::barrier_init(umma::shared_address(&bar_read), 4);
        umma::barrier_init(umma::shared_address(&bar_p), 4);
        failed_slot = dirty = 0;
        umma::barrier_init_done();
    }
    if (warp == 5) umma::tensor_columns_take<256>(umma::shared_address(&tensor_base_slot));
    umma::fence_before();
    __syncthreads();
    umma::fence_after();
    const uint32_t s_at = tensor_base_slot, o_at = s_at + kTile, p_at = kAhead ? o_at + 64 : s_at;

    if (warp == 4) {
        // ---- copies in; the tile on the diagonal comes first
        const int kv = head / P.group;
        bool ok = true;
        if (umma::elected()) {
            umma::barrier_expect(umma::shared_address(&bar_q), kTileBytes);
            for (int h = 0; h < HALVES; ++h)
                umma::tensor_load3(q_at + h * kHalfBytes, &map_q, h * 64, head, first, umma::shared_address(&bar_q));
        }
        __syncwarp();
        for (int j = 0; j <= tile && ok; ++j) {
            const int token = first - j * kTile, stage = j % kStages;
            const uint32_t phase = (j / kStages & 1) ^ 1;
            ok = wait_all(&bar_k_empty[stage], phase, failed);
            if (!ok) break;
            if (umma::elected()) {
                umma::barrier_expect(umma::shared_address(&bar_k_full[stage]), kTileBytes);
                for (int h = 0; h < HALVES; ++h)
                    umma::tensor_load3(k_at + stage * kTileBytes + h * kHalfBytes, &map_k, h * 64, kv, token, umma::shared_address(&bar_k_full[stage]));
            }
            __syncwarp();
            ok = wait_all(&bar_v_empty[stage], phase, failed);
            if (!ok) break;
            if (umma::elected()) {
                umma::barrier_expect(umma::shared_address(&bar_v_full[stage]), kTileBytes);
                for (int h = 0; h < HALVES; ++h)
                    umma::tensor_load3(v_at + stage * kTileBytes + h * kHalfBytes, &map_v, h * 64, kv, token, umma::shared_address(&bar_v_full[stage]));
            }
            __syncwarp();
        }
        if (!ok) __nanosleep(1000000);           // copies in flight land long before
    } else if (warp == 5) {
        // ---- products; they run in the order in which they are issued, so S may follow P V without a wait
        const int steps = (P.dim + 15) / 16;
        const uint32_t instr_s = umma::instruction(kBf16, false, false, kTile, kTile);
        const uint32_t instr_o = umma::instruction(kBf16, false, true, kTile, steps * 16);
        const uint64_t dq = umma::operand(q_at, false), dk = umma::operand(k_at, false), dv = umma::operand(v_at, true, kHalfBytes);
        auto scores = [&](int j) {
            const int stage = j % kStages;
            if (!wait_all(&bar_k_full[stage], j / kStages & 1, failed)) return false;
            if (kAhead && j > 0 && !wait_all(&bar_read, (j & 1) ^ 1, failed)) return false;
            umma::fence_after();
            if (umma::elected()) {
                for (int s = 0; s < steps; ++s) {
                    const uint32_t on = (s >> 2) * (kHalfBytes >> 4) + (s & 3) * 2;
                    umma::multiply<false>(s_at, dq + on, dk + stage * (kTileBytes >> 4) + on, instr_s, s > 0);
                }
                umma::products_arrive<false>(umma::shared_address(&bar_s));
                umma::products_arrive<false>(umma::shared_address(&bar_k_empty[stage]));
            }
            __syncwarp();
            return true;
        };
        bool ok = wait_all(&bar_q, 0, failed) && scores(0);
        for (int j = 0; j <= tile && ok; ++j) {
            const int stage = j % kStages;
            if (kAhead && j < tile && !scores(j + 1)) break;
            ok = wait_all(&bar_v_full[stage], j / kStages & 1, failed) && wait_all(&bar_p, j & 1, failed);
            if (!ok) break;
            umma::fence_after();
            if (umma::elected()) {
#pragma unroll
                for (int s = 0; s < kTile / 16; ++s)
                    umma::multiply_from_tensor_memory(o_at, p_at + s * 8, dv + stage * (kTileBytes >> 4) + s * 128, instr_o, j > 0 || s > 0);
                umma::products_arrive<false>(umma::shared_address(&bar_v_empty[stage]));
                umma::products_arrive<false>(umma::shared_address(&bar_o));
            }
            __syncwarp();
            if (!kAhead && j < tile) ok = scores(j + 1);
        }
    } else {
        // ---- softmax: one query a thread
        const int row = threadIdx.x;
        const uint32_t lanes = (uint32_t)(warp * 32) << 16;
        float far = 0.0f;
        const float *table = nullptr;
        if constexpr (BIAS) {
            if (threadIdx.x < kMostBuckets) tables.value[threadIdx.x] = threadIdx.x < P.bias.buckets ? bias_at<T>(P.bias, threadIdx.x, P.heads, head) : 0.0f;
            make_tables<kTile, true>(P.bias, tables);
            table = tables.distance + kBefore;
            far = tables.value[P.bias.buckets - 1];
        }
        float top = -INFINITY, sum = 0.0f;       // top: what is subtracted, base 2
        bool ok = true;
        for (int j = 0; j <= tile; ++j) {
            ok = wait_all(&bar_s, j & 1, failed);
            if (!ok) break;
            umma::fence_after();
            const bool diagonal = j == 0, near = BIAS && j * kTile - (kTile - 1) < P.bias.last;
            const float *distance = table + j * kTile + row;                  // - column
            // the row, in two halves so that the second is on its way under the first's maximum; with a bias it becomes
            // the whole exponent here, else scale and bias come with the exponential
            uint32_t s[kTile];
            float most[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            umma::tensor_memory_load(s_at + lanes, s);
            umma::tensor_memory_load(s_at + lanes + 32, s + 32);
            umma::tensor_memory_loaded<64>(s);
            umma::tensor_memory_load(s_at + lanes + 64, s + 64);
            umma::tensor_memory_load(s_at + lanes + 96, s + 96);
#pragma unroll
            for (int c = 0; c < kTile; c += 64) {
                if (c > 0) umma::tensor_memory_loaded<64>(s + c);
                if (near) {
#pragma unroll
                    for (int i = c; i < c + 64; ++i) s[i] = __float_as_uint(__fmaf_rn(__uint_as_float(s[i]), P.scale2, distance[-i]));
                }
                if (diagonal) {
#pragma unroll
                    for (int i = c; i < c + 64; ++i)
                        if (i > row) s[i] = 0xff800000u;                     // -inf
                }
#pragma unroll
                for (int i = c; i < c + 64; i += 8)
#pragma unroll
                    for (int n = 0; n < 4; ++n) most[n] = max3(most[n], __uint_as_float(s[i + 2 * n]), __uint_as_float(s[i + 2 * n + 1]));
            }
            if (kAhead) {
                umma::fence_before();
                __syncwarp();
                if (lane == 0) umma::barrier_arrive(umma::shared_address(&bar_read));
            }
            float higher = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
            if (!near) higher = __fmaf_rn(higher, P.scale2, far);
            if (kAhead && j > 0) {               // else bar_s has said so: the sums of the tile before are complete
                ok = wait_all(&bar_o, (j & 1) ^ 1, failed);
                if (!ok) break;
                umma::fence_after();
            }
            if (__any_sync(0xffffffffu, higher > top + kLazy)) {
                higher = fmaxf(higher, top);
                const float factor = higher > -INFINITY ? exp2_fast(top - higher) : 1.0f;
                top = higher;
                sum *= factor;
                if (j > 0) {
                    for (int c = 0; c < P.dim; c += 16) {
                        uint32_t u[16];
                        umma::tensor_memory_load16(o_at + lanes + c, u);
                        umma::tensor_memory_loaded<16>(u);
#pragma unroll
                        for (int i = 0; i < 16; ++i) u[i] = __float_as_uint(__uint_as_float(u[i]) * factor);
                        umma::tensor_memory_store16(o_at + lanes + c, u);
                    }
                }
            }
            const float base = (near ? 0.0f : far) + kShift - (top > -INFINITY ? top : 0.0f);
            const uint64_t times = both(near ? 1.0f : P.scale2), plus = both(base);
            uint64_t parts[4] = {0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < kTile; c += 32) {
                uint32_t p[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint64_t x = fma_both(pair_of(s[c + 2 * i], s[c + 2 * i + 1]), times, plus);
                    const float2 e = make_float2(exp2_fast(low_of(x)), exp2_fast(high_of(x)));
                    parts[i & 3] = add_both(parts[i & 3], pair_of(__float_as_uint(e.x), __float_as_uint(e.y)));
                    p[i] = pack2<T>(e.x, e.y);
                }
                umma::tensor_memory_store16(p_at + lanes + c / 2, p);
            }
            const uint64_t all = add_both(add_both(parts[0], parts[1]), add_both(parts[2], parts[3]));
            const float here = low_of(all) + high_of(all);
            sum += here;
            if (diagonal) {
                // keys that are masked here may hold anything: rows of the next sequence, or of none
                ok = wait_all(&bar_v_full[0], 0, failed);
                if (!ok) break;
                if (clean_row<T>(tiles + (1 + kStages) * kTileBytes, row, HALVES)) dirty = 1;
                umma::copies_see_shared();
            }
            umma::tensor_memory_stored();
            umma::fence_before();
            __syncwarp();
            if (lane == 0) umma::barrier_arrive(umma::shared_address(&bar_p));
        }
        if (ok) ok = wait_all(&bar_o, tile & 1, failed);
        umma::fence_after();
        barrier_named(1, kTile);
        const bool poisoned = *(volatile int *)&dirty != 0;
        const int left = item.length - tile * kTile;                          // queries of this tile
        const float unit = !ok || *failed ? NAN : sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
        const long long token = first + row;
        uint16_t *out = (uint16_t *)P.out.p + token * P.out.token + head * P.out.head;
        const uint16_t *v = (const uint16_t *)P.v.p + (long long)first * P.v.token + head / P.group * P.v.head;
        for (int c = 0; c < P.dim; c += 16) {
            uint32_t u[16];
            umma::tensor_memory_load16(o_at + lanes + c, u);
            umma::tensor_memory_loaded<16>(u);
            if (row < left) {
                float x[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = __uint_as_float(u[i]) * unit;
                if (poisoned) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (c + i < P.dim) x[i] += taken_away<T>(v + c + i, P.v.token, 0, row + 1);
                }
                put8<T>(out + c, x);
                if (c + 8 < P.dim) put8<T>(out + c + 8, x + 8);
            }
            __syncwarp();
        }
        if (row < left) P.lse[(long long)head * P.tokens + token] = !ok || *failed ? NAN : sum == 0.0f ? -INFINITY : (top + (log2f(sum) - kShift)) * kLn2;
    }
    __syncwarp();
    umma::fence_before();
    __syncthreads();
    umma::fence_after();
    if (warp == 5) umma::tensor_columns_give<256>(tensor_base_slot);
}

// ---------------------------------------------------------------------------
// Backward
// ---------------------------------------------------------------------------

struct BackwardParams {
    const Item *items;
    const int *count;
    int tokens, heads, group, dim;
    float scale, scale2;
    Heads q, k, grad;                        // read where numbers are not finite
    Heads out0, out1;                        // dq; or dk and dv
    const float *lse, *delta;
    const float2 *norms;                     // NULL, or `blocks` of them
    int blocks;
    Bias bias;
    float *partials;                         // dbias by slot, head and bucket; NULL: not wanted
};

constexpr int kBackwardThreads = 320;        // eight warps of softmax, one of copies, one of products
constexpr int kSoftmaxThreads = 256;
constexpr int kStripe = 16;                  // columns of ds that are summed along their diagonals at a time
constexpr int kStripeFloats = 32 * (kStripe + 1);

template <int HALVES, bool KEYS, bool BIAS>
constexpr int backward_shared()
{
    return 1024 + 6 * HALVES * kHalfBytes + (BIAS && !KEYS ? 8 * (kStripeFloats + kMostBuckets) * 4 : 0);
}

// One kernel, two uses.  A CTA keeps two tiles of 128 rows (A0, A1) and meets
// pairs of tiles of 128 rows (B0, B1) one after the other:
//              A0  A1  B0  B1     S = A0 B0^T   T = A1 B1^T   sums
//   !KEYS      q   do  k   v      scores        dp            dq += ds B0
//   KEYS       k   v   q   do     scores^T      dp^T          dk += ds^T B0, dv += p^T B1
// The scores are computed in both: seven products instead of the five that a
// single pass needs, and in exchange no sum passes between CTAs, so that all
// gradients are the same in every run and dq needs no fp32 sums in memory.
// KEYS goes through all query heads that share its keys.  p and ds go back into
// tensor memory, in place of the scores and of dp, as left operands.  Softmax
// threads have one row and 64 columns each.  While they form p, the products of
// ds of the tile before and of dp run; while they form ds, those of p and of the
// next scores.
template <class T, int HALVES, bool KEYS, bool BIAS>
__global__ void __launch_bounds__(kBackwardThreads, 1)
psops_attention_backward_kernel(const __grid_constant__ CUtensorMap map_a0, const __grid_constant__ CUtensorMap map_a1,
                                const __grid_constant__ CUtensorMap map_b0, const __grid_constant__ CUtensorMap map_b1,
                                const __grid_constant__ BackwardParams P)
{
    constexpr bool kBf16 = __is_same(T, __nv_bfloat16);
    constexpr int kTileBytes = HALVES * kHalfBytes;
    // fp16: probabilities are kept 2^14 times as large (dv is scaled back), ds by a power of two from the norms
    constexpr float kShift = kBf16 ? 0.0f : 14.0f;
    extern __shared__ uint8_t raw[];
    __shared__ alignas(8) uint64_t bar_a, bar_b_full[2], bar_b_empty[2], bar_s, bar_t, bar_p, bar_ds, bar_sums;
    __shared__ uint32_t tensor_base_slot;
    __shared__ int failed_slot, dirty0, dirty1;
    __shared__ float2 most[kBackwardThreads / 32];
    __shared__ float by_column[KEYS ? 2 : 1][2][kTile];                     // lse and delta of the queries
    __shared__ typename Choose<BIAS>::Type tables;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int *failed = &failed_slot;
    umma::after_the_kernel_before();
    const int kv_heads = P.heads / P.group;
    const int grid_heads = KEYS ? kv_heads : P.heads;
    const int head = blockIdx.x % grid_heads;                               // of A0
    const int index = blockIdx.x / grid_heads;
    if (index >= *P.count) return;
    const Item item = P.items[index];
    if (item.length <= 0) return;
    const int tiles_of = (item.length + kTile - 1) / kTile;
    const int tile = KEYS ? tiles_of - 1 - item.level : item.level;         // the work is level + 1 tiles (of each head)
    const int first = item.first + tile * kTile;
    const int meets = item.level + 1, rounds = KEYS ? meets * P.group : meets;
    uint8_t *tiles = raw + (((umma::shared_address(raw) + 1023u) & ~1023u) - umma::shared_address(raw));
    const uint32_t a_at = umma::shared_address(tiles), b_at = a_at + 2 * kTileBytes;
    float *stripes = (float *)(tiles + 6 * kTileBytes), *bucket_sums = stripes + 8 * kStripeFloats;

    if (threadIdx.x == 0) {
        for (uint64_t *b : {&bar_a, &bar_b_full[0], &bar_b_full[1], &bar_b_empty[0], &bar_b_empty[1], &bar_s, &bar_t, &bar_sums})
            umma::barrier_init(umma::shared_address(b), 1);
        umma::barrier_init(umma::shared_address(&bar_p), 8);
        umma::barrier_init(umma::shared_address(&bar_ds), 8);
        failed_slot = dirty0 = dirty1 = 0;
        umma::barrier_init_done();
    }
    if (warp == 9) umma::tensor_columns_take<512>(umma::shared_address(&tensor_base_slot));
    if (BIAS && !KEYS)
        for (int i = threadIdx.x; i < 8 * kMostBuckets; i += kBackwardThreads) bucket_sums[i] = 0.0f;
    if (!kBf16) {
        float2 m = make_float2(0.0f, 0.0f);
        for (int i = threadIdx.x; i < P.blocks; i += kBackwardThreads) m = make_float2(fmaxf(m.x, P.norms[i].x), fmaxf(m.y, P.norms[i].y));
#pragma unroll
        for (int d = 16; d > 0; d /= 2)
            m = make_float2(fmaxf(m.x, __shfl_xor_sync(0xffffffffu, m.x, d)), fmaxf(m.y, __shfl_xor_sync(0xffffffffu, m.y, d)));
        if (lane == 0) most[warp] = m;
    }
    umma::fence_before();
    __syncthreads();
    umma::fence_after();
    const uint32_t s_at = tensor_base_slot, t_at = s_at + kTile, sum0_at = t_at + kTile, sum1_at = sum0_at + HALVES * 64;
    // the tile of B in round j: !KEYS from the diagonal down, KEYS from the diagonal up, head after head
    auto token_of = [&](int j) { return KEYS ? first + (j % meets) * kTile : first - j * kTile; };

    if (warp == 8) {
        // ---- copies in
        bool ok = true;
        if (umma::elected()) {
            umma::barrier_expect(umma::shared_address(&bar_a), 2 * kTileBytes);
            for (int h = 0; h < HALVES; ++h) {
                umma::tensor_load3(a_at + h * kHalfBytes, &map_a0, h * 64, head, first, umma::shared_address(&bar_a));
                umma::tensor_load3(a_at + kTileBytes + h * kHalfBytes, &map_a1, h * 64, head, first, umma::shared_address(&bar_a));
            }
        }
        __syncwarp();
        for (int j = 0; j < rounds && ok; ++j) {
            const int stage = j & 1, token = token_of(j), b_head = KEYS ? head * P.group + j / meets : head / P.group;
            ok = wait_all(&bar_b_empty[stage], (j >> 1 & 1) ^ 1, failed);
            if (!ok) break;
            if (umma::elected()) {
                const uint32_t to = b_at + stage * 2 * kTileBytes, full = umma::shared_address(&bar_b_full[stage]);
                umma::barrier_expect(full, 2 * kTileBytes);
                for (int h = 0; h < HALVES; ++h) {
                    umma::tensor_load3(to + h * kHalfBytes, &map_b0, h * 64, b_head, token, full);
                    umma::tensor_load3(to + kTileBytes + h * kHalfBytes, &map_b1, h * 64, b_head, token, full);
                }
            }
            __syncwarp();
        }
        if (!ok) __nanosleep(1000000);           // copies in flight land long before
    } else if (warp == 9) {
        // ---- products, in the order in which they are issued
        const int steps = (P.dim + 15) / 16;
        const uint32_t instr_s = umma::instruction(kBf16, false, false, kTile, kTile);
        const uint32_t instr_sum = umma::instruction(kBf16, false, true, kTile, steps * 16);
        const uint64_t da = umma::operand(a_at, false), db = umma::operand(b_at, false);
        const uint64_t db_across = umma::operand(b_at, true, kHalfBytes);
        constexpr uint32_t kNext = kTileBytes >> 4;                          // from A0 to A1, from B0 to B1
        // which: 0 scores, 1 dp
        auto scores = [&](int j, int which) {
            const uint32_t stage = (j & 1) * 2 * kNext + which * kNext;
            if (umma::elected()) {
                for (int s = 0; s < steps; ++s) {
                    const uint32_t on = (s >> 2) * (kHalfBytes >> 4) + (s & 3) * 2;
                    umma::multiply<false>(which ? t_at : s_at, da + which * kNext + on, db + stage + on, instr_s, s > 0);
                }
                umma::products_arrive<false>(umma::shared_address(which ? &bar_t : &bar_s));
            }
            __syncwarp();
        };
        auto add = [&](int j, int which, uint32_t from, uint32_t to) {
            if (umma::elected()) {
#pragma unroll
                for (int s = 0; s < kTile / 16; ++s)        // columns 0-31 and 64-95 hold the halves
                    umma::multiply_from_tensor_memory(to, from + (s >> 2) * 64 + (s & 3) * 8, db_across + (j & 1) * 2 * kNext + which * kNext + s * 128,
                                                      instr_sum, j > 0 || s > 0);
            }
            __syncwarp();
        };
        bool ok = wait_all(&bar_a, 0, failed) && wait_all(&bar_b_full[0], 0, failed);
        if (ok) {
            umma::fence_after();
            scores(0, 0);
            scores(0, 1);
        }
        for (int j = 0; j < rounds && ok; ++j) {
            ok = wait_all(&bar_p, j & 1, failed);
            if (!ok) break;
            umma::fence_after();
            if (KEYS) add(j, 1, s_at, sum1_at);
            if (j + 1 < rounds) {
                ok = wait_all(&bar_b_full[(j + 1) & 1], (j + 1) >> 1 & 1, failed);
                if (!ok) break;
                umma::fence_after();
                scores(j + 1, 0);
            }
            ok = wait_all(&bar_ds, j & 1, failed);
            if (!ok) break;
            umma::fence_after();
            add(j, 0, t_at, sum0_at);
            if (umma::elected()) {
                umma::products_arrive<false>(umma::shared_address(&bar_b_empty[j & 1]));
                if (j + 1 == rounds) umma::products_arrive<false>(umma::shared_address(&bar_sums));
            }
            __syncwarp();
            if (j + 1 < rounds) scores(j + 1, 1);
        }
    } else {
        // ---- softmax: row and 64 columns of each tile
        const int half = warp >> 2, row = threadIdx.x & (kTile - 1), col0 = half * 64;
        const uint32_t lanes = ((uint32_t)((warp & 3) * 32) << 16) + col0;
        const int left = item.length - tile * kTile;                        // rows of A that exist
        float unit = 1.0f;                                                  // of ds
        if (!kBf16) {
            float2 m = make_float2(0.0f, 0.0f);
            for (int w = 0; w < kBackwardThreads / 32; ++w) m = make_float2(fmaxf(m.x, most[w].x), fmaxf(m.y, most[w].y));
            const float bound = 2.0f * sqrtf(m.x) * sqrtf(m.y);             // |ds| <= p (|dp| + |delta|)
            if (bound > 0.0f && bound < INFINITY) {
                int e;
                frexpf(bound, &e);
                unit = ldexpf(1.0f, min(max(14 - e, -100), 100));
            }
        }
        const float unit_p = kBf16 ? 1.0f : unit * 0x1p-14f;
        // the bias of the (first) query head
        float far = 0.0f, next_value = 0.0f;
        const float *table = nullptr;
        auto value = [&](int q_head) { return threadIdx.x < P.bias.buckets ? bias_at<T>(P.bias, threadIdx.x, P.heads, q_head) : 0.0f; };
        if constexpr (BIAS) {
            if (threadIdx.x < kMostBuckets) tables.value[threadIdx.x] = value(KEYS ? head * P.group : head);
            make_tables<kSoftmaxThreads, true>(P.bias, tables);
            table = tables.distance + kBefore;
            far = tables.value[P.bias.buckets - 1];
        }
        float row_lse = 0.0f, row_delta = 0.0f, far_sum = 0.0f;
        // a row whose scores are all -inf has no probabilities
        auto base2 = [](float lse) { return lse == -INFINITY ? INFINITY : lse * kLog2e; };
        if (!KEYS && row < left) {
            const long long at = (long long)head * P.tokens + first + row;
            row_lse = base2(P.lse[at]);
            row_delta = -P.delta[at] * unit_p;
        }
        auto fetch = [&](int j) {                                            // this thread's part of by_column
            const int token = token_of(j) + row, q_head = head * P.group + j / meets;
            if (token >= item.first + item.length) return 0.0f;
            const long long at = (long long)q_head * P.tokens + token;
            return half == 0 ? base2(P.lse[at]) : -P.delta[at] * unit_p;
        };
        float coming = KEYS ? fetch(0) : 0.0f;
        bool ok = true;                          // where it is not, all rounds are gone through all the same, for the barriers in them
        for (int j = 0; j < rounds; ++j) {
            const int apart = KEYS ? j % meets : j;                         // tiles between queries and keys
            const bool diagonal = apart == 0;
            const int columns = KEYS ? min(item.length - (tile + apart) * kTile, kTile) : kTile;   // columns that exist
            if (KEYS) {
                by_column[j & 1][half][row] = coming;
                if constexpr (BIAS) {
                    if (j > 0 && j % meets == 0) {
                        barrier_named(1, kSoftmaxThreads);                  // nobody reads the tables of the head before
                        if (threadIdx.x < kMostBuckets) tables.value[threadIdx.x] = next_value;
                        make_tables<kSoftmaxThreads, false>(P.bias, tables);
                        far = tables.value[P.bias.buckets - 1];
                    }
                    if (j % meets == 0 && j + meets < rounds) next_value = value(head * P.group + j / meets + 1);
                }
                barrier_named(1, kSoftmaxThreads);
                if (j + 1 < rounds) coming = fetch(j + 1);
            }
            const bool near = BIAS && apart * kTile - (kTile - 1) < P.bias.last;
            const bool masked = diagonal || columns < kTile;
            // distance of column c: of a query row to keys it falls with c, of a key row to queries it grows
            const float *distance = table + apart * kTile + (KEYS ? col0 - row : row - col0);
            ok &= wait_all(&bar_s, j & 1, failed);
            if (masked) {
                // what is masked may hold anything: it must not meet a zero in a product to come
                ok &= wait_all(&bar_t, j & 1, failed);
                uint8_t *b = tiles + (2 + (j & 1) * 2 + (KEYS ? half : 0)) * kTileBytes;
                if ((KEYS || half == 0) && (diagonal || row >= columns) && clean_row<T>(b, row, HALVES) && diagonal) {
                    if (KEYS && half == 1) dirty1 = 1;
                    else dirty0 = 1;
                }
                umma::copies_see_shared();
            }
            umma::fence_after();
            float p[64];
            auto counts = [&](int c) { return KEYS ? (!diagonal || col0 + c >= row) && col0 + c < columns : !diagonal || col0 + c <= row; };
            uint32_t s[64];
            umma::tensor_memory_load(s_at + lanes, s);
            umma::tensor_memory_load(s_at + lanes + 32, s + 32);
            umma::tensor_memory_loaded<64>(s);
            const uint64_t times = both(P.scale2);
#pragma unroll
            for (int c = 0; c < 64; c += 32) {
#pragma unroll
                for (int i = c; i < c + 32; i += 4) {
                    uint64_t plus[2] = {both(far + (kShift - row_lse)), 0};
                    plus[1] = plus[0];
                    if (KEYS || near) {
                        float4 lse = make_float4(row_lse, row_lse, row_lse, row_lse);
                        if (KEYS) lse = *(const float4 *)&by_column[j & 1][0][col0 + i];
                        float of[4] = {kShift - lse.x, kShift - lse.y, kShift - lse.z, kShift - lse.w};
#pragma unroll
                        for (int n = 0; n < 4; ++n) of[n] += near ? distance[KEYS ? i + n : -(i + n)] : far;
                        plus[0] = pair_of(__float_as_uint(of[0]), __float_as_uint(of[1]));
                        plus[1] = pair_of(__float_as_uint(of[2]), __float_as_uint(of[3]));
                    }
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        const uint64_t x = fma_both(pair_of(s[i + 2 * n], s[i + 2 * n + 1]), times, plus[n]);
                        p[i + 2 * n] = exp2_fast(low_of(x));
                        p[i + 2 * n + 1] = exp2_fast(high_of(x));
                    }
                }
                if (masked) {
#pragma unroll
                    for (int i = c; i < c + 32; ++i)
                        if (!counts(i)) p[i] = 0.0f;
                }
                if (KEYS) {
                    uint32_t w[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) w[i] = pack2<T>(p[c + 2 * i], p[c + 2 * i + 1]);
                    umma::tensor_memory_store16(s_at + lanes + c / 2, w);
                }
            }
            if (KEYS) umma::tensor_memory_stored();
            umma::fence_before();
            __syncwarp();
            if (lane == 0) umma::barrier_arrive(umma::shared_address(&bar_p));
            ok &= wait_all(&bar_t, j & 1, failed);
            umma::fence_after();
#pragma unroll
            for (int c = 0; c < 64; c += 32) {
                uint32_t u[32];
                umma::tensor_memory_load(t_at + lanes + c, u);
                umma::tensor_memory_loaded<32>(u);
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    // delta has its sign turned
                    uint64_t minus[2] = {both(row_delta), both(row_delta)};
                    if (KEYS) {
                        const uint4 delta = *(const uint4 *)&by_column[j & 1][1][col0 + c + i];
                        minus[0] = pair_of(delta.x, delta.y);
                        minus[1] = pair_of(delta.z, delta.w);
                    }
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        const int at = c + i + 2 * n;
                        const uint64_t dp = pair_of(u[i + 2 * n], u[i + 2 * n + 1]);
                        const uint64_t x = mul_both(kBf16 ? add_both(dp, minus[n]) : fma_both(dp, both(unit_p), minus[n]),
                                                    pair_of(__float_as_uint(p[at]), __float_as_uint(p[at + 1])));
                        p[at] = low_of(x);
                        p[at + 1] = high_of(x);
                    }
                }
                if (masked) {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (!counts(c + i)) p[c + i] = 0.0f;
                }
                uint32_t w[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = pack2<T>(p[c + 2 * i], p[c + 2 * i + 1]);
                umma::tensor_memory_store16(t_at + lanes + c / 2, w);
            }
            umma::tensor_memory_stored();
            umma::fence_before();
            __syncwarp();
            if (lane == 0) umma::barrier_arrive(umma::shared_address(&bar_ds));
            if (BIAS && !KEYS && P.partials != nullptr) {
                if (!near) {
                    uint64_t part[4] = {0, 0, 0, 0};
#pragma unroll
                    for (int c = 0; c < 64; c += 2) part[c / 2 & 3] = add_both(part[c / 2 & 3], pair_of(__float_as_uint(p[c]), __float_as_uint(p[c + 1])));
                    const uint64_t all = add_both(add_both(part[0], part[1]), add_both(part[2], part[3]));
                    far_sum += low_of(all) + high_of(all);
                } else if constexpr (BIAS) {
                    // The warp's 32 rows x 64 columns have 95 diagonals, one distance each: lane l sums those of numbers l,
                    // l + 32 and l + 64, read askew from shared memory 16 columns at a time (row r, column c: number
                    // r - c + 63).  Then equal buckets are neighbours, summed across lanes in a fixed order.
                    float *stripe = stripes + warp * kStripeFloats, *mine = bucket_sums + warp * kMostBuckets;
                    float sums[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int c = 0; c < 64; c += kStripe) {
#pragma unroll
                        for (int i = 0; i < kStripe; ++i) stripe[lane * (kStripe + 1) + i] = row < left ? p[c + i] : 0.0f;
                        __syncwarp();
                        // in columns 32 k .. 32 k + 31, row l + (c - 32 k) - 31 of lane l has number l + 32 (1 - k), and
                        // 32 rows further down (where that is negative) number l + 32 (2 - k)
                        const int high = c < 32 ? 2 : 1;
#pragma unroll
                        for (int i = 0; i < kStripe; ++i) {
                            const int r = lane + (c & 31) + i - 31;
                            const float x = stripe[(r & 31) * (kStripe + 1) + i];
                            if (r >= 0) sums[high - 1] += x;
                            else sums[high] += x;
                        }
                        __syncwarp();
                    }
                    const int zero = apart * kTile + (warp & 3) * 32 - col0 - 63;            // distance of diagonal 0
#pragma unroll
                    for (int n = 0; n < 3; ++n) {
                        const int d = zero + lane + n * 32;
                        const int bucket = d < 0 || n == 2 && lane == 31 ? -1 : tables.bucket[d];
                        float sum = sums[n];
#pragma unroll
                        for (int k = 1; k < 32; k *= 2) {
                            const float other = __shfl_down_sync(0xffffffffu, sum, k);
                            const int its = __shfl_down_sync(0xffffffffu, bucket, k);
                            if (lane + k < 32 && its == bucket) sum += other;
                        }
                        const int before = __shfl_up_sync(0xffffffffu, bucket, 1);
                        if (bucket >= 0 && (lane == 0 || before != bucket)) mine[bucket] += sum;
                        __syncwarp();
                    }
                }
            }
        }
        if (ok) ok = wait_all(&bar_sums, 0, failed);
        umma::fence_after();
        barrier_named(1, kSoftmaxThreads);
        const bool gone = !ok || *failed;
        const long long token = first + row;
        // half of the columns of each sum
        const int begin = half * 32 * HALVES, end = min(begin + 32 * HALVES, P.dim);
#pragma unroll
        for (int which = 0; which < (KEYS ? 2 : 1); ++which) {
            const bool poisoned = *(volatile int *)(which ? &dirty1 : &dirty0) != 0;
            const Heads &O = which ? P.out1 : P.out0;
            if (O.p == nullptr) continue;
            const float times = gone ? NAN : which ? (kBf16 ? 1.0f : 0x1p-14f) : P.scale / unit;
            uint16_t *out = (uint16_t *)O.p + token * O.token + head * O.head;
            for (int c = begin; c < end; c += 16) {
                uint32_t u[16];
                umma::tensor_memory_load16((which ? sum1_at : sum0_at) + lanes - col0 + c, u);
                umma::tensor_memory_loaded<16>(u);
                if (row < left) {
                    float x[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = __uint_as_float(u[i]) * times;
                    if (poisoned) {
                        // !KEYS: the keys of this tile up to the query; KEYS: queries (do) of this tile from the key on, all heads
                        for (int g = 0; g < (KEYS ? P.group : 1); ++g) {
                            const Heads &B = !KEYS ? P.k : which ? P.grad : P.q;
                            const uint16_t *b = (const uint16_t *)B.p + (long long)first * B.token + (KEYS ? head * P.group + g : head / P.group) * B.head;
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                if (c + i < end) x[i] += taken_away<T>(b + c + i, B.token, KEYS ? row : 0, KEYS ? min(left, kTile) : row + 1);
                        }
                    }
                    put8<T>(out + c, x);
                    if (c + 8 < end) put8<T>(out + c + 8, x + 8);
                }
                __syncwarp();
            }
        }
        if (BIAS && !KEYS && P.partials != nullptr) {
            if (row >= left) far_sum = 0.0f;
#pragma unroll
            for (int d = 16; d > 0; d /= 2) far_sum += __shfl_xor_sync(0xffffffffu, far_sum, d);
            if (lane == 0) bucket_sums[warp * kMostBuckets + P.bias.buckets - 1] += far_sum;
            barrier_named(1, kSoftmaxThreads);
            if (threadIdx.x < P.bias.buckets) {
                float sum = 0.0f;
                for (int w = 0; w < 8; ++w) sum += bucket_sums[w * kMostBuckets + threadIdx.x];
                P.partials[((long long)item.slot * P.heads + head) * P.bias.buckets + threadIdx.x] = gone ? NAN : sum / unit;
            }
        }
    }
    __syncwarp();
    umma::fence_before();
    __syncthreads();
    umma::fence_after();
    if (warp == 9) umma::tensor_columns_give<512>(tensor_base_slot);
}

// dbias: the slots of all tiles joined in their order, in double.
constexpr int kJoinParts = 16;
struct JoinParams {
    const float *partials;
    const int *used;
    int slots, heads, buckets, fp32;
    void *out;                               // buckets x heads
};
template <class T>
__global__ void __launch_bounds__(32 * kJoinParts) psops_attention_join_kernel(const JoinParams P)
{
    __shared__ double sums[kJoinParts][32];
    umma::after_the_kernel_before();
    const int per_slot = P.heads * P.buckets, at = blockIdx.x * 32 + (threadIdx.x & 31), part = threadIdx.x >> 5;
    double sum = 0.0;
    if (at < per_slot)
        for (int s = part; s < P.slots; s += kJoinParts)
            if (P.used[s]) sum += (double)P.partials[(long long)s * per_slot + at];
    sums[part][threadIdx.x & 31] = sum;
    __syncthreads();
    if (part != 0 || at >= per_slot) return;
    for (int p = 1; p < kJoinParts; ++p) sum += sums[p][threadIdx.x];
    const int head = at / P.buckets, bucket = at % P.buckets;
    const long long to = (long long)bucket * P.heads + head;
    if (P.fp32) ((float *)P.out)[to] = (float)sum;
    else ((T *)P.out)[to] = (T)(float)sum;
}

} // namespace psops_attention_k
