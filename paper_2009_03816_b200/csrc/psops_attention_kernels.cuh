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
// The tensor cores cut off what does not fit into a running sum.  After so many
// tiles (16,384 terms) a sum goes to memory, where fp32 additions carry it on.
constexpr int kChain = 128;
constexpr int kFoldFloats = kTile * kMostDim;    // room of a CTA for one of them
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Division of numbers below 2^31 by a number that the host knows.
struct Divisor {
    uint32_t by, factor, shift;
};
__device__ __forceinline__ uint32_t divide(uint32_t x, const Divisor &d) { return (uint32_t)(((uint64_t)x * d.factor) >> d.shift); }

// A tile of a sequence.
struct alignas(16) Item {
    int first, length;       // first token and tokens of its sequence
    int level;               // its number, counted so that its work grows with it
    int slot;                // the same for the same tile of the same batch in any call
};

struct Heads {               // tokens x heads x dim, elements of a head consecutive
    void *p;
    long long token, head;   // strides in elements
};

struct Bias {
    const void *p;                           // buckets x heads, NULL for none
    int fp32;                                // else of the call's 16-bit type
    int buckets, last;                       // last: the first distance of the last bucket
    int first[kMostBuckets];                 // the first distance of each bucket
};

// What lies below -1e30, such as the lowest number of bf16 and fp32, takes its pairs
// out as -inf does.
template <class T>
__device__ __forceinline__ float bias_at(const Bias &B, int bucket, int heads, int head)
{
    const long long i = (long long)bucket * heads + head;
    const float b = B.fp32 ? ((const float *)B.p)[i] : (float)((const T *)B.p)[i];
    return b < -1e30f ? -INFINITY : b;
}

// Beside a bias of -1e9 a score has no digits left in fp32, and a logarithm none in
// lse.  So the level of a row is the largest bias of the buckets that it meets, those
// up to the one of its position, where that lies beyond kPlain (an exponent of that
// size is off by 2^-16); else 0.  It is taken off the row's biases before a score is
// added, and off its lse, which the backward pass sums up once more for that (lse
// itself is rounded as a whole); rows whose lse is not beyond kPlain need none of it
// there.  Levels are rare (a mask of -1e9 over all that a sequence's first tokens
// meet) and have code of their own, out of line: within the usual code they cost it 3
// to 7 % of its time.
constexpr float kPlain = 256.0f;
__device__ __forceinline__ bool beyond_plain(float x) { return fabsf(x) > kPlain && fabsf(x) < INFINITY; }
__device__ __forceinline__ float level_of(float most) { return beyond_plain(most) ? most : 0.0f; }

struct PrepParams {
    const int *offsets;
    int sequences, tokens, capacity;
    Item *items;
    int *count;
    int *used;               // NULL, or by slot whether a tile has it
    int *ticket;             // NULL, or becomes zero
    int *zero;               // so many numbers that become zero
    int zeros;
    int heads, kv_heads, dim;
    int fill;                // how many of `rest` are to be zeroed where no sequence is
    Heads rest[3];
    int rest_heads[3];
    float *rest_lse;
    // backward
    Heads out, grad, v;
    float *delta;            // NULL in a forward pass
    int blocks;              // for these two; those beyond are for
    int *levels;             // ... whether any row can have a level, and
    float *beside;           // (NULL in a forward pass) base 2: the log-sum-exps of rows with levels, beside those
    const float *lse;
    Heads q, k;
    float scale2;
    Bias bias;
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

// Both to about 2^-23, relative and, of the logarithm of numbers near 1, absolute.
__device__ __forceinline__ float reciprocal(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float log2_fast(float x)
{
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
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
// 2^x of two numbers without the special-function unit, which has 16 results a clock
// where a tile of products of dim 128 takes 16 scores a clock: 2^n times a
// polynomial for 2^f, f in [-1/2, 1/2] (least largest relative error at degree 5, by
// Remez's exchange: 1.6e-7 with these coefficients, 2.2e-7 evaluated in fp32).
// Below 2^-126 it is zero; NaN stays NaN.
__device__ __forceinline__ uint64_t exp2_both(uint64_t x)
{
    float a = low_of(x), b = high_of(x);
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(a) : "f"(-127.0f));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(b) : "f"(-127.0f));
    x = pair_of(__float_as_uint(a), __float_as_uint(b));
    const uint64_t t = add_both(x, both(12582912.0f));                       // 1.5 2^23 + n
    const uint64_t f = fma_both(add_both(t, both(-12582912.0f)), both(-1.0f), x);
    uint64_t p = both(0x1.5c08e6p-10f);
    p = fma_both(p, f, both(0x1.3d0c52p-7f));
    p = fma_both(p, f, both(0x1.c6b6e4p-5f));
    p = fma_both(p, f, both(0x1.ebf918p-3f));
    p = fma_both(p, f, both(0x1.62e428p-1f));
    p = fma_both(p, f, both(1.0f));
    return mul_both(p, pair_of(((uint32_t)t << 23) + 0x3f800000u, ((uint32_t)(t >> 32) << 23) + 0x3f800000u));
}
// Two probabilities; every OWN-th of 16 pairs by the polynomial.
template <int OWN>
__device__ __forceinline__ uint64_t exp2_pair(uint64_t x, int i)
{
    if (i % OWN == OWN - 1) return exp2_both(x);
    return pair_of(__float_as_uint(exp2_fast(low_of(x))), __float_as_uint(exp2_fast(high_of(x))));
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

__device__ __forceinline__ void bounds_of(const PrepParams &P, int b, int &first, int &length)
{
    first = clamped(P.offsets[b], 0, P.tokens);
    length = max(clamped(P.offsets[b + 1], 0, P.tokens) - first, 0);
}

// One block.  Tiles go into bins by level (several levels to a bin only beyond
// kBins of them); within a bin the order is left to chance, which changes when
// a tile is done and nothing else.  There are capacity - 1 tiles at most, which grids
// count on; offsets that decrease could make more, which are left out.
__device__ __forceinline__ void make_list(const PrepParams &P)
{
    __shared__ int sequences_at[kBins + 1], rest_at[kBins + 1], next[kBins];
    const int most = (P.tokens + kTile - 1) / kTile;
    int shift = 0;
    while ((most >> shift) >= kBins) ++shift;
    const int bins = (most >> shift) + 1;
    for (int i = threadIdx.x; i <= bins; i += kPrepThreads) sequences_at[i] = rest_at[i] = 0;
    if (P.ticket != nullptr && threadIdx.x == 0) *P.ticket = 0;
    for (int i = threadIdx.x; i < P.zeros; i += kPrepThreads) P.zero[i] = 0;
    if (P.used != nullptr)
        for (int i = threadIdx.x; i < P.capacity; i += kPrepThreads) P.used[i] = 0;
    __syncthreads();
    for (int b = threadIdx.x; b < P.sequences; b += kPrepThreads) {
        int first, length;
        bounds_of(P, b, first, length);
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
        if (lane == 31) *P.count = min(before, P.capacity - 1);
    }
    __syncthreads();
    auto place = [&](int first, int length, int slot, int level) {
        const int at = atomicAdd(&next[level >> shift], 1);
        if (at < P.capacity - 1 && slot + level < P.capacity) {
            P.items[at] = Item{first, length, level, slot + level};
            if (P.used != nullptr) P.used[slot + level] = 1;
        } else if (at < P.capacity - 1) {
            P.items[at] = Item{0, 0, 0, 0};                  // its slot belongs to another
        }
    };
    // a team of threads for each sequence: as many as there are for each, a warp at most
    int team = 32;
    while (team > 1 && team * P.sequences > kPrepThreads) team /= 2;
    for (int b = threadIdx.x / team; b < P.sequences; b += kPrepThreads / team) {
        int first, length;
        bounds_of(P, b, first, length);
        for (int l = threadIdx.x % team; l * kTile < length; l += team) place(first, length, first / kTile + b, l);
    }
}

// Zeroes what the call's own tensors hold where no sequence is.
template <int THREADS>
__device__ __forceinline__ void fill_rest(const PrepParams &P, int block, int blocks)
{
    const int low = P.sequences > 0 ? clamped(P.offsets[0], 0, P.tokens) : 0;
    const int high = P.sequences > 0 ? max(clamped(P.offsets[P.sequences], 0, P.tokens), low) : 0;
    const int count = low + P.tokens - high, words = P.dim / 8;
    for (int t = 0; t < P.fill; ++t) {
        const int per_token = P.rest_heads[t] * words;
        for (long long i = (long long)block * THREADS + threadIdx.x; i < (long long)count * per_token; i += (long long)blocks * THREADS) {
            const int n = (int)(i / per_token), w = (int)(i % per_token), token = n < low ? n : high + n - low;
            uint16_t *row = (uint16_t *)P.rest[t].p + token * P.rest[t].token + (w / words) * P.rest[t].head;
            *(uint4 *)(row + (w % words) * 8) = make_uint4(0, 0, 0, 0);
        }
    }
    if (P.rest_lse != nullptr)
        for (long long i = (long long)block * THREADS + threadIdx.x; i < (long long)count * P.heads; i += (long long)blocks * THREADS) {
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
// largest squared norm of a row of do and of v (rows that are not finite or of no
// sequence left out): together they bound ds.
template <class T>
__device__ __forceinline__ void make_delta(const PrepParams &P, int block, int blocks)
{
    const int lane = threadIdx.x & 15, teams = kPrepThreads / 16;
    const bool on = lane * 8 < P.dim;
    const long long rows = (long long)P.tokens * P.heads, step = (long long)blocks * teams;
    float most_grad = 0.0f, most_v = 0.0f;
    int low = 0, high = 0;                                   // tokens of sequences
    if (P.norms != nullptr && P.sequences > 0) {
        low = clamped(P.offsets[0], 0, P.tokens);
        high = max(clamped(P.offsets[P.sequences], 0, P.tokens), low);
    }
    constexpr int U = 4;
    for (long long r0 = (long long)block * teams + threadIdx.x / 16; r0 - threadIdx.x / 16 < rows; r0 += U * step) {
        uint4 g[U], o[U];
        long long to[U];
        bool counts[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long r = r0 + u * step;
            g[u] = o[u] = make_uint4(0, 0, 0, 0);
            to[u] = -1;
            counts[u] = false;
            if (r < rows) {
                const int token = (int)(r / P.heads), head = (int)(r % P.heads);
                to[u] = (long long)head * P.tokens + token;
                counts[u] = token >= low && token < high;
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
            if (counts[u] && square < INFINITY) most_grad = fmaxf(most_grad, square);
        }
    }
    if (P.norms == nullptr) return;
    const long long v_rows = (long long)high * P.kv_heads, v_first = (long long)low * P.kv_heads;
    for (long long r = v_first + (long long)block * teams + threadIdx.x / 16; r - threadIdx.x / 16 < v_rows; r += step) {
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

// The log-sum-exp of one row beside its level, if it has one, key by key; by 16 lanes
// (`team`).
template <class T>
__device__ __noinline__ void sum_beside_level(const PrepParams &P, int token, int head, uint32_t team)
{
    const int lane = threadIdx.x & 15;
    // the last sequence that begins at the token or before
    int low = 0, high = P.sequences;
    while (low < high) {
        const int mid = (low + high) / 2;
        if (P.offsets[mid] <= token) low = mid + 1;
        else high = mid;
    }
    if (low == 0 || token >= P.offsets[low]) return;
    const int first = clamped(P.offsets[low - 1], 0, token);
    float most = -INFINITY;
    for (int b = lane; b < P.bias.buckets; b += 16)
        if (P.bias.first[b] <= token - first) most = fmaxf(most, bias_at<T>(P.bias, b, P.heads, head));
#pragma unroll
    for (int d = 8; d > 0; d /= 2) most = fmaxf(most, __shfl_xor_sync(team, most, d));
    const float level = level_of(most);
    if (level == 0.0f) return;
    const bool on = lane * 8 < P.dim;
    const uint16_t *keys = (const uint16_t *)P.k.p + head / (P.heads / P.kv_heads) * P.k.head + lane * 8;
    uint4 q = make_uint4(0, 0, 0, 0);
    if (on) q = *(const uint4 *)((const uint16_t *)P.q.p + token * P.q.token + head * P.q.head + lane * 8);
    int bucket = P.bias.buckets;
    float beside = 0.0f, top = -INFINITY, sum = 0.0f;
    constexpr int U = 4;                     // keys under way
    for (int j0 = first; j0 <= token; j0 += U) {
        uint4 k[U];
        float x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            k[u] = make_uint4(0, 0, 0, 0);
            if (on) k[u] = *(const uint4 *)(keys + min(j0 + u, token) * P.k.token);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x[u] = dot8<T>(q, k[u]);
#pragma unroll
            for (int d = 8; d > 0; d /= 2) x[u] += __shfl_xor_sync(team, x[u], d);
        }
        float higher = top;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int distance = token - j0 - u;
            if (distance >= 0 && (bucket == P.bias.buckets || distance < P.bias.first[bucket])) {
                do --bucket;
                while (distance < P.bias.first[bucket]);
                beside = (bias_at<T>(P.bias, bucket, P.heads, head) - level) * kLog2e;
            }
            x[u] = distance >= 0 ? __fmaf_rn(x[u], P.scale2, beside) : -INFINITY;
            higher = fmaxf(higher, x[u]);
        }
        if (higher > -INFINITY) {
            sum *= exp2_fast(top - higher);
#pragma unroll
            for (int u = 0; u < U; ++u) sum += exp2_fast(x[u] - higher);
        }
        top = higher;
    }
    // a row without any score has no probabilities
    if (lane == 0) P.beside[(long long)head * P.tokens + token] = top > -INFINITY ? top + log2_fast(sum) : INFINITY;
}

// By blocks of their own, which end where no row can have a level.
template <class T>
__device__ __forceinline__ void make_beside(const PrepParams &P, int block, int blocks)
{
    bool some = false;
    const int entries = P.bias.buckets * P.heads;
    for (int i = threadIdx.x; i < entries; i += kPrepThreads) some |= beyond_plain(bias_at<T>(P.bias, i / P.heads, P.heads, i % P.heads));
    if (__syncthreads_or(some)) {
        some = false;
        for (int h = threadIdx.x; h < P.heads; h += kPrepThreads) {
            float most = -INFINITY;
            for (int b = 0; b < P.bias.buckets; ++b) {
                most = fmaxf(most, bias_at<T>(P.bias, b, P.heads, h));
                some |= level_of(most) != 0.0f;
            }
        }
        some = __syncthreads_or(some);
    }
    if (block == 0 && threadIdx.x == 0) *P.levels = some;
    if (!some || P.beside == nullptr) return;
    const long long rows = (long long)P.tokens * P.heads;
    for (long long r = (long long)block * (kPrepThreads / 16) + threadIdx.x / 16; r < rows; r += (long long)blocks * (kPrepThreads / 16)) {
        // a block's rows are neighbours and read the same keys
        const int token = (int)(r % P.tokens), head = (int)(r / P.tokens);
        if (beyond_plain(P.lse[r])) sum_beside_level<T>(P, token, head, 0xffffu << (threadIdx.x & 16));
    }
}

template <class T>
__global__ void __launch_bounds__(kPrepThreads, 2) psops_attention_prepare_kernel(const __grid_constant__ PrepParams P)
{
    umma::after_the_kernel_before();
    if (blockIdx.x == 0) {
        make_list(P);
        return;
    }
    const int block = blockIdx.x - 1, more = gridDim.x - 1 - P.blocks;
    if (block >= P.blocks) {
        make_beside<T>(P, block - P.blocks, more);
        return;
    }
    if (P.fill > 0) fill_rest<kPrepThreads>(P, block, P.blocks);
    if (P.delta != nullptr) make_delta<T>(P, block, P.blocks);
}

// ---------------------------------------------------------------------------
// What the two tensor-core kernels share
// ---------------------------------------------------------------------------

__device__ __forceinline__ void barrier_named(int id, int threads)
{
    asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
// The same; whether x is true in any of the threads.
__device__ __forceinline__ bool barrier_any(int id, int threads, bool x)
{
    uint32_t any;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(any)
                 : "r"((uint32_t)x), "r"(id), "r"(threads)
                 : "memory");
    return any != 0;
}

// What the softmax threads of a CTA keep of the bias; distances up to a tile's
// reach beyond the last bucket's beginning.
struct Tables {
    float value[kMostBuckets];               // of the head at hand, base 2; LEVELS: as given
    float level[kMostBuckets];               // LEVELS: of rows whose position is in a bucket
    int first[kMostBuckets];
    uint8_t bucket[kMostDistance + 2 * kTile];
    float distance[kTableFloats];            // [kBefore + d]: the bias of distance d, as in `value`

    __device__ __forceinline__ float level_at(const Bias &B, int position) const { return level[bucket[min(position, B.last)]]; }
    // LEVELS: the bias of distance d beside a level, base 2; of distances below 0 any number
    __device__ __forceinline__ float beside(int d, float level) const { return (distance[kBefore + d] - level) * kLog2e; }
};
// By one warp, two buckets a lane: running maxima over the buckets.
__device__ __noinline__ void make_levels(Tables &t, int buckets)
{
    const int lane = threadIdx.x & 31, b = 2 * lane;
    const float one = b < buckets ? t.value[b] : -INFINITY, two = b + 1 < buckets ? t.value[b + 1] : -INFINITY;
    float most = fmaxf(one, two);
    for (int d = 1; d < 32; d *= 2) {
        const float n = __shfl_up_sync(0xffffffffu, most, d);
        if (lane >= d) most = fmaxf(most, n);
    }
    float before = __shfl_up_sync(0xffffffffu, most, 1);
    if (lane == 0) before = -INFINITY;
    t.level[b] = level_of(fmaxf(before, one));
    t.level[b + 1] = level_of(most);
}
// By THREADS threads that share barrier 1; mine: of the first ones the bias of bucket threadIdx.x.
template <int THREADS, bool BUCKETS, bool LEVELS>
__device__ __forceinline__ void make_tables(const Bias &B, Tables &t, float mine)
{
    const int many = B.last + 2 * kTile;
    if (threadIdx.x < kMostBuckets) t.value[threadIdx.x] = LEVELS ? mine : mine * kLog2e;
    if (BUCKETS && threadIdx.x < kMostBuckets) t.first[threadIdx.x] = threadIdx.x < B.buckets ? B.first[threadIdx.x] : INT32_MAX;
    barrier_named(1, THREADS);
    if (LEVELS && threadIdx.x < 32) make_levels(t, B.buckets);
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

// acc + 0 x: stays zero as long as both halves of x are finite.
template <class T> __device__ __forceinline__ uint32_t add_nothing(uint32_t acc, uint32_t x)
{
    if (__is_same(T, __half)) asm("fma.rn.f16x2 %0, %1, %2, %0;" : "+r"(acc) : "r"(x), "r"(0u));
    else asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(acc) : "r"(x), "r"(0u));
    return acc;
}
// Whether there are numbers that are not finite among 64 elements of a row of a
// tile.  The eight 16-byte words are taken in the swizzle's order.
template <class T>
__device__ __forceinline__ bool not_clean(const uint8_t *half_tile, int row)
{
    const uint4 *at = (const uint4 *)(half_tile + row * 128);
    uint32_t acc = 0;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const uint4 w = at[c ^ (row & 7)];
        acc = add_nothing<T>(add_nothing<T>(add_nothing<T>(add_nothing<T>(acc, w.x), w.y), w.z), w.w);
    }
    return (acc & 0x7fff7fffu) != 0;
}
// Makes zeros of them, so that a probability of zero meets none.
template <class T>
__device__ __noinline__ void clean_row(uint8_t *half_tile, int row)
{
    constexpr uint32_t kExponent = __is_same(T, __half) ? 0x7c00u : 0x7f80u;
#pragma unroll 1
    for (int c = 0; c < 32; ++c) {
        uint32_t &x = ((uint32_t *)(half_tile + row * 128))[c];
        if ((x & kExponent) == kExponent) x &= 0xffff0000u;
        if (((x >> 16) & kExponent) == kExponent) x &= 0xffffu;
    }
    umma::copies_see_shared();
}
// Bits 0 to n - 1 of 32.
__device__ __forceinline__ uint32_t below(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }

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

// What a CTA does in turn k: tiles of the list, each with all heads before the
// next, dealt out to the CTAs to and fro.  The list is in order of work, so that
// all get about the same.
struct Work {
    Item item;
    int head;
    bool some;
};
__device__ __forceinline__ Work work_at(const Item *items, int total, const Divisor &heads, int k)
{
    const uint32_t many = gridDim.x, i = k * many + (k & 1 ? many - 1 - blockIdx.x : blockIdx.x);
    Work w{};
    w.some = i < (uint32_t)total;
    if (w.some) {
        const uint32_t of = divide(i, heads);
        const int4 x = *(const int4 *)(items + of);
        w.item = Item{x.x, x.y, x.z, x.w};
        w.head = (int)(i - of * heads.by);
    }
    return w;
}

// The same without a list, where there are no more works than CTAs: each warp
// looks for its CTA's one itself.
__device__ __forceinline__ Work own_work(const PrepParams &P, const Divisor &heads)
{
    const int lane = threadIdx.x & 31;
    const uint32_t of = divide(blockIdx.x, heads);
    Work w{};
    w.head = (int)(blockIdx.x - of * heads.by);
    int before = 0;                          // tiles of the sequences before
    for (int b = 0; b < P.sequences && !w.some; b += 32) {
        int first = 0, length = 0;
        if (b + lane < P.sequences) bounds_of(P, b + lane, first, length);
        const int tiles = (length + kTile - 1) / kTile;
        int up_to = tiles;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int n = __shfl_up_sync(0xffffffffu, up_to, d);
            if (lane >= d) up_to += n;
        }
        const uint32_t found = __ballot_sync(0xffffffffu, before + up_to > (int)of);
        if (found != 0) {
            const int at = __ffs(found) - 1;
            w.some = true;
            w.item.first = __shfl_sync(0xffffffffu, first, at);
            w.item.length = __shfl_sync(0xffffffffu, length, at);
            w.item.level = (int)of - before - __shfl_sync(0xffffffffu, up_to - tiles, at);
        }
        before += __shfl_sync(0xffffffffu, up_to, 31);
    }
    return w;
}

// 32 columns from column c of a warp's 32 rows, out of tensor memory into rows of
// 16-bit numbers.  A lane has a row; after four lanes have traded their quarters
// of it (a transposition of 4 x 4 words of 16 bytes) they store 64 consecutive
// bytes of one row together.  Row r is at to + r stride, `rows` of them exist.
// fix(x): what else becomes of the lane's own row.
template <class T, class Fix>
__device__ __forceinline__ void put_rows(uint32_t from, float times, uint16_t *to, long long stride, int c, int dim, int rows, Fix &&fix)
{
    const int lane = threadIdx.x & 31;
    uint32_t u[32];
    umma::tensor_memory_load(from + c, u);
    umma::tensor_memory_loaded<32>(u);
    float x[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(u[i]) * times;
    fix(x);
    uint32_t w[4][4];
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i / 4][i % 4] = pack2<T>(x[2 * i], x[2 * i + 1]);
#pragma unroll
    for (int bit = 1; bit <= 2; bit *= 2) {
        const bool upper = lane & bit;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (q & bit) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t theirs = __shfl_xor_sync(0xffffffffu, upper ? w[q][i] : w[q | bit][i], bit);
                if (upper) w[q][i] = theirs;
                else w[q | bit][i] = theirs;
            }
        }
    }
    const int column = c + (lane & 3) * 8;
    if (column < dim) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int r = (lane & ~3) + q;
            if (r < rows) *(uint4 *)(to + r * stride + column) = make_uint4(w[q][0], w[q][1], w[q][2], w[q][3]);
        }
    }
    __syncwarp();
}

// ---------------------------------------------------------------------------
// Forward
// ---------------------------------------------------------------------------

// The place of a thread's row in a CTA's room; column c is at [c * kTile].
__device__ __forceinline__ float *room_of(float *fold, int which, int row) { return fold + (long long)which * kFoldFloats + row; }

// Columns begin to end of this thread's row in tensor memory are added to what is
// in its room, times a factor, or put there.
__device__ __noinline__ void add_to_room(float *room, uint32_t from, int begin, int end, float factor, bool add)
{
#pragma unroll 1
    for (int c = begin; c < end; c += 16) {
        uint32_t u[16];
        umma::tensor_memory_load16(from + c, u);
        umma::tensor_memory_loaded<16>(u);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float *at = room + (c + i) * kTile;
            *at = add ? __fmaf_rn(*at, factor, __uint_as_float(u[i])) : __uint_as_float(u[i]);
        }
    }
}

struct None {};
template <bool BIAS> struct Choose { using Type = Tables; };
template <> struct Choose<false> { using Type = None; };

struct ForwardParams {
    const Item *items;
    const int *count;
    const int *levels;                       // with a list: whether any row can have a level
    int tokens, heads, dim;
    Divisor by_heads, by_group;
    float scale2;                            // scale, base 2
    Heads out, v;
    float *lse;
    Bias bias;
    float *fold;                             // room for sums of more than kChain tiles, kFoldFloats for each CTA
    int own;                                 // works without a list, and rows of no sequence zeroed here
    PrepParams prep;
};

template <int HALVES, bool BIAS>
struct ForwardShared {
    static constexpr int kStages = HALVES == 1 ? 2 : 1;
    alignas(8) uint64_t q_full[kStages], q_empty[kStages], k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages], s, read, p[2], o;
    int failed, dirty[2];
    float other[2][2][kTile], other_sum[2][kTile], fold_top[2][kTile];   // maxima (by parity of the tile) and sums of the rows' halves
    typename Choose<BIAS>::Type tables;
};

constexpr int kForwardThreads = 320;         // eight warps of softmax, one of copies, one of products
constexpr int kSoftmaxThreads = 256;
constexpr float kLazy = 8.0f;                // a maximum moves only when it grows by more than this (base 2)

template <int HALVES>
constexpr int forward_shared() { return 1024 + (HALVES == 1 ? 6 : 3) * HALVES * kHalfBytes; }

// Whether rows whose position is in bucket threadIdx.x have a level.
template <class T>
__device__ __forceinline__ bool head_has_levels(const Bias &B, int heads, int head)
{
    if (threadIdx.x >= B.buckets || !beyond_plain(bias_at<T>(B, threadIdx.x, heads, head))) return false;
    float most = -INFINITY;
    for (int b = 0; b <= (int)threadIdx.x; ++b) most = fmaxf(most, bias_at<T>(B, b, heads, head));
    return level_of(most) != 0.0f;
}

// What the softmax threads of a CTA do, half a row each.
template <class T, int HALVES, bool BIAS, bool LEVELS>
__device__ __forceinline__ void forward_rows(const ForwardParams &P, ForwardShared<HALVES, BIAS> &M, uint8_t *tiles, uint32_t tensor_base, Work coming, int total)
{
    constexpr bool kBf16 = __is_same(T, __nv_bfloat16);
    constexpr int kTileBytes = HALVES * kHalfBytes;
    constexpr bool kAhead = HALVES == 1;
    constexpr int kStages = kAhead ? 2 : 1;
    // of 16 pairs, 8,192 tokens, 16 heads: dim 64 four 208 us, two 199, one 215, none 220; dim 128 two 258, the 12th 254, the last 259, none 265
    constexpr int kOwn = kAhead ? 8 : 12;
    // fp16 has no numbers below 2^-24: probabilities, at most 2^kLazy, are kept higher up
    constexpr float kShift = kBf16 ? 0.0f : 7.0f;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int half = warp >> 2, row = threadIdx.x & (kTile - 1), col0 = half * 64;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t s_at = tensor_base, o_at = s_at + kTile, p_at = kAhead ? o_at + 64 : s_at;
    const int o_begin = half * 32 * HALVES, o_end = min(o_begin + 32 * HALVES, P.dim);      // its columns of O
    volatile int *failed = &M.failed;
    auto kv_of = [&](int head) { return (int)divide(head, P.by_group); };
    float far = 0.0f;
    const float *table = nullptr;
    if constexpr (BIAS) table = M.tables.distance + kBefore;
    // where it is not, all works are gone through all the same, without waits, for the barriers in them
    bool ok = true;
    int t = 0, n = 0, head_before = -1;
    for (int turn = 1; coming.some; ++turn) {
        const Work w = coming;
        coming = work_at(P.items, total, P.by_heads, turn);
        if (w.item.length <= 0) continue;
        const int tile = w.item.level, first = w.item.first + tile * kTile;
        if constexpr (BIAS) {
            if (w.head != head_before) {
                const float mine = threadIdx.x < P.bias.buckets ? bias_at<T>(P.bias, threadIdx.x, P.heads, w.head) : 0.0f;
                if (n == 0) make_tables<kSoftmaxThreads, true, LEVELS>(P.bias, M.tables, mine);
                else make_tables<kSoftmaxThreads, false, LEVELS>(P.bias, M.tables, mine);
                far = M.tables.value[P.bias.buckets - 1];
                head_before = w.head;
            }
            if constexpr (LEVELS) far = M.tables.beside(P.bias.last, M.tables.level_at(P.bias, tile * kTile + row));
        }
        float top = -INFINITY, sum = 0.0f;   // top: what is subtracted, base 2
        for (int j = 0; j <= tile; ++j, ++t) {
            ok = ok && wait_all(&M.s, t & 1, failed);
            umma::fence_after();
            if (j > 0 && j % kChain == 0) {
                // a chain of sums ends: what lies in memory, of another maximum, and this one
                if (kAhead) {
                    ok = ok && wait_all(&M.o, (t & 1) ^ 1, failed);
                    umma::fence_after();
                }
                float *folded = room_of(P.fold, blockIdx.x, row);
                const float factor = top > -INFINITY ? exp2_fast(M.fold_top[half][row] - top) : 1.0f;
                add_to_room(folded, o_at + lanes, o_begin, o_end, factor, j > kChain);
                M.fold_top[half][row] = top;
            }
            const bool diagonal = j == 0, near = BIAS && j * kTile - (kTile - 1) < P.bias.last;
            const float *distance = table + j * kTile + row - col0;           // - column
            // half a row; with a bias it becomes the whole exponent here, else scale and bias come with the exponential
            uint32_t s[64];
            float most[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            umma::tensor_memory_load(s_at + lanes + col0, s);
            umma::tensor_memory_load(s_at + lanes + col0 + 32, s + 32);
            umma::tensor_memory_loaded<64>(s);
            if constexpr (LEVELS) {
                if (near) {
                    const float level = M.tables.level_at(P.bias, tile * kTile + row);
#pragma unroll
                    for (int i = 0; i < 64; ++i)
                        s[i] = __float_as_uint(__fmaf_rn(__uint_as_float(s[i]), P.scale2, M.tables.beside(j * kTile + row - col0 - i, level)));
                }
            }
            if (near && !LEVELS) {
#pragma unroll
                for (int i = 0; i < 64; ++i) s[i] = __float_as_uint(__fmaf_rn(__uint_as_float(s[i]), P.scale2, distance[-i]));
            }
            if (diagonal) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const uint32_t keep = below(row - col0 + 1 - 32 * c);
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (!(keep >> i & 1)) s[32 * c + i] = 0xff800000u;   // -inf
                }
            }
#pragma unroll
            for (int i = 0; i < 64; i += 8)
#pragma unroll
                for (int m = 0; m < 4; ++m) most[m] = max3(most[m], __uint_as_float(s[i + 2 * m]), __uint_as_float(s[i + 2 * m + 1]));
            if (kAhead) {
                umma::fence_before();
                __syncwarp();
                if (lane == 0) umma::barrier_arrive(umma::shared_address(&M.read));
            }
            float higher = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
            M.other[t & 1][half][row] = higher;
            barrier_named(2 + (warp & 3), 64);                           // the two warps that have these rows
            higher = fmaxf(higher, M.other[t & 1][half ^ 1][row]);
            if (!near) higher = __fmaf_rn(higher, P.scale2, far);
            if (kAhead && t > 0) {           // else M.s has said so: the product of the tile before is complete
                ok = ok && wait_all(&M.o, (t & 1) ^ 1, failed);
                umma::fence_after();
            }
            if (__any_sync(0xffffffffu, higher > top + kLazy)) {
                higher = fmaxf(higher, top);
                const float factor = higher > -INFINITY ? exp2_fast(top - higher) : 1.0f;
                top = higher;
                sum *= factor;
                if (j % kChain > 0) {
                    for (int c = o_begin; c < o_end; c += 16) {
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
            for (int c = 0; c < 64; c += 32) {
                uint32_t p[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint64_t x = fma_both(pair_of(s[c + 2 * i], s[c + 2 * i + 1]), times, plus);
                    const uint64_t e = exp2_pair<kOwn>(x, i);
                    parts[i & 3] = add_both(parts[i & 3], e);
                    p[i] = pack2<T>(low_of(e), high_of(e));
                }
                umma::tensor_memory_store16(p_at + lanes + (kAhead ? half * 32 : col0) + c / 2, p);
                if (!diagonal) {
                    umma::tensor_memory_stored();
                    umma::fence_before();
                    __syncwarp();
                    if (lane == 0) umma::barrier_arrive(umma::shared_address(&M.p[c / 32]));
                }
            }
            const uint64_t all = add_both(add_both(parts[0], parts[1]), add_both(parts[2], parts[3]));
            sum += low_of(all) + high_of(all);
            if (diagonal) {
                // keys that are masked here may hold anything: rows of the next sequence, or of none
                ok = ok && wait_all(&M.v_full[t % kStages], t / kStages & 1, failed);
                uint8_t *v = tiles + (2 * kStages + t % kStages) * kTileBytes + half * kHalfBytes;
                if (half < HALVES && not_clean<T>(v, row)) {
                    clean_row<T>(v, row);
                    M.dirty[n & 1] = 1;
                }
                umma::tensor_memory_stored();
                umma::fence_before();
                __syncwarp();
                if (lane == 0)
                    for (int i = 0; i < 2; ++i) umma::barrier_arrive(umma::shared_address(&M.p[i]));
            }
        }
        // while the last product runs: the sum, and all that does not need O
        const int left = w.item.length - tile * kTile;                        // queries of this tile
        uint16_t *out = (uint16_t *)P.out.p + (long long)(first + (warp & 3) * 32) * P.out.token + w.head * P.out.head;
        M.other_sum[half][row] = sum;
        barrier_named(2 + (warp & 3), 64);
        sum += M.other_sum[half ^ 1][row];
        float unit = sum > 0.0f || sum != sum ? reciprocal(sum) : 0.0f;
        if (half == 0 && row < left) {
            float lse = sum == 0.0f ? -INFINITY : (top + (log2_fast(sum) - kShift)) * kLn2;
            if constexpr (LEVELS) lse += M.tables.level_at(P.bias, tile * kTile + row);
            P.lse[(long long)w.head * P.tokens + first + row] = lse;
        }
        ok = ok && wait_all(&M.o, (t & 1) ^ 1, failed);
        umma::fence_after();
        if (threadIdx.x == 0) M.dirty[(n & 1) ^ 1] = 0;                         // read by all in the work before
        barrier_named(1, kSoftmaxThreads);
        const bool poisoned = *(volatile int *)&M.dirty[n & 1] != 0;
        if (!ok || *failed) {
            unit = NAN;
            if (half == 0 && row < left) P.lse[(long long)w.head * P.tokens + first + row] = NAN;
        }
        for (int c = o_begin; c < o_end; c += 32)
            put_rows<T>(o_at + lanes, unit, out, P.out.token, c, P.dim, left - (warp & 3) * 32, [&](float *x) {
                if (tile >= kChain) {
                    const float *folded = room_of(P.fold, blockIdx.x, row);
                    const float factor = top > -INFINITY ? exp2_fast(M.fold_top[half][row] - top) * unit : unit;
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (c + i < o_end) x[i] = __fmaf_rn(folded[(c + i) * kTile], factor, x[i]);
                }
                if (!poisoned) return;
                const uint16_t *v = (const uint16_t *)P.v.p + (long long)first * P.v.token + kv_of(w.head) * P.v.head;
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (c + i < o_end && row < left) x[i] += taken_away<T>(v + c + i, P.v.token, 0, row + 1);
            });
        ++n;
    }
}
template <class T, int HALVES>
__device__ __noinline__ void forward_rows_with_levels(const ForwardParams &P, ForwardShared<HALVES, true> &M, uint8_t *tiles, uint32_t tensor_base, Work coming,
                                                      int total)
{
    forward_rows<T, HALVES, true, true>(P, M, tiles, tensor_base, coming, total);
}

// A CTA has 128 queries of one head; two CTAs share an SM, so that one's softmax
// runs under the other's products.  Per tile of 128 keys: S = Q K^T into tensor
// memory; two threads have a row of it, 64 columns each, and tell one another
// their maxima; P goes back into tensor memory as the left operand of O += P V,
// 32 columns of each half ahead of the others.  For dim <= 64 the half of an SM's
// tensor memory that a CTA has holds P beside S: the next scores are computed as
// soon as S has been read, with two tiles of K and V under way.  For more, P takes
// the place of S.
// 8,192 tokens, 16 heads (bf16, one sequence): dim 128 0.25 to 0.28 ms, 0.98 to 1.08
// PFLOP/s, where exponentials and products take the same time and wait for one
// another (54 % of each unit); dim 64 0.21 ms, 0.65 PFLOP/s, bound by the exponentials
// and the issue slots about them (57 % of both).  37 sequences of some 440 tokens
// have works of 3.5 tiles, whose beginnings and ends cost as much as the tiles.
template <class T, int HALVES, bool BIAS>
__global__ void __launch_bounds__(kForwardThreads, 2)
psops_attention_forward_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                               const __grid_constant__ CUtensorMap map_v, const __grid_constant__ ForwardParams P)
{
    constexpr bool kBf16 = __is_same(T, __nv_bfloat16);
    constexpr int kTileBytes = HALVES * kHalfBytes;
    constexpr bool kAhead = HALVES == 1;
    constexpr int kStages = kAhead ? 2 : 1;
    extern __shared__ uint8_t raw[];
    __shared__ ForwardShared<HALVES, BIAS> M;
    __shared__ uint32_t tensor_base_slot;

    const int warp = threadIdx.x >> 5;
    volatile int *failed = &M.failed;
    uint8_t *tiles = raw + (((umma::shared_address(raw) + 1023u) & ~1023u) - umma::shared_address(raw));
    const uint32_t q_at = umma::shared_address(tiles), k_at = q_at + kStages * kTileBytes, v_at = k_at + kStages * kTileBytes;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i)
            for (uint64_t *b : {&M.q_full[i], &M.q_empty[i], &M.k_full[i], &M.k_empty[i], &M.v_full[i], &M.v_empty[i]})
                umma::barrier_init(umma::shared_address(b), 1);
        umma::barrier_init(umma::shared_address(&M.s), 1);
        umma::barrier_init(umma::shared_address(&M.o), 1);
        umma::barrier_init(umma::shared_address(&M.read), 8);
        for (int i = 0; i < 2; ++i) umma::barrier_init(umma::shared_address(&M.p[i]), 8);
        M.failed = M.dirty[0] = M.dirty[1] = 0;
        umma::barrier_init_done();
        umma::prefetch_map(&map_q);
        umma::prefetch_map(&map_k);
        umma::prefetch_map(&map_v);
    }
    if (warp == 9) umma::tensor_columns_take<256>(umma::shared_address(&tensor_base_slot));
    umma::fence_before();
    __syncthreads();
    umma::fence_after();
    const uint32_t s_at = tensor_base_slot, o_at = s_at + kTile, p_at = kAhead ? o_at + 64 : s_at;

    umma::after_the_kernel_before();
    auto kv_of = [&](int head) { return (int)divide(head, P.by_group); };
    int total = 0;
    Work coming;
    if (P.own) {
        coming = own_work(P.prep, P.by_heads);
        if (P.prep.fill > 0) fill_rest<kForwardThreads>(P.prep, blockIdx.x, gridDim.x);
    } else {
        total = *P.count * P.heads;
        coming = work_at(P.items, total, P.by_heads, 0);
    }

    if (warp == 8) {
        // ---- copies in; the tile on the diagonal comes first
        bool ok = true;
        int t = 0, n = 0;                        // tiles and works before this one
        for (int turn = 1; coming.some && ok; ++turn) {
            const Work w = coming;
            coming = work_at(P.items, total, P.by_heads, turn);
            if (w.item.length <= 0) continue;
            const int first = w.item.first + w.item.level * kTile, kv = kv_of(w.head), q_stage = n % kStages;
            ok = wait_all(&M.q_empty[q_stage], (n / kStages & 1) ^ 1, failed);
            if (!ok) break;
            if (umma::elected()) {
                umma::barrier_expect(umma::shared_address(&M.q_full[q_stage]), kTileBytes);
                for (int h = 0; h < HALVES; ++h)
                    umma::tensor_load3(q_at + q_stage * kTileBytes + h * kHalfBytes, &map_q, h * 64, w.head, first, umma::shared_address(&M.q_full[q_stage]));
            }
            __syncwarp();
            ++n;
            for (int j = 0; j <= w.item.level; ++j, ++t) {
                const int token = first - j * kTile, stage = t % kStages;
                const uint32_t phase = (t / kStages & 1) ^ 1;
                ok = wait_all(&M.k_empty[stage], phase, failed);
                if (!ok) break;
                if (umma::elected()) {
                    umma::barrier_expect(umma::shared_address(&M.k_full[stage]), kTileBytes);
                    for (int h = 0; h < HALVES; ++h)
                        umma::tensor_load3(k_at + stage * kTileBytes + h * kHalfBytes, &map_k, h * 64, kv, token, umma::shared_address(&M.k_full[stage]));
                }
                __syncwarp();
                ok = wait_all(&M.v_empty[stage], phase, failed);
                if (!ok) break;
                if (umma::elected()) {
                    umma::barrier_expect(umma::shared_address(&M.v_full[stage]), kTileBytes);
                    for (int h = 0; h < HALVES; ++h)
                        umma::tensor_load3(v_at + stage * kTileBytes + h * kHalfBytes, &map_v, h * 64, kv, token, umma::shared_address(&M.v_full[stage]));
                }
                __syncwarp();
            }
        }
        if (!ok) __nanosleep(1000000);           // copies in flight land long before
    } else if (warp == 9) {
        // ---- products; they run in the order in which they are issued, so S may follow P V without a wait
        const int steps = (P.dim + 15) / 16;
        const uint32_t instr_s = umma::instruction(kBf16, false, false, kTile, kTile);
        const uint32_t instr_o = umma::instruction(kBf16, false, true, kTile, steps * 16);
        const uint64_t dq = umma::operand(q_at, false), dk = umma::operand(k_at, false), dv = umma::operand(v_at, true, kHalfBytes);
        constexpr uint32_t kNext = kTileBytes >> 4;
        // scores of tile t, the `j`th of work n
        auto scores = [&](int t, int n, int j, int last) {
            const int stage = t % kStages, q_stage = n % kStages;
            if (j == 0 && !wait_all(&M.q_full[q_stage], n / kStages & 1, failed)) return false;
            if (!wait_all(&M.k_full[stage], t / kStages & 1, failed)) return false;
            if (kAhead && t > 0 && !wait_all(&M.read, (t & 1) ^ 1, failed)) return false;
            umma::fence_after();
            if (umma::elected()) {
                for (int s = 0; s < steps; ++s) {
                    const uint32_t on = (s >> 2) * (kHalfBytes >> 4) + (s & 3) * 2;
                    umma::multiply<false>(s_at, dq + q_stage * kNext + on, dk + stage * kNext + on, instr_s, s > 0);
                }
                umma::products_arrive<false>(umma::shared_address(&M.s));
                umma::products_arrive<false>(umma::shared_address(&M.k_empty[stage]));
                if (j == last) umma::products_arrive<false>(umma::shared_address(&M.q_empty[q_stage]));
            }
            __syncwarp();
            return true;
        };
        int t = 0, n = 0, turn = 1;
        auto next_work = [&]() {                 // the next one with tokens
            Work w = coming;
            while (w.some) {
                coming = work_at(P.items, total, P.by_heads, turn++);
                if (w.item.length > 0) break;
                w = coming;
            }
            return w;
        };
        Work w = next_work();
        bool ok = !w.some || scores(0, 0, 0, w.item.level);
        while (w.some && ok) {
            const Work then = next_work();
            for (int j = 0; j <= w.item.level; ++j, ++t) {
                const int stage = t % kStages;
                // the scores after these: of the next tile, or of the next work's first one
                auto ahead = [&]() {
                    return j < w.item.level ? scores(t + 1, n, j + 1, w.item.level) : !then.some || scores(t + 1, n + 1, 0, then.item.level);
                };
                if (kAhead) ok = ahead();
                ok = ok && wait_all(&M.v_full[stage], t / kStages & 1, failed);
                // the first 32 columns of both halves of a row, then the others
                for (int part = 0; part < 2 && ok; ++part) {
                    ok = wait_all(&M.p[part], t & 1, failed);
                    if (!ok) break;
                    umma::fence_after();
                    if (umma::elected()) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            // 16 keys s of the tile; P's columns are 0-63, or 0-31 and 64-95 where it lies in S
                            const int s = (i >> 1) * 4 + part * 2 + (i & 1);
                            umma::multiply_from_tensor_memory(o_at, p_at + (i >> 1) * (kAhead ? 32 : 64) + (part * 2 + (i & 1)) * 8,
                                                              dv + stage * kNext + s * 128, instr_o, j % kChain > 0 || part > 0 || i > 0);
                        }
                        if (part == 1) {
                            umma::products_arrive<false>(umma::shared_address(&M.v_empty[stage]));
                            umma::products_arrive<false>(umma::shared_address(&M.o));
                        }
                    }
                    __syncwarp();
                }
                if (!ok) break;
                if (!kAhead && !(ok = ahead())) break;
            }
            ++n;
            w = then;
        }
    } else {
        // ---- softmax
        bool levels = false;
        if constexpr (BIAS) {
            if (P.own) levels = barrier_any(1, kSoftmaxThreads, coming.some && head_has_levels<T>(P.bias, P.heads, coming.head));
            else levels = *P.levels != 0;
            if (levels) forward_rows_with_levels<T, HALVES>(P, M, tiles, tensor_base_slot, coming, total);
        }
        if (!levels) forward_rows<T, HALVES, BIAS, false>(P, M, tiles, tensor_base_slot, coming, total);
    }
    __syncwarp();
    umma::fence_before();
    __syncthreads();
    umma::fence_after();
    if (warp == 9) umma::tensor_columns_give<256>(tensor_base_slot);
}

// ---------------------------------------------------------------------------
// Backward
// ---------------------------------------------------------------------------

// dbias's sums: by slot (only used ones count), head and bucket.
constexpr int kJoinParts = 16;
struct JoinParams {
    const float *partials;
    const int *used;
    int slots, heads, buckets, fp32;
    void *out;                               // buckets x heads
    int *ticket;
};
// Slots from, from + step, ... of one of them, eight loads under way at a time.
__device__ __forceinline__ double sum_of_slots(const JoinParams &P, int at, int from, int step)
{
    const int per_slot = P.heads * P.buckets;
    double sum = 0.0;
    for (int s = from; s < P.slots; s += 8 * step) {
        float x[8];
        int used[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int slot = min(s + i * step, P.slots - 1);
            used[i] = s + i * step < P.slots ? P.used[slot] : 0;
            x[i] = __ldcg(P.partials + (long long)slot * per_slot + at);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (used[i]) sum += (double)x[i];
    }
    return sum;
}
template <class T>
__device__ __forceinline__ void put_dbias(const JoinParams &P, int at, double sum)
{
    const long long to = (long long)(at % P.buckets) * P.heads + at / P.buckets;
    if (P.fp32) ((float *)P.out)[to] = (float)sum;
    else ((T *)P.out)[to] = (T)(float)sum;
}

struct BackwardParams {
    const Item *items;
    const int *count;
    int tokens, heads, group, dim;
    Divisor by_heads, by_kv_heads, by_group;
    int keys;
    int split;                               // KEYS: a work has one query head only, and the last of a key head's CTAs adds them up
    int *arrived, *unclean;                  // for that, by slot and key head, from zero: CTAs that are done; which of dk, dv met no number
    float scale, scale2;
    Heads q, k, grad;                        // read where numbers are not finite
    Heads dq, dk, dv;                        // an address is NULL where the result is not wanted
    const float *lse, *beside;               // beside: of rows with levels
    const int *levels;                       // whether there can be any
    float *delta;                            // !KEYS makes it exact, for KEYS after it
    const float2 *norms;                     // NULL, or `blocks` of them
    int blocks;
    Bias bias;
    float *partials;                         // dbias by slot, head and bucket; NULL: not wanted
    float *fold;                             // room for sums of more than kChain tiles, twice kFoldFloats for each CTA
    JoinParams join;                         // ticket NULL: a kernel of its own joins them
};

constexpr int kBackwardThreads = 320;        // as above
// columns of ds that are summed along their diagonals at a time: as many as there is shared memory for
template <int HALVES> constexpr int kStripe = HALVES == 1 ? 32 : 16;
constexpr int kFewBuckets = 3;               // fewer buckets in a warp's part of a tile are summed one by one: 185 to 181 us
                                             // of a launch with 12,345 tokens, 12 heads and a bias to 512 (5: the same)
template <int HALVES> constexpr int kStripeFloats = 32 * (kStripe<HALVES> + 1);

template <int HALVES, bool BIAS>
constexpr int backward_shared() { return 1024 + 6 * HALVES * kHalfBytes + (BIAS ? 8 * (kStripeFloats<HALVES> + kMostBuckets) * 4 : 0); }

struct Barriers {
    uint64_t a_full, a_empty, b_full[2], b_empty[2], s[2], t, p, ds, sums;
};
template <bool BIAS>
struct BackwardShared {
    Barriers bars;
    int dirty[2][2];                         // by parity of the work, and which of B
    alignas(16) float by_column[2][2][kTile];        // lse and delta of the queries
    float level[BIAS ? 2 : 1][BIAS ? kTile : 1];     // and their levels
    float of_half[2][kTile];
    int last, unclean;
    typename Choose<BIAS>::Type tables;
};

// One kernel, two uses, one launch each.  A CTA keeps two tiles of 128 rows
// (A0, A1) and meets pairs of tiles of 128 rows (B0, B1) one after the other:
//              A0  A1  B0  B1     S = A0 B0^T   T = A1 B1^T   sums
//   !KEYS      q   do  k   v      scores        dp            dq += ds B0, mean key += p B0
//   KEYS       k   v   q   do     scores^T      dp^T          dk += ds^T B0, dv += p^T B1, dbias
// The scores are computed in both: eight products instead of the five that a
// single pass needs, and in exchange no sum passes between CTAs, so that all
// gradients are the same in every run and dq needs no fp32 sums in memory.
// KEYS goes through all query heads that share its keys.  p and ds go back into
// tensor memory, in place of the scores and of dp, as left operands.  Softmax
// threads have one row and 64 columns each.  While they form p, the products of
// ds of the tile before and of dp run; while they form ds, those of p and of the
// next scores.
// delta = do . out comes with out's rounding and its probabilities', which would be
// common to a row's ds (dq was off by 2.1 times what its own rounding leaves, dk by
// 1.8).  But a row's ds have the sum zero: what they sum up to is what delta is off
// by, and what their own rounding has in common.  !KEYS takes it out, in dq by the
// mean key (one more product, p k; dq and dk are off by 1.3 to 1.5 times their
// rounding then, for a tenth of the time), and leaves the corrected delta to KEYS.
// Where a row has but one tile, delta is made from p and dp first.
// 8,192 tokens, 16 heads of 128 on 4 (bf16, one sequence): queries 0.43 ms, keys 0.46,
// 1.2 PFLOP/s: tensor unit 64 % of the time, fed from shared memory at its 128
// bytes a clock in the scores' products; longer calls meet the power cap.  dim 64:
// 0.35 and 0.39 ms, the softmax threads' latency (one CTA an SM).
template <class T, int HALVES, bool KEYS, bool BIAS, bool LEVELS>
__device__ __forceinline__ void backward_part(const CUtensorMap &map_a0, const CUtensorMap &map_a1, const CUtensorMap &map_b0, const CUtensorMap &map_b1,
                                              const BackwardParams &P, BackwardShared<BIAS> &M, uint8_t *tiles, uint32_t tensor_base, float unit,
                                              volatile int *failed)
{
    constexpr bool kBf16 = __is_same(T, __nv_bfloat16);
    constexpr int kTileBytes = HALVES * kHalfBytes;
    constexpr int kOwn = 4;                  // queries and keys of 8,192 tokens, 16 heads x 64: 780 us, every 8th pair 800, none 808
    // scores in two places by turns, where tensor memory has room for them: the next ones need not wait for these
    constexpr bool kTwice = KEYS && HALVES == 1;
    constexpr uint32_t kSecond = 3 * kTile;                                 // columns 384 to 511
    // fp16: probabilities are kept 2^14 times as large (dv is scaled back), ds by a power of two from the norms
    constexpr float kShift = kBf16 ? 0.0f : 14.0f;
    Barriers &bars = M.bars;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t a_at = umma::shared_address(tiles), b_at = a_at + 2 * kTileBytes;
    float *stripes = (float *)(tiles + 6 * kTileBytes), *bucket_sums = stripes + 8 * kStripeFloats<HALVES>;

    if (threadIdx.x == 0) {
        for (uint64_t *b : {&bars.a_full, &bars.a_empty, &bars.b_full[0], &bars.b_full[1], &bars.b_empty[0], &bars.b_empty[1], &bars.s[0],
                            &bars.s[1], &bars.t, &bars.sums})
            umma::barrier_init(umma::shared_address(b), 1);
        umma::barrier_init(umma::shared_address(&bars.p), 8);
        umma::barrier_init(umma::shared_address(&bars.ds), 8);
        M.dirty[0][0] = M.dirty[0][1] = M.dirty[1][0] = M.dirty[1][1] = 0;
        umma::barrier_init_done();
    }
    if (BIAS && KEYS)
        for (int i = threadIdx.x; i < 8 * kMostBuckets; i += kBackwardThreads) bucket_sums[i] = 0.0f;
    umma::fence_before();
    __syncthreads();
    umma::fence_after();
    const uint32_t s_at = tensor_base, t_at = s_at + kTile, sum0_at = t_at + kTile, sum1_at = sum0_at + HALVES * 64;

    const Divisor &heads = KEYS ? P.by_kv_heads : P.by_heads;               // of A0
    const int total = *P.count * (int)heads.by;
    auto work_of = [&](int turn) { return work_at(P.items, total, heads, turn); };
    Work coming = work_of(0);
    auto kv_of = [&](int head) { return (int)divide(head, P.by_group); };
    // KEYS: the key head of a work, its first query head and how many
    auto key_head_of = [&](const Work &w) { return P.split ? kv_of(w.head) : w.head; };
    auto query_head_of = [&](const Work &w) { return P.split ? w.head : w.head * P.group; };
    const int query_heads = P.split ? 1 : P.group;
    // A tile meets level + 1 tiles of B (of each head): !KEYS from the diagonal down, KEYS from the diagonal up.
    auto tile_of = [](const Work &w) { return KEYS ? (w.item.length + kTile - 1) / kTile - 1 - w.item.level : w.item.level; };
    auto token_of = [](int first, int meets, int j) { return KEYS ? first + (j % meets) * kTile : first - j * kTile; };

    if (warp == 8) {
        // ---- copies in
        bool ok = true;
        int r = 0, n = 0;                        // rounds and works before this one
        for (int turn = 1; coming.some && ok; ++turn) {
            const Work w = coming;
            coming = work_of(turn);
            if (w.item.length <= 0) continue;
            const int first = w.item.first + tile_of(w) * kTile, meets = w.item.level + 1, rounds = KEYS ? meets * query_heads : meets;
            const int a_head = KEYS ? key_head_of(w) : w.head;
            ok = wait_all(&bars.a_empty, (n & 1) ^ 1, failed);
            if (!ok) break;
            if (umma::elected()) {
                umma::barrier_expect(umma::shared_address(&bars.a_full), 2 * kTileBytes);
                for (int h = 0; h < HALVES; ++h) {
                    umma::tensor_load3(a_at + h * kHalfBytes, &map_a0, h * 64, a_head, first, umma::shared_address(&bars.a_full));
                    umma::tensor_load3(a_at + kTileBytes + h * kHalfBytes, &map_a1, h * 64, a_head, first, umma::shared_address(&bars.a_full));
                }
            }
            __syncwarp();
            ++n;
            for (int j = 0; j < rounds; ++j, ++r) {
                const int stage = r & 1, token = token_of(first, meets, j), b_head = KEYS ? query_head_of(w) + j / meets : kv_of(w.head);
                ok = wait_all(&bars.b_empty[stage], (r >> 1 & 1) ^ 1, failed);
                if (!ok) break;
                if (umma::elected()) {
                    const uint32_t to = b_at + stage * 2 * kTileBytes, full = umma::shared_address(&bars.b_full[stage]);
                    umma::barrier_expect(full, 2 * kTileBytes);
                    for (int h = 0; h < HALVES; ++h) {
                        umma::tensor_load3(to + h * kHalfBytes, &map_b0, h * 64, b_head, token, full);
                        umma::tensor_load3(to + kTileBytes + h * kHalfBytes, &map_b1, h * 64, b_head, token, full);
                    }
                }
                __syncwarp();
            }
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
        auto scores = [&](int r, int which) {
            const uint32_t stage = (r & 1) * 2 * kNext + which * kNext;
            if (umma::elected()) {
                for (int s = 0; s < steps; ++s) {
                    const uint32_t on = (s >> 2) * (kHalfBytes >> 4) + (s & 3) * 2;
                    umma::multiply<false>(which ? t_at : s_at + (kTwice && (r & 1) ? kSecond : 0), da + which * kNext + on, db + stage + on, instr_s, s > 0);
                }
                umma::products_arrive<false>(umma::shared_address(which ? &bars.t : &bars.s[kTwice ? r & 1 : 0]));
            }
            __syncwarp();
        };
        auto add = [&](int r, int j, int which, uint32_t from, uint32_t to) {
            if (umma::elected()) {
#pragma unroll
                for (int s = 0; s < kTile / 16; ++s)        // columns 0-31 and 64-95 hold the halves
                    umma::multiply_from_tensor_memory(to, from + (s >> 2) * 64 + (s & 3) * 8, db_across + (r & 1) * 2 * kNext + which * kNext + s * 128,
                                                      instr_sum, j % kChain > 0 || s > 0);
            }
            __syncwarp();
        };
        bool ok = true;
        int r = 0, n = 0;
        for (int turn = 1; coming.some && ok; ++turn) {
            const Work w = coming;
            coming = work_of(turn);
            if (w.item.length <= 0) continue;
            const int meets = w.item.level + 1, rounds = KEYS ? meets * query_heads : meets;
            auto loaded = [&](int r) { return wait_all(&bars.b_full[r & 1], r >> 1 & 1, failed); };
            auto last_scores = [&](int j) {                                  // A is read no more
                if (j == rounds - 1 && umma::elected()) umma::products_arrive<false>(umma::shared_address(&bars.a_empty));
                __syncwarp();
            };
            ok = wait_all(&bars.a_full, n & 1, failed) && loaded(r);
            if (!ok) break;
            umma::fence_after();
            scores(r, 0);
            scores(r, 1);
            last_scores(0);
            for (int j = 0; j < rounds; ++j, ++r) {
                auto next_scores = [&]() {
                    if (j + 1 == rounds) return true;
                    if (!loaded(r + 1)) return false;
                    umma::fence_after();
                    scores(r + 1, 0);
                    return true;
                };
                // the place of the next scores has been read: bar_ds of the round before says so
                if (kTwice && !(ok = next_scores())) break;
                ok = wait_all(&bars.p, r & 1, failed);
                if (!ok) break;
                umma::fence_after();
                add(r, j, KEYS ? 1 : 0, s_at + (kTwice && (r & 1) ? kSecond : 0), sum1_at);
                if (!kTwice) {
                    // ... or follows in the order of the products
                    if (!(ok = next_scores())) break;
                }
                ok = wait_all(&bars.ds, r & 1, failed);
                if (!ok) break;
                umma::fence_after();
                add(r, j, 0, t_at, sum0_at);
                if (umma::elected()) {
                    umma::products_arrive<false>(umma::shared_address(&bars.b_empty[r & 1]));
                    if (j + 1 == rounds || (j + 1) % kChain == 0) umma::products_arrive<false>(umma::shared_address(&bars.sums));
                }
                __syncwarp();
                if (j + 1 < rounds) {
                    scores(r + 1, 1);
                    last_scores(j + 1);
                }
            }
            ++n;
        }
    } else {
        // ---- softmax: row and 64 columns of each tile
        const int half = warp >> 2, row = threadIdx.x & (kTile - 1), col0 = half * 64;
        const uint32_t lanes = ((uint32_t)((warp & 3) * 32) << 16) + col0;
        const float unit_p = kBf16 ? 1.0f : unit * 0x1p-14f;
        // a row whose scores are all -inf has no probabilities
        auto base2 = [](float lse) { return lse == -INFINITY ? INFINITY : lse * kLog2e; };
        float far = 0.0f;
        const float *table = nullptr;
        if constexpr (BIAS) table = M.tables.distance + kBefore;
        // what the two threads of a row have, together
        auto both_halves = [&](float x) {
            barrier_named(2 + (warp & 3), 64);                              // what they had before has been read
            M.of_half[half][row] = x;
            barrier_named(2 + (warp & 3), 64);
            return M.of_half[0][row] + M.of_half[1][row];
        };
        // where it is not, all works are gone through all the same, without waits, for the barriers in them
        bool ok = true;
        int r = 0, n = 0, chains = 0, head_before = -1;                     // rounds, works and chains of sums before
        for (int turn = 1; coming.some; ++turn) {
            const Work w = coming;
            coming = work_of(turn);
            if (w.item.length <= 0) continue;
            const Item item = w.item;
            const int head = KEYS ? key_head_of(w) : w.head, tile = tile_of(w), first = item.first + tile * kTile, meets = item.level + 1;
            const int rounds = KEYS ? meets * query_heads : meets;
            const int left = item.length - tile * kTile;                        // rows of A that exist
            float row_base = 0.0f, row_delta = 0.0f, row_sum = 0.0f, far_sum = 0.0f, next_value = 0.0f;
            if (!KEYS && row < left) {
                const long long at = (long long)head * P.tokens + first + row;
                row_base = kShift - base2(P.lse[at]);
                row_delta = -P.delta[at] * unit_p;
            }
            // KEYS: lse or delta of one query of a round, as it is in memory, a round ahead; 0 where there is none
            auto fetch = [&](int apart, int q_head) {
                const int token = first + apart * kTile + row;
                if (token >= item.first + item.length) return 0.0f;
                return (half == 0 ? P.lse : P.delta)[(long long)q_head * P.tokens + token];
            };
            int apart = 0, q_head = KEYS ? query_head_of(w) : head;             // tiles between queries and keys; KEYS: the query head
            float column = KEYS ? fetch(0, q_head) : 0.0f;
            // the bias of the (first) query head
            auto value = [&](int q_head) { return threadIdx.x < P.bias.buckets ? bias_at<T>(P.bias, threadIdx.x, P.heads, q_head) : 0.0f; };
            if constexpr (BIAS) {
                if (q_head != head_before) {
                    if (n > 0) barrier_named(1, kSoftmaxThreads);               // nobody reads the M.tables of the head before
                    const float mine = value(q_head);
                    if (n == 0) make_tables<kSoftmaxThreads, true, LEVELS>(P.bias, M.tables, mine);
                    else make_tables<kSoftmaxThreads, false, LEVELS>(P.bias, M.tables, mine);
                    far = LEVELS ? M.tables.beside(P.bias.last, 0.0f) : M.tables.value[P.bias.buckets - 1];
                    head_before = q_head;
                }
            }
            float row_level = 0.0f;
            if constexpr (LEVELS && !KEYS) {
                if (row < left) {
                    const long long at = (long long)head * P.tokens + first + row;
                    if (beyond_plain(P.lse[at])) row_level = M.tables.level_at(P.bias, tile * kTile + row);
                    if (row_level != 0.0f) row_base = kShift - P.beside[at];
                }
                far = M.tables.beside(P.bias.last, row_level);
            }
            for (int j = 0; j < rounds; ++j, ++r) {
                if (j > 0 && j % kChain == 0) {
                    // before p and ds of this round let the next chain begin
                    ok = ok && wait_all(&bars.sums, chains++ & 1, failed);
                    umma::fence_after();
                    for (int which = 0; which < 2; ++which)
                        add_to_room(room_of(P.fold, blockIdx.x * 2 + which, row), (which ? sum1_at : sum0_at) + lanes - col0, half * 32 * HALVES,
                                    min((half + 1) * 32 * HALVES, P.dim), 1.0f, j > kChain);
                    umma::fence_before();
                }
                const bool diagonal = apart == 0;
                const bool near = BIAS && apart * kTile - (kTile - 1) < P.bias.last;
                const int columns = KEYS ? min(item.length - (tile + apart) * kTile, kTile) : kTile;   // columns that exist
                if (KEYS) {
                    if constexpr (BIAS) {
                        if (j > 0 && diagonal) {
                            barrier_named(1, kSoftmaxThreads);                  // nobody reads the M.tables of the head before
                            make_tables<kSoftmaxThreads, false, LEVELS>(P.bias, M.tables, next_value);
                            far = LEVELS ? M.tables.beside(P.bias.last, 0.0f) : M.tables.value[P.bias.buckets - 1];
                            head_before = q_head;
                        }
                        if (diagonal && j + meets < rounds) next_value = value(q_head + 1);
                    }
                    float of = half == 0 ? kShift - base2(column) + (near ? 0.0f : far) : -column * unit_p;
                    if constexpr (LEVELS) {
                        if (half == 0) {
                            // (where there is no query, column is 0)
                            const float level = beyond_plain(column) ? M.tables.level_at(P.bias, (tile + apart) * kTile + row) : 0.0f;
                            M.level[r & 1][row] = level;
                            if (level != 0.0f)
                                of = kShift - P.beside[(long long)q_head * P.tokens + first + apart * kTile + row] +
                                     (near ? 0.0f : M.tables.beside(P.bias.last, level));
                        }
                    }
                    M.by_column[r & 1][half][row] = of;
                    barrier_named(1, kSoftmaxThreads);
                    const bool last = apart + 1 == meets;
                    if (j + 1 < rounds) column = fetch(last ? 0 : apart + 1, last ? q_head + 1 : q_head);
                }
                const bool masked = diagonal || columns < kTile;
                // distance of column c: of a query row to keys it falls with c, of a key row to queries it grows
                const float *distance = table + apart * kTile + (KEYS ? col0 - row : row - col0);
                ok = ok && wait_all(&bars.s[kTwice ? r & 1 : 0], (kTwice ? r >> 1 : r) & 1, failed);
                if (masked) {
                    // What is masked may hold anything: it must not meet a zero in a product to come.  KEYS: one half of the
                    // threads looks at q, the other at do; else both at k.
                    uint8_t *b = tiles + (2 + (r & 1) * 2 + (KEYS ? half : 0)) * kTileBytes;
                    bool any = false;
                    if (diagonal || row >= columns)
#pragma unroll
                        for (int h = 0; h < HALVES; ++h)
                            if (KEYS || h == half) any |= not_clean<T>(b + h * kHalfBytes, row);
                    if (__any_sync(0xffffffffu, any)) {
                        ok = ok && wait_all(&bars.t, r & 1, failed);            // the scores' products have read them
                        if (any) {
                            for (int h = 0; h < HALVES; ++h)
                                if (KEYS || h == half) clean_row<T>(b + h * kHalfBytes, row);
                            if (diagonal) M.dirty[n & 1][KEYS ? half : 0] = 1;
                        }
                        __syncwarp();
                    }
                }
                umma::fence_after();
                float p[64];
                // the columns that count, a bit each: !KEYS up to the row, KEYS from the row on, and those that exist
                uint32_t keep[2] = {~0u, ~0u};
                if (masked) {
                    const int from = KEYS && diagonal ? row - col0 : 0, to = KEYS ? columns - col0 : row - col0 + 1;
#pragma unroll
                    for (int c = 0; c < 2; ++c) keep[c] = below(to - 32 * c) & ~below(from - 32 * c);
                }
                const uint32_t here = s_at + lanes + (kTwice && (r & 1) ? kSecond : 0);
                uint32_t s[64];
                umma::tensor_memory_load(here, s);
                umma::tensor_memory_load(here + 32, s + 32);
                umma::tensor_memory_loaded<64>(s);
                const uint64_t times = both(P.scale2), even = both(row_base + far);
#pragma unroll
                for (int c = 0; c < 64; c += 32) {
                    // what a score's product is added to: shift, bias, -lse
                    if (LEVELS && near) {
                        if constexpr (LEVELS) {
#pragma unroll
                            for (int i = c; i < c + 32; ++i) {
                                const int d = KEYS ? apart * kTile + col0 + i - row : apart * kTile + row - col0 - i;
                                p[i] = (KEYS ? M.by_column[r & 1][0][col0 + i] : row_base) +
                                       M.tables.beside(d, KEYS ? M.level[r & 1][col0 + i] : row_level);
                            }
                        }
                    } else if (KEYS && near) {
#pragma unroll
                        for (int i = c; i < c + 32; i += 4) {
                            const float4 of = *(const float4 *)&M.by_column[r & 1][0][col0 + i];
                            p[i] = of.x + distance[i];
                            p[i + 1] = of.y + distance[i + 1];
                            p[i + 2] = of.z + distance[i + 2];
                            p[i + 3] = of.w + distance[i + 3];
                        }
                    } else if (KEYS) {
#pragma unroll
                        for (int i = c; i < c + 32; i += 4) {
                            const float4 of = *(const float4 *)&M.by_column[r & 1][0][col0 + i];
                            p[i] = of.x;
                            p[i + 1] = of.y;
                            p[i + 2] = of.z;
                            p[i + 3] = of.w;
                        }
                    } else if (near) {
#pragma unroll
                        for (int i = c; i < c + 32; ++i) p[i] = row_base + distance[-i];
                    } else {
#pragma unroll
                        for (int i = c; i < c + 32; ++i) p[i] = low_of(even);
                    }
#pragma unroll
                    for (int i = c; i < c + 32; i += 2) {
                        const uint64_t x = fma_both(pair_of(s[i], s[i + 1]), times, pair_of(__float_as_uint(p[i]), __float_as_uint(p[i + 1])));
                        const uint64_t e = exp2_pair<kOwn>(x, i / 2);
                        p[i] = low_of(e);
                        p[i + 1] = high_of(e);
                    }
                    if (masked) {
#pragma unroll
                        for (int i = c; i < c + 32; ++i)
                            if (!(keep[c / 32] >> (i - c) & 1)) p[i] = 0.0f;
                    }
                    uint32_t w[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) w[i] = pack2<T>(p[c + 2 * i], p[c + 2 * i + 1]);
                    umma::tensor_memory_store16(here + c / 2, w);
                }
                umma::tensor_memory_stored();
                umma::fence_before();
                __syncwarp();
                // (a warp arrives but once in a round: KEYS has a barrier in each, else the next scores wait for all to arrive)
                if (lane == 0) umma::barrier_arrive(umma::shared_address(&bars.p));
                ok = ok && wait_all(&bars.t, r & 1, failed);
                umma::fence_after();
                uint64_t rounded[4] = {0, 0, 0, 0};                             // sums of ds as it enters the products
                if (!KEYS && rounds == 1) {
                    // all of the row is here: delta from p and dp themselves
                    float sum = 0.0f;
#pragma unroll
                    for (int c = 0; c < 64; c += 32) {
                        uint32_t u[32];
                        umma::tensor_memory_load(t_at + lanes + c, u);
                        umma::tensor_memory_loaded<32>(u);
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (keep[c / 32] >> i & 1) sum = __fmaf_rn(p[c + i], __uint_as_float(u[i]), sum);
                    }
                    row_delta = -both_halves(sum) * (kBf16 ? 1.0f : unit_p * 0x1p-14f);
                }
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
                            const uint4 delta = *(const uint4 *)&M.by_column[r & 1][1][col0 + c + i];
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
                            if (!(keep[c / 32] >> i & 1)) p[c + i] = 0.0f;
                    }
                    uint32_t w[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) w[i] = pack2<T>(p[c + 2 * i], p[c + 2 * i + 1]);
                    umma::tensor_memory_store16(t_at + lanes + c / 2, w);
                    if (!KEYS) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float2 x = unpack2<T>(w[i]);
                            rounded[i & 3] = add_both(rounded[i & 3], pair_of(__float_as_uint(x.x), __float_as_uint(x.y)));
                        }
                    }
                }
                umma::tensor_memory_stored();
                umma::fence_before();
                __syncwarp();
                if (lane == 0) umma::barrier_arrive(umma::shared_address(&bars.ds));
                if (!KEYS) {
                    const uint64_t all = add_both(add_both(rounded[0], rounded[1]), add_both(rounded[2], rounded[3]));
                    row_sum += low_of(all) + high_of(all);
                }
                if (BIAS && KEYS && P.partials != nullptr) {
                    if (!near) {
                        uint64_t part[4] = {0, 0, 0, 0};
#pragma unroll
                        for (int c = 0; c < 64; c += 2) part[c / 2 & 3] = add_both(part[c / 2 & 3], pair_of(__float_as_uint(p[c]), __float_as_uint(p[c + 1])));
                        const uint64_t all = add_both(add_both(part[0], part[1]), add_both(part[2], part[3]));
                        far_sum += low_of(all) + high_of(all);
                    } else if constexpr (BIAS) {
                        // the warp's 32 rows x 64 columns have 95 diagonals, one distance each; diagonal 0's, and the buckets of all
                        const int zero = apart * kTile + col0 - (warp & 3) * 32 - 31;
                        const int low = M.tables.bucket[max(zero, 0)], high = zero + 94 < 0 ? low - 1 : M.tables.bucket[max(zero + 94, 0)];
                        float *mine = bucket_sums + warp * kMostBuckets;
                        if (high - low < kFewBuckets) {
                            // farther out a bucket is wide: its part of each row, as bits, one bucket after the other
                            for (int bucket = low; bucket <= high; ++bucket) {
                                // distance of column c: row_zero + c
                                const int row_zero = zero + 31 - lane;
                                const int from = M.tables.first[bucket] - row_zero;
                                const int to = bucket == P.bias.buckets - 1 ? 64 : M.tables.first[bucket + 1] - row_zero;
                                float part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                                for (int c = 0; c < 64; c += 32) {
                                    const uint32_t of = row < left ? below(to - c) & ~below(from - c) : 0u;
#pragma unroll
                                    for (int i = 0; i < 32; ++i)
                                        if (of >> i & 1) part[i & 3] += p[c + i];
                                }
                                float sum = (part[0] + part[1]) + (part[2] + part[3]);
#pragma unroll
                                for (int k = 16; k > 0; k /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, k);
                                if (lane == 0) mine[bucket] += sum;
                                __syncwarp();
                            }
                        } else {
                            // lane l sums the diagonals of numbers l, l + 32 and l + 64, read askew from shared memory some columns at a time (row r, column c: number
                            // c - r + 31).  Then equal buckets are neighbours, summed across lanes in a fixed order.
                            float *stripe = stripes + warp * kStripeFloats<HALVES>;
                            float sums[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
                            for (int c = 0; c < 64; c += kStripe<HALVES>) {
#pragma unroll
                                for (int i = 0; i < kStripe<HALVES>; ++i) stripe[lane * (kStripe<HALVES> + 1) + i] = row < left ? p[c + i] : 0.0f;
                                __syncwarp();
                                // column 32 k + c of lane l: row c - l - 1 has number l + 32 (k + 1), or where that is negative the
                                // row 32 further down number l + 32 k
                                const int k = c / 32;
#pragma unroll
                                for (int i = 0; i < kStripe<HALVES>; ++i) {
                                    const int r = (c & 31) + i - lane - 1;
                                    const float x = stripe[(r & 31) * (kStripe<HALVES> + 1) + i];
                                    if (r >= 0) sums[k + 1] += x;
                                    else sums[k] += x;
                                }
                                __syncwarp();
                            }
                            int bucket[3], before[3];
#pragma unroll
                            for (int n = 0; n < 3; ++n) {
                                const int d = zero + lane + n * 32;
                                bucket[n] = d < 0 || n == 2 && lane == 31 ? -1 : M.tables.bucket[d];
                                before[n] = __shfl_up_sync(0xffffffffu, bucket[n], 1);
                            }
#pragma unroll
                            for (int k = 1; k < 32; k *= 2)
#pragma unroll
                                for (int n = 0; n < 3; ++n) {
                                    const float theirs = __shfl_down_sync(0xffffffffu, sums[n], k);
                                    const int its = __shfl_down_sync(0xffffffffu, bucket[n], k);
                                    if (lane + k < 32 && its == bucket[n]) sums[n] += theirs;
                                }
#pragma unroll
                            for (int n = 0; n < 3; ++n) {
                                if (bucket[n] >= 0 && (lane == 0 || before[n] != bucket[n])) mine[bucket[n]] += sums[n];
                                __syncwarp();
                            }
                        }
                    }
                }
                if (BIAS && KEYS && P.partials != nullptr && apart + 1 == meets) {
                    // the sums of this query head
                    far_sum = row < left ? far_sum : 0.0f;
#pragma unroll
                    for (int d = 16; d > 0; d /= 2) far_sum += __shfl_xor_sync(0xffffffffu, far_sum, d);
                    if (lane == 0) bucket_sums[warp * kMostBuckets + P.bias.buckets - 1] += far_sum;
                    far_sum = 0.0f;
                    barrier_named(1, kSoftmaxThreads);
                    if (threadIdx.x < P.bias.buckets) {
                        float sum = 0.0f;
                        for (int of = 0; of < 8; ++of) {
                            sum += bucket_sums[of * kMostBuckets + threadIdx.x];
                            bucket_sums[of * kMostBuckets + threadIdx.x] = 0.0f;
                        }
                        P.partials[((long long)item.slot * P.heads + q_head) * P.bias.buckets + threadIdx.x] = !ok || *failed ? NAN : sum / unit;
                    }
                    barrier_named(1, kSoftmaxThreads);                          // the next sums start from zero
                }
                if (++apart == meets) {
                    apart = 0;
                    ++q_head;
                }
            }
            if (!KEYS) {
                row_sum = both_halves(row_sum);
                if (half == 0 && row < left) {
                    const long long at = (long long)head * P.tokens + first + row;
                    P.delta[at] = rounds > 1 ? P.delta[at] + row_sum / unit : -row_delta / unit_p;
                }
            }
            ok = ok && wait_all(&bars.sums, chains++ & 1, failed);
            umma::fence_after();
            if (threadIdx.x < 2) M.dirty[(n & 1) ^ 1][threadIdx.x] = 0;           // read by all in the work before
            barrier_named(1, kSoftmaxThreads);
            const bool gone = !ok || *failed;
            // half of the columns of each sum
            const int begin = half * 32 * HALVES, end = min(begin + 32 * HALVES, P.dim);
            int unclean = *(volatile int *)&M.dirty[n & 1][0] | *(volatile int *)&M.dirty[n & 1][1] << 1;
            if (KEYS && P.split) {
                // sums to this CTA's room; the last CTA of the key head reads them all, in the order of the heads
                for (int which = 0; which < 2; ++which)
                    add_to_room(room_of(P.fold, blockIdx.x * 2 + which, row), (which ? sum1_at : sum0_at) + lanes - col0, begin, end, 1.0f, rounds > kChain);
                __threadfence();
                barrier_named(1, kSoftmaxThreads);
                const int at = item.slot * (int)divide(P.heads, P.by_group) + head;
                if (threadIdx.x == 0) {
                    if (gone) unclean |= 4;
                    if (unclean != 0) atomicOr(P.unclean + at, unclean);
                    __threadfence();
                    M.last = atomicAdd(P.arrived + at, 1) == P.group - 1;
                    __threadfence();
                    M.unclean = *(volatile int *)(P.unclean + at);
                }
                barrier_named(1, kSoftmaxThreads);
                unclean = M.unclean;
                if (!M.last) continue;                                          // its only work
            }
#pragma unroll
            for (int which = 0; which < (KEYS ? 2 : 1); ++which) {
                const bool poisoned = unclean >> which & 1;
                const Heads &O = !KEYS ? P.dq : which ? P.dv : P.dk;
                if (O.p == nullptr) continue;
                const float times = gone || unclean & 4 ? NAN : which ? (kBf16 ? 1.0f : 0x1p-14f) : P.scale / unit;
                uint16_t *out = (uint16_t *)O.p + (long long)(first + (warp & 3) * 32) * O.token + head * O.head;
                for (int c = begin; c < end; c += 32)
                    put_rows<T>((which ? sum1_at : sum0_at) + lanes - col0, times, out, O.token, c, P.dim, left - (warp & 3) * 32, [&](float *x) {
                        if (KEYS && P.split) {
                            const int cta = (int)blockIdx.x - (w.head - head * P.group);                // of the first head; work i is CTA i's
#pragma unroll
                            for (int i = 0; i < 32; ++i) x[i] = 0.0f;
#pragma unroll 1
                            for (int g = 0; g < P.group; ++g) {
                                const float *from = room_of(P.fold, (cta + g) * 2 + which, row);
#pragma unroll
                                for (int i = 0; i < 32; ++i)
                                    if (c + i < end) x[i] += __ldcg(from + (c + i) * kTile);
                            }
#pragma unroll
                            for (int i = 0; i < 32; ++i) x[i] *= times;
                        } else if (rounds > kChain) {
                            const float *folded = room_of(P.fold, blockIdx.x * 2 + which, row);
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (c + i < end) x[i] = __fmaf_rn(folded[(c + i) * kTile], times, x[i]);
                        }
                        if (!KEYS) {
                            // what the sum of the row's ds is off zero by, times the mean key
                            const float off = -row_sum * times * (kBf16 ? 1.0f : 0x1p-14f);
                            const float *folded = room_of(P.fold, blockIdx.x * 2 + 1, row);
                            uint32_t u[32];
                            umma::tensor_memory_load(sum1_at + lanes - col0 + c, u);
                            umma::tensor_memory_loaded<32>(u);
#pragma unroll
                            for (int i = 0; i < 32; ++i) {
                                const float mean = __uint_as_float(u[i]) + (rounds > kChain && c + i < end ? folded[(c + i) * kTile] : 0.0f);
                                x[i] = __fmaf_rn(mean, off, x[i]);
                            }
                        }
                        if (!poisoned || row >= left) return;
                        // !KEYS: the keys of this tile up to the query; KEYS: queries (do) of this tile from the key on, all heads
                        for (int g = 0; g < (KEYS ? P.group : 1); ++g) {
                            const Heads &B = !KEYS ? P.k : which ? P.grad : P.q;
                            const uint16_t *b = (const uint16_t *)B.p + (long long)first * B.token + (KEYS ? head * P.group + g : kv_of(head)) * B.head;
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (c + i < end) x[i] += taken_away<T>(b + c + i, B.token, KEYS ? row : 0, KEYS ? min(left, kTile) : row + 1);
                        }
                    });
            }
            ++n;
        }
    }
}

template <class T, int HALVES, bool KEYS>
__device__ __noinline__ void backward_part_with_levels(const CUtensorMap &map_a0, const CUtensorMap &map_a1, const CUtensorMap &map_b0, const CUtensorMap &map_b1,
                                                       const BackwardParams &P, BackwardShared<true> &M, uint8_t *tiles, uint32_t tensor_base, float unit,
                                                       volatile int *failed)
{
    backward_part<T, HALVES, KEYS, true, true>(map_a0, map_a1, map_b0, map_b1, P, M, tiles, tensor_base, unit, failed);
}

template <class T, int HALVES, bool BIAS>
__global__ void __launch_bounds__(kBackwardThreads, 1)
psops_attention_backward_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                                const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_grad,
                                const __grid_constant__ BackwardParams P)
{
    extern __shared__ uint8_t raw[];
    __shared__ BackwardShared<BIAS> shared;
    __shared__ uint32_t tensor_base_slot;
    __shared__ int failed_slot;
    __shared__ float2 most[kBackwardThreads / 32];

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t *tiles = raw + (((umma::shared_address(raw) + 1023u) & ~1023u) - umma::shared_address(raw));
    if (threadIdx.x == 0) {
        failed_slot = 0;
        umma::prefetch_map(&map_q);
        umma::prefetch_map(&map_k);
        umma::prefetch_map(&map_v);
        umma::prefetch_map(&map_grad);
    }
    if (warp == 9) umma::tensor_columns_take<512>(umma::shared_address(&tensor_base_slot));
    __syncthreads();                                                        // it has them before the next kernel may come
    umma::after_the_kernel_before();
    float unit = 1.0f;                                                      // of ds
    if (__is_same(T, __half)) {
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
    if (__is_same(T, __half)) {
        float2 m = make_float2(0.0f, 0.0f);
        for (int w = 0; w < kBackwardThreads / 32; ++w) m = make_float2(fmaxf(m.x, most[w].x), fmaxf(m.y, most[w].y));
        const float bound = 2.0f * sqrtf(m.x) * sqrtf(m.y);                 // |ds| <= p (|dp| + |delta|)
        if (bound > 0.0f && bound < INFINITY) {
            int e;
            frexpf(bound, &e);
            unit = ldexpf(1.0f, min(max(14 - e, -100), 100));
        }
    }
    const uint32_t tensor_base = tensor_base_slot;
    bool levels = false;
    if constexpr (BIAS) {
        levels = *P.levels != 0;
        if (levels) {
            if (P.keys) backward_part_with_levels<T, HALVES, true>(map_k, map_v, map_q, map_grad, P, shared, tiles, tensor_base, unit, &failed_slot);
            else backward_part_with_levels<T, HALVES, false>(map_q, map_grad, map_k, map_v, P, shared, tiles, tensor_base, unit, &failed_slot);
        }
    }
    if (!levels) {
        if (P.keys) backward_part<T, HALVES, true, BIAS, false>(map_k, map_v, map_q, map_grad, P, shared, tiles, tensor_base, unit, &failed_slot);
        else backward_part<T, HALVES, false, BIAS, false>(map_q, map_grad, map_k, map_v, P, shared, tiles, tensor_base, unit, &failed_slot);
    }
    __syncwarp();
    umma::fence_before();
    __syncthreads();
    umma::fence_after();
    if (warp == 9) umma::tensor_columns_give<512>(tensor_base);
    if (!P.keys || P.join.ticket == nullptr) return;
    // few sums: the CTA that is done last joins them
    __shared__ int last;
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicAdd(P.join.ticket, 1) == (int)gridDim.x - 1;
        __threadfence();
    }
    __syncthreads();
    if (last)
        for (int at = threadIdx.x; at < P.join.heads * P.join.buckets; at += kBackwardThreads)
            put_dbias<T>(P.join, at, sum_of_slots(P.join, at, 0, 1));
}

// dbias: the slots of all tiles joined in their order, in double.
template <class T>
__global__ void __launch_bounds__(32 * kJoinParts) psops_attention_join_kernel(const JoinParams P)
{
    __shared__ double sums[kJoinParts][32];
    umma::after_the_kernel_before();
    const int per_slot = P.heads * P.buckets, at = blockIdx.x * 32 + (threadIdx.x & 31), part = threadIdx.x >> 5;
    double sum = at < per_slot ? sum_of_slots(P, at, part, kJoinParts) : 0.0;
    sums[part][threadIdx.x & 31] = sum;
    __syncthreads();
    if (part != 0 || at >= per_slot) return;
    for (int p = 1; p < kJoinParts; ++p) sum += sums[p][threadIdx.x];
    put_dbias<T>(P, at, sum);
}

} // namespace psops_attention_k
