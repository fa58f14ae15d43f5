// psops_optim_kernels.cuh -- AdamW over many tensors and the 2-norm of many
// gradients (C entries: psops_optim.cu).
//
// Both are streaming passes over a list of tensors.  The list lies in device
// memory as one entry per tensor, and beside it a list of chunks (tensor, index
// of the chunk within it), so that one launch covers tensors of any size: a
// block takes chunks c, c + gridDim.x, ...
//
// Within a tensor a warp works on 256 consecutive elements at a time, eight per
// lane.  Where all arrays of a tensor are misaligned alike -- by the same
// number `lo` < 8 of elements against a group of eight -- their pointers are
// moved back by lo and the elements are numbered lo .. hi - 1; a group of eight
// that lies within [lo, hi) then moves in one access of 16 or 32 bytes, and
// only a tensor's first and last group go element by element.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "psops_umma.cuh"

namespace {

constexpr int kOptThreads = 256;
constexpr int kOptWarps = kOptThreads / 32;
constexpr int kGroup = 256;                     // elements of a warp's step, and of an 8-bit moment's scale

struct AdamwEntry {
    float *p;
    const void *g;
    void *copy, *m, *v;
    float *m_scale, *v_scale;
    long long lo, hi;
    double weight_decay;
    int vec;                                    // groups of eight are aligned in every array
    int pad_;
};

struct AdamwState {
    double pow1, pow2;                          // beta^t with t the number of the next step
    long long steps;                            // steps taken
    unsigned tickets;
};

struct AdamwParams {
    const AdamwEntry *entries;
    const uint2 *chunks;                        // {tensor, chunk within it}
    AdamwState *state;
    const float *scale;
    double lr, beta1, beta2;
    float b1, b1c, b2, b2c, eps;                // beta, 1 - beta
    unsigned n_chunks;
};

// Eight elements as they lie in memory, and as numbers.
template <class T> struct Eight { uint32_t w[2 * sizeof(T)]; };

__device__ __forceinline__ void load_eight(const void *p, uint32_t (&w)[8])
{
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p));
}
__device__ __forceinline__ void load_eight(const void *p, uint32_t (&w)[4])
{
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
}
__device__ __forceinline__ void load_eight(const void *p, uint32_t (&w)[2])
{
    asm volatile("ld.global.L1::no_allocate.v2.b32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
}
__device__ __forceinline__ void store_eight(float *p, const float (&x)[8])
{
    asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]),
                 "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7])
                 : "memory");
}
__device__ __forceinline__ float2 widen(const __half2 h) { return __half22float2(h); }
__device__ __forceinline__ float2 widen(const __nv_bfloat162 h) { return __bfloat1622float2(h); }
template <class T2>
__device__ __forceinline__ void widen_eight(const uint32_t (&w)[4], float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        T2 h;
        memcpy(&h, &w[i], 4);
        const float2 f = widen(h);
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ void numbers(const Eight<float> &e, float (&x)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(e.w[j]);
}
__device__ __forceinline__ void numbers(const Eight<__half> &e, float (&x)[8]) { widen_eight<__half2>(e.w, x); }
__device__ __forceinline__ void numbers(const Eight<__nv_bfloat16> &e, float (&x)[8]) { widen_eight<__nv_bfloat162>(e.w, x); }

__device__ __forceinline__ __half2 narrow2(const __half *, float a, float b) { return __floats2half2_rn(a, b); }
__device__ __forceinline__ __nv_bfloat162 narrow2(const __nv_bfloat16 *, float a, float b) { return __floats2bfloat162_rn(a, b); }
template <class T>
__device__ __forceinline__ void store_eight(T *p, const float (&x)[8])
{
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const auto h = narrow2((const T *)nullptr, x[2 * i], x[2 * i + 1]);
        memcpy(&w[i], &h, 4);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ float one_in(const float *p) { return *p; }
__device__ __forceinline__ float one_in(const __half *p) { return __half2float(*p); }
__device__ __forceinline__ float one_in(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ void one_out(float *p, float x) { *p = x; }
__device__ __forceinline__ void one_out(__half *p, float x) { *p = __float2half_rn(x); }
__device__ __forceinline__ void one_out(__nv_bfloat16 *p, float x) { *p = __float2bfloat16_rn(x); }

// 8-bit e4m3 numbers
struct Q8 { uint8_t b; };
__device__ __forceinline__ float2 q8_decode2(unsigned short two)
{
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
    return __half22float2(__half2(h));
}
__device__ __forceinline__ unsigned short q8_encode2(float a, float b)
{
    return (unsigned short)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ void numbers(const Eight<Q8> &e, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = q8_decode2((unsigned short)(e.w[i >> 1] >> (16 * (i & 1))));
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ void store_eight(Q8 *p, const float (&x)[8])
{
    unsigned w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        w[i] = (unsigned)q8_encode2(x[4 * i], x[4 * i + 1]) | ((unsigned)q8_encode2(x[4 * i + 2], x[4 * i + 3]) << 16);
    *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
}
__device__ __forceinline__ float one_in(const Q8 *p) { return q8_decode2(p->b).x; }
__device__ __forceinline__ void one_out(Q8 *p, float x) { p->b = (uint8_t)q8_encode2(x, 0.0f); }

// The elements of one lane where they do not move as a group of eight: element
// first + j * stride for every bit j of the mask.  Strides are 1, or 32 where
// the arrays of the tensor are not aligned alike.
struct Lane {
    long long first;
    int stride;
    unsigned mask;
};

__device__ __forceinline__ Lane lane_of(long long group, int lane, bool vec, long long lo, long long hi)
{
    Lane L;
    L.first = vec ? group + lane * 8 : group + lane;
    L.stride = vec ? 1 : 32;
    L.mask = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const long long i = L.first + j * L.stride;
        L.mask |= (i >= lo && i < hi) ? 1u << j : 0u;
    }
    return L;
}

template <class T>
__device__ __forceinline__ void load_lane(const T *base, const Lane &L, float (&x)[8])
{
    const T *at = base + L.first;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (L.mask >> j & 1u) ? one_in(at + j * L.stride) : 0.0f;
}
template <class T>
__device__ __forceinline__ void store_lane(T *base, const Lane &L, const float (&x)[8])
{
    T *at = base + L.first;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (L.mask >> j & 1u) one_out(at + j * L.stride, x[j]);
}

__device__ __forceinline__ float max_or_nan(float a, float b)
{
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}
// Largest magnitude of a warp's 256 values, NaN if there is one.  Across the
// lanes magnitudes are compared as bit patterns, which order alike, with NaN
// above everything.
__device__ __forceinline__ float top_of(const float (&x)[8])
{
    float t = fabsf(x[0]);
#pragma unroll
    for (int j = 1; j < 8; ++j) t = max_or_nan(t, fabsf(x[j]));
    return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(t) & 0x7fffffffu));
}

template <int BITS> struct MomentOf;
template <> struct MomentOf<32> { using T = float; };
template <> struct MomentOf<8> { using T = Q8; };

// What a step multiplies with, the same for every element of a tensor.
struct AdamwFactors { float scale, rate, spread, decay; };

// The step for eight elements of a lane: weights and moments in, weights and
// moments out; for 8 bits the moments come out as they are kept, and the
// block's two scales beside them.
template <int BITS>
__device__ __forceinline__ void adamw_eight(const AdamwParams &P, const AdamwFactors &F, float (&p)[8], const float (&g_in)[8],
                                            float (&m_io)[8], float (&v_io)[8], float &m_scale, float &v_scale)
{
    float root[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float g = __fmul_rn(g_in[j], F.scale);
        float m = m_io[j], v = v_io[j];
        if (BITS == 8) {
            m = __fmul_rn(m, m_scale);
            v = __fmul_rn(v, v_scale);
            v = __fmul_rn(v, v);
        }
        m = __fadd_rn(__fmul_rn(m, P.b1), __fmul_rn(g, P.b1c));
        v = __fadd_rn(__fmul_rn(v, P.b2), __fmul_rn(__fmul_rn(g, g), P.b2c));
        root[j] = __fsqrt_rn(v);
        const float step = __fdiv_rn(__fmul_rn(m, F.rate), __fadd_rn(__fmul_rn(root[j], F.spread), P.eps));
        p[j] = __fsub_rn(__fmul_rn(p[j], F.decay), step);
        m_io[j] = m;
        v_io[j] = v;
    }
    if (BITS == 8) {
        // elements that do not exist came in as zeros and stay zeros: they do not raise a block's top
        const float tm = top_of(m_io), tr = top_of(root);
        const bool some_m = tm >= 0x1p-100f, some_r = tr >= 0x1p-100f;
        // four quotients, one division: every lane does one of them
        const int lane = threadIdx.x & 31;
        const float mine = lane & 2 ? tr : tm;
        const float quotient = __fdiv_rn(lane & 1 ? mine : 448.0f, lane & 1 ? 448.0f : mine);
        const float inv_m = some_m ? __shfl_sync(0xffffffffu, quotient, 0) : 0.0f;
        const float new_m = some_m ? __shfl_sync(0xffffffffu, quotient, 1) : 0.0f;
        const float inv_r = some_r ? __shfl_sync(0xffffffffu, quotient, 2) : 0.0f;
        const float new_r = some_r ? __shfl_sync(0xffffffffu, quotient, 3) : 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            m_io[j] = __fmul_rn(m_io[j], inv_m);
            const float r = __fmul_rn(root[j], inv_r);
            v_io[j] = root[j] > 0.0f ? fmaxf(r, 0x1p-9f) : r;         // 2^-9: the smallest e4m3 number
        }
        m_scale = new_m;
        v_scale = new_r;
    }
}

// A whole, aligned group.
template <int BITS, class G, class C>
__device__ __forceinline__ void adamw_whole(const AdamwEntry *E, long long group, int lane, const AdamwParams &P, const AdamwFactors &F)
{
    using M = typename MomentOf<BITS>::T;
    using CT = typename std::conditional<__is_same(C, void), __half, C>::type;
    const long long at = group + lane * 8;
    Eight<float> p8;
    Eight<G> g8;
    Eight<M> m8, v8;
    float p[8], g[8], m[8], v[8], m_scale = 0.0f, v_scale = 0.0f;
    load_eight(E->p + at, p8.w);
    load_eight((const G *)E->g + at, g8.w);
    load_eight((const M *)E->m + at, m8.w);
    load_eight((const M *)E->v + at, v8.w);
    if (BITS == 8) {
        m_scale = E->m_scale[group / kGroup];
        v_scale = E->v_scale[group / kGroup];
    }
    numbers(p8, p);
    numbers(g8, g);
    numbers(m8, m);
    numbers(v8, v);
    adamw_eight<BITS>(P, F, p, g, m, v, m_scale, v_scale);
    store_eight(E->p + at, p);
    store_eight((M *)E->m + at, m);
    store_eight((M *)E->v + at, v);
    if (!__is_same(C, void) && E->copy != nullptr) store_eight((CT *)E->copy + at, p);
    if (BITS == 8 && lane == 0) {                 // the reductions in between have every lane past its reads
        E->m_scale[group / kGroup] = m_scale;
        E->v_scale[group / kGroup] = v_scale;
    }
}

// A group that is cut off by the tensor's ends, or of a tensor whose arrays are not aligned alike.
template <int BITS, class G, class C>
__device__ __noinline__ void adamw_broken(const AdamwEntry *E, long long group, int lane, const AdamwParams &P, const AdamwFactors F)
{
    using M = typename MomentOf<BITS>::T;
    using CT = typename std::conditional<__is_same(C, void), __half, C>::type;
    if (group >= E->hi) return;
    const Lane L = lane_of(group, lane, E->vec != 0, E->lo, E->hi);
    float p[8], g[8], m[8], v[8], m_scale = 0.0f, v_scale = 0.0f;
    load_lane(E->p, L, p);
    load_lane((const G *)E->g, L, g);
    load_lane((const M *)E->m, L, m);
    load_lane((const M *)E->v, L, v);
    if (BITS == 8) {
        m_scale = E->m_scale[group / kGroup];
        v_scale = E->v_scale[group / kGroup];
    }
    __syncwarp();                                 // every lane has the old scales before one writes the new ones
    adamw_eight<BITS>(P, F, p, g, m, v, m_scale, v_scale);
    store_lane(E->p, L, p);
    store_lane((M *)E->m, L, m);
    store_lane((M *)E->v, L, v);
    if (!__is_same(C, void) && E->copy != nullptr) store_lane((CT *)E->copy, L, p);
    if (BITS == 8 && lane == 0) {
        E->m_scale[group / kGroup] = m_scale;
        E->v_scale[group / kGroup] = v_scale;
    }
}

constexpr int kAdamwChunk = kOptWarps * kGroup;                     // elements: a group for each warp

// Blocks of an SM.  With 8-bit moments a group is some 70 instructions per
// element for 14 bytes, and more warps hide one another's latencies; with fp32
// moments fewer of them keep the streams of HBM longer.  Measured on 134 M
// elements, 2 / 3 / 4 / 5 blocks: 8 bits with bf16 gradients 549 / 424 / 386 /
// 383 us; fp32 572 / 594 / 616 / 617 us, but 204 M elements of 1,288 tensors
// 969 / 867 us with 2 / 3, and 11 M with bf16 gradients 61 / 56 us.
template <int BITS> constexpr int kAdamwBlocks = BITS == 8 ? 4 : 3;

// One step of AdamW (the formula is in psops.h).  What bounds it is HBM
// traffic: 28 bytes per element with fp32 moments and gradients (204 M elements
// of 1,288 tensors: 850 to 877 us, 6.5 to 6.7 TB/s, what a plain copy reaches);
// 14 to 16 with 8-bit moments and 16-bit gradients, where the instructions weigh
// as much (268 M of 291 tensors with bf16 copies: 797 to 839 us, 5.1 to 5.4 TB/s).  Keeping the next
// group's loads in registers under the arithmetic was slower (its registers cost
// more warps than the overlap gave: 473 us against 378 us for 134 M elements).
template <int BITS, class G, class C>
__global__ void __launch_bounds__(kOptThreads, kAdamwBlocks<BITS>) psops_adamw_kernel(const __grid_constant__ AdamwParams P)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    umma::after_the_kernel_before();
    AdamwFactors F;
    F.scale = P.scale != nullptr ? *P.scale : 1.0f;
    if (!(fabsf(F.scale) < INFINITY)) return;                       // skipped: nothing changes, t stays
    const double pow1 = P.state->pow1, pow2 = P.state->pow2;
    F.rate = (float)(P.lr * (1.0 / (1.0 - pow1)));
    F.spread = (float)(1.0 / sqrt(1.0 - pow2));
    for (unsigned c = blockIdx.x; c < P.n_chunks; c += gridDim.x) {
        const uint2 chunk = P.chunks[c];
        const AdamwEntry *E = P.entries + chunk.x;
        const long long group = (long long)chunk.y * kAdamwChunk + warp * kGroup;
        F.decay = (float)(1.0 - P.lr * E->weight_decay);
        if (E->vec != 0 && group >= E->lo && group + kGroup <= E->hi) adamw_whole<BITS, G, C>(E, group, lane, P, F);
        else adamw_broken<BITS, G, C>(E, group, lane, P, F);
    }
    // The block that comes last moves the state on to the next step: every
    // block has used the values it read by then.
    __syncthreads();
    if (threadIdx.x == 0 && atomicAdd(&P.state->tickets, 1u) == gridDim.x - 1) {
        P.state->pow1 = pow1 * P.beta1;
        P.state->pow2 = pow2 * P.beta2;
        P.state->steps += 1;
        P.state->tickets = 0;
    }
}

// ---------------------------------------------------------------------------
// 2-norm
// ---------------------------------------------------------------------------

struct NormEntry {
    const void *g;                              // moved back by lo elements, so that the address is a multiple of 32
    long long lo, hi;
};

struct NormParams {
    const NormEntry *entries;
    const uint2 *chunks;
    double *partials;                           // one per block
    unsigned *tickets;
    float *out;
    float max_norm;
    unsigned n_chunks;
};

template <class G> struct NormShape {
    static constexpr int kPer = 32 / (int)sizeof(G);                // elements of a 32-byte access
    static constexpr int kDeep = 4;                                 // accesses of a thread in flight
    static constexpr int kChunk = kOptThreads * kPer * kDeep;       // elements
};

__device__ __forceinline__ float sum_squares(const float *, const uint4 a, const uint4 b)
{
    const unsigned w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(__uint_as_float(w[i]), __uint_as_float(w[i]), s);
    return s;
}
template <class T2>
__device__ __forceinline__ float sum_squares_16(const uint4 a, const uint4 b)
{
    const unsigned w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        T2 h;
        memcpy(&h, &w[i], 4);
        const float2 f = widen(h);
        s = fmaf(f.x, f.x, s);
        s = fmaf(f.y, f.y, s);
    }
    return s;
}
__device__ __forceinline__ float sum_squares(const __half *, const uint4 a, const uint4 b) { return sum_squares_16<__half2>(a, b); }
__device__ __forceinline__ float sum_squares(const __nv_bfloat16 *, const uint4 a, const uint4 b) { return sum_squares_16<__nv_bfloat162>(a, b); }

__device__ __forceinline__ void load_32(const void *p, uint4 &a, uint4 &b)
{
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w)
                 : "l"(p));
}

// Sum over a block in a fixed order; the result is in thread 0.
__device__ __forceinline__ double block_sum(double x, double *shared)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = x;
    __syncthreads();
    double s = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < kOptWarps; ++w) s += shared[w];
    return s;
}

// Each block adds up the squares of its chunks; the block that draws the last
// ticket adds the blocks' sums, always in the same order, and writes the norm
// and the factor.  Bound by reading the gradients once.
template <class G>
__global__ void __launch_bounds__(kOptThreads) psops_gradnorm_kernel(const NormParams P)
{
    using S = NormShape<G>;
    __shared__ double shared[kOptWarps];
    __shared__ bool last;
    umma::after_the_kernel_before();
    double sum = 0.0;
    for (unsigned c = blockIdx.x; c < P.n_chunks; c += gridDim.x) {
        const uint2 chunk = P.chunks[c];
        const NormEntry E = P.entries[chunk.x];
        const G *g = (const G *)E.g;
        const long long first = (long long)chunk.y * S::kChunk + (long long)threadIdx.x * S::kPer;
        uint4 a[S::kDeep], b[S::kDeep];
#pragma unroll
        for (int i = 0; i < S::kDeep; ++i) {
            const long long at = first + (long long)i * kOptThreads * S::kPer;
            if (at >= E.lo && at + S::kPer <= E.hi) load_32(g + at, a[i], b[i]);
        }
#pragma unroll
        for (int i = 0; i < S::kDeep; ++i) {
            const long long at = first + (long long)i * kOptThreads * S::kPer;
            if (at >= E.lo && at + S::kPer <= E.hi) {
                sum += (double)sum_squares((const G *)nullptr, a[i], b[i]);
            } else {
                float s = 0.0f;
                for (int j = 0; j < S::kPer; ++j)
                    if (at + j >= E.lo && at + j < E.hi) {
                        const float x = one_in(g + at + j);
                        s = fmaf(x, x, s);
                    }
                sum += (double)s;
            }
        }
    }
    const double mine = block_sum(sum, shared);
    if (threadIdx.x == 0) {
        P.partials[blockIdx.x] = mine;
        __threadfence();
        last = atomicAdd(P.tickets, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double total = 0.0;
    for (unsigned b = threadIdx.x; b < gridDim.x; b += kOptThreads) total += __ldcg(P.partials + b);
    total = block_sum(total, shared);
    if (threadIdx.x == 0) {
        const float norm = (float)sqrt(total);
        const bool finite = norm < INFINITY;
        P.out[0] = norm;
        P.out[1] = finite ? fminf(1.0f, P.max_norm / (norm + 1e-6f)) : NAN;
        *P.tickets = 0;
    }
}

} // namespace
