// psops_keep_kernels.cuh -- activations kept in 8 bits for the backward pass.
//
// A row's blocks of 128 elements share a scale: s = top / 127 with top the largest
// magnitude, code = x / s rounded to the nearest, ties away from zero.
// All of it is bound by memory, and close to it by instructions: a warp does four
// blocks at a time (two where rows are not aligned to 8 bytes).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <cstring>

#include "psops_umma.cuh"

namespace psops_keep_k {

constexpr int kBlock = 128;
constexpr int kThreads = 256;
constexpr int kPitch = 16;                       // rows of codes begin on multiples of it
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kGeluA = 1.5957691216057308f, kGeluB = 0.044715f;     // 2 sqrt(2 / pi)

// Which block of which row: division by the blocks of a row, for numbers below 2^31.
struct Blocks {
    uint32_t count;                              // in all
    uint32_t of_row;
    uint32_t factor, shift;
};
__device__ __forceinline__ uint32_t row_of(const Blocks &B, uint32_t i) { return (uint32_t)(((uint64_t)i * B.factor) >> B.shift); }

template <class T> __device__ __forceinline__ float to_float(uint32_t low16);
template <> __device__ __forceinline__ float to_float<__half>(uint32_t u)
{
    const __half_raw r{(unsigned short)u};
    return __half2float(__half(r));
}
template <> __device__ __forceinline__ float to_float<__nv_bfloat16>(uint32_t u) { return __uint_as_float(u << 16); }
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

// The elements of a lane, as pairs.  W consecutive ones lie together, (lane +
// lanes k) W on: with W = 8 16-byte accesses (rows aligned to that), with W = 4, 2 or
// 1 (rows aligned to 8, 4 or 2 bytes) every access of a block's lanes is still to
// consecutive memory.  Eight lanes a block spread what a block costs over 16 elements
// each (6.4 TB/s of a copy's 6.5 where 16 lanes gave 4.9); with narrow accesses 16
// lanes touch fewer sectors at a time (odd widths: 3.4 TB/s, with eight 2.3).
template <int W> constexpr int kLanes = W >= 4 ? 8 : 16;
template <int W> constexpr int kOf = kBlock / kLanes<W>;
template <int W> struct Some { uint32_t pair[kOf<W> / 2]; };
template <int W> struct Codes { uint32_t four[kOf<W> / 4]; };

template <int BYTES> struct Word;
template <> struct Word<16> { using Type = uint4; };
template <> struct Word<8> { using Type = uint2; };
template <> struct Word<4> { using Type = uint32_t; };

// n: elements of the block that exist; WHOLE: all of them do.
template <int W, bool WHOLE>
__device__ __forceinline__ Some<W> load(const uint16_t *p, int lane, int n)
{
    Some<W> e{};
#pragma unroll
    for (int k = 0; k < kOf<W> / W; ++k) {
        const int at = (lane + kLanes<W> * k) * W;
        if constexpr (W > 1) {
            if (WHOLE || at + W <= n) {
                const auto w = __ldcs((const typename Word<2 * W>::Type *)(p + at));
                memcpy(&e.pair[k * W / 2], &w, 2 * W);
                continue;
            }
        }
        if (!WHOLE) {
#pragma unroll
            for (int i = 0; i < W; ++i)
                if (at + i < n) e.pair[(k * W + i) / 2] |= (uint32_t)__ldcs(p + at + i) << ((k * W + i) % 2 * 16);
        }
    }
    return e;
}
template <int W, bool WHOLE>
__device__ __forceinline__ void store(uint16_t *p, int lane, int n, const Some<W> &e)
{
#pragma unroll
    for (int k = 0; k < kOf<W> / W; ++k) {
        const int at = (lane + kLanes<W> * k) * W;
        if constexpr (W > 1) {
            if (WHOLE || at + W <= n) {
                typename Word<2 * W>::Type w;
                memcpy(&w, &e.pair[k * W / 2], 2 * W);
                *(typename Word<2 * W>::Type *)(p + at) = w;
                continue;
            }
        }
        if (!WHOLE) {
#pragma unroll
            for (int i = 0; i < W; ++i)
                if (at + i < n) p[at + i] = (uint16_t)(e.pair[(k * W + i) / 2] >> ((k * W + i) % 2 * 16));
        }
    }
}
// Codes of the same sixteen.  Rows of codes are padded to whole groups of 16, which
// a block's stores fill with zeros.
template <int W, bool WHOLE>
__device__ __forceinline__ void store_codes(uint8_t *p, int lane, int padded, const Codes<W> &c)
{
#pragma unroll
    for (int k = 0; k < kOf<W> / W; ++k) {
        const int at = (lane + kLanes<W> * k) * W;
        if (!WHOLE && at >= padded) continue;
        if constexpr (W == 8) *(uint2 *)(p + at) = make_uint2(c.four[2 * k], c.four[2 * k + 1]);
        if constexpr (W == 4) *(uint32_t *)(p + at) = c.four[k];
        if constexpr (W == 2) *(uint16_t *)(p + at) = (uint16_t)(c.four[k / 2] >> (k % 2 * 16));
        if constexpr (W == 1) p[at] = (uint8_t)(c.four[k / 4] >> (k % 4 * 8));
    }
}
template <int W, bool WHOLE>
__device__ __forceinline__ Codes<W> load_codes(const uint8_t *p, int lane, int padded)
{
    Codes<W> c{};
#pragma unroll
    for (int k = 0; k < kOf<W> / W; ++k) {
        const int at = (lane + kLanes<W> * k) * W;
        if (!WHOLE && at >= padded) continue;
        if constexpr (W == 8) {
            const uint2 w = __ldcs((const uint2 *)(p + at));
            c.four[2 * k] = w.x;
            c.four[2 * k + 1] = w.y;
        }
        if constexpr (W == 4) c.four[k] = __ldcs((const uint32_t *)(p + at));
        if constexpr (W == 2) c.four[k / 2] |= (uint32_t)__ldcs((const uint16_t *)(p + at)) << (k % 2 * 16);
        if constexpr (W == 1) c.four[k / 4] |= (uint32_t)__ldcs(p + at) << (k % 4 * 8);
    }
    return c;
}

// Codes and scale of a block, by its lanes.  Ties are exact quotients of two numbers
// of 11 bits at most by 127; any other quotient is 2^-19 off a tie or more.  The
// factor 1 + 2^-21 moves ties away from zero, since the reciprocal, its factor and
// their product are off by 2^-22 together at most, and moves nothing else across one.
// A block with a number that is not finite has the scale NaN; one below 2^-100 is zeros.
template <class T, int W>
__device__ __forceinline__ Codes<W> quantise(const Some<W> &e, float *scale)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kOf<W> / 2; ++i) top = __vmaxu2(top, e.pair[i] & 0x7fff7fffu);
#pragma unroll
    for (int d = kLanes<W> / 2; d > 0; d /= 2) top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, d));
    const uint32_t bits = max(top & 0xffffu, top >> 16);
    const float most = to_float<T>(bits);
    const bool some = most >= 0x1p-100f, finite = most < INFINITY;
    *scale = finite ? (some ? __fdiv_rn(most, 127.0f) : 0.0f) : NAN;
    float inverse;                           // 2^8 / top, within 2^-23, is a normal number for any top
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inverse) : "f"(most * 0x1p-8f));
    inverse = some ? inverse * (127.0f * 0x1p-8f * (1.0f + 0x1p-21f)) : 0.0f;
    Codes<W> c;
#pragma unroll
    for (int i = 0; i < kOf<W> / 4; ++i) {
        const float2 x = unpack2<T>(e.pair[2 * i]), y = unpack2<T>(e.pair[2 * i + 1]);
        // the sum's low byte is the nearest whole number
        const uint32_t code[4] = {__float_as_uint(__fmaf_rn(x.x, inverse, 12582912.0f)), __float_as_uint(__fmaf_rn(x.y, inverse, 12582912.0f)),
                                  __float_as_uint(__fmaf_rn(y.x, inverse, 12582912.0f)), __float_as_uint(__fmaf_rn(y.y, inverse, 12582912.0f))};
        c.four[i] = __byte_perm(__byte_perm(code[0], code[1], 0x0040), __byte_perm(code[2], code[3], 0x0040), 0x5410);
        if (!finite) c.four[i] = 0;
    }
    return c;
}
template <int W>
__device__ __forceinline__ void values(const Codes<W> &c, float scale, float *x)
{
#pragma unroll
    for (int h = 0; h < kOf<W> / 4; ++h) {
        const uint32_t w = c.four[h] ^ 0x80808080u;                         // code + 128
#pragma unroll
        for (int i = 0; i < 4; ++i)
            x[4 * h + i] = (__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7440 + i)) - 8388736.0f) * scale;
    }
}

// ---- the activation ----------------------------------------------------------
constexpr int kRelu = 0, kSilu = 1, kGelu = 2;

__device__ __forceinline__ float sigmoid(float z)
{
    float e, s;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -kLog2e));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.0f + e));
    return s;
}
// f(a), and its derivative where asked for
template <int KIND, bool SLOPE>
__device__ __forceinline__ float activation(float a, float *slope)
{
    if (KIND == kRelu) {
        if (SLOPE) *slope = a <= 0.0f ? 0.0f : a > 0.0f ? 1.0f : a;
        return a <= 0.0f ? 0.0f : a;
    }
    const float square = a * a;
    const float z = KIND == kSilu ? a : a * __fmaf_rn(square, kGeluA * kGeluB, kGeluA);
    const float s = sigmoid(z);
    if (SLOPE) {
        // far out z' overflows where s (1 - s) has long been zero
        const float bend = s * (1.0f - s);
        const float dz = KIND == kSilu ? 1.0f : __fmaf_rn(square, 3.0f * kGeluA * kGeluB, kGeluA);
        *slope = bend == 0.0f ? s : __fmaf_rn(a * bend, dz, s);
    }
    return a * s;
}

// ---- kernels -------------------------------------------------------------------
struct KeepParams {
    Blocks blocks;
    int cols;
    const uint16_t *x[2];                        // pack: x; forward: a, b; unpack: -; backward: dy
    long long x_ld[2];
    uint16_t *y[3];                              // unpack: x; forward: y; backward: da, db, y (the last two may be NULL)
    long long y_ld[3];
    uint8_t *codes[2];
    float *scales[2];
};
constexpr int kPack = 0, kUnpack = 1, kForward = 2, kBackward = 3;
template <int JOB, bool WHOLE> constexpr int kTimes = JOB == kPack || JOB == kUnpack || (JOB == kBackward && WHOLE) ? 2 : 1;

// `GATED` doubles the inputs.  A warp has a few blocks, U times over.  U: what kept
// most bytes under way without costing warps their registers.
template <class T, int JOB, int KIND, bool GATED, int W, bool WHOLE>
__global__ void __launch_bounds__(kThreads) psops_keep_kernel(const KeepParams P)
{
    constexpr int N = GATED ? 2 : 1;
    constexpr int U = kTimes<JOB, WHOLE>;
    constexpr int kOfWarp = 32 / kLanes<W>;
    umma::after_the_kernel_before();
    const int lane = threadIdx.x % kLanes<W>;
    const long long pitch = (P.cols + kPitch - 1) / kPitch * kPitch;
    const uint32_t step = gridDim.x * (kThreads / kLanes<W>) * U;
    // whole warps go round together: all lanes take part in every shuffle; what a warp does at a time lies together
    for (uint32_t first = (blockIdx.x * (kThreads / 32) + threadIdx.x / 32) * kOfWarp * U; first < P.blocks.count; first += step) {
        uint32_t row[U];
        int col[U], n[U];
        Some<W> in[U][N];
        Codes<W> code[U][N];
        float scale[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t i = first + u * kOfWarp + threadIdx.x % 32 / kLanes<W>;
            const bool there = i < P.blocks.count;
            row[u] = there ? row_of(P.blocks, i) : 0;
            const uint32_t of = there ? i - row[u] * P.blocks.of_row : 0;
            col[u] = (int)of * kBlock;
            n[u] = there ? (WHOLE ? kBlock : min(P.cols - col[u], kBlock)) : 0;
            if (JOB != kUnpack) {
#pragma unroll
                for (int t = 0; t < (JOB == kForward ? N : 1); ++t)
                    in[u][t] = load<W, WHOLE>(P.x[t] + row[u] * P.x_ld[t] + col[u], lane, n[u]);
            }
            if (JOB == kUnpack || JOB == kBackward) {
#pragma unroll
                for (int t = 0; t < N; ++t) {
                    code[u][t] = load_codes<W, WHOLE>(P.codes[t] + row[u] * pitch + col[u], lane, n[u]);
                    scale[u][t] = __ldcs(P.scales[t] + (long long)row[u] * P.blocks.of_row + of);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool there = n[u] > 0;
            Codes<W> kept[N];
            float s[N];
            if (JOB == kPack || JOB == kForward) {
#pragma unroll
                for (int t = 0; t < N; ++t) kept[t] = quantise<T, W>(in[u][t], &s[t]);
            }
            if (!there) continue;
            if (JOB == kPack || JOB == kForward) {
                const int padded = (n[u] + kPitch - 1) / kPitch * kPitch;
#pragma unroll
                for (int t = 0; t < N; ++t) {
                    store_codes<W, WHOLE>(P.codes[t] + row[u] * pitch + col[u], lane, padded, kept[t]);
                    if (lane == 0) P.scales[t][(long long)row[u] * P.blocks.of_row + col[u] / kBlock] = s[t];
                }
            }
            if (JOB == kForward) {
                Some<W> y;
#pragma unroll
                for (int i = 0; i < kOf<W> / 2; ++i) {
                    const float2 a = unpack2<T>(in[u][0].pair[i]);
                    float2 f = make_float2(activation<KIND, false>(a.x, nullptr), activation<KIND, false>(a.y, nullptr));
                    if (GATED) {
                        const float2 b = unpack2<T>(in[u][N - 1].pair[i]);
                        f = make_float2(f.x * b.x, f.y * b.y);
                    }
                    y.pair[i] = pack2<T>(f.x, f.y);
                }
                store<W, WHOLE>(P.y[0] + row[u] * P.y_ld[0] + col[u], lane, n[u], y);
            }
            if (JOB == kUnpack) {
                float x[kOf<W>];
                values<W>(code[u][0], scale[u][0], x);
                Some<W> y;
#pragma unroll
                for (int i = 0; i < kOf<W> / 2; ++i) y.pair[i] = pack2<T>(x[2 * i], x[2 * i + 1]);
                store<W, WHOLE>(P.y[0] + row[u] * P.y_ld[0] + col[u], lane, n[u], y);
            }
            if (JOB == kBackward) {
                float a[kOf<W>], b[kOf<W>];
                values<W>(code[u][0], scale[u][0], a);
                if (GATED) values<W>(code[u][N - 1], scale[u][N - 1], b);
                Some<W> da, db, y;
#pragma unroll
                for (int i = 0; i < kOf<W> / 2; ++i) {
                    const float2 g = unpack2<T>(in[u][0].pair[i]);
                    float2 slope, f;
                    f.x = activation<KIND, true>(a[2 * i], &slope.x);
                    f.y = activation<KIND, true>(a[2 * i + 1], &slope.y);
                    if (GATED) {
                        db.pair[i] = pack2<T>(g.x * f.x, g.y * f.y);
                        slope = make_float2(slope.x * b[2 * i], slope.y * b[2 * i + 1]);
                        f = make_float2(f.x * b[2 * i], f.y * b[2 * i + 1]);
                    }
                    da.pair[i] = pack2<T>(g.x * slope.x, g.y * slope.y);
                    y.pair[i] = pack2<T>(f.x, f.y);
                }
                if (P.y[0] != nullptr) store<W, WHOLE>(P.y[0] + row[u] * P.y_ld[0] + col[u], lane, n[u], da);
                if (GATED && P.y[1] != nullptr) store<W, WHOLE>(P.y[1] + row[u] * P.y_ld[1] + col[u], lane, n[u], db);
                if (P.y[2] != nullptr) store<W, WHOLE>(P.y[2] + row[u] * P.y_ld[2] + col[u], lane, n[u], y);
            }
        }
    }
}

} // namespace psops_keep_k
