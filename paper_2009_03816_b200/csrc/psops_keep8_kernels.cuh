// psops_keep8_kernels.cuh -- activations kept in 8 bits for the backward pass.
//
// A row's blocks of 128 elements share a scale: s = top / 127 with top the largest
// magnitude, code = x / s rounded to the nearest, ties away from zero.
// All of it is bound by memory: a warp does two blocks at a time, 16 lanes with 8
// elements each, several blocks in flight.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <cstring>

#include "psops_umma.cuh"

namespace psops_keep8_k {

constexpr int kBlock = 128;
constexpr int kThreads = 256, kTeams = kThreads / 16;
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

// The eight elements of a lane, as four pairs.  W consecutive ones lie together,
// (lane + 16 k) W on: with W = 8 all of them (16-byte aligned rows), with W = 2 or 1
// (4-byte or 2-byte aligned ones) every access of 16 lanes is still to consecutive
// memory.
struct Eight { uint32_t pair[4]; };

template <int W>
__device__ __forceinline__ Eight load(const uint16_t *p, int lane, int n)
{
    Eight e{};
    if constexpr (W == 8) {
        const int at = lane * 8;
        if (at + 8 <= n) {
            const uint4 w = __ldcs((const uint4 *)(p + at));
            e = Eight{{w.x, w.y, w.z, w.w}};
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (at + i < n) e.pair[i / 2] |= (uint32_t)p[at + i] << (i % 2 * 16);
        }
    } else if constexpr (W == 2) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int at = (lane + 16 * k) * 2;
            if (at + 2 <= n) e.pair[k] = __ldcs((const uint32_t *)(p + at));
            else if (at < n) e.pair[k] = p[at];
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int at = lane + 16 * k;
            if (at < n) e.pair[k / 2] |= (uint32_t)__ldcs(p + at) << (k % 2 * 16);
        }
    }
    return e;
}
template <int W>
__device__ __forceinline__ void store(uint16_t *p, int lane, int n, const Eight &e)
{
    if constexpr (W == 8) {
        const int at = lane * 8;
        if (at + 8 <= n) {
            *(uint4 *)(p + at) = make_uint4(e.pair[0], e.pair[1], e.pair[2], e.pair[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (at + i < n) p[at + i] = (uint16_t)(e.pair[i / 2] >> (i % 2 * 16));
        }
    } else if constexpr (W == 2) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int at = (lane + 16 * k) * 2;
            if (at + 2 <= n) *(uint32_t *)(p + at) = e.pair[k];
            else if (at < n) p[at] = (uint16_t)e.pair[k];
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int at = lane + 16 * k;
            if (at < n) p[at] = (uint16_t)(e.pair[k / 2] >> (k % 2 * 16));
        }
    }
}
// Codes of the same eight: x is elements 0-3, y is 4-7.  Rows of codes are padded
// to whole groups of 16, which a block's stores fill with zeros.
template <int W>
__device__ __forceinline__ void store_codes(uint8_t *p, int lane, int padded, uint2 c)
{
    if constexpr (W == 8) {
        if (lane * 8 < padded) *(uint2 *)(p + lane * 8) = c;
    } else if constexpr (W == 2) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int at = (lane + 16 * k) * 2;
            if (at < padded) *(uint16_t *)(p + at) = (uint16_t)((k < 2 ? c.x : c.y) >> (k % 2 * 16));
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (lane + 16 * k < padded) p[lane + 16 * k] = (uint8_t)((k < 4 ? c.x : c.y) >> (k % 4 * 8));
    }
}
template <int W>
__device__ __forceinline__ uint2 load_codes(const uint8_t *p, int lane, int padded)
{
    uint2 c = make_uint2(0, 0);
    if constexpr (W == 8) {
        if (lane * 8 < padded) c = __ldcs((const uint2 *)(p + lane * 8));
    } else if constexpr (W == 2) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int at = (lane + 16 * k) * 2;
            if (at < padded) (k < 2 ? c.x : c.y) |= (uint32_t)__ldcs((const uint16_t *)(p + at)) << (k % 2 * 16);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (lane + 16 * k < padded) (k < 4 ? c.x : c.y) |= (uint32_t)__ldcs(p + lane + 16 * k) << (k % 4 * 8);
    }
    return c;
}

// Codes and scale of a block, 16 lanes.  Ties are exact quotients of two numbers
// of 11 bits at most by 127; any other quotient is 2^-19 off a tie or more, so the
// factor 1 + 2^-21 moves ties away from zero and nothing else across one.  A block
// with a number that is not finite has the scale NaN; one below 2^-100 is zeros.
template <class T>
__device__ __forceinline__ uint2 quantise(const Eight &e, float *scale)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = __vmaxu2(top, e.pair[i] & 0x7fff7fffu);
#pragma unroll
    for (int d = 8; d > 0; d /= 2) top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, d));
    const uint32_t bits = max(top & 0xffffu, top >> 16);
    const float most = to_float<T>(bits);
    const bool some = most >= 0x1p-100f, finite = most < INFINITY;
    *scale = finite ? (some ? __fdiv_rn(most, 127.0f) : 0.0f) : NAN;
    const float inverse = some && finite ? __fmul_rn(__fdiv_rn(127.0f, most), 1.0f + 0x1p-21f) : 0.0f;
    uint32_t code[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 x = unpack2<T>(e.pair[i]);
        // the sum's low byte is the nearest whole number
        code[2 * i] = __float_as_uint(__fmaf_rn(x.x, inverse, 12582912.0f));
        code[2 * i + 1] = __float_as_uint(__fmaf_rn(x.y, inverse, 12582912.0f));
    }
    uint2 c;
    c.x = __byte_perm(__byte_perm(code[0], code[1], 0x0040), __byte_perm(code[2], code[3], 0x0040), 0x5410);
    c.y = __byte_perm(__byte_perm(code[4], code[5], 0x0040), __byte_perm(code[6], code[7], 0x0040), 0x5410);
    return finite ? c : make_uint2(0, 0);
}
__device__ __forceinline__ void values(uint2 c, float scale, float *x)
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t w = (h ? c.y : c.x) ^ 0x80808080u;                  // code + 128
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

// `GATED` doubles the inputs.  U blocks of a team are in flight at a time.
template <class T, int JOB, int KIND, bool GATED, int W>
__global__ void __launch_bounds__(kThreads) psops_keep8_kernel(const KeepParams P)
{
    constexpr int N = GATED ? 2 : 1;
    constexpr int U = JOB == kPack || JOB == kUnpack ? 4 : 2;
    umma::after_the_kernel_before();
    const int lane = threadIdx.x & 15;
    const uint32_t teams = gridDim.x * kTeams;
    const long long pitch = (P.cols + kPitch - 1) / kPitch * kPitch;
    // whole warps go round together: both teams take part in every shuffle
    for (uint32_t first = blockIdx.x * kTeams + (threadIdx.x >> 5) * 2; first < P.blocks.count; first += teams * U) {
        uint32_t row[U];
        int col[U], n[U];
        Eight in[U][N];
        uint2 code[U][N];
        float scale[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t i = first + u * teams + (threadIdx.x >> 4 & 1);
            row[u] = row_of(P.blocks, i);
            col[u] = (int)(i - row[u] * P.blocks.of_row) * kBlock;
            n[u] = i < P.blocks.count ? min(P.cols - col[u], kBlock) : 0;
            if (n[u] == 0) row[u] = 0, col[u] = 0;
            if (JOB != kUnpack) {
#pragma unroll
                for (int t = 0; t < (JOB == kForward ? N : 1); ++t) in[u][t] = load<W>(P.x[t] + row[u] * P.x_ld[t] + col[u], lane, n[u]);
            }
            if (JOB == kUnpack || JOB == kBackward) {
#pragma unroll
                for (int t = 0; t < N; ++t) {
                    code[u][t] = load_codes<W>(P.codes[t] + row[u] * pitch + col[u], lane, n[u]);
                    scale[u][t] = n[u] > 0 ? __ldcs(P.scales[t] + (long long)row[u] * P.blocks.of_row + col[u] / kBlock) : 0.0f;
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int padded = (n[u] + kPitch - 1) / kPitch * kPitch;
            if (JOB == kPack || JOB == kForward) {
#pragma unroll
                for (int t = 0; t < N; ++t) {
                    float s;
                    const uint2 c = quantise<T>(in[u][t], &s);
                    if (n[u] > 0) {
                        store_codes<W>(P.codes[t] + row[u] * pitch + col[u], lane, padded, c);
                        if (lane == 0) P.scales[t][(long long)row[u] * P.blocks.of_row + col[u] / kBlock] = s;
                    }
                }
            }
            if (JOB == kForward) {
                Eight y;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 a = unpack2<T>(in[u][0].pair[i]);
                    float2 f = make_float2(activation<KIND, false>(a.x, nullptr), activation<KIND, false>(a.y, nullptr));
                    if (GATED) {
                        const float2 b = unpack2<T>(in[u][N - 1].pair[i]);
                        f = make_float2(f.x * b.x, f.y * b.y);
                    }
                    y.pair[i] = pack2<T>(f.x, f.y);
                }
                store<W>(P.y[0] + row[u] * P.y_ld[0] + col[u], lane, n[u], y);
            }
            if (JOB == kUnpack) {
                float x[8];
                values(code[u][0], scale[u][0], x);
                Eight y;
#pragma unroll
                for (int i = 0; i < 4; ++i) y.pair[i] = pack2<T>(x[2 * i], x[2 * i + 1]);
                store<W>(P.y[0] + row[u] * P.y_ld[0] + col[u], lane, n[u], y);
            }
            if (JOB == kBackward) {
                float a[8], b[8];
                values(code[u][0], scale[u][0], a);
                if (GATED) values(code[u][N - 1], scale[u][N - 1], b);
                Eight da, db, y;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
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
                if (P.y[0] != nullptr) store<W>(P.y[0] + row[u] * P.y_ld[0] + col[u], lane, n[u], da);
                if (GATED && P.y[1] != nullptr) store<W>(P.y[1] + row[u] * P.y_ld[1] + col[u], lane, n[u], db);
                if (P.y[2] != nullptr) store<W>(P.y[2] + row[u] * P.y_ld[2] + col[u], lane, n[u], y);
            }
        }
    }
}

} // namespace psops_keep8_k
