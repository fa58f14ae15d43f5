// psops_keep.cu -- C entries of activations kept in 8 bits.
#include "psops.h"

#include <cuda_runtime.h>

#include <algorithm>
#include <new>

#include "psops_host.cuh"
#include "psops_keep_kernels.cuh"

using namespace psops_keep_k;
using psops_host::ceil_div;
using psops_host::launch;
using psops_host::OnDevice;

struct psops_keep : psops_host::Base {};

namespace {

constexpr int64_t kCtasOfSm = 64;                            // dealt out as they end, beyond what runs at once
constexpr int64_t kMostBlocksOfRows = (int64_t)1 << 30;      // blocks of 128 in a call, so that numbers of blocks stay below 2^31

using Kernel = void (*)(const KeepParams);

template <class T, int JOB, int KIND, bool GATED>
Kernel by_width(int width)
{
    return width == 16  ? psops_keep_kernel<T, JOB, KIND, GATED, 8, true>
           : width == 8 ? psops_keep_kernel<T, JOB, KIND, GATED, 8, false>
           : width == 4 ? psops_keep_kernel<T, JOB, KIND, GATED, 4, false>
           : width == 2 ? psops_keep_kernel<T, JOB, KIND, GATED, 2, false> : psops_keep_kernel<T, JOB, KIND, GATED, 1, false>;
}
template <class T, int JOB>
Kernel by_kind(int kind, bool gated, int width)
{
    if (kind == PSOPS_RELU) return gated ? by_width<T, JOB, kRelu, true>(width) : by_width<T, JOB, kRelu, false>(width);
    if (kind == PSOPS_SILU) return gated ? by_width<T, JOB, kSilu, true>(width) : by_width<T, JOB, kSilu, false>(width);
    return gated ? by_width<T, JOB, kGelu, true>(width) : by_width<T, JOB, kGelu, false>(width);
}
template <class T>
Kernel kernel_of(int job, int kind, bool gated, int width)
{
    return job == kPack     ? by_width<T, kPack, 0, false>(width)
           : job == kUnpack ? by_width<T, kUnpack, 0, false>(width)
           : job == kForward ? by_kind<T, kForward>(kind, gated, width) : by_kind<T, kBackward>(kind, gated, width);
}

int run(psops_keep *k, int job, int kind, int32_t type, int64_t rows, int64_t cols, bool gated, KeepParams P)
{
    P.cols = (int)cols;
    const uint32_t of_row = (uint32_t)ceil_div(cols, kBlock);
    int shift = 0;
    while (((uint32_t)1 << shift) < of_row) ++shift;
    P.blocks = Blocks{(uint32_t)(rows * of_row), of_row, (uint32_t)((((uint64_t)1 << (31 + shift)) + of_row - 1) / of_row), (uint32_t)(31 + shift)};
    // the widest access that all rows allow
    int width = 8;
    auto look = [&](const void *p, int64_t ld) {
        if (p == nullptr) return;
        while (width > 1 && (((uintptr_t)p & (2 * width - 1)) || (rows > 1 && ld % width))) width /= 2;
    };
    for (int i = 0; i < 2; ++i) look(P.x[i], P.x_ld[i]);
    for (int i = 0; i < 3; ++i) look(P.y[i], P.y_ld[i]);
    if (width == 8 && cols % kBlock == 0) width = 16;            // and no block is short
    const int times = job == kPack ? kTimes<kPack, false> : job == kUnpack ? kTimes<kUnpack, false> : job == kForward ? kTimes<kForward, false>
                      : width == 16 ? kTimes<kBackward, true> : kTimes<kBackward, false>;
    const int64_t of_cta = kThreads / (width >= 4 ? kLanes<4> : kLanes<1>) * times;
    const int64_t grid = std::min<int64_t>(ceil_div(rows * of_row, of_cta), (int64_t)k->sms * kCtasOfSm);
    return launch(k, "psops_keep_kernel",
                  type == PSOPS_F16 ? kernel_of<__half>(job, kind, gated, width) : kernel_of<__nv_bfloat16>(job, kind, gated, width),
                  dim3((unsigned)grid), kThreads, 0, 1, P);
}

int check(const psops_keep *k, int32_t type, int64_t rows, int64_t cols)
{
    if (k == nullptr || (type != PSOPS_F16 && type != PSOPS_BF16) || rows < 0 || cols < 1 || cols > INT32_MAX - kBlock ||
        rows > kMostBlocksOfRows / ceil_div(cols, kBlock))
        return PSOPS_EINVAL;
    return PSOPS_OK;
}
int check_rows(const void *p, int64_t ld, int64_t rows, int64_t cols)
{
    if (rows > 0 && p == nullptr) return PSOPS_EINVAL;
    if ((rows > 1 && ld < cols) || ld > (int64_t)1 << 40) return PSOPS_EINVAL;
    return (uintptr_t)p & 1u ? PSOPS_EALIGN : PSOPS_OK;
}
int check_kept(const void *codes, const void *scales, int64_t rows)
{
    if (rows > 0 && (codes == nullptr || scales == nullptr)) return PSOPS_EINVAL;
    return ((uintptr_t)codes & 15u) || ((uintptr_t)scales & 3u) ? PSOPS_EALIGN : PSOPS_OK;
}

#define PSOPS_DO(call)                     \
    do {                                   \
        const int rc_ = (call);            \
        if (rc_ != PSOPS_OK) return rc_;   \
    } while (0)

} // namespace

extern "C" {

int psops_keep_create(psops_keep **out, void *cuda_stream)
{
    if (out == nullptr) return PSOPS_EINVAL;
    *out = nullptr;
    psops_keep *k = new (std::nothrow) psops_keep();
    if (k == nullptr) return PSOPS_ENOMEM;
    k->stream = (cudaStream_t)cuda_stream;
    int rc = psops_host::not_capturing(k);
    cudaError_t e = rc == PSOPS_OK ? cudaGetDevice(&k->device) : cudaSuccess;
    if (rc == PSOPS_OK && e == cudaSuccess) e = cudaDeviceGetAttribute(&k->sms, cudaDevAttrMultiProcessorCount, k->device);
    if (e != cudaSuccess) rc = PSOPS_ECUDA;
    if (rc != PSOPS_OK) {
        delete k;
        return rc;
    }
    *out = k;
    return PSOPS_OK;
}

int psops_keep_pack(psops_keep *k, int32_t type, int64_t rows, int64_t cols, const void *d_x, int64_t x_ld, void *d_codes, float *d_scales)
{
    PSOPS_DO(check(k, type, rows, cols));
    PSOPS_DO(check_rows(d_x, x_ld, rows, cols));
    PSOPS_DO(check_kept(d_codes, d_scales, rows));
    if (rows == 0) return PSOPS_OK;
    OnDevice guard(k);
    KeepParams P{};
    P.x[0] = (const uint16_t *)d_x; P.x_ld[0] = x_ld;
    P.codes[0] = (uint8_t *)d_codes; P.scales[0] = d_scales;
    return run(k, kPack, 0, type, rows, cols, false, P);
}

int psops_keep_unpack(psops_keep *k, int32_t type, int64_t rows, int64_t cols, const void *d_codes, const float *d_scales, void *d_x, int64_t x_ld)
{
    PSOPS_DO(check(k, type, rows, cols));
    PSOPS_DO(check_rows(d_x, x_ld, rows, cols));
    PSOPS_DO(check_kept(d_codes, d_scales, rows));
    if (rows == 0) return PSOPS_OK;
    OnDevice guard(k);
    KeepParams P{};
    P.codes[0] = (uint8_t *)d_codes; P.scales[0] = (float *)d_scales;
    P.y[0] = (uint16_t *)d_x; P.y_ld[0] = x_ld;
    return run(k, kUnpack, 0, type, rows, cols, false, P);
}

int psops_keep_activate(psops_keep *k, int32_t kind, int32_t type, int64_t rows, int64_t cols, const void *d_a, int64_t a_ld, const void *d_b,
                         int64_t b_ld, void *d_y, int64_t y_ld, void *d_a_codes, float *d_a_scales, void *d_b_codes, float *d_b_scales)
{
    PSOPS_DO(check(k, type, rows, cols));
    if (kind < PSOPS_RELU || kind > PSOPS_GELU) return PSOPS_EINVAL;
    PSOPS_DO(check_rows(d_a, a_ld, rows, cols));
    PSOPS_DO(check_rows(d_y, y_ld, rows, cols));
    PSOPS_DO(check_kept(d_a_codes, d_a_scales, rows));
    if (d_b != nullptr) {
        PSOPS_DO(check_rows(d_b, b_ld, rows, cols));
        PSOPS_DO(check_kept(d_b_codes, d_b_scales, rows));
    }
    if (rows == 0) return PSOPS_OK;
    OnDevice guard(k);
    KeepParams P{};
    P.x[0] = (const uint16_t *)d_a; P.x_ld[0] = a_ld;
    P.x[1] = (const uint16_t *)d_b; P.x_ld[1] = b_ld;
    P.y[0] = (uint16_t *)d_y; P.y_ld[0] = y_ld;
    P.codes[0] = (uint8_t *)d_a_codes; P.scales[0] = d_a_scales;
    P.codes[1] = (uint8_t *)d_b_codes; P.scales[1] = d_b_scales;
    return run(k, kForward, kind, type, rows, cols, d_b != nullptr, P);
}

int psops_keep_activate_backward(psops_keep *k, int32_t kind, int32_t type, int64_t rows, int64_t cols, const void *d_a_codes, const float *d_a_scales,
                                  const void *d_b_codes, const float *d_b_scales, const void *d_dy, int64_t dy_ld, void *d_da, int64_t da_ld,
                                  void *d_db, int64_t db_ld, void *d_y, int64_t y_ld)
{
    PSOPS_DO(check(k, type, rows, cols));
    if (kind < PSOPS_RELU || kind > PSOPS_GELU || (d_db != nullptr && d_b_codes == nullptr)) return PSOPS_EINVAL;
    PSOPS_DO(check_rows(d_dy, dy_ld, rows, cols));
    PSOPS_DO(check_kept(d_a_codes, d_a_scales, rows));
    if (d_b_codes != nullptr) PSOPS_DO(check_kept(d_b_codes, d_b_scales, rows));
    if (d_da != nullptr) PSOPS_DO(check_rows(d_da, da_ld, rows, cols));
    if (d_db != nullptr) PSOPS_DO(check_rows(d_db, db_ld, rows, cols));
    if (d_y != nullptr) PSOPS_DO(check_rows(d_y, y_ld, rows, cols));
    if (rows == 0 || (d_da == nullptr && d_db == nullptr && d_y == nullptr)) return PSOPS_OK;
    OnDevice guard(k);
    KeepParams P{};
    P.x[0] = (const uint16_t *)d_dy; P.x_ld[0] = dy_ld;
    P.y[0] = (uint16_t *)d_da; P.y_ld[0] = da_ld;
    P.y[1] = (uint16_t *)d_db; P.y_ld[1] = db_ld;
    P.y[2] = (uint16_t *)d_y; P.y_ld[2] = y_ld;
    P.codes[0] = (uint8_t *)d_a_codes; P.scales[0] = (float *)d_a_scales;
    P.codes[1] = (uint8_t *)d_b_codes; P.scales[1] = (float *)d_b_scales;
    return run(k, kBackward, kind, type, rows, cols, d_b_codes != nullptr, P);
}

int psops_keep_set_stream(psops_keep *k, void *cuda_stream) { return psops_host::set_stream(k, cuda_stream); }
int64_t psops_keep_launch_count(const psops_keep *k) { return k ? k->launches : 0; }
const char *psops_keep_last_error(const psops_keep *k) { return k ? k->err : ""; }

int psops_keep_destroy(psops_keep *k)
{
    if (k == nullptr) return PSOPS_EINVAL;
    OnDevice guard(k);
    const int rc = cudaStreamSynchronize(k->stream) == cudaSuccess ? PSOPS_OK : PSOPS_ECUDA;
    delete k;
    return rc;
}

} // extern "C"
