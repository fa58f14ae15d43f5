// psops_host.cuh -- host-side helpers shared by the training operators' C entries.
#pragma once

#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>
#include <cstdio>

namespace psops_host {

inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

#define PSOPS_TRY(base, call)                                             \
    do {                                                                  \
        const cudaError_t e_ = (call);                                    \
        if (e_ != cudaSuccess) return (base)->fail(e_, #call);            \
    } while (0)

// What every training-operator context has: its GPU, its stream, its launch
// count and the text of the last CUDA error.
struct Base {
    cudaStream_t stream = nullptr;
    int device = 0;
    int sms = 0;
    int64_t launches = 0;
    cudaEvent_t moved = nullptr;       // orders a new stream behind the old one
    char err[256] = {0};

    ~Base()
    {
        if (moved) cudaEventDestroy(moved);
    }

    int fail(cudaError_t e, const char *what)
    {
        std::snprintf(err, sizeof(err), "%s: %s", what, cudaGetErrorString(e));
        return PSOPS_ECUDA;
    }
};

// Work of a context belongs to the GPU that was current at its creation; the
// entry points switch to it for their duration if another one is current.
class OnDevice {
public:
    explicit OnDevice(const Base *b) : previous_(-1)
    {
        int now = -1;
        if (b != nullptr && cudaGetDevice(&now) == cudaSuccess && now != b->device &&
            cudaSetDevice(b->device) == cudaSuccess)
            previous_ = now;
    }
    ~OnDevice()
    {
        if (previous_ >= 0) cudaSetDevice(previous_);
    }
    OnDevice(const OnDevice &) = delete;
    OnDevice &operator=(const OnDevice &) = delete;

private:
    int previous_;
};

// Launches a kernel that begins with umma::after_the_kernel_before.
template <typename... Params, typename... Args>
int launch(Base *b, const char *name, void (*kernel)(Params...), dim3 grid, int threads, size_t shared, int cluster, Args &&...args)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = b->stream;
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
    if (e != cudaSuccess) return b->fail(e, name);
    b->launches += 1;
    return PSOPS_OK;
}

inline int set_stream(Base *b, void *cuda_stream)
{
    if (b == nullptr) return PSOPS_EINVAL;
    const cudaStream_t to = (cudaStream_t)cuda_stream;
    if (to == b->stream) return PSOPS_OK;
    OnDevice guard(b);
    cudaStreamCaptureStatus from_capture = cudaStreamCaptureStatusNone, to_capture = cudaStreamCaptureStatusNone;
    unsigned long long from_id = 0, to_id = 0;
    PSOPS_TRY(b, cudaStreamGetCaptureInfo(to, &to_capture, &to_id));
    PSOPS_TRY(b, cudaStreamGetCaptureInfo(b->stream, &from_capture, &from_id));
    // both outside captures, or two branches of one
    if (to_capture == from_capture && (to_capture == cudaStreamCaptureStatusNone || to_id == from_id)) {
        if (b->moved == nullptr) PSOPS_TRY(b, cudaEventCreateWithFlags(&b->moved, cudaEventDisableTiming));
        PSOPS_TRY(b, cudaEventRecord(b->moved, b->stream));
        PSOPS_TRY(b, cudaStreamWaitEvent(to, b->moved, 0));
    }
    b->stream = to;
    return PSOPS_OK;
}

// What must not become part of a captured graph: a table that is sent from the
// staging below (every replay would send what the staging holds by then), the
// setting up of a context (it would be done at the replay only), a wait for the host.
inline int not_capturing(Base *b)
{
    cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
    PSOPS_TRY(b, cudaStreamIsCapturing(b->stream, &status));
    return status == cudaStreamCaptureStatusNone ? PSOPS_OK : PSOPS_ESTATE;
}

// Page-locked staging of a small table that is sent to the device again and
// again: the copy is asynchronous, and the staging is not overwritten before
// the copy that read it has run.
class Staging {
public:
    ~Staging()
    {
        if (event_) cudaEventDestroy(event_);
        if (host_) cudaFreeHost(host_);
    }
    cudaError_t reserve(size_t bytes)
    {
        cudaError_t e = cudaHostAlloc(&host_, bytes ? bytes : 1, cudaHostAllocDefault);
        if (e == cudaSuccess) e = cudaEventCreateWithFlags(&event_, cudaEventDisableTiming);
        return e;
    }
    cudaError_t wait() { return sent_ ? cudaEventSynchronize(event_) : cudaSuccess; }
    void *host() { return host_; }
    cudaError_t send(void *dst, size_t bytes, cudaStream_t stream)
    {
        cudaError_t e = cudaMemcpyAsync(dst, host_, bytes, cudaMemcpyHostToDevice, stream);
        if (e == cudaSuccess) e = cudaEventRecord(event_, stream);
        sent_ = sent_ || e == cudaSuccess;
        return e;
    }

private:
    void *host_ = nullptr;
    cudaEvent_t event_ = nullptr;
    bool sent_ = false;
};

} // namespace psops_host
