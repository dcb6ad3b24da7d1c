// op_host.h - what the host sides of the entry points share: the guard that makes a device current
// for a call, and argument checks that end in a message and a code.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "rpd_internal.h"

namespace rpd {

// Entry points that touch the GPU run with their device current and its primary context bound to
// the calling thread - cudaSetDevice does both; a host thread that has not used the CUDA runtime yet
// has no context, and the driver's tensor-map encoder then fails - and give the thread its previous
// device back when they return.
struct DeviceGuard {
    int prev = -1;
    cudaError_t err = cudaSuccess;
    explicit DeviceGuard(int dev) {
        if (cudaGetDevice(&prev) != cudaSuccess) prev = -1;
        err = cudaSetDevice(dev);
    }
    ~DeviceGuard() {
        int now = -1;
        if (prev >= 0 && cudaGetDevice(&now) == cudaSuccess && now != prev) cudaSetDevice(prev);
    }
    DeviceGuard(const DeviceGuard &) = delete;
    DeviceGuard &operator=(const DeviceGuard &) = delete;
};

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *,
                                  const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                  const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's tensor-map encoder, looked up once; null where the driver does not have it.
inline EncodeTiledFn encode_fn() {
    static const EncodeTiledFn fn = [] {  // initialised once, thread-safely
        void *ptr = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &ptr, 12000,
                                             cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            return reinterpret_cast<EncodeTiledFn>(ptr);
        return static_cast<EncodeTiledFn>(nullptr);
    }();
    return fn;
}

inline int op_fail(int code, const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    set_last_error(buf);
    return code;
}

inline int op_cuda_fail(cudaError_t e, const char *what) {
    cudaGetLastError();  // reported here: it is not the next call's
    return op_fail(e == cudaErrorMemoryAllocation ? RPD_ERR_OUT_OF_MEMORY : RPD_ERR_CUDA, "%s: %s", what,
                   cudaGetErrorString(e));
}

// While it lives, this thread's allocations and frees are allowed although some stream is being captured in the global mode
// (without it they would fail, and end that capture).
struct RelaxedCapture {
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    RelaxedCapture() { cudaThreadExchangeStreamCaptureMode(&mode); }
    ~RelaxedCapture() { cudaThreadExchangeStreamCaptureMode(&mode); }
    RelaxedCapture(const RelaxedCapture &) = delete;
    RelaxedCapture &operator=(const RelaxedCapture &) = delete;
};

constexpr int64_t kWaitCyclesPerUs = 2000;  // the limit of a wait in a kernel is counted in cycles of some 2 GHz
constexpr int64_t kMaxWaitUs = 60000000;

// Bytes of an element of one of the RPD_TYPE_* types, 0 for anything else.
inline int type_size(int type) {
    return type == RPD_TYPE_F32 ? 4 : type == RPD_TYPE_BF16 || type == RPD_TYPE_F16 ? 2 : 0;
}

inline bool aligned_to(const void *p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// The library's kernels are sm_103a code: any other device is refused before a launch.
inline int check_device(int device) {
    int major = 0, minor = 0;
    cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, device);
    cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, device);
    if (major != 10 || minor != 3)
        return op_fail(RPD_ERR_UNSUPPORTED, "device is sm_%d%d; this library is built for sm_103a", major, minor);
    return RPD_OK;
}

// A launch without attributes, with its own error (not one that an earlier call has left behind).
template <typename... KArgs, typename... Args>
cudaError_t launch_plain(void (*kernel)(KArgs...), int grid, int block, cudaStream_t s, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.stream = s;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// The largest of 16, 8, 4 and 2 that divides an address (and whatever is or-ed into it).
inline int common_align(uintptr_t bits) { return bits & 2 ? 2 : bits & 4 ? 4 : bits & 8 ? 8 : 16; }

}  // namespace rpd
