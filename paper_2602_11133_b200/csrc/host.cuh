// Host side of a launch, shared by the translation units: status codes from CUDA errors, the launch itself, device facts.
#pragma once
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstddef>
#include <cstdint>

#include "../../include/jot.h"

namespace jot {

inline thread_local int g_last_cuda_error = 0;
inline std::atomic<int64_t> g_launches{0};

#define JOT_CUDA(expr)                                  \
    do {                                                \
        cudaError_t e_ = (expr);                        \
        if (e_ != cudaSuccess) {                        \
            g_last_cuda_error = (int)e_;                \
            return JOT_ERR_CUDA;                        \
        }                                               \
    } while (0)
#define JOT_TRY(expr)              \
    do {                           \
        int s_ = (expr);           \
        if (s_ != JOT_OK) return s_; \
    } while (0)

inline int launch_check() {
    g_launches.fetch_add(1, std::memory_order_relaxed);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) {
        g_last_cuda_error = (int)e;
        return JOT_ERR_CUDA;
    }
    return JOT_OK;
}

// Every kernel goes out through here: programmatic stream serialization lets a kernel's launch and
// on-chip prologue overlap the tail of its predecessor (see pdl.cuh for the device side).
template <typename... KArgs, typename... Args>
void launch_k(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);     // errors are picked up by launch_check()
}

// ---------------------------------------------------------------- device facts
struct DeviceInfo {
    int ok = 0, sms = 0, status = JOT_OK;
    PFN_cuTensorMapEncodeTiled_v12000 encode = nullptr;
};

inline int device_info(DeviceInfo** out) {
    static thread_local DeviceInfo cache[64];
    int dev = 0;
    JOT_CUDA(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) return JOT_ERR_DEVICE;
    DeviceInfo& di = cache[dev];
    if (!di.ok) {
        int major = 0;
        JOT_CUDA(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev));
        JOT_CUDA(cudaDeviceGetAttribute(&di.sms, cudaDevAttrMultiProcessorCount, dev));
        if (major != 10) return JOT_ERR_DEVICE;
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult qres;
        JOT_CUDA(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres));
        if (qres != cudaDriverEntryPointSuccess || fn == nullptr) return JOT_ERR_DEVICE;
        di.encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
        di.ok = 1;
    }
    *out = &di;
    return JOT_OK;
}

inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

}  // namespace jot
