// What the operators around the mask (process.cu, sample.cu, head.cu, norm.cu, mx4.cu, mx4_head.cu) share:
// the C entries' error path, launches, and small device helpers.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <string>

#include "../../include/psc_ops.h"

namespace psc {
// Sets the message psc_last_error returns (never throws) and gives back `code`.
psc_status ops_fail(psc_status code, const char* what, const char* why) noexcept;
}  // namespace psc

namespace {

using psc::ops_fail;

constexpr unsigned FULL = 0xffffffffu;

inline psc_status ops_check(cudaError_t e, const char* what) {
    if (e == cudaSuccess) return PSC_OK;
    return ops_fail(e == cudaErrorMemoryAllocation ? PSC_ERR_OOM : PSC_ERR_CUDA, what, cudaGetErrorString(e));
}

// SMs of the current device (asked once per device and thread).
inline int current_sms() {
    static thread_local int of = -1, n = 0;
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev != of) {
        cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
        of = dev;
    }
    return n > 0 ? n : 1;
}

// Lets a kernel use all the dynamic shared memory of the current device beside its own (once
// per kernel, device and thread; always the same amount, so that threads cannot undo each
// other's setting).
inline psc_status allow_smem(const void* kernel, const char* what) {
    struct Allowed {
        const void* kernel;
        int dev;
    };
    static thread_local Allowed known[64];
    static thread_local int n = 0;
    int dev = 0, most = 0;
    cudaGetDevice(&dev);
    for (int i = 0; i < n; i++)
        if (known[i].kernel == kernel && known[i].dev == dev) return PSC_OK;
    cudaFuncAttributes of = {};
    psc_status s = ops_check(cudaDeviceGetAttribute(&most, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev), what);
    if (s == PSC_OK) s = ops_check(cudaFuncGetAttributes(&of, kernel), what);
    if (s == PSC_OK)
        s = ops_check(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                           most - (int)of.sharedSizeBytes), what);
    if (s == PSC_OK && n < 64) known[n++] = {kernel, dev};
    return s;
}

inline bool is_dtype(psc_dtype d) { return d == PSC_F32 || d == PSC_BF16; }
inline bool is_aligned(const void* p, int64_t stride_bytes, int64_t to) {
    return (uintptr_t)p % to == 0 && stride_bytes % to == 0;
}
// Whether rows of a dtype start at multiples of its size (as torch's do).
inline bool is_whole(const void* p, psc_dtype d) { return (uintptr_t)p % (d == PSC_BF16 ? 2 : 4) == 0; }

// Launch that may start while the stream's previous kernel finishes (programmatic
// dependent launch; the kernel waits for its results itself), as clusters of
// `cluster` blocks where that is over 1.
template <typename... KArgs, typename... Args>
psc_status ops_launch(void (*kernel)(KArgs...), dim3 grid, int block, size_t smem, int cluster, cudaStream_t cs,
                      const char* what, Args... args) {
    if (smem > 16 * 1024) {                     // with what a kernel declares itself, 48 KB need no asking
        psc_status s = allow_smem((const void*)kernel, what);
        if (s != PSC_OK) return s;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = cs;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return ops_check(cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...), what);
}

__device__ __forceinline__ void dep_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void dep_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ float load_f32(const float* p) { return *p; }
__device__ __forceinline__ float load_f32(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store_f32(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_f32(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

}  // namespace
