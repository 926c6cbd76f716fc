// What the operators around the mask (process.cu, sample.cu, head.cu) share:
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

// Allows `smem` bytes of dynamic shared memory for a kernel on the
// current device; what this thread has already allowed is not asked for again.
inline psc_status allow_smem(const void* kernel, int smem, const char* what) {
    struct Allowed {
        const void* kernel;
        int dev, smem;
    };
    static thread_local Allowed known[64];
    static thread_local int n = 0;
    int dev = 0;
    cudaGetDevice(&dev);
    Allowed* a = nullptr;
    for (int i = 0; i < n && !a; i++)
        if (known[i].kernel == kernel && known[i].dev == dev) a = &known[i];
    if (a && a->smem >= smem) return PSC_OK;
    psc_status s = ops_check(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem), what);
    if (s != PSC_OK) return s;
    if (!a && n < 64) a = &known[n++];
    if (a) *a = {kernel, dev, smem};
    return PSC_OK;
}

inline bool is_dtype(psc_dtype d) { return d == PSC_F32 || d == PSC_BF16; }
inline bool is_aligned(const void* p, int64_t stride_bytes, int64_t to) {
    return (uintptr_t)p % to == 0 && stride_bytes % to == 0;
}

// Launch that may start while the stream's previous kernel finishes (programmatic
// dependent launch; the kernel waits for its results itself), as clusters of
// `cluster` blocks where that is over 1.
template <typename... KArgs, typename... Args>
psc_status ops_launch(void (*kernel)(KArgs...), dim3 grid, int block, size_t smem, int cluster, cudaStream_t cs,
                      const char* what, Args... args) {
    if (smem > 16 * 1024) {                     // with what a kernel declares itself, 48 KB need no asking
        psc_status s = allow_smem((const void*)kernel, (int)smem, what);
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

// Whether the packed mask row (NULL: no mask) allows token v.
__device__ __forceinline__ bool allows(const uint32_t* row, int v) { return !row || (row[v >> 5] >> (v & 31)) & 1; }

}  // namespace
