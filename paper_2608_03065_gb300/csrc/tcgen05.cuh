// What the tensor-core kernels (head.cu, mx4_head.cu) share: barriers in shared memory with bounded
// waits, TMA copies and their maps, operand descriptors, the accumulators' way back.
#pragma once

#include <cuda.h>
#include <cudaTypedefs.h>

#include "ops_common.cuh"

namespace {

constexpr int SMEM_MAX = 227 * 1024;

__device__ __forceinline__ uint32_t smem_addr(const void* p) {
    return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_arrive_tx(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
// The same without waiting a while for the answer (mbar_try does for up to 4 us).
__device__ __forceinline__ bool mbar_look(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
constexpr int WAIT_POLLS = 1 << 22;
// Bounded wait: gives up after some seconds (16), or soon after any other wait of the block did.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* failed) {
    for (int it = 0; it < WAIT_POLLS; it++) {
        if (mbar_try(bar, parity)) return true;
        if ((it & 1023) == 1023 && *failed) return false;
    }
    *failed = 1;
    return false;
}
// The same by a whole warp, with one answer for all lanes; and for two barriers at once
// (a poll takes about a hundred cycles to answer, so both are asked before either is looked at).
// CHECK: one that gives up after `polls` looks, for a kernel's self-test.
template <bool CHECK = false>
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* failed, int polls = 0) {
    for (int it = 0; it < (CHECK ? polls : WAIT_POLLS); it++) {
        if (__all_sync(FULL, CHECK ? mbar_look(bar, parity) : mbar_try(bar, parity))) return true;
        if ((it & 1023) == 1023 && __any_sync(FULL, *failed)) return false;
    }
    *failed = 1;
    return false;
}
template <bool CHECK = false>
__device__ __forceinline__ bool warp_wait2(uint32_t bar0, uint32_t parity0, uint32_t bar1, uint32_t parity1,
                                           volatile int* failed, int polls = 0) {
    if (!CHECK) {
        const bool a = mbar_try(bar0, parity0), b = mbar_try(bar1, parity1);
        if (__all_sync(FULL, a && b)) return true;
    }
    return warp_wait<CHECK>(bar0, parity0, failed, polls) && warp_wait<CHECK>(bar1, parity1, failed, polls);
}
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(p));
    return p != 0;
}
// A place in a ring of n slots: the slot and the parity of its current use.
struct Place {
    int s = 0;
    uint32_t parity = 0;
    __device__ __forceinline__ void next(int n) {
        if (++s == n) s = 0, parity ^= 1;
    }
};
__device__ __forceinline__ void tma_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
        ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
// Shared-memory operand descriptor: rows of 128 bytes in the 128-byte swizzle, 8 rows per 1024 bytes.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr) {
    return (uint64_t)((addr & 0x3FFFF) >> 4) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// Arrives at the barrier (of both blocks of a pair) when the products so far are done.
template <bool PAIR>
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    if (PAIR)
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
            ::"r"(bar), "h"((uint16_t)3)
            : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
}
// Arrives at the first block's barrier of that place.
__device__ __forceinline__ void arrive_at_first(uint32_t bar) {
    asm volatile(
        "{\n .reg .b32 r;\n mapa.shared::cluster.u32 r, %0, 0;\n"
        " mbarrier.arrive.shared::cluster.b64 _, [r];\n}" ::"r"(bar)
        : "memory");
}
// 16 columns of the warp's 32 lanes; complete after tmem_wait.
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t r[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_wait(uint32_t r[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; i++) asm volatile("" : "+r"(r[i]));      // no use of r before the wait
}

// A tensor map over rows of `stride` bytes, boxes of `cols` x `rows`.
bool tensor_map(CUtensorMap* m, CUtensorMapDataType type, const void* p, uint64_t cols, uint64_t rows, uint64_t stride,
                uint32_t box_cols, uint32_t box_rows, CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B) {
    static PFN_cuTensorMapEncodeTiled_v12000 encode = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &r) != cudaSuccess ||
            r != cudaDriverEntryPointSuccess)
            f = nullptr;
        return (PFN_cuTensorMapEncodeTiled_v12000)f;
    }();
    if (!encode) return false;
    const cuuint64_t dims[2] = {cols, rows}, strides[1] = {stride};
    const cuuint32_t box[2] = {box_cols, box_rows}, step[2] = {1, 1};
    return encode(m, type, 2, const_cast<void*>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
