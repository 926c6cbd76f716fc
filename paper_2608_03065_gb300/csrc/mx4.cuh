// The microscaled 4-bit format (psc_mx4.h) on the device: eight columns at a time in a thread,
// four neighbouring threads a block of 32 columns, sixteen a row's piece of a tile of exponents.
#pragma once

#include "../../include/psc_mx4.h"
#include "ops_common.cuh"

namespace {

constexpr int MAX_QUANTIZE_K = 1 << 30;

// Eight values of a row from column k on, zeros past K.  vec: 16-byte loads are in place (then K
// is a multiple of 8).
__device__ __forceinline__ void load8(const float* row, int k, int K, bool vec, float v[8]) {
    if (vec) {
        const float4 a = *reinterpret_cast<const float4*>(row + k), b = *reinterpret_cast<const float4*>(row + k + 4);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] = k + j < K ? row[k + j] : 0.f;
    }
}
__device__ __forceinline__ void load8(const __nv_bfloat16* row, int k, int K, bool vec, float v[8]) {
    if (vec) {
        const uint4 a = *reinterpret_cast<const uint4*>(row + k);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int j = 0; j < 4; j++) {
            v[2 * j] = __uint_as_float(w[j] << 16);
            v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] = k + j < K ? __bfloat162float(row[k + j]) : 0.f;
    }
}
__device__ __forceinline__ void store8(float* row, int k, int K, bool vec, const float v[8]) {
    if (vec) {
        *reinterpret_cast<float4*>(row + k) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4*>(row + k + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; j++)
            if (k + j < K) row[k + j] = v[j];
    }
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ void store8(__nv_bfloat16* row, int k, int K, bool vec, const float v[8]) {
    if (vec) {
        *reinterpret_cast<uint4*>(row + k) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]),
                                                        pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    } else {
#pragma unroll
        for (int j = 0; j < 8; j++)
            if (k + j < K) row[k + j] = __float2bfloat16_rn(v[j]);
    }
}
// Whether rows of these elements take load8's and store8's 16-byte accesses.
template <typename T>
inline bool wide_rows(const void* p, int64_t stride, int K) {
    return !p || (K % 8 == 0 && is_aligned(p, stride * (int64_t)sizeof(T), 16));
}

// The magnitudes' bit patterns order as the magnitudes do, with infinities and NaN above all.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
constexpr uint32_t INF_BITS = 0x7f800000u;

// Where the exponent of row r's block b is; n_tiles = ceil(K / 128).
__host__ __device__ __forceinline__ int64_t block_at(int r, int b, int n_tiles) {
    return 512 * ((int64_t)(r / 128) * n_tiles + b / 4) + 16 * (r % 32) + 4 * (r % 128 / 32) + b % 4;
}

// Of a block whose largest magnitude has these bits: the byte e + 127, and 2^-e.  The largest
// magnitude lies in [4, 8) 2^e (below where e is -127), so x 2^-e is exact and codes reach 4 or 6.
__device__ __forceinline__ uint32_t block_byte(uint32_t top) {
    return top >= INF_BITS ? 255u : (uint32_t)max((int)(top >> 23) - 2, 0);
}
__device__ __forceinline__ float block_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
// 2^e, NaN for a NaN block.
__device__ __forceinline__ float block_value(uint32_t byte) {
    return __uint_as_float(byte == 255 ? 0x7fc00000u : byte ? byte << 23 : 1u << 22);
}

// Eight values as codes, the first in the lowest bits (ties to even, 6 at most).
__device__ __forceinline__ uint32_t codes8(const float v[8], float inverse) {
    uint32_t out;
    asm("{\n .reg .b8 a, b, c, d;\n"
        " cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
        " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n"
        " mov.b32 %0, {a, b, c, d};\n}"
        : "=r"(out)
        : "f"(v[0] * inverse), "f"(v[1] * inverse), "f"(v[2] * inverse), "f"(v[3] * inverse), "f"(v[4] * inverse),
          "f"(v[5] * inverse), "f"(v[6] * inverse), "f"(v[7] * inverse));
    return out;
}

// A thread's eight columns from 8 c on of a row, to codes and exponents.  All 32 lanes of a warp
// call it for neighbouring chunks c, lane 0's a multiple of 16; what lies past the row's last
// tile stores nothing.
__device__ __forceinline__ void quantize8(const float v[8], int c, int K, int row, uint8_t* q_row, uint8_t* blocks) {
    const int lane = threadIdx.x & 31;
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; j++) top = max(top, magnitude(v[j]));
    top = max(top, __shfl_xor_sync(FULL, top, 1));
    top = max(top, __shfl_xor_sync(FULL, top, 2));
    const uint32_t byte = block_byte(top);
    if (c < (K + 31) / 32 * 4)
        *reinterpret_cast<uint32_t*>(q_row + c * 4) = byte == 255 ? 0u : codes8(v, block_inverse(byte));
    // the four blocks of a tile's row, by one of its sixteen lanes
    uint32_t word = byte << (8 * ((lane >> 2) & 3));
    word |= __shfl_xor_sync(FULL, word, 4);
    word |= __shfl_xor_sync(FULL, word, 8);
    const int n_tiles = (K + 127) / 128;
    if (!(lane & 15) && c < n_tiles * 16)
        *reinterpret_cast<uint32_t*>(blocks + block_at(row, c / 4, n_tiles)) = word;
}

inline bool is_mx4(const void* q, int64_t stride, const void* blocks, int K) {
    return is_aligned(q, stride, 16) && (uintptr_t)blocks % 16 == 0 && stride >= ((int64_t)K + 31) / 32 * 16;
}

}  // namespace
