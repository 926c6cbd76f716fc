// psc_quantize_mx4 and psc_dequantize_mx4: matrices into microscaled 4-bit floating point and back.
#include <cuda_fp16.h>

#include <algorithm>

#include "mx4.cuh"

namespace {

constexpr int AT_ONCE = 2;              // pieces that a thread has under way

// Both ways a thread has eight neighbouring columns.  I: what counts a matrix's pieces.
template <typename T, bool WIDE, typename I>
__global__ void __launch_bounds__(256) k_quantize_mx4(const T* x, int64_t stride, I items, int n_tiles, int K, uint8_t* q,
                                                      int64_t q_stride, uint8_t* blocks) {
    dep_wait();
    dep_launch();
    // sixteen lanes a tile of a row; whole warps go round together, as their lanes share blocks and tiles
    const I step = (I)gridDim.x * 16, end = (items + 1) / 2 * 2;
    for (I i0 = (I)blockIdx.x * 16 + (threadIdx.x >> 4); i0 < end; i0 += step * AT_ONCE) {
        float v[AT_ONCE][8];
        int row[AT_ONCE], c[AT_ONCE];
#pragma unroll
        for (int j = 0; j < AT_ONCE; j++) {
            const I i = i0 + j * step;
            row[j] = (int)(i / (I)n_tiles), c[j] = (int)(i - (I)row[j] * n_tiles) * 16 + (threadIdx.x & 15);
#pragma unroll
            for (int e = 0; e < 8; e++) v[j][e] = 0.f;
            if (i < items && c[j] * 8 < K) load8<WIDE>(x + (size_t)row[j] * stride, c[j] * 8, K, v[j]);
        }
#pragma unroll
        for (int j = 0; j < AT_ONCE; j++)
            if (i0 + j * step < end)            // of both of the warp's tiles
                quantize8(v[j], c[j], i0 + j * step < items ? K : 0, row[j], q + (size_t)row[j] * q_stride, blocks);
    }
}

// The values of a byte's two codes.
__device__ __forceinline__ float2 values2(uint32_t codes) {
    uint32_t pair;
    asm("{\n .reg .b8 a, b;\n .reg .b16 h;\n cvt.u16.u32 h, %1;\n mov.b16 {a, b}, h;\n cvt.rn.f16x2.e2m1x2 %0, a;\n}"
        : "=r"(pair)
        : "r"(codes));
    return __half22float2(*reinterpret_cast<const __half2*>(&pair));
}

template <typename T, bool WIDE, typename I>
__global__ void __launch_bounds__(256) k_dequantize_mx4(const uint8_t* q, int64_t q_stride, const uint8_t* blocks,
                                                        const float* scale, I items, int chunks, int K, T* y,
                                                        int64_t stride) {
    dep_wait();
    dep_launch();
    const I step = (I)gridDim.x * 256, end = (items + 31) / 32 * 32;
    for (I i0 = (I)blockIdx.x * 256 + threadIdx.x; i0 < end; i0 += step * AT_ONCE) {
        uint32_t codes[AT_ONCE], byte[AT_ONCE];
        int row[AT_ONCE], c[AT_ONCE];
        float s[AT_ONCE];
#pragma unroll
        for (int j = 0; j < AT_ONCE; j++) {
            const I i = i0 + j * step;
            row[j] = i < items ? (int)(i / (I)chunks) : 0, c[j] = i < items ? (int)(i - (I)row[j] * chunks) : 0;
            codes[j] = *reinterpret_cast<const uint32_t*>(q + (size_t)row[j] * q_stride + c[j] * 4);
            byte[j] = blocks[block_at(row[j], c[j] / 4, (K + 127) / 128)];
            s[j] = scale ? scale[row[j]] : 1.f;
        }
#pragma unroll
        for (int j = 0; j < AT_ONCE; j++) {
            const float top = block_value(byte[j]);
            float v[8];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const float2 f = values2(codes[j] >> (8 * e));
                v[2 * e] = f.x * top * s[j];
                v[2 * e + 1] = f.y * top * s[j];
            }
            store8<WIDE>(y + (size_t)row[j] * stride, c[j] * 8, K, v, i0 + j * step < items, c[j] > 0);
        }
    }
}

template <typename T, bool WIDE>
psc_status quantize(const T* x, int64_t stride, int T_, int K, uint8_t* q, int64_t q_stride, uint8_t* blocks,
                    cudaStream_t cs) {
    const int n_tiles = (K + 127) / 128;
    const int64_t items = (int64_t)T_ * n_tiles;
    const dim3 grid((unsigned)std::min<int64_t>((items + 16 * AT_ONCE - 1) / (16 * AT_ONCE), 1 << 22));
    if (items < (1ll << 30))
        return ops_launch(k_quantize_mx4<T, WIDE, uint32_t>, grid, 256, 0, 1, cs, "k_quantize_mx4", x, stride,
                          (uint32_t)items, n_tiles, K, q, q_stride, blocks);
    return ops_launch(k_quantize_mx4<T, WIDE, int64_t>, grid, 256, 0, 1, cs, "k_quantize_mx4", x, stride, items, n_tiles,
                      K, q, q_stride, blocks);
}

template <typename T, bool WIDE>
psc_status dequantize(const uint8_t* q, int64_t q_stride, const uint8_t* blocks, const float* scale, int T_, int K, T* y,
                      int64_t stride, cudaStream_t cs) {
    const int chunks = (K + 7) / 8;
    const int64_t items = (int64_t)T_ * chunks;
    const dim3 grid((unsigned)std::min<int64_t>((items + 256 * AT_ONCE - 1) / (256 * AT_ONCE), 1 << 22));
    if (items < (1ll << 30))
        return ops_launch(k_dequantize_mx4<T, WIDE, uint32_t>, grid, 256, 0, 1, cs, "k_dequantize_mx4", q, q_stride,
                          blocks, scale, (uint32_t)items, chunks, K, y, stride);
    return ops_launch(k_dequantize_mx4<T, WIDE, int64_t>, grid, 256, 0, 1, cs, "k_dequantize_mx4", q, q_stride, blocks,
                      scale, items, chunks, K, y, stride);
}

template <typename T>
psc_status quantize(const void* x, int64_t stride, int T_, int K, uint8_t* q, int64_t q_stride, uint8_t* blocks,
                    cudaStream_t cs) {
    if (wide_rows<T>(x, stride, K)) return quantize<T, true>((const T*)x, stride, T_, K, q, q_stride, blocks, cs);
    return quantize<T, false>((const T*)x, stride, T_, K, q, q_stride, blocks, cs);
}

template <typename T>
psc_status dequantize(const uint8_t* q, int64_t q_stride, const uint8_t* blocks, const float* scale, int T_, int K,
                      void* y, int64_t stride, cudaStream_t cs) {
    if (wide_rows<T>(y, stride, K))
        return dequantize<T, true>(q, q_stride, blocks, scale, T_, K, (T*)y, stride, cs);
    return dequantize<T, false>(q, q_stride, blocks, scale, T_, K, (T*)y, stride, cs);
}

}  // namespace

extern "C" {

int64_t psc_mx4_block_bytes(int32_t rows, int32_t K) {
    if (rows <= 0 || K <= 0 || K > MAX_QUANTIZE_K) return 0;
    return 512 * (((int64_t)rows + 127) / 128) * (((int64_t)K + 127) / 128);
}

psc_status psc_quantize_mx4(const void* d_x, psc_dtype dtype, int64_t row_stride, int32_t T, int32_t K, uint8_t* d_q,
                            int64_t q_stride, uint8_t* d_blocks, void* stream) {
    const char* me = "psc_quantize_mx4";
    if (T < 0 || K <= 0 || row_stride < K || !is_dtype(dtype) || (T && (!d_x || !d_q || !d_blocks)))
        return ops_fail(PSC_ERR_ARG, me, "bad arguments");
    if (K > MAX_QUANTIZE_K) return ops_fail(PSC_ERR_LIMIT, me, "K over 2^30");
    if (!is_mx4(d_q, q_stride, d_blocks, K))
        return ops_fail(PSC_ERR_ARG, me, "codes or blocks with a bad stride or alignment");
    if (T == 0) return PSC_OK;
    if (dtype == PSC_BF16)
        return quantize<__nv_bfloat16>(d_x, row_stride, T, K, d_q, q_stride, d_blocks, (cudaStream_t)stream);
    return quantize<float>(d_x, row_stride, T, K, d_q, q_stride, d_blocks, (cudaStream_t)stream);
}

psc_status psc_dequantize_mx4(const uint8_t* d_q, int64_t q_stride, const uint8_t* d_blocks, const float* d_scale,
                              int32_t T, int32_t K, void* d_y, psc_dtype dtype, int64_t row_stride, void* stream) {
    const char* me = "psc_dequantize_mx4";
    if (T < 0 || K <= 0 || row_stride < K || !is_dtype(dtype) || (T && (!d_y || !d_q || !d_blocks)))
        return ops_fail(PSC_ERR_ARG, me, "bad arguments");
    if (K > MAX_QUANTIZE_K) return ops_fail(PSC_ERR_LIMIT, me, "K over 2^30");
    if (!is_mx4(d_q, q_stride, d_blocks, K))
        return ops_fail(PSC_ERR_ARG, me, "codes or blocks with a bad stride or alignment");
    if (T == 0) return PSC_OK;
    if (dtype == PSC_BF16)
        return dequantize<__nv_bfloat16>(d_q, q_stride, d_blocks, d_scale, T, K, d_y, row_stride, (cudaStream_t)stream);
    return dequantize<float>(d_q, q_stride, d_blocks, d_scale, T, K, d_y, row_stride, (cudaStream_t)stream);
}

}  // extern "C"
