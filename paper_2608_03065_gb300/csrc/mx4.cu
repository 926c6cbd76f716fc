// psc_quantize_mx4 and psc_dequantize_mx4: matrices into microscaled 4-bit floating point and back.
#include <cuda_fp16.h>

#include <algorithm>

#include "mx4.cuh"

namespace {

// Sixteen lanes per tile of a row (128 columns).
template <typename T>
__global__ void __launch_bounds__(256) k_quantize_mx4(const T* x, int64_t stride, int64_t items, int n_tiles, int K,
                                                      uint8_t* q, int64_t q_stride, uint8_t* blocks, bool wide) {
    dep_wait();
    dep_launch();
    // whole warps go round together: their lanes share blocks and tiles
    for (int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); i < (items + 1) / 2 * 2; i += (int64_t)gridDim.x * 16) {
        const int row = (int)(i / n_tiles), tile = (int)(i - (int64_t)row * n_tiles);
        const int c = tile * 16 + (threadIdx.x & 15);
        float v[8] = {};
        const bool there = i < items;
        if (there && c * 8 < K) load8(x + (size_t)row * stride, c * 8, K, wide, v);
        quantize8(v, c, there ? K : 0, row, q + (size_t)row * q_stride, blocks);
    }
}

template <typename T>
__global__ void __launch_bounds__(256) k_dequantize_mx4(const uint8_t* q, int64_t q_stride, const uint8_t* blocks,
                                                        const float* scale, int64_t items, int chunks, int K, T* y,
                                                        int64_t stride, bool wide) {
    dep_wait();
    dep_launch();
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < items; i += (int64_t)gridDim.x * 256) {
        const int row = (int)(i / chunks), c = (int)(i - (int64_t)row * chunks);
        const uint32_t codes = *reinterpret_cast<const uint32_t*>(q + (size_t)row * q_stride + c * 4);
        const float top = block_value(blocks[block_at(row, c / 4, (K + 127) / 128)]);
        const float s = scale ? scale[row] : 1.f;
        float v[8];
#pragma unroll
        for (int j = 0; j < 4; j++) {
            uint32_t pair;
            asm("{\n .reg .b8 a, b;\n .reg .b16 h;\n cvt.u16.u32 h, %1;\n mov.b16 {a, b}, h;\n"
                " cvt.rn.f16x2.e2m1x2 %0, a;\n}"
                : "=r"(pair)
                : "r"(codes >> (8 * j)));
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&pair));
            v[2 * j] = f.x * top * s;
            v[2 * j + 1] = f.y * top * s;
        }
        store8(y + (size_t)row * stride, c * 8, K, wide, v);
    }
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
    const int n_tiles = (K + 127) / 128;
    const int64_t items = (int64_t)T * n_tiles;
    const dim3 grid((unsigned)std::min<int64_t>((items + 15) / 16, 1 << 30));
    if (dtype == PSC_BF16)
        return ops_launch(k_quantize_mx4<__nv_bfloat16>, grid, 256, 0, 1, (cudaStream_t)stream, "k_quantize_mx4",
                          (const __nv_bfloat16*)d_x, row_stride, items, n_tiles, K, d_q, q_stride, d_blocks,
                          wide_rows<__nv_bfloat16>(d_x, row_stride, K));
    return ops_launch(k_quantize_mx4<float>, grid, 256, 0, 1, (cudaStream_t)stream, "k_quantize_mx4", (const float*)d_x,
                      row_stride, items, n_tiles, K, d_q, q_stride, d_blocks, wide_rows<float>(d_x, row_stride, K));
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
    const int chunks = (K + 7) / 8;
    const int64_t items = (int64_t)T * chunks;
    const dim3 grid((unsigned)std::min<int64_t>((items + 255) / 256, 1 << 30));
    if (dtype == PSC_BF16)
        return ops_launch(k_dequantize_mx4<__nv_bfloat16>, grid, 256, 0, 1, (cudaStream_t)stream, "k_dequantize_mx4",
                          d_q, q_stride, d_blocks, d_scale, items, chunks, K, (__nv_bfloat16*)d_y, row_stride,
                          wide_rows<__nv_bfloat16>(d_y, row_stride, K));
    return ops_launch(k_dequantize_mx4<float>, grid, 256, 0, 1, (cudaStream_t)stream, "k_dequantize_mx4", d_q, q_stride,
                      d_blocks, d_scale, items, chunks, K, (float*)d_y, row_stride, wide_rows<float>(d_y, row_stride, K));
}

}  // extern "C"
