// psc_quantize_mx4 and psc_dequantize_mx4: matrices into microscaled 4-bit floating point and back.
#include <cuda_fp16.h>

#include <algorithm>

#include "mx4.cuh"

namespace {

// Both ways sixteen lanes have a tile of a row (128 columns), eight neighbouring columns each, and go from row to
// row in steps of rows_step (n_tiles * rows_step sixteens of lanes in all; whole warps go round
// together, as their lanes share blocks and tiles).  AT_ONCE rows of a lane are under way together.
constexpr int AT_ONCE = 2, TURNS = 2;

struct Lane {
    uint32_t row;                           // the first
    int c;                                  // the chunk
    bool there;
};
__device__ __forceinline__ Lane lane_of(int n_tiles, uint32_t rows_step) {
    const uint32_t i = blockIdx.x * 16u + (threadIdx.x >> 4), row = i / (uint32_t)n_tiles;
    return {row, (int)(i - row * n_tiles) * 16 + (int)(threadIdx.x & 15), row < rows_step};
}

template <typename T, bool WIDE>
__global__ void __launch_bounds__(256) k_quantize_mx4(const T* x, int64_t stride, uint32_t rows, int n_tiles,
                                                      uint32_t rows_step, int K, uint8_t* q, int64_t q_stride, uint8_t* blocks) {
    const Lane l = lane_of(n_tiles, rows_step);
    const bool inside = l.c * 8 < K;
    dep_wait();
    dep_launch();
    for (uint32_t r0 = l.row; __any_sync(FULL, r0 < rows); r0 += rows_step * AT_ONCE) {
        float v[AT_ONCE][8];
#pragma unroll
        for (int j = 0; j < AT_ONCE; j++) {
            const uint32_t row = r0 + j * rows_step;
#pragma unroll
            for (int e = 0; e < 8; e++) v[j][e] = 0.f;
            if (l.there && inside && row < rows) load8<WIDE>(x + (size_t)row * stride, l.c * 8, K, v[j]);
        }
#pragma unroll
        for (int j = 0; j < AT_ONCE; j++) {
            const uint32_t row = r0 + j * rows_step;
            quantize8(v[j], largest8(v[j]), l.c, l.there && row < rows ? K : 0, row, q + (size_t)row * q_stride, blocks);
        }
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

template <typename T, bool WIDE>
__global__ void __launch_bounds__(256) k_dequantize_mx4(const uint8_t* q, int64_t q_stride, const uint8_t* blocks,
                                                        const float* scale, uint32_t rows, int n_tiles,
                                                        uint32_t rows_step, int K,
                                                        T* y, int64_t stride) {
    const Lane l = lane_of(n_tiles, rows_step);
    const bool inside = l.there && l.c * 8 < K;
    dep_wait();
    dep_launch();
    for (uint32_t r0 = l.row; __any_sync(FULL, r0 < rows); r0 += rows_step * AT_ONCE) {
        uint32_t codes[AT_ONCE], byte[AT_ONCE];
        float s[AT_ONCE];
#pragma unroll
        for (int j = 0; j < AT_ONCE; j++) {
            const uint32_t row = r0 + j * rows_step;
            codes[j] = byte[j] = 0;
            s[j] = 1.f;
            if (!inside || row >= rows) continue;
            codes[j] = *reinterpret_cast<const uint32_t*>(q + (size_t)row * q_stride + l.c * 4);
            byte[j] = blocks[block_at(row, l.c / 4, n_tiles)];
            if (scale) s[j] = scale[row];
        }
#pragma unroll
        for (int j = 0; j < AT_ONCE; j++) {
            const uint32_t row = r0 + j * rows_step;
            const float top = block_value(byte[j]);
            float v[8];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const float2 f = values2(codes[j] >> (8 * e));
                v[2 * e] = f.x * top * s[j];
                v[2 * e + 1] = f.y * top * s[j];
            }
            store8<WIDE>(y + (size_t)row * stride, l.c * 8, K, v, inside && row < rows, l.c & 15);
        }
    }
}

// Rows under way at a time: enough for some waves of blocks over the GPU, of which none ends much later than
// the others, each lane with a few turns.
struct Grid {
    int n_tiles, rows_step;
    dim3 blocks;
};
Grid grid_of(int rows, int K) {
    const int n_tiles = (K + 127) / 128, wave = (current_sms() * 8 * 16 + n_tiles - 1) / n_tiles;
    const int step = std::max(1, std::min(std::max(wave, rows / (AT_ONCE * TURNS)), (rows + AT_ONCE - 1) / AT_ONCE));
    return {n_tiles, step, dim3((unsigned)(((int64_t)n_tiles * step + 15) / 16))};
}

template <typename T>
psc_status quantize(const void* x, int64_t stride, int rows, int K, uint8_t* q, int64_t q_stride, uint8_t* blocks,
                    cudaStream_t cs) {
    const Grid g = grid_of(rows, K);
    return ops_launch(wide_rows<T>(x, stride, K) ? k_quantize_mx4<T, true> : k_quantize_mx4<T, false>, g.blocks, 256, 0, 1,
                      cs, "k_quantize_mx4", (const T*)x, stride, rows, g.n_tiles, g.rows_step, K, q, q_stride, blocks);
}

template <typename T>
psc_status dequantize(const uint8_t* q, int64_t q_stride, const uint8_t* blocks, const float* scale, int rows, int K,
                      void* y, int64_t stride, cudaStream_t cs) {
    const Grid g = grid_of(rows, K);
    return ops_launch(wide_rows<T>(y, stride, K) ? k_dequantize_mx4<T, true> : k_dequantize_mx4<T, false>, g.blocks, 256, 0,
                      1, cs, "k_dequantize_mx4", q, q_stride, blocks, scale, rows, g.n_tiles, g.rows_step, K, (T*)y, stride);
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
