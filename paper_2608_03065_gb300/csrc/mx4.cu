// psc_quantize_mx4 and psc_dequantize_mx4: matrices into microscaled 4-bit floating point and back.
#include <cuda_fp16.h>

#include <algorithm>

#include "mx4.cuh"

namespace {

// Both ways sixteen lanes have a tile of a row (128 columns), eight neighbouring columns each, and go from row to
// row in steps of rows_step (n_tiles * rows_step sixteens of lanes in all; whole warps go round
// together, as their lanes share blocks and tiles).  AT_ONCE rows of a lane are under way together.
// In f32 memory bounds them, read and written once: 151,936 x 1,024 into 4 bits and back 214 us (1.41 GB: 97 % of a
// copy's rate).  In bf16 their instructions do, a column costing what it does in f32: 32,768 x 2,048 into 4 bits 40 us
// (4.3 TB/s), back 32 (5.3).
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
            quantize8(v[j], largest8(v[j], 0.f), l.c, l.there && row < rows ? K : 0, q + (size_t)row * q_stride,
                      blocks + block_at(row, 0, n_tiles));
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

// WIDE false: chunks at columns 8 c - shift, as y's rows lie (load8_at); their codes come from two words, their
// exponents from up to two blocks.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(256) k_dequantize_mx4(const uint8_t* q, int64_t q_stride, const uint8_t* blocks,
                                                        const float* scale, uint32_t rows, int n_tiles, int lane_tiles,
                                                        uint32_t rows_step, int K, T* y, int64_t stride) {
    const Lane l = lane_of(lane_tiles, rows_step);
    const int words = (K + 31) / 32 * 4;
    dep_wait();
    dep_launch();
    if (!l.there) return;
    for (uint32_t r0 = l.row; r0 < rows; r0 += rows_step * AT_ONCE) {
        uint32_t codes[AT_ONCE], byte[AT_ONCE], byte2[AT_ONCE];
        float s[AT_ONCE];
        int k[AT_ONCE];
#pragma unroll
        for (int j = 0; j < AT_ONCE; j++) {
            const uint32_t row = r0 + j * rows_step;
            codes[j] = byte[j] = byte2[j] = 0;
            s[j] = 1.f;
            const int shift = WIDE ? 0 : row_shift(y + (size_t)row * stride);
            k[j] = l.c * 8 - shift;
            if (k[j] >= K || row >= rows) continue;
            const uint32_t* from = reinterpret_cast<const uint32_t*>(q + (size_t)row * q_stride);
            if (shift) {
                const uint32_t lo = l.c > 0 ? from[l.c - 1] : 0u, hi = l.c < words ? from[l.c] : 0u;
                codes[j] = __funnelshift_r(lo, hi, 4 * (8 - shift));
                byte2[j] = blocks[block_at(row, min(k[j] + 7, K - 1) / 32, n_tiles)];
            } else {
                codes[j] = from[l.c];
            }
            byte[j] = blocks[block_at(row, max(k[j], 0) / 32, n_tiles)];
            if (scale) s[j] = scale[row];
        }
#pragma unroll
        for (int j = 0; j < AT_ONCE; j++) {
            const uint32_t row = r0 + j * rows_step;
            if (k[j] >= K || row >= rows) continue;
            const float top = block_value(byte[j]), top2 = block_value(byte2[j]);
            const int second = WIDE || (k[j] & 31) < 25 ? 8 : 32 - (k[j] & 31);     // the first column of the next block
            float v[8];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const float2 f = values2(codes[j] >> (8 * e));
                v[2 * e] = f.x * (2 * e < second ? top : top2) * s[j];
                v[2 * e + 1] = f.y * (2 * e + 1 < second ? top : top2) * s[j];
            }
            store8_at(y + (size_t)row * stride, k[j], K, true, v);
        }
    }
}

// Rows under way at a time: enough for some waves of blocks over the GPU, of which none ends much later than
// the others, each lane with a few turns.
struct Grid {
    int n_tiles, rows_step;
    dim3 blocks;
};
Grid grid_of(int rows, int n_tiles) {
    const int64_t wave = (current_sms() * 8 * 16 + n_tiles - 1) / n_tiles, most = (1ll << 31) / n_tiles;
    const int64_t step = std::min({std::max<int64_t>(wave, rows / (AT_ONCE * TURNS)), ((int64_t)rows + AT_ONCE - 1) / AT_ONCE, most});
    return {n_tiles, (int)step, dim3((unsigned)((n_tiles * step + 15) / 16))};
}

template <typename T>
psc_status quantize(const void* x, int64_t stride, int rows, int K, uint8_t* q, int64_t q_stride, uint8_t* blocks,
                    cudaStream_t cs) {
    const Grid g = grid_of(rows, (K + 127) / 128);
    return ops_launch(wide_rows<T>(x, stride, K) ? k_quantize_mx4<T, true> : k_quantize_mx4<T, false>, g.blocks, 256, 0, 1,
                      cs, "k_quantize_mx4", (const T*)x, stride, rows, g.n_tiles, g.rows_step, K, q, q_stride, blocks);
}

template <typename T>
psc_status dequantize(const uint8_t* q, int64_t q_stride, const uint8_t* blocks, const float* scale, int rows, int K,
                      void* y, int64_t stride, cudaStream_t cs) {
    const bool wide = wide_rows<T>(y, stride, K);
    const Grid g = grid_of(rows, (K + (wide ? 0 : 7) + 127) / 128);
    return ops_launch(wide ? k_dequantize_mx4<T, true> : k_dequantize_mx4<T, false>, g.blocks, 256, 0, 1, cs,
                      "k_dequantize_mx4", q, q_stride, blocks, scale, rows, (K + 127) / 128, g.n_tiles, g.rows_step, K, (T*)y,
                      stride);
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
    if (!is_whole(d_x, dtype)) return ops_fail(PSC_ERR_ARG, me, "an address that is no multiple of its elements' size");
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
    if (!is_whole(d_y, dtype) || (uintptr_t)d_scale % 4)
        return ops_fail(PSC_ERR_ARG, me, "an address that is no multiple of its elements' size");
    if (T == 0) return PSC_OK;
    if (dtype == PSC_BF16)
        return dequantize<__nv_bfloat16>(d_q, q_stride, d_blocks, d_scale, T, K, d_y, row_stride, (cudaStream_t)stream);
    return dequantize<float>(d_q, q_stride, d_blocks, d_scale, T, K, d_y, row_stride, (cudaStream_t)stream);
}

}  // extern "C"
