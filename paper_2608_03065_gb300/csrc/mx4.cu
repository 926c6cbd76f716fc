// psc_quantize_mx4, psc_dequantize_mx4 and psc_head_logits_mx4: matrices in microscaled
// 4-bit floating point, and the vocabulary projection on them under the grammar's mask.
#include <cuda_fp16.h>

#include <algorithm>

#include "mx4.cuh"

namespace {

constexpr int MAX_K = 131072;
constexpr int MAX_V = 1 << 30, MAX_T = 1 << 24;

// ------------------------------------------------------------- into 4 bits and back
//
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

// --------------------------------------------------------------------- the projection
struct Head {
    const uint8_t* q;
    int64_t q_stride;
    const uint8_t* q_blocks;
    const float* scale;
    int T;
    const uint8_t* w;
    int64_t w_stride;
    const uint8_t* w_blocks;
    const float* w_scale;
    int V, K;
    const uint32_t* bitmask;
    int W;                              // mask words of a row
    int64_t row_stride;
};

// Eight codes as bytes of twice their values, in order.
__device__ __forceinline__ uint2 doubled8(uint32_t codes) {
    const uint32_t m = codes & 0x77777777u, side = ((codes >> 1) & 0x44444444u) | 0x32103210u;
    uint2 out;
    // the magnitudes' bytes, their negatives, and of each byte the one that its sign picks
    out.x = __byte_perm(__byte_perm(0x03020100u, 0x0C080604u, m), __byte_perm(0xFDFEFF00u, 0xF4F8FAFCu, m), side);
    out.y = __byte_perm(__byte_perm(0x03020100u, 0x0C080604u, m >> 16), __byte_perm(0xFDFEFF00u, 0xF4F8FAFCu, m >> 16),
                        side >> 16);
    return out;
}
// The smaller and the larger; NaN if one is.
__device__ __forceinline__ float min_nan(float a, float b) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// k_mx4_rows: a warp per 32 vocabulary rows (a word of the masks), of which those that some of up
// to N tokens allow are read, 4 at once, a lane per block of 32 columns.  A block's products are
// summed in whole numbers (quarters; exact), then scaled: the smaller power of two first, so that
// nothing leaves f32 on the way to a sum that does not.
constexpr int ROWS = 4;
constexpr int ROWS_THREADS = 256;

template <typename T, int N>
__global__ void __launch_bounds__(ROWS_THREADS) k_mx4_rows(Head h, int t0, T* logits) {
    extern __shared__ __align__(16) uint8_t dyn[];
    __shared__ float s_out[ROWS_THREADS / 32][N * 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int nb = (h.K + 31) / 32, n_tiles = (h.K + 127) / 128, n = min(N, h.T - t0);
    uint2* xs = reinterpret_cast<uint2*>(dyn);                          // [N][4][nb]: doubled codes, eight a piece
    float* xe = reinterpret_cast<float*>(dyn + (size_t)N * nb * 32);    // [N][nb]
    dep_wait();
    dep_launch();
    for (int i = threadIdx.x; i < N * nb * 4; i += ROWS_THREADS) {
        const int t = i / (nb * 4), c = i - t * nb * 4, b = c >> 2;
        const bool there = t < n;
        xs[(t * 4 + (c & 3)) * nb + b] =
            there ? doubled8(*reinterpret_cast<const uint32_t*>(h.q + (size_t)(t0 + t) * h.q_stride + c * 4))
                  : make_uint2(0, 0);
        if (!(c & 3)) xe[t * nb + b] = there ? block_value(h.q_blocks[block_at(t0 + t, b, n_tiles)]) : 0.f;
    }
    __syncthreads();
    float* out = s_out[warp];
    for (int item = blockIdx.x * (ROWS_THREADS / 32) + warp; item < h.W; item += gridDim.x * (ROWS_THREADS / 32)) {
        const int v0 = item * 32, v = v0 + lane;
        const uint32_t mine = lane >= n ? 0u : h.bitmask ? h.bitmask[(size_t)(t0 + lane) * h.W + item] : FULL;
        uint32_t rows = __reduce_or_sync(FULL, mine);
        if (h.V - v0 < 32) rows &= (1u << (h.V - v0)) - 1;
        while (rows) {
            int r[ROWS];
#pragma unroll
            for (int i = 0; i < ROWS; i++) {
                r[i] = __ffs(rows) - 1;             // -1: none left
                rows &= rows - 1;
            }
            float acc[ROWS][N] = {};
            for (int b = lane; b < nb; b += 32) {
                uint4 w[ROWS];
                float e[ROWS];
#pragma unroll
                for (int i = 0; i < ROWS; i++) {
                    w[i] = make_uint4(0, 0, 0, 0);
                    e[i] = 0.f;
                    if (r[i] < 0) continue;
                    w[i] = __ldcs(reinterpret_cast<const uint4*>(h.w + (size_t)(v0 + r[i]) * h.w_stride + b * 16));
                    e[i] = block_value(h.w_blocks[block_at(v0 + r[i], b, n_tiles)]);
                }
#pragma unroll
                for (int i = 0; i < ROWS; i++) {
                    const uint32_t c[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
                    uint2 d[4];
#pragma unroll
                    for (int j = 0; j < 4; j++) d[j] = doubled8(c[j]);
#pragma unroll
                    for (int t = 0; t < N; t++) {
                        int s = 0;
#pragma unroll
                        for (int j = 0; j < 4; j++) {
                            const uint2 x = xs[(t * 4 + j) * nb + b];
                            s = __dp4a((int)d[j].x, (int)x.x, s);
                            s = __dp4a((int)d[j].y, (int)x.y, s);
                        }
                        const float f = xe[t * nb + b];
                        acc[i][t] = fmaf((float)s * 0.25f * min_nan(e[i], f), max_nan(e[i], f), acc[i][t]);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < ROWS; i++)
#pragma unroll
                for (int t = 0; t < N; t++) {
                    float s = acc[i][t];
#pragma unroll
                    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(FULL, s, o);
                    if (lane == 0 && r[i] >= 0) out[t * 32 + r[i]] = s;
                }
        }
        __syncwarp();
        const float sw = v < h.V && h.w_scale ? h.w_scale[v] : 1.f;
        for (int t = 0; t < n; t++) {
            const uint32_t bits = __shfl_sync(FULL, mine, t);
            const float st = h.scale ? h.scale[t0 + t] : 1.f;
            if (v < h.V)
                store_f32(logits + (size_t)(t0 + t) * h.row_stride + v,
                          (bits >> lane) & 1 ? out[t * 32 + lane] * st * sw : __uint_as_float(0xFF800000u));
        }
        __syncwarp();
    }
}

template <typename T, int N>
psc_status head_rows(const Head& h, T* logits, cudaStream_t cs) {
    const int nb = (h.K + 31) / 32;
    for (int t0 = 0; t0 < h.T; t0 += N) {
        psc_status s = ops_launch(k_mx4_rows<T, N>, dim3(std::min((h.W + 7) / 8, current_sms() * 2)), ROWS_THREADS,
                                  (size_t)N * nb * 36, 1, cs, "k_mx4_rows", h, t0, logits);
        if (s != PSC_OK) return s;
    }
    return PSC_OK;
}

template <typename T>
psc_status head(const Head& h, T* logits, uint8_t* work, cudaStream_t cs) {
    psc_status s = ops_check(cudaMemsetAsync(work, 0, 4, cs), "psc_head_logits_mx4");
    if (s != PSC_OK) return s;
    if (h.K <= 4096) return head_rows<T, 16>(h, logits, cs);
    if (h.K <= 32768) return head_rows<T, 4>(h, logits, cs);
    return head_rows<T, 1>(h, logits, cs);
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

int64_t psc_head_mx4_work_bytes(int32_t T, int32_t V, int32_t K) {
    (void)T, (void)V, (void)K;
    return 256;
}

psc_status psc_head_logits_mx4(const uint8_t* d_q, int64_t q_stride, const uint8_t* d_q_blocks, const float* d_scale,
                               int32_t T, const uint8_t* d_w, int64_t w_stride, const uint8_t* d_w_blocks,
                               const float* d_w_scale, int32_t V, int32_t K, const uint32_t* d_bitmask, void* d_logits,
                               psc_dtype dtype, int64_t row_stride, void* d_work, int64_t work_bytes, void* stream) {
    const char* me = "psc_head_logits_mx4";
    if (T < 0 || V <= 0 || K <= 0 || row_stride < V || !is_dtype(dtype) || !d_w || !d_w_blocks ||
        (T && (!d_q || !d_q_blocks || !d_logits)))
        return ops_fail(PSC_ERR_ARG, me, "bad arguments");
    if (K > MAX_K) return ops_fail(PSC_ERR_LIMIT, me, "K over 131,072");
    if (T > MAX_T || V > MAX_V) return ops_fail(PSC_ERR_LIMIT, me, "too many rows");
    if (!is_mx4(d_w, w_stride, d_w_blocks, K) || (T && !is_mx4(d_q, q_stride, d_q_blocks, K)))
        return ops_fail(PSC_ERR_ARG, me, "codes or blocks with a bad stride or alignment");
    if (T == 0) return PSC_OK;
    if (!d_work || (uintptr_t)d_work % 256 || work_bytes < psc_head_mx4_work_bytes(T, V, K))
        return ops_fail(PSC_ERR_ARG, me, "workspace missing, unaligned or too small");
    const Head h{d_q, q_stride, d_q_blocks, d_scale, T, d_w, w_stride, d_w_blocks, d_w_scale, V, K, d_bitmask,
                 (V + 31) / 32, row_stride};
    if (dtype == PSC_BF16) return head(h, (__nv_bfloat16*)d_logits, (uint8_t*)d_work, (cudaStream_t)stream);
    return head(h, (float*)d_logits, (uint8_t*)d_work, (cudaStream_t)stream);
}

}  // extern "C"
