// psc_quantize_rows and psc_head_logits: the vocabulary projection in 8-bit
// integers with a scale per token and per vocabulary row, under the grammar's mask.
#include <algorithm>

#include "ops_common.cuh"

namespace {

constexpr int MAX_K = 131072;           // K * 127 * 128 stays below 2^31

// One block per row: the largest magnitude, then the quotients.
template <typename T>
__global__ void __launch_bounds__(256) k_quantize_rows(const T* x, int64_t stride, int K, int8_t* q, int64_t q_stride,
                                                       float* scale) {
    __shared__ float s_max[8];
    __shared__ int s_bad[8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    dep_wait();
    dep_launch();
    const T* row = x + (size_t)blockIdx.x * stride;
    float mx = 0.f;
    int bad = 0;
    for (int k = threadIdx.x; k < K; k += blockDim.x) {
        const float a = fabsf(load_f32(row + k));
        bad |= !(a <= 3.402823466e+38f);
        mx = fmaxf(mx, a);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, o));
    bad = __any_sync(FULL, bad);
    if (lane == 0) s_max[warp] = mx, s_bad[warp] = bad;
    __syncthreads();
    for (int w = 0; w < 8; w++) mx = fmaxf(mx, s_max[w]), bad |= s_bad[w];
    const float sc = bad ? __uint_as_float(0x7fc00000u) : __fmul_rn(mx, 1.f / 127.f);
    if (threadIdx.x == 0) scale[blockIdx.x] = sc;
    for (int k = threadIdx.x; k < K; k += blockDim.x) {
        const float v = sc > 0.f ? rintf(__fdiv_rn(load_f32(row + k), sc)) : 0.f;
        q[(size_t)blockIdx.x * q_stride + k] = (int8_t)fminf(fmaxf(v, -127.f), 127.f);
    }
}

struct Head {
    const int8_t* q;
    int64_t q_stride;
    const float* scale;
    int T;
    const int8_t* w;
    int64_t w_stride;
    const float* w_scale;
    int V, K;
    const uint32_t* bitmask;
    int W;
    int64_t row_stride;
};

// Integer dot products at any alignment: a block per 64 tokens x 64 vocabulary
// rows, 4 x 4 sums a thread, 64 bytes of K at a time through shared memory.
template <typename T>
__global__ void __launch_bounds__(256) k_head_dot(Head h, T* logits, int aligned4) {
    constexpr int TILE = 64, KB = 16, LD = KB + 1;      // words of K per step; odd row length: no bank conflicts
    __shared__ int sw[TILE * LD], sq[TILE * LD];
    dep_wait();
    dep_launch();
    const int v0 = blockIdx.x * TILE, t0 = blockIdx.y * TILE;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    int any = !h.bitmask;
    if (h.bitmask && threadIdx.x < TILE * 2) {
        const int t = t0 + (threadIdx.x >> 1), wi = (v0 >> 5) + (threadIdx.x & 1);
        any = t < h.T && wi < h.W && h.bitmask[(size_t)t * h.W + wi] != 0;
    }
    any = __syncthreads_or(any);
    int acc[4][4] = {};
    auto load = [&](int* dst, const int8_t* src, int64_t stride, int r0, int rows, int k0) {
        for (int i = threadIdx.x; i < TILE * KB; i += 256) {
            const int r = i / KB, k = k0 + (i % KB) * 4;
            int word = 0;
            if (r0 + r < rows && k < h.K) {
                const int8_t* p = src + (size_t)(r0 + r) * stride + k;
                if (aligned4 && k + 4 <= h.K) word = *reinterpret_cast<const int*>(p);
                else
                    for (int j = 0; j < 4 && k + j < h.K; j++) word |= (int)(uint8_t)p[j] << (8 * j);
            }
            dst[r * LD + i % KB] = word;
        }
    };
    if (any) {
        for (int k0 = 0; k0 < h.K; k0 += KB * 4) {
            load(sw, h.w, h.w_stride, v0, h.V, k0);
            load(sq, h.q, h.q_stride, t0, h.T, k0);
            __syncthreads();
#pragma unroll
            for (int k = 0; k < KB; k++) {
                int a[4], c[4];
#pragma unroll
                for (int i = 0; i < 4; i++) a[i] = sw[(tx + 16 * i) * LD + k], c[i] = sq[(ty + 16 * i) * LD + k];
#pragma unroll
                for (int i = 0; i < 4; i++)
#pragma unroll
                    for (int j = 0; j < 4; j++) acc[i][j] = __dp4a(a[i], c[j], acc[i][j]);
            }
            __syncthreads();
        }
    }
    for (int j = 0; j < 4; j++) {
        const int t = t0 + ty + 16 * j;
        if (t >= h.T) break;
        const float st = h.scale[t];
        const uint32_t* mask = h.bitmask ? h.bitmask + (size_t)t * h.W : nullptr;
        for (int i = 0; i < 4; i++) {
            const int v = v0 + tx + 16 * i;
            if (v >= h.V) continue;
            const float y = allows(mask, v) ? (float)acc[i][j] * st * h.w_scale[v] : __uint_as_float(0xFF800000u);
            store_f32(logits + (size_t)t * h.row_stride + v, y);
        }
    }
}

template <typename T>
psc_status head(const Head& h, T* logits, cudaStream_t cs) {
    const int aligned4 = is_aligned(h.w, h.w_stride, 4) && is_aligned(h.q, h.q_stride, 4);
    return ops_launch(k_head_dot<T>, dim3((h.V + 63) / 64, (h.T + 63) / 64), 256, 0, 1, cs, "k_head_dot", h, logits,
                      aligned4);
}

}  // namespace

extern "C" {

psc_status psc_quantize_rows(const void* d_x, psc_dtype dtype, int64_t row_stride, int32_t T, int32_t K, int8_t* d_q,
                             int64_t q_stride, float* d_scale, void* stream) {
    const char* me = "psc_quantize_rows";
    if (T < 0 || K <= 0 || row_stride < K || q_stride < K || !is_dtype(dtype) || (T && (!d_x || !d_q || !d_scale)))
        return ops_fail(PSC_ERR_ARG, me, "bad arguments");
    if (T == 0) return PSC_OK;
    cudaStream_t cs = (cudaStream_t)stream;
    if (dtype == PSC_BF16)
        return ops_launch(k_quantize_rows<__nv_bfloat16>, dim3(T), 256, 0, 1, cs, "k_quantize_rows",
                          (const __nv_bfloat16*)d_x, row_stride, K, d_q, q_stride, d_scale);
    return ops_launch(k_quantize_rows<float>, dim3(T), 256, 0, 1, cs, "k_quantize_rows", (const float*)d_x, row_stride,
                      K, d_q, q_stride, d_scale);
}

int64_t psc_head_work_bytes(int32_t T, int32_t V, int32_t K) {
    (void)T, (void)V, (void)K;
    return 256;
}

psc_status psc_head_logits(const int8_t* d_q, int64_t q_stride, const float* d_scale, int32_t T, const int8_t* d_w,
                           int64_t w_stride, const float* d_w_scale, int32_t V, int32_t K, const uint32_t* d_bitmask,
                           void* d_logits, psc_dtype dtype, int64_t row_stride, void* d_work, int64_t work_bytes,
                           void* stream) {
    const char* me = "psc_head_logits";
    if (T < 0 || V <= 0 || K <= 0 || q_stride < K || w_stride < K || row_stride < V || !is_dtype(dtype) || !d_w ||
        !d_w_scale || (T && (!d_q || !d_scale || !d_logits)))
        return ops_fail(PSC_ERR_ARG, me, "bad arguments");
    if (K > MAX_K) return ops_fail(PSC_ERR_LIMIT, me, "K over 131,072");
    if (T > 65535 * 64) return ops_fail(PSC_ERR_LIMIT, me, "too many rows");
    if (T == 0) return PSC_OK;
    if (!d_work || (uintptr_t)d_work % 256 || work_bytes < psc_head_work_bytes(T, V, K))
        return ops_fail(PSC_ERR_ARG, me, "workspace missing, unaligned or too small");
    const Head h{d_q, q_stride, d_scale, T, d_w, w_stride, d_w_scale, V, K, d_bitmask, (V + 31) / 32, row_stride};
    if (dtype == PSC_BF16) return head(h, (__nv_bfloat16*)d_logits, (cudaStream_t)stream);
    return head(h, (float*)d_logits, (cudaStream_t)stream);
}

}  // extern "C"
