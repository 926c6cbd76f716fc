// psc_norm_quantize_rows and psc_norm_quantize_mx4: the last residual addition, the
// root-mean-square norm, and its output in 8 or 4 bits.
//
// The normalised row is r (h gain) with one number r = 1 / sqrt(mean h^2 + eps) for the whole
// row.  Quantisation by the row's (or a block's) own largest magnitude does not see such a
// factor, so the codes are made of v = h gain and r goes into the row's scale: the codes
// need not wait for the sum of squares, and do not carry its rounding.
#include <cfloat>
#include <cmath>

#include "../../include/psc_norm.h"
#include "mx4.cuh"

namespace {

struct Norm {
    const void* x;
    int64_t x_stride;
    const void* residual;
    int64_t residual_stride;
    void* sum;
    int64_t sum_stride;
    const float* gain;
    float eps;
    int T, K;
    uint8_t* q;
    int64_t q_stride;
    uint8_t* blocks;
    float* scale;
    bool wide, wide_gain, wide_q;               // 16-byte accesses are in place
};

constexpr int NORM_WARPS = 32;

struct RowStats {
    float squares;
    uint32_t h, v;                              // the largest magnitudes' bits
};

// Over the block, the same in every thread; the order of the sum depends on the block's size alone.
__device__ __forceinline__ RowStats over_block(RowStats s) {
    __shared__ float s_squares[NORM_WARPS];
    __shared__ uint32_t s_h[NORM_WARPS], s_v[NORM_WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = blockDim.x >> 5;
#pragma unroll
    for (int o = 16; o; o >>= 1) s.squares += __shfl_xor_sync(FULL, s.squares, o);
    s.h = __reduce_max_sync(FULL, s.h);
    s.v = __reduce_max_sync(FULL, s.v);
    if (n == 1) return s;
    if (lane == 0) s_squares[warp] = s.squares, s_h[warp] = s.h, s_v[warp] = s.v;
    __syncthreads();
    s.squares = lane < n ? s_squares[lane] : 0.f;
    s.h = lane < n ? s_h[lane] : 0u;
    s.v = lane < n ? s_v[lane] : 0u;
#pragma unroll
    for (int o = 16; o; o >>= 1) s.squares += __shfl_xor_sync(FULL, s.squares, o);
    s.h = __reduce_max_sync(FULL, s.h);
    s.v = __reduce_max_sync(FULL, s.v);
    return s;
}

// A block per row, eight columns (a chunk) at a time in a thread.  NV chunks of a thread are kept in
// registers (0: any number, read again for what comes after the sums).
template <typename T, bool MX4, int NV>
__global__ void __launch_bounds__(1024) k_norm(Norm a) {
    const int row = blockIdx.x, chunks = (a.K + 7) / 8;
    dep_wait();
    dep_launch();
    const T* x = (const T*)a.x + (size_t)row * a.x_stride;
    const T* res = a.residual ? (const T*)a.residual + (size_t)row * a.residual_stride : nullptr;
    T* sum = a.sum ? (T*)a.sum + (size_t)row * a.sum_stride : nullptr;
    uint8_t* q = a.q + (size_t)row * a.q_stride;
    auto load_h = [&](int c, float h[8]) {
        load8(x, c * 8, a.K, a.wide, h);
        if (res) {
            float r[8];
            load8(res, c * 8, a.K, a.wide, r);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                h[j] += r[j];
                if (sizeof(T) == 2) h[j] = __bfloat162float(__float2bfloat16_rn(h[j]));    // as the stream holds it
            }
        }
        if (sum) store8(sum, c * 8, a.K, a.wide, h);
    };
    auto load_gain = [&](int c, float g[8]) {
        if (a.gain) load8(a.gain, c * 8, a.K, a.wide_gain, g);
        else
#pragma unroll
            for (int j = 0; j < 8; j++) g[j] = 1.f;
    };
    auto add = [&](const float h[8], const float v[8], RowStats& s) {
#pragma unroll
        for (int j = 0; j < 8; j++) {
            s.squares = fmaf(h[j], h[j], s.squares);
            s.h = max(s.h, magnitude(h[j]));
            s.v = max(s.v, magnitude(v[j]));
        }
    };
    auto store_q = [&](int c, const float v[8], float s) {              // v / s in whole numbers
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const float y = s > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(v[j], s)), -127.f), 127.f) : 0.f;
            w[j >> 2] |= (uint32_t)(uint8_t)(int8_t)(int)y << (8 * (j & 3));
        }
        if (a.wide_q) *reinterpret_cast<uint2*>(q + c * 8) = make_uint2(w[0], w[1]);
        else
#pragma unroll
            for (int j = 0; j < 8; j++)
                if (c * 8 + j < a.K) q[c * 8 + j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
    };

    constexpr int KEPT = NV ? NV : 1;
    float h[KEPT][8], v[KEPT][8];
    RowStats s = {0.f, 0u, 0u};
    // whole warps go round together: a warp's lanes share blocks and tiles
    const int rounds = (chunks + blockDim.x - 1) / blockDim.x;
#pragma unroll
    for (int i = 0; i < (NV ? NV : rounds); i++) {
        const int c = i * blockDim.x + threadIdx.x, at = NV ? i : 0;
        float g[8] = {};
#pragma unroll
        for (int j = 0; j < 8; j++) h[at][j] = 0.f;
        if (c < chunks) load_h(c, h[at]), load_gain(c, g);
#pragma unroll
        for (int j = 0; j < 8; j++) v[at][j] = h[at][j] * g[j];
        add(h[at], v[at], s);
        if (MX4) quantize8(v[at], c, a.K, row, q, a.blocks);
    }
    s = over_block(s);

    const bool bad = s.h >= INF_BITS || s.v >= INF_BITS;
    double r;
    if (!bad && s.h && (s.h > 0x57800000u || s.h < 0x2b800000u)) {
        // beyond 2^48 or below 2^-40 the squares (or r) may leave f32: again, with the largest magnitude near 1
        const int e = max(1, min(253, (int)(s.h >> 23)));
        const float f = __uint_as_float((uint32_t)(254 - e) << 23);
        float again = 0.f;
        for (int i = 0; i < rounds; i++) {
            const int c = i * blockDim.x + threadIdx.x;
            float y[8] = {};
            if (c < chunks) {
                if (NV) {
#pragma unroll
                    for (int n = 0; n < KEPT; n++)
                        if (n == i)
#pragma unroll
                            for (int j = 0; j < 8; j++) y[j] = h[n][j];
                } else if (sum) load8(sum, c * 8, a.K, a.wide, y);
                else load_h(c, y);
            }
#pragma unroll
            for (int j = 0; j < 8; j++) again = fmaf(y[j] * f, y[j] * f, again);
        }
        __syncthreads();
        const RowStats t = over_block({again, 0u, 0u});
        r = 1.0 / sqrt((double)t.squares / a.K / ((double)f * f) + a.eps);
    } else {
        r = __fdiv_rn(1.f, __fsqrt_rn(__fdiv_rn(s.squares, (float)a.K) + a.eps));
    }
    const float nan = __uint_as_float(0x7fc00000u);
    if (MX4) {
        // 1 / sqrt(0): a row of zeros with eps 0
        if (threadIdx.x == 0) a.scale[row] = bad ? nan : s.h == 0 && a.eps == 0.f ? 0.f : (float)r;
        return;
    }
    const float unit = bad ? nan : __fmul_rn(__uint_as_float(s.v), 1.f / 127.f);
    if (threadIdx.x == 0) a.scale[row] = unit == 0.f ? 0.f : (float)(unit * r);
#pragma unroll
    for (int i = 0; i < (NV ? NV : rounds); i++) {
        const int c = i * blockDim.x + threadIdx.x, at = NV ? i : 0;
        if (c >= chunks) break;
        if (!NV) {
            float g[8];
            if (sum) load8(sum, c * 8, a.K, a.wide, h[0]);
            else load_h(c, h[0]);
            load_gain(c, g);
#pragma unroll
            for (int j = 0; j < 8; j++) v[0][j] = h[0][j] * g[j];
        }
        store_q(c, v[at], unit);
    }
}

template <typename T, bool MX4>
psc_status norm(Norm a, const char* me, cudaStream_t cs) {
    a.wide = wide_rows<T>(a.x, a.x_stride, a.K) && wide_rows<T>(a.residual, a.residual_stride, a.K) &&
             wide_rows<T>(a.sum, a.sum_stride, a.K);
    a.wide_gain = wide_rows<float>(a.gain, 0, a.K);
    a.wide_q = a.K % 8 == 0 && is_aligned(a.q, a.q_stride, 8);
    const int chunks = (a.K + 7) / 8;
    const int threads = chunks < 1024 ? (chunks + 31) / 32 * 32 : 1024, rounds = (chunks + threads - 1) / threads;
    auto kernel = rounds == 1 ? k_norm<T, MX4, 1> : rounds == 2 ? k_norm<T, MX4, 2> : k_norm<T, MX4, 0>;
    return ops_launch(kernel, dim3(a.T), threads, 0, 1, cs, me, a);
}

template <bool MX4>
psc_status norm_entry(const char* me, const Norm& a, psc_dtype dtype, void* stream) {
    if (a.T < 0 || a.K <= 0 || !is_dtype(dtype) || a.x_stride < a.K || (a.residual && a.residual_stride < a.K) ||
        (a.sum && a.sum_stride < a.K) || !(a.eps >= 0.f && a.eps <= FLT_MAX) ||
        (a.T && (!a.x || !a.q || !a.scale || (MX4 && !a.blocks))))
        return ops_fail(PSC_ERR_ARG, me, "bad arguments");
    if ((a.sum == a.x && a.sum && a.sum_stride != a.x_stride && a.T > 1) ||
        (a.sum == a.residual && a.sum && a.sum_stride != a.residual_stride && a.T > 1))
        return ops_fail(PSC_ERR_ARG, me, "the sum in place of an input has another stride");
    if (a.K > MAX_QUANTIZE_K) return ops_fail(PSC_ERR_LIMIT, me, "K over 2^30");
    if (MX4 ? !is_mx4(a.q, a.q_stride, a.blocks, a.K) : a.q_stride < a.K)
        return ops_fail(PSC_ERR_ARG, me, "codes or blocks with a bad stride or alignment");
    if (a.T == 0) return PSC_OK;
    if (dtype == PSC_BF16) return norm<__nv_bfloat16, MX4>(a, me, (cudaStream_t)stream);
    return norm<float, MX4>(a, me, (cudaStream_t)stream);
}

}  // namespace

extern "C" {

psc_status psc_norm_quantize_rows(const void* d_x, psc_dtype dtype, int64_t row_stride, const void* d_residual,
                                  int64_t residual_stride, void* d_sum, int64_t sum_stride, const float* d_gain,
                                  float eps, int32_t T, int32_t K, int8_t* d_q, int64_t q_stride, float* d_scale,
                                  void* stream) {
    return norm_entry<false>("psc_norm_quantize_rows",
                             Norm{d_x, row_stride, d_residual, residual_stride, d_sum, sum_stride, d_gain, eps, T, K,
                                  (uint8_t*)d_q, q_stride, nullptr, d_scale, false, false, false},
                             dtype, stream);
}

psc_status psc_norm_quantize_mx4(const void* d_x, psc_dtype dtype, int64_t row_stride, const void* d_residual,
                                 int64_t residual_stride, void* d_sum, int64_t sum_stride, const float* d_gain,
                                 float eps, int32_t T, int32_t K, uint8_t* d_q, int64_t q_stride, uint8_t* d_blocks,
                                 float* d_scale, void* stream) {
    return norm_entry<true>("psc_norm_quantize_mx4",
                            Norm{d_x, row_stride, d_residual, residual_stride, d_sum, sum_stride, d_gain, eps, T, K,
                                 d_q, q_stride, d_blocks, d_scale, false, false, false},
                            dtype, stream);
}

}  // extern "C"
