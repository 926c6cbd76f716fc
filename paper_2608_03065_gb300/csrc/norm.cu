// psc_norm_quantize_rows and psc_norm_quantize_mx4: the last residual addition, the
// root-mean-square norm, and its output in 8 or 4 bits.
//
// The normalised row is r (h gain) with one number r = 1 / sqrt(mean h^2 + eps) for the whole
// row.  Quantisation by the row's (or a block's) own largest magnitude does not see such a
// factor, so the codes are made of v = h gain and r goes into the row's scale: the codes
// need not wait for the sum of squares, and do not carry its rounding.
#include <algorithm>
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
    float most;                                 // sums of squares up to which their mean with eps stays in f32
};

struct RowStats {
    float squares;                              // of h
    uint32_t top;                               // the largest magnitude's bits (of v, in the first pass)
};

// Over the block, the same in every thread.
__device__ __forceinline__ void over_warp(RowStats& s) {
#pragma unroll
    for (int o = 16; o; o >>= 1) s.squares += __shfl_xor_sync(FULL, s.squares, o);
    s.top = __reduce_max_sync(FULL, s.top);
}
// Of n warps, which have over_warp's.  turn: counts a block's calls (what one reads, the next but one writes).
__device__ __forceinline__ void over_warps(RowStats& s, int n, int turn) {
    __shared__ RowStats s_both[2][32];
    RowStats* s_all = s_both[turn & 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (n == 1 && blockDim.x == 32) return;
    if (lane == 0 && warp < n) s_all[warp] = s;
    __syncthreads();
    s = lane < n ? s_all[lane] : RowStats{0.f, 0u};
    over_warp(s);
}
// The same where SHARES threads stand for each of a smaller block (and have a chunk each of what it would have),
// the sums in its order.
template <int SHARES>
__device__ __forceinline__ void over_block(RowStats& s, int turn) {
    const int warps = blockDim.x / 32 / SHARES;
    if (SHARES > 1) {
        __shared__ float s_squares[1024];
        __shared__ uint32_t s_top[32];
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = blockDim.x / SHARES;
        s_squares[threadIdx.x] = s.squares;
        s.top = __reduce_max_sync(FULL, s.top);
        if (lane == 0) s_top[warp] = s.top;
        __syncthreads();
        const int at = threadIdx.x % n;
        s.squares = s_squares[at];
#pragma unroll
        for (int i = 1; i < SHARES; i++) s.squares += s_squares[at + i * n];
        s.top = lane < (int)blockDim.x / 32 ? s_top[lane] : 0u;
    }
    over_warp(s);
    if (SHARES == 1 || warps > 1) over_warps(s, warps, turn);
}

// How a kernel's chunks lie: WIDE, whole and aligned; SHIFTED, at columns 8 c - shift (load8_at); BLOCKS, at columns
// 8 c as the blocks of 32 columns ask for, aligned or not.
enum Chunks { WIDE, SHIFTED, BLOCKS };

// A row of the inputs, a chunk (eight columns from k on) at a time; all lanes of a warp call these.
template <typename T, Chunks C>
struct Row {
    const T *x, *residual;
    T* sum;
    uint8_t* q;
    const float* gain;
    int K, shift;
    bool in_place;
    __device__ __forceinline__ Row(const Norm& a, int row, int width)
        : x((const T*)a.x + (size_t)row * a.x_stride),
          residual(a.residual ? (const T*)a.residual + (size_t)row * a.residual_stride : nullptr),
          sum(a.sum ? (T*)a.sum + (size_t)row * a.sum_stride : nullptr), q(a.q + (size_t)row * a.q_stride), gain(a.gain),
          K(width), shift(0), in_place(true) {
        if (C != SHIFTED) return;
        shift = row_shift(x);
        in_place = (!residual || row_shift(residual) == shift) && (!sum || row_shift(sum) == shift) &&
                   row_shift(q) == shift;
    }
    __device__ __forceinline__ int column(int c) const { return C == SHIFTED ? c * 8 - shift : c * 8; }
    __device__ __forceinline__ void load(const T* from, int k, float h[8]) const {
        if (C == SHIFTED) load8_at(from, k, K, in_place, h);
        else load8<C == WIDE>(from, k, K, h);
    }
    // h; again: the second time, when the sum may have replaced an input
    __device__ __forceinline__ void load_h(int k, float h[8], bool again = false) const {
#pragma unroll
        for (int j = 0; j < 8; j++) h[j] = 0.f;
        if (k >= K) return;
        if (again && sum) return load(sum, k, h);
        load(x, k, h);
        if (residual) {
            float r[8];
            load(residual, k, r);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                h[j] += r[j];
                if (sizeof(T) == 2) h[j] = __bfloat162float(__float2bfloat16_rn(h[j]));       // as the stream holds it
            }
        }
    }
    __device__ __forceinline__ void store_h(int k, const float h[8]) const {
        if (!sum) return;
        if (C == SHIFTED) {
            if (k < K) store8_at(sum, k, K, in_place, h);
        } else {
            store8<C == WIDE>(sum, k, K, h, k < K, k > 0);
        }
    }
    __device__ __forceinline__ void load_gain(int k, float g[8]) const {
#pragma unroll
        for (int j = 0; j < 8; j++) g[j] = 1.f;
        if (!gain || k >= K) return;
        if (C == SHIFTED && k < 0) load8_at(gain, k, K, false, g);
        else load8<C == WIDE>(gain, k, K, g);
    }
    __device__ __forceinline__ void store_codes(int k, uint2 w) const {
        if (k >= K) return;
        if (C == WIDE || (in_place && k >= 0 && k + 8 <= K)) {
            *reinterpret_cast<uint2*>(q + k) = w;
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++)
                if (k + j >= 0 && k + j < K) q[k + j] = (uint8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
        }
    }
};

// What a row's sums give.
struct Factor {
    float unit;                                 // of the 8-bit codes; NaN: the row is not finite
    float scale;                                // the row's, for 8 or for 4 bits
};
// again(f): this thread's part of the sum of (h f)^2, and the largest |h f|.
template <bool MX4, int SHARES, typename Again>
__device__ __forceinline__ Factor factor_of(const Norm& a, const RowStats& s, int& turn, Again again) {
    const float unit = s.top >= INF_BITS ? __uint_as_float(0x7fc00000u) : __fmul_rn(__uint_as_float(s.top), 1.f / 127.f);
    if (isnan(unit)) return {unit, unit};
    if (s.squares >= 0x1p-76f && s.squares <= a.most) {
        const float r = __fdiv_rn(1.f, __fsqrt_rn(__fdiv_rn(s.squares, (float)a.K) + a.eps));
        return {unit, MX4 ? r : unit * r};
    }
    // the squares, their mean with eps, or r, may leave f32 (squares of less than 2^-126 lose bits, but not of a sum from 2^-76
    // on): once more, with the largest magnitude near 1.  It reads the sums again, of which a lane may have stored
    // another's (store_shifted), and no barrier need have come since in a block of one warp.
    __syncthreads();
    RowStats t = again(1.f);
    __syncthreads();
    over_block<SHARES>(t, turn++);
    const int e = max(1, min(253, (int)(t.top >> 23)));
    const bool zeros = t.top == 0;
    const float f = __uint_as_float((uint32_t)(254 - e) << 23);
    t = again(f);
    __syncthreads();
    over_block<SHARES>(t, turn++);
    const double r = 1.0 / sqrt((double)t.squares / a.K / ((double)f * f) + a.eps);
    // a row of zeros with eps 0, or of no unit: 0, not the product with an infinite r
    if (MX4) return {unit, zeros && a.eps == 0.f ? 0.f : (float)r};
    return {unit, unit == 0.f ? 0.f : (float)(unit * r)};
}

// Eight codes v / unit in two words.  A quotient within 127 is v * inverse to 2^-16 (inverse is the rounded
// 1 / unit, 2^-24 of it off, and the quotient has its own rounding), so the nearest whole number to that product is
// the code unless the product is that close to a half; it is rounded to a whole number by adding 1.5 * 2^23,
// whose low byte then is the code.
__device__ __forceinline__ uint2 codes_of(const float v[8], float unit, float inverse) {
    constexpr float BIG = 12582912.f, NEAR = 0.5f - 0x1p-15f;
    uint32_t w[8];
    bool sure = true;
#pragma unroll
    for (int j = 0; j < 8; j++) {
        const float m = fmaf(v[j], inverse, BIG);
        sure &= fabsf(fmaf(v[j], inverse, BIG - m)) <= NEAR;
        w[j] = __float_as_uint(m);
    }
    if (!sure)                                  // near a half, or the unit is 0 or NaN or has no inverse
#pragma unroll
        for (int j = 0; j < 8; j++)
            w[j] = unit > 0.f ? (uint32_t)(int)fminf(fmaxf(rintf(__fdiv_rn(v[j], unit)), -127.f), 127.f) : 0u;
    return make_uint2(__byte_perm(__byte_perm(w[0], w[1], 0x0040), __byte_perm(w[2], w[3], 0x0040), 0x5410),
                      __byte_perm(__byte_perm(w[4], w[5], 0x0040), __byte_perm(w[6], w[7], 0x0040), 0x5410));
}

// h of a chunk from its words.
__device__ __forceinline__ void unpack_h(const uint32_t (&x)[4], const uint32_t (&r)[4], bool residual, float h[8],
                                         const __nv_bfloat16*) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; j++) {
        // a sum of two bf16 rounded to bf16 at once is the one rounded to f32 on the way: where that rounding is
        // not exact, the smaller is below 2^-16 of the larger, and the sum far from where bf16's rounding turns
        __nv_bfloat162 s = *reinterpret_cast<const __nv_bfloat162*>(&x[j]);
        if (residual) s = __hadd2_rn(s, *reinterpret_cast<const __nv_bfloat162*>(&r[j]));
        w[j] = *reinterpret_cast<const uint32_t*>(&s);
    }
    unpack8(w, h, (const __nv_bfloat16*)nullptr);
}
__device__ __forceinline__ void unpack_h(const uint32_t (&x)[8], const uint32_t (&r)[8], bool residual, float h[8],
                                         const float*) {
#pragma unroll
    for (int j = 0; j < 8; j++) h[j] = residual ? __uint_as_float(x[j]) + __uint_as_float(r[j]) : __uint_as_float(x[j]);
}

// Many aligned rows: blocks stay and go from row to row, and each thread copies its chunks of the next `stages`
// rows into shared memory ahead (cp.async; nobody else reads them, so that only their own thread waits).  In k_norm
// a block's loads all come at its beginning, and half of its time nothing is under way: 16,384 rows of
// 4,096 bf16 columns with residual 114 us, this way 75.  FULL_ROWS: every thread has its four chunks (rows of whole
// multiples of 1,024 columns), which leaves out checks where instructions bound it: without residual
// 62.0 us with this and the residual known at run time only, 48.9 this way; into 4 bits with residual, and back, 111 and
// 105 (there alone 71, with 93 % of its bytes at a copy's rate; without residual 50, half of it instructions).
template <typename T, bool MX4, bool RESIDUAL, bool FULL_ROWS>
__global__ void __launch_bounds__(768, 1) k_norm_many(Norm a, int stages) {
    constexpr int NV = 4, N = sizeof(T) * 2, PIECES = N / 4;           // words, 16-byte pieces of a chunk
    constexpr int parts = RESIDUAL ? 2 : 1;
    extern __shared__ uint4 s_ring[];
    const int step = blockDim.x, chunks = FULL_ROWS ? NV * step : a.K / 8, K = chunks * 8;
    dep_wait();
    dep_launch();
    // a thread's pieces of a stage, one of each thread after the other
    auto place = [&](int stage, int part, int i, int piece) {
        return s_ring + stage * (parts * NV * PIECES * step) + threadIdx.x + ((part * NV + i) * PIECES + piece) * step;
    };
    auto copy = [&](int stage, uint32_t r) {
        if (r < (uint32_t)a.T) {
            const T* x = (const T*)a.x + (size_t)r * a.x_stride + threadIdx.x * 8;
            const T* residual = RESIDUAL ? (const T*)a.residual + (size_t)r * a.residual_stride + threadIdx.x * 8 : nullptr;
#pragma unroll
            for (int i = 0; i < NV; i++) {
                if (!FULL_ROWS && i * step + (int)threadIdx.x >= chunks) break;
#pragma unroll
                for (int part = 0; part < parts; part++)
#pragma unroll
                    for (int piece = 0; piece < PIECES; piece++)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(
                                         (uint32_t)__cvta_generic_to_shared(place(stage, part, i, piece))),
                                     "l"((const char*)((part ? residual : x) + i * step * 8) + 16 * piece)
                                     : "memory");
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto read = [&](int stage, int part, int i, uint32_t (&w)[N]) {
#pragma unroll
        for (int piece = 0; piece < PIECES; piece++) {
            const uint4 x = *place(stage, part, i, piece);
            w[4 * piece] = x.x, w[4 * piece + 1] = x.y, w[4 * piece + 2] = x.z, w[4 * piece + 3] = x.w;
        }
    };
    for (int i = 0; i < stages; i++) copy(i, blockIdx.x + i * gridDim.x);
    int stage = 0, turn = 0;
    for (uint32_t r = blockIdx.x; r < (uint32_t)a.T; r += gridDim.x, stage = stage + 1 == stages ? 0 : stage + 1) {
        const Row<T, WIDE> row(a, r, K);
        uint8_t* blocks = MX4 ? a.blocks + block_at(r, 0, (a.K + 127) / 128) : nullptr;
        // this row's copies, the oldest of `stages` groups
        if (stages == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else if (stages == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
        else asm volatile("cp.async.wait_group 3;" ::: "memory");
        float v[NV][8];
        RowStats s = {0.f, 0u};
        float top = 0.f;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int c = i * step + threadIdx.x;
            uint32_t x[N] = {}, res[N] = {};
            if (FULL_ROWS || c < chunks) {
                read(stage, 0, i, x);
                if (parts == 2) read(stage, 1, i, res);
            }
            unpack_h(x, res, parts == 2, v[i], (const T*)nullptr);
            float g[8], squares = 0.f;
            row.load_gain(c * 8, g);
            row.store_h(c * 8, v[i]);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                squares = fmaf(v[i][j], v[i][j], squares);
                v[i][j] *= g[j];
            }
            s.squares += squares;
            const float most = largest8(v[i], top);
            if (MX4) bad |= quantize8<FULL_ROWS>(v[i], most, c, K, row.q, blocks);
            else top = most;
        }
        copy(stage, r + stages * gridDim.x);
        s.top = MX4 ? (bad ? INF_BITS : 0u) : __float_as_uint(top) & 0x7fffffffu;
        over_block<1>(s, turn++);
        const Factor f = factor_of<MX4, 1>(a, s, turn, [&](float by) {
            RowStats t = {0.f, 0u};
            for (int c = threadIdx.x; c < chunks; c += step) {
                float h[8], part = 0.f;
                row.load_h(c * 8, h, true);
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    part = fmaf(h[j] * by, h[j] * by, part);
                    t.top = max(t.top, __float_as_uint(h[j] * by) & 0x7fffffffu);
                }
                t.squares += part;
            }
            return t;
        });
        if (threadIdx.x == 0) a.scale[r] = f.scale;
        if (MX4) continue;
        const float inverse = __fdiv_rn(1.f, f.unit);
#pragma unroll
        for (int i = 0; i < NV; i++) row.store_codes((i * step + threadIdx.x) * 8, codes_of(v[i], f.unit, inverse));
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// A block per row, NV chunks of it in a thread's registers (0: any number, read again for what comes after
// the sums).  Small blocks whose threads have four chunks each keep most loads under way (16,384 rows of 4,096
// bf16 columns: 128 threads 111 us, 512 threads 141); where there are too few rows for that, four times as many
// threads, a chunk each, are done sooner (2,048 columns with residual: 1 row 4.1 us with 64 threads, 1.9 with 256;
// 600 rows 5.0 and 3.2).  Both add up in the same order (SHARES).
template <typename T, bool MX4, Chunks C, int NV, int SHARES, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) k_norm(Norm a) {
    dep_wait();
    dep_launch();
    const Row<T, C> row(a, blockIdx.x, a.K);
    const int chunks = (a.K + row.shift + 7) / 8;
    // whole warps go round together: a warp's lanes share blocks and tiles
    const int rounds = NV ? NV : (chunks + blockDim.x - 1) / blockDim.x;
    constexpr int KEPT = NV ? NV : 1;
    float v[KEPT][8];
    RowStats s = {0.f, 0u};
    float top = 0.f;
    bool bad = false;
    uint8_t* blocks = MX4 ? a.blocks + block_at(blockIdx.x, 0, (a.K + 127) / 128) : nullptr;
    auto column = [&](int i) { return row.column(i * blockDim.x + threadIdx.x); };
#pragma unroll
    for (int i = 0; i < (NV ? NV : 0); i++) row.load_h(column(i), v[i]);       // all on their way before any is used
#pragma unroll
    for (int i = 0; i < rounds; i++) {
        const int k = column(i), at = NV ? i : 0;
        float g[8], squares = 0.f;
        if (!NV) row.load_h(k, v[0]);
        row.load_gain(k, g);
        row.store_h(k, v[at]);
#pragma unroll
        for (int j = 0; j < 8; j++) {
            squares = fmaf(v[at][j], v[at][j], squares);
            v[at][j] *= g[j];
        }
        s.squares += squares;
        const float most = largest8(v[at], top);
        if (MX4) bad |= quantize8(v[at], most, k / 8, a.K, row.q, blocks);
        else top = most;
    }
    s.top = MX4 ? (bad ? INF_BITS : 0u) : __float_as_uint(top) & 0x7fffffffu;
    int turn = 0;
    over_block<SHARES>(s, turn++);
    const Factor f = factor_of<MX4, SHARES>(a, s, turn, [&](float by) {
        RowStats t = {0.f, 0u};
        for (int i = 0; i * (int)blockDim.x < chunks; i++) {
            float h[8], part = 0.f;
            row.load_h(column(i), h, true);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                part = fmaf(h[j] * by, h[j] * by, part);
                t.top = max(t.top, __float_as_uint(h[j] * by) & 0x7fffffffu);
            }
            t.squares += part;
        }
        return t;
    });
    if (threadIdx.x == 0) a.scale[blockIdx.x] = f.scale;
    if (MX4) return;
    const float inverse = __fdiv_rn(1.f, f.unit);
#pragma unroll
    for (int i = 0; i < rounds; i++) {
        const int k = column(i), at = NV ? i : 0;
        if (!NV) {
            float g[8];
            row.load_h(k, v[0], true);
            row.load_gain(k, g);
#pragma unroll
            for (int j = 0; j < 8; j++) v[0][j] *= g[j];
        }
        row.store_codes(k, codes_of(v[at], f.unit, inverse));
    }
}

constexpr int RING_BYTES = 200 * 1024;            // of an SM's shared memory, for rows under way

template <typename T, bool MX4, Chunks C>
psc_status norm(const Norm& a, const char* me, cudaStream_t cs) {
    // a thread's share goes by the width and by where x's rows start (a chunk more where those are shifted), and so do
    // the sums' orders; not by how the other tensors lie
    const bool shifted = C == SHIFTED && !wide_rows<T>(a.x, a.x_stride, a.K);
    const int chunks = (a.K + (shifted ? 14 : 7)) / 8, quarter = (chunks + 3) / 4;
    const int threads = quarter < 1024 ? (quarter + 31) / 32 * 32 : 1024;
    // a chunk a thread while that fits the GPU at once (1024 threads an SM)
    if (threads <= 256 && (int64_t)a.T * 4 * threads <= 1024ll * current_sms())
        return ops_launch(k_norm<T, MX4, C, 1, 4, 1024>, dim3(a.T), 4 * threads, 0, 1, cs, me, a);
    if (C == WIDE && threads <= 512) {
        // as many blocks as registers leave room for, as many rows ahead as shared memory does; into 8 bits with a
        // residual memory bounds many rows, and fewer blocks with more rows ahead are faster (768 and 512 threads an SM:
        // 16,384 rows of 4,096 bf16 columns 77.8 and 75.2 us, 65,536 of 2,048 157 and 143; without the residual
        // 48.9 and 67.0, into 4 bits and back with it 104.7 and 113.6;
        // few rows a block: 8,192 of 2,048 with residual 22.2 and 23.1)
        const int stage = threads * 4 * 8 * (int)sizeof(T) * (a.residual ? 2 : 1);
        const bool fewer = a.residual && !MX4 && a.T >= 8 * (768 / threads) * current_sms();
        const int most = std::max(1, (fewer ? 512 : 768) / threads);
        const int blocks = std::max(1, std::min(most, RING_BYTES / (2 * stage))), stages = std::min(4, RING_BYTES / (blocks * stage));
        if (stages >= 2 && a.T >= 2 * blocks * current_sms())
            return ops_launch(!a.residual          ? chunks == 4 * threads ? k_norm_many<T, MX4, false, true>
                                                                           : k_norm_many<T, MX4, false, false>
                              : chunks == 4 * threads ? k_norm_many<T, MX4, true, true>
                                                      : k_norm_many<T, MX4, true, false>,
                              dim3(blocks * current_sms()), threads, (size_t)stages * stage, 1, cs, me, a, stages);
    }
    return ops_launch(threads <= 256         ? k_norm<T, MX4, C, 4, 1, 256>
                      : chunks <= 4 * threads ? k_norm<T, MX4, C, 4, 1, 1024>
                                              : k_norm<T, MX4, C, 0, 1, 1024>,
                      dim3(a.T), threads, 0, 1, cs, me, a);
}

template <typename T, bool MX4>
psc_status norm(const Norm& a, const char* me, cudaStream_t cs) {
    const bool wide = wide_rows<T>(a.x, a.x_stride, a.K) && wide_rows<T>(a.residual, a.residual_stride, a.K) &&
                      wide_rows<T>(a.sum, a.sum_stride, a.K) && wide_rows<float>(a.gain, 0, a.K) && a.K % 8 == 0 &&
                      is_aligned(a.q, a.q_stride, 8);
    return wide ? norm<T, MX4, WIDE>(a, me, cs) : norm<T, MX4, MX4 ? BLOCKS : SHIFTED>(a, me, cs);
}

template <bool MX4>
psc_status norm_entry(const char* me, Norm a, psc_dtype dtype, void* stream) {
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
    if (!is_whole(a.x, dtype) || !is_whole(a.residual, dtype) || !is_whole(a.sum, dtype) || (uintptr_t)a.gain % 4 ||
        (uintptr_t)a.scale % 4)
        return ops_fail(PSC_ERR_ARG, me, "an address that is no multiple of its elements' size");
    if (a.T == 0) return PSC_OK;
    a.most = a.eps <= 0x1p126f ? 0x1p126f : 0.f;
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
                                  (uint8_t*)d_q, q_stride, nullptr, d_scale, 0.f},
                             dtype, stream);
}

psc_status psc_norm_quantize_mx4(const void* d_x, psc_dtype dtype, int64_t row_stride, const void* d_residual,
                                 int64_t residual_stride, void* d_sum, int64_t sum_stride, const float* d_gain,
                                 float eps, int32_t T, int32_t K, uint8_t* d_q, int64_t q_stride, uint8_t* d_blocks,
                                 float* d_scale, void* stream) {
    return norm_entry<true>("psc_norm_quantize_mx4",
                            Norm{d_x, row_stride, d_residual, residual_stride, d_sum, sum_stride, d_gain, eps, T, K,
                                 d_q, q_stride, d_blocks, d_scale, 0.f},
                            dtype, stream);
}

}  // extern "C"
