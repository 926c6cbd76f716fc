// psc_quantize_rows and psc_head_logits: the vocabulary projection in 8-bit
// integers with a scale per token and per vocabulary row, under the grammar's mask.
//
// The product is sum_k q[t][k] w[v][k] over whole numbers of 8 bits.  This GPU's
// integer tensor rate is far below its 16-bit one, and whole numbers up to 2^11 are
// exact in f16, so the tensor cores take both operands as f16 and add in f32: the
// sums are those of the integers while they stay below 2^24.  What it has to move
// is the weights, one byte each, so they stay bytes up to the SM and are widened
// there, on the way from the TMA's buffers to the tensor core's.
#include <cuda_fp16.h>

#include <algorithm>

#include "tcgen05.cuh"

namespace {

constexpr int MAX_K = 131072;           // K * 127 * 128 stays below 2^31
constexpr int MAX_V = 1 << 30, MAX_T = 1 << 24;     // and numbers of rows, rounded up to tiles, too
constexpr int MAX_QUANTIZE_K = 1 << 30;

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
    int W;                              // mask words of a row here, and from row to row
    int mask_stride;
    int64_t row_stride;
    int first;                          // the call's first slab: the fault word starts at 0
};

// Sixteen bytes at any address, of which the first n (if fewer) are there; zeros behind them.
__device__ __forceinline__ uint4 load_bytes(const int8_t* p, int n) {
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 16; j++)
        if (j < n) w[j >> 2] |= (uint32_t)(uint8_t)p[j] << (8 * (j & 3));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Rows at any address -> rows of `pitch` bytes (a multiple of 16) at aligned ones, zeros past
// K: a warp per row, 16 bytes a lane, put together from the two aligned pieces that hold
// them.  [begin, end) are the source's bytes; pieces that are not all inside go byte by byte.
__global__ void __launch_bounds__(256) k_pack_rows(const int8_t* w, int64_t stride, int rows, int K, int pitch,
                                                   const int8_t* begin, const int8_t* end, int8_t* out) {
    const int lane = threadIdx.x & 31, n_warps = gridDim.x * 8;
    dep_wait();
    dep_launch();
    for (int r = blockIdx.x * 8 + (threadIdx.x >> 5); r < rows; r += n_warps) {
        const int8_t* row = w + (size_t)r * stride;
        const int off = (int)((uintptr_t)row & 15);
        const int8_t* base = row - off;
        for (int c0 = 0; c0 < pitch / 16; c0 += 32) {
            const int c = c0 + lane, left = K - c * 16;
            const int8_t* at = base + c * 16;
            uint4 v;
            if (off && left >= 16 && at >= begin && at + 32 <= end) {
                const uint4 a = *reinterpret_cast<const uint4*>(at), b = *reinterpret_cast<const uint4*>(at + 16);
                const uint32_t x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
                const int words = off >> 2, bits = 8 * (off & 3);
                uint32_t y[5];
#pragma unroll
                for (int i = 0; i < 5; i++)
                    y[i] = words == 0 ? x[i] : words == 1 ? x[i + 1] : words == 2 ? x[i + 2] : i < 4 ? x[i + 3] : x[7];
                v = make_uint4(__funnelshift_r(y[0], y[1], bits), __funnelshift_r(y[1], y[2], bits),
                               __funnelshift_r(y[2], y[3], bits), __funnelshift_r(y[3], y[4], bits));
            } else {
                v = off == 0 && left >= 16 ? *reinterpret_cast<const uint4*>(at) : load_bytes(row + c * 16, left);
            }
            if (c < pitch / 16) *reinterpret_cast<uint4*>(out + (size_t)r * pitch + c * 16) = v;
        }
    }
}

// ------------------------------------------------------------------ few tokens
//
// k_head_rows: a warp per 4 vocabulary rows, integer dot products of their bytes (a lane's
// 16 at once) with up to N tokens in shared memory.  With few tokens the weights' bytes are
// all that counts; a tensor core would spend its time on 128-row operands that hardly any
// column uses (about 56 cycles per product of 16 columns of K, whatever N).  Under a mask,
// rows that no token allows are not read.  Measured without a mask on 128,256 x 2048 (with
// k_head_mma in brackets): 1 token 45 us (64), 4 tokens 49 (62), 8 tokens 71 (62).  One token
// over 262,144 x 4096: 167 us, 6.4 TB/s.
constexpr int ROWS = 4;
constexpr int ROWS_THREADS = 256;
constexpr int ROWS_X_MAX = 64 * 1024;         // bytes of tokens held in shared memory

// Whether a mask leaves so few rows (up to a quarter) that reading them one by one wins:
// 16 tokens over 128,256 x 2048 take 174 us by rows and 64 us by k_head_mma when all are
// needed, 17 and 47 us when some 300 are.  flags: of every tile, the rows that some token allows.
__device__ __forceinline__ bool few_rows(const uint8_t* flags, int n_tiles, int V) {
    int sum = 0;
    for (int i = threadIdx.x; i < n_tiles; i += blockDim.x) sum += flags[i];
    __shared__ int s_sum[32];
    sum = __reduce_add_sync(FULL, sum);
    if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
    __syncthreads();
    sum = __reduce_add_sync(FULL, (threadIdx.x & 31) < blockDim.x / 32 ? s_sum[threadIdx.x & 31] : 0);
    return 4 * (int64_t)sum <= V;
}

template <typename T, int N, bool MASKED>
__global__ void __launch_bounds__(ROWS_THREADS) k_head_rows(Head h, T* logits, int* faults, const uint8_t* flags,
                                                            int n_tiles) {
    constexpr int WIDTH = MASKED ? 32 : ROWS;           // vocabulary rows of a warp's item
    extern __shared__ __align__(16) uint8_t dyn[];
    __shared__ float s_out[ROWS_THREADS / 32][N * WIDTH];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int chunks = (h.K + 15) / 16;                 // 16-byte pieces of a row
    uint4* xs = reinterpret_cast<uint4*>(dyn);          // [N][chunks], zero past K and T
    dep_wait();
    dep_launch();
    if (flags && !few_rows(flags, n_tiles, h.V)) return;        // k_head_mma's
    if (!flags && h.first && blockIdx.x == 0 && threadIdx.x == 0) *faults = 0;
    for (int i = threadIdx.x; i < N * chunks; i += ROWS_THREADS) {
        const int t = i / chunks, k = (i - t * chunks) * 16;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (t < h.T) {
            const int8_t* p = h.q + (size_t)t * h.q_stride + k;
            x = k + 16 <= h.K && !((uintptr_t)p & 15) ? *reinterpret_cast<const uint4*>(p) : load_bytes(p, h.K - k);
        }
        xs[i] = x;
    }
    __syncthreads();
    // a row's last piece past K: within its stride, except perhaps in the last row
    const bool ragged = h.K % 16 != 0;
    // sums over K of the rows v0 + r[i] (none where r[i] < 0), to out[t * WIDTH + r[i]]
    float* out = s_out[warp];
    auto dots = [&](int v0, const int (&r)[ROWS]) {
        int acc[ROWS][N] = {};
#pragma unroll 2
        for (int c = lane; c < chunks; c += 32) {
            uint4 w[ROWS];
#pragma unroll
            for (int i = 0; i < ROWS; i++) {
                w[i] = make_uint4(0, 0, 0, 0);
                if (r[i] < 0) continue;
                const int8_t* p = h.w + (size_t)(v0 + r[i]) * h.w_stride + c * 16;
                if (ragged && c == chunks - 1 && v0 + r[i] == h.V - 1) w[i] = load_bytes(p, h.K - c * 16);
                else w[i] = __ldcs(reinterpret_cast<const uint4*>(p));
            }
#pragma unroll
            for (int t = 0; t < N; t++) {
                const uint4 x = xs[t * chunks + c];
#pragma unroll
                for (int i = 0; i < ROWS; i++) {
                    acc[i][t] = __dp4a((int)w[i].x, (int)x.x, acc[i][t]);
                    acc[i][t] = __dp4a((int)w[i].y, (int)x.y, acc[i][t]);
                    acc[i][t] = __dp4a((int)w[i].z, (int)x.z, acc[i][t]);
                    acc[i][t] = __dp4a((int)w[i].w, (int)x.w, acc[i][t]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < ROWS; i++)
#pragma unroll
            for (int t = 0; t < N; t++) {
                const int sum = __reduce_add_sync(FULL, acc[i][t]);
                if (lane == 0 && r[i] >= 0) out[t * WIDTH + r[i]] = (float)sum;
            }
    };
    const int n_items = (h.V + WIDTH - 1) / WIDTH, n_warps = gridDim.x * (ROWS_THREADS / 32);
    const int me = blockIdx.x * (ROWS_THREADS / 32) + warp;
    if (!MASKED) {                                      // neighbouring rows, the same number for all warps
        const int to = (int)((int64_t)(me + 1) * n_items / n_warps);
        for (int item = (int)((int64_t)me * n_items / n_warps); item < to; item++) {
            const int v0 = item * ROWS;
            int r[ROWS];
#pragma unroll
            for (int i = 0; i < ROWS; i++) r[i] = v0 + i < h.V ? i : -1;
            dots(v0, r);
            __syncwarp();
            for (int t0 = 0; t0 < h.T; t0 += 32 / ROWS) {
                const int t = t0 + lane / ROWS, v = v0 + lane % ROWS;
                if (t < h.T && v < h.V)
                    store_f32(logits + (size_t)t * h.row_stride + v,
                              out[t * ROWS + lane % ROWS] * h.scale[t] * h.w_scale[v]);
            }
            __syncwarp();
        }
    } else {                                            // a mask word each; what masks allow may lie together
        for (int item = me; item < n_items; item += n_warps) {
            const int v0 = item * 32, v = v0 + lane;
            const uint32_t mine = lane < h.T ? h.bitmask[(size_t)lane * h.mask_stride + item] : 0u;
            uint32_t rows = __reduce_or_sync(FULL, mine);
            if (h.V - v0 < 32) rows &= (1u << (h.V - v0)) - 1;
            while (rows) {
                int r[ROWS];
#pragma unroll
                for (int i = 0; i < ROWS; i++) {
                    r[i] = __ffs(rows) - 1;             // -1: none left
                    rows &= rows - 1;
                }
                dots(v0, r);
            }
            __syncwarp();
            const float sw = v < h.V ? h.w_scale[v] : 0.f;
            for (int t = 0; t < h.T; t++) {
                const uint32_t bits = __shfl_sync(FULL, mine, t);
                if (v < h.V)
                    store_f32(logits + (size_t)t * h.row_stride + v, (bits >> lane) & 1
                                                                         ? out[t * WIDTH + lane] * h.scale[t] * sw
                                                                         : __uint_as_float(0xFF800000u));
            }
            __syncwarp();
        }
    }
}

template <typename T, int N>
psc_status head_rows(const Head& h, T* logits, uint8_t* work, cudaStream_t cs, const uint8_t* flags = nullptr,
                     int n_tiles = 0) {
    const size_t smem = (size_t)N * ((h.K + 15) / 16) * 16;
    const int per_sm = N > 4 ? 2 : 3, items = h.bitmask ? h.W : (h.V + ROWS - 1) / ROWS;     // as their registers allow
    return ops_launch(h.bitmask ? k_head_rows<T, N, true> : k_head_rows<T, N, false>,
                      dim3(std::min((items + 7) / 8, current_sms() * per_sm)), ROWS_THREADS, smem, 1, cs,
                      "k_head_rows", h, logits, (int*)work, flags, n_tiles);
}

// ------------------------------------------------------------ the tensor-core path
//
// k_head_mma: a persistent block per SM over tiles of 128 vocabulary rows (the
// tensor core's M) by up to 256 tokens (its N).  The weights are the large operand
// and every one is used for all tokens of the batch at once, so each is loaded and
// widened once per 256 tokens.  Per 64 columns of K:
//   warp 0        TMA: 128 x 128 bytes of weights into the byte ring (128 columns at a time)
//   warps 8-15    bytes -> f16 into the operand ring, in the tensor core's 128-byte swizzle
//   warp 2        TMA: the tokens' f16 rows (k_head_prep widened them) beside them
//   warp 1        four tcgen05.mma of 128 x N x 16 into one of two accumulators in TMEM (of a
//                 pair: the first block's, 256 x N x 16; the second's says when its operands are there)
//   warps 4-7     the other accumulator: scales, mask, logits (a lane per vocabulary row)
// With many tokens what bounds it is shared memory: per 64 columns of K and 256 tokens a block
// on its own moves 112 KB through it (bytes in and out 16, widened weights in and out 32,
// tokens in and out 64), 875 cycles where the products take 512.  So blocks pair up (PAIR):
// 256 rows of weights, 128 in each, by the same tokens, half in each (tcgen05's
// cta_group::2), which leaves 80 KB.  256 tokens over 262,144 x 4096: 424 -> 366 us, 1502
// TFLOP/s; 64 tokens over 128,256 x 2048: 66 us alone, 77 in pairs; 128 tokens over 128,256 x
// 4096: 157 alone, 149 in pairs.  1024 tokens over 262,144 x 2048: 681 us, 1615 TFLOP/s.
// Byte b becomes f16 without a conversion: b + 128 under the exponent of 1024 is
// 1152 + b, minus 1152; five instructions for four bytes.
constexpr int VT = 128;                       // vocabulary rows of a tile
constexpr int NT_MAX = 256;                   // tokens of a tile at most
constexpr int KB = 64;                        // columns of K per operand stage (128 bytes of f16)
constexpr int RAW_BYTES = VT * 128;           // a stage of the byte ring: 128 columns
constexpr int A_BYTES = VT * KB * 2;
constexpr int MAX_RAW = 8, N_A = 4, MAX_X = 4;     // stages of the rings: bytes, widened weights, tokens
constexpr int MMA_THREADS = 512;

struct Plan {
    int N, n_nt, n_vt;                        // tokens per tile, tiles of tokens and of vocabulary rows
    bool pair;                                // two blocks work on 256 vocabulary rows together
    int n_raw, n_x, x_group;                  // stages of the byte ring, of the tokens' ring; K stages in one of those
    int Kp;                                   // K rounded up to whole stages
    int tmem;                                 // TMEM columns
    size_t smem;
    int64_t x_at, flags_at, bytes;            // in the workspace: the fault word, the f16 tokens, the tile flags
};

constexpr int PAIR_N = 128;                   // tokens of a tile from which blocks pair up

Plan plan_of(int T, int V, int K) {
    Plan p;
    p.n_nt = (T + NT_MAX - 1) / NT_MAX;
    p.N = ((T + p.n_nt - 1) / p.n_nt + 15) / 16 * 16;
    p.n_vt = (V + VT - 1) / VT;
    p.pair = p.N >= PAIR_N && p.n_vt > 1;
    if (p.pair) p.N = (p.N + 31) / 32 * 32;
    p.Kp = (K + KB - 1) / KB * KB;
    // A stage of the tokens' ring holds several columns' stages where those are small, so
    // that the issuing warp waits and releases seldom (16 tokens over 128,256 x 2048: 63 us, with
    // one a stage 79); the byte ring, which covers the memory's latency, gets the shared memory
    // that is left.
    const int own = p.pair ? p.N / 2 : p.N;   // tokens in a block's shared memory
    p.x_group = own <= 32 ? 4 : own <= 64 ? 2 : 1;
    const int x_bytes = own * KB * 2 * p.x_group;
    p.n_x = own <= 128 ? MAX_X : 3;
    p.n_raw = std::min(MAX_RAW, (SMEM_MAX - 2048 - N_A * A_BYTES - p.n_x * x_bytes) / RAW_BYTES);
    p.smem = 1024 + (size_t)N_A * A_BYTES + (size_t)p.n_x * x_bytes + (size_t)p.n_raw * RAW_BYTES;
    p.tmem = 32;
    while (p.tmem < 2 * p.N) p.tmem <<= 1;
    p.x_at = 256;
    p.flags_at = p.x_at + ((int64_t)T * p.Kp * 2 + 255) / 256 * 256;
    p.bytes = p.flags_at + ((int64_t)p.n_vt * p.n_nt + 255) / 256 * 256;
    return p;
}

// D (+)= A B; of a pair: 256 rows, A's 128 and half of B's columns from each block.
template <bool PAIR>
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
    if (PAIR)
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
            " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(add)
            : "memory");
    else
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
            " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(add)
            : "memory");
}
// Four signed bytes as four f16.
__device__ __forceinline__ uint2 widen4(uint32_t b) {
    const uint32_t u = b ^ 0x80808080u, base = 0x64646464u;
    uint32_t lo = __byte_perm(u, base, 0x4140), hi = __byte_perm(u, base, 0x4342);
    const __half2 off = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));
    __half2 l = __hsub2(*reinterpret_cast<__half2*>(&lo), off), h = __hsub2(*reinterpret_cast<__half2*>(&hi), off);
    return make_uint2(*reinterpret_cast<uint32_t*>(&l), *reinterpret_cast<uint32_t*>(&h));
}

// The tokens' rows in f16, zero past K; how many rows of each tile some token allows; the fault word.
__global__ void __launch_bounds__(256) k_head_prep(Head h, int Kp, int N, int n_vt, int n_nt, int x_blocks,
                                                   int* faults, __half* x, uint8_t* flags) {
    dep_wait();
    dep_launch();
    if (h.first && blockIdx.x == 0 && threadIdx.x == 0) *faults = 0;
    if ((int)blockIdx.x < x_blocks) {                 // 16 columns a thread
        const int per = Kp / 16;
        const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
        if (i >= (int64_t)h.T * per) return;
        const int t = (int)(i / per), k = (int)(i - (int64_t)t * per) * 16;
        const int8_t* src = h.q + (size_t)t * h.q_stride + k;
        const uint4 v = k + 16 <= h.K && !((uintptr_t)src & 15) ? *reinterpret_cast<const uint4*>(src)
                                                                : load_bytes(src, h.K - k);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        uint4* dst = reinterpret_cast<uint4*>(x + (size_t)t * Kp + k);
#pragma unroll
        for (int j = 0; j < 2; j++) {
            const uint2 a = widen4(w[2 * j]), c = widen4(w[2 * j + 1]);
            dst[j] = make_uint4(a.x, a.y, c.x, c.y);
        }
        return;
    }
    const int item = (blockIdx.x - x_blocks) * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (item >= n_vt * n_nt) return;
    const int vt = item / n_nt, t0 = (item - vt * n_nt) * N, t1 = min(h.T, t0 + N);
    uint32_t any = 0;
    // a lane per word of a token's four, eight tokens at a time
    for (int t = t0 + (lane >> 2); t < t1; t += 8) {
        const int wi = vt * 4 + (lane & 3);
        if (wi < h.W) any |= h.bitmask[(size_t)t * h.mask_stride + wi];
    }
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) any |= __shfl_xor_sync(FULL, any, o);
    const int rows = __reduce_add_sync(FULL, lane < 4 ? __popc(any) : 0);
    if (lane == 0) flags[item] = (uint8_t)rows;
}

template <typename T, bool PAIR>
__global__ void __launch_bounds__(MMA_THREADS, 1) k_head_mma(const __grid_constant__ CUtensorMap w_map,
                                                             const __grid_constant__ CUtensorMap x_map, Head h,
                                                             T* logits, int N, int n_nt, int n_vt, int Kp, int n_raw,
                                                             int n_x, int x_group, int tmem_cols, int* faults,
                                                             const uint8_t* flags, int leave_few) {
    if (leave_few) {                                  // few rows are k_head_rows'
        dep_wait();
        if (few_rows(flags, n_vt * n_nt, h.V)) return;
    }
    constexpr int PER = 8 / N_A, ROWS = VT / PER;      // converting warps of a group, rows of each
    extern __shared__ uint8_t dyn[];
    __shared__ __align__(8) uint64_t s_bars[2 * (MAX_RAW + N_A + MAX_X) + 5 + N_A];
    __shared__ uint32_t s_tmem;
    __shared__ int s_failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t base = (smem_addr(dyn) + 1023) & ~1023u;
    // of a pair, the blocks have 128 vocabulary rows and half of the tokens each
    constexpr int SIDES = PAIR ? 2 : 1;
    const int side = PAIR ? (int)cluster_rank() : 0, own_n = N / SIDES;
    const int n_items = (n_vt + SIDES - 1) / SIDES * n_nt;
    const int first = blockIdx.x / SIDES, step = gridDim.x / SIDES;
    const int x_block = own_n * KB * 2, x_bytes = x_block * x_group;
    auto a_at = [&](int s) { return base + s * A_BYTES; };
    auto x_at = [&](int s) { return base + N_A * A_BYTES + s * x_bytes; };
    auto raw_at = [&](int s) { return base + N_A * A_BYTES + n_x * x_bytes + s * RAW_BYTES; };
    const uint32_t bars = smem_addr(s_bars);
    auto raw_full = [&](int s) { return bars + 8 * s; };
    auto raw_empty = [&](int s) { return bars + 8 * (MAX_RAW + s); };
    auto a_full = [&](int s) { return bars + 8 * (2 * MAX_RAW + s); };
    auto a_empty = [&](int s) { return bars + 8 * (2 * MAX_RAW + N_A + s); };
    auto x_full = [&](int s) { return bars + 8 * (2 * (MAX_RAW + N_A) + s); };
    auto x_empty = [&](int s) { return bars + 8 * (2 * (MAX_RAW + N_A) + MAX_X + s); };
    constexpr int LAST = 2 * (MAX_RAW + N_A + MAX_X);
    auto acc_full = [&](int s) { return bars + 8 * (LAST + s); };
    auto acc_empty = [&](int s) { return bars + 8 * (LAST + 2 + s); };
    const uint32_t drained = bars + 8 * (LAST + 4);
    auto other_full = [&](int s) { return bars + 8 * (LAST + 5 + s); };    // the second block's operands are there

    if (threadIdx.x == 0) {
        s_failed = 0;
        for (int s = 0; s < n_raw; s++) mbar_init(raw_full(s), 1), mbar_init(raw_empty(s), 2 * PER);
        for (int s = 0; s < N_A; s++) mbar_init(a_full(s), PER), mbar_init(a_empty(s), 1);
        for (int s = 0; s < n_x; s++) mbar_init(x_full(s), 1), mbar_init(x_empty(s), 1);
        for (int s = 0; s < 2; s++) mbar_init(acc_full(s), 1), mbar_init(acc_empty(s), 4 * SIDES);
        for (int s = 0; s < N_A; s++) mbar_init(other_full(s), 1);
        mbar_init(drained, SIDES > 1 ? 2 : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (PAIR) cluster_sync();
    if (warp == 3) {
        if (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&s_tmem)),
                         "r"(tmem_cols)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&s_tmem)),
                         "r"(tmem_cols)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (PAIR) cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = s_tmem;
    volatile int* failed = &s_failed;
    const int n_k = Kp / KB, n_k2 = (n_k + 1) / 2;
    // k_head_prep began once every earlier kernel had completed, and this one after it had
    // begun: only what k_head_prep writes (flags, f16 tokens) has to be waited for.
    const bool masked = h.bitmask != nullptr;
    if (warp != 0 || masked) dep_wait();
    // whether an item's tiles (of all its blocks) hold an allowed token
    auto is_active = [&](int item) {
        if (!masked) return true;
        if (!PAIR) return flags[item] != 0;
        const int vt = item / n_nt * 2, nt = item % n_nt;
        return (flags[vt * n_nt + nt] | (vt + 1 < n_vt ? flags[(vt + 1) * n_nt + nt] : 0)) != 0;
    };

    if (warp == 0) {
        if (lane == 0) {
            Place p;
            int c = 0;
            for (int item = first; item < n_items && !*failed; item += step) {
                if (!is_active(item)) continue;
                const int v0 = (item / n_nt * SIDES + side) * VT;
                for (int k = 0; k < n_k2; k++, c++, p.next(n_raw)) {
                    if (!mbar_wait(raw_empty(p.s), p.parity ^ 1, failed)) break;
                    mbar_arrive_tx(raw_full(p.s), RAW_BYTES);
                    tma_2d(raw_at(p.s), &w_map, k * 128, v0, raw_full(p.s));
                }
            }
            if (*failed)                              // let the copies in flight land
                for (int i = max(0, c - n_raw); i < c; i++)
                    for (int it = 0; it < (1 << 20) && !mbar_try(raw_full(i % n_raw), (i / n_raw) & 1); it++) {}
        }
    } else if (warp == 2) {
        if (lane == 0) {
            Place p;
            int c = 0;
            for (int item = first; item < n_items && !*failed; item += step) {
                if (!is_active(item)) continue;
                const int t0 = item % n_nt * N + side * own_n;
                for (int k = 0; k < n_k; k += x_group, c++, p.next(n_x)) {
                    if (!mbar_wait(x_empty(p.s), p.parity ^ 1, failed)) break;
                    const int n = min(x_group, n_k - k);
                    mbar_arrive_tx(x_full(p.s), n * x_block);
                    for (int j = 0; j < n; j++)
                        tma_2d(x_at(p.s) + j * x_block, &x_map, (k + j) * KB, t0, x_full(p.s));
                }
            }
            if (*failed)
                for (int i = max(0, c - n_x); i < c; i++)
                    for (int it = 0; it < (1 << 20) && !mbar_try(x_full(i % n_x), (i / n_x) & 1); it++) {}
        }
    } else if (warp == 1) {
        // The whole warp waits, so that addresses and descriptors stay in uniform registers; one
        // lane issues.  Of a pair the first block issues, and the second tells it of its operands.
        // D f32, A and B f16, both along K; N and M.
        const uint32_t idesc = (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(VT * SIDES >> 4) << 24);
        const bool issuer = elect_one();
        Place pa, px, acc;
        bool ok = true;
        for (int item = first; item < n_items && ok; item += step) {
            if (!is_active(item)) continue;
            if (side == 0 && !(ok = warp_wait(acc_empty(acc.s), acc.parity ^ 1, failed))) break;
            const uint32_t d = tmem + acc.s * N;
            int in_group = 0;
            for (int k = 0; k < n_k; k++, pa.next(N_A)) {
                if (!(ok = in_group ? warp_wait(a_full(pa.s), pa.parity, failed)
                                    : warp_wait2(x_full(px.s), px.parity, a_full(pa.s), pa.parity, failed)))
                    break;
                const bool last = in_group + 1 == x_group || k + 1 == n_k;
                if (side == 0) {
                    if (PAIR && !(ok = warp_wait(other_full(pa.s), pa.parity, failed))) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t da = operand_desc(a_at(pa.s)), db = operand_desc(x_at(px.s) + in_group * x_block);
                    if (issuer) {
#pragma unroll
                        for (int j = 0; j < KB / 16; j++) mma_f16<PAIR>(d, da + 2 * j, db + 2 * j, idesc, k | j);
                        mma_commit<PAIR>(a_empty(pa.s));
                        if (last) mma_commit<PAIR>(x_empty(px.s));
                        if (k + 1 == n_k) mma_commit<PAIR>(acc_full(acc.s));
                    }
                } else if (issuer) {
                    arrive_at_first(other_full(pa.s));
                }
                in_group++;
                if (last) in_group = 0, px.next(n_x);
            }
            acc.next(2);
        }
        if (!ok && issuer && side == 0) {             // let the products in flight finish
            mma_commit<PAIR>(drained);
            if (PAIR) mma_commit<PAIR>(drained);
            for (int it = 0; it < (1 << 20) && !mbar_try(drained, 0); it++) {}
        }
    } else if (warp >= 8) {
        // N_A groups of warps, a group per slot of the operand ring: what one stage waits for (its
        // slot, its bytes, its stores to become visible) passes while others are converted.
        // A parity names one phase only to whom the phase before is known to be complete.  Of its
        // own slot a group sees every phase.  A byte slot goes round among the groups, so the
        // wait for the operand slot comes first: it ends when the products of the stage N_A before
        // are done, so every byte stage up to that one has landed, and with at least N_A byte
        // slots the last use of this stage's slot is one of those.
        const int group = (warp - 8) / PER, r0 = (warp % PER) * ROWS + (lane >> 3) + ((lane >> 2) & 1) * 4;
        int c = 0, cr = 0, at = 0;                    // stages of both rings before this item; pr is number `at`
        Place pr;
        uint32_t parity = 1;                          // of the group's slot's next release
        bool ok = true;                               // the same in all lanes
        for (int item = first; item < n_items && ok; item += step) {
            if (!is_active(item)) continue;
            for (int k = (group - c) & (N_A - 1); k < n_k; k += N_A) {
                const int s = group;
                for (; at < cr + (k >> 1); at++) pr.next(n_raw);
                const int sr = pr.s;
                if (!(ok = warp_wait(a_empty(s), parity, failed))) break;
                parity ^= 1;
                if (!(ok = warp_wait(raw_full(sr), pr.parity, failed))) break;
                // lanes 0-3 and 4-7 take rows 4 apart, so that eight lanes touch all 32
                // banks in both swizzles
                uint4 v[ROWS / 8];
#pragma unroll
                for (int j = 0; j < ROWS / 8; j++) {
                    const int r = r0 + j * 8;
                    const uint32_t from = raw_at(sr) + r * 128 + ((((k & 1) * 4 + (lane & 3)) ^ (r & 7)) << 4);
                    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                                 : "=r"(v[j].x), "=r"(v[j].y), "=r"(v[j].z), "=r"(v[j].w)
                                 : "r"(from));
                }
                const int odd = (lane >> 2) & 1, col = (lane & 3) * 2;
#pragma unroll
                for (int j = 0; j < ROWS / 8; j++) {
                    const int r = r0 + j * 8;
                    const uint2 a = widen4(v[j].x), b = widen4(v[j].y), d = widen4(v[j].z), e = widen4(v[j].w);
                    const uint32_t to = a_at(s) + r * 128;
                    const uint4 first = odd ? make_uint4(d.x, d.y, e.x, e.y) : make_uint4(a.x, a.y, b.x, b.y);
                    const uint4 second = odd ? make_uint4(a.x, a.y, b.x, b.y) : make_uint4(d.x, d.y, e.x, e.y);
                    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(to + (((col + odd) ^ (r & 7)) << 4)),
                                 "r"(first.x), "r"(first.y), "r"(first.z), "r"(first.w)
                                 : "memory");
                    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(to + (((col + 1 - odd) ^ (r & 7)) << 4)),
                                 "r"(second.x), "r"(second.y), "r"(second.z), "r"(second.w)
                                 : "memory");
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(a_full(s));
                    mbar_arrive(raw_empty(sr));       // each warp of both halves' groups
                    if (!(k & 1) && k + 1 == n_k) mbar_arrive(raw_empty(sr));
                }
            }
            c += n_k;
            cr += n_k2;
        }
    } else if (warp >= 4) {
        const int quad = warp & 3;
        Place acc;
        for (int item = first; item < n_items; item += step) {
            const bool active = is_active(item);
            const int vt = item / n_nt * SIDES + side, t0 = item % n_nt * N, n = min(N, h.T - t0);
            const int v = vt * VT + quad * 32 + lane, wi = vt * 4 + quad;
            // the tile's scales and mask words (a lane per token), read while its products run
            const float sw = v < h.V ? h.w_scale[v] : 0.f;
            float st[NT_MAX / 32];
            uint32_t word[NT_MAX / 32];
#pragma unroll
            for (int i = 0; i < NT_MAX / 32; i++) {
                const int t = i * 32 + lane;
                st[i] = t < n ? h.scale[t0 + t] : 0.f;
                const bool there = active && t < n && wi < h.W;
                word[i] = !masked ? FULL : there ? h.bitmask[(size_t)(t0 + t) * h.mask_stride + wi] : 0u;
            }
            if (active) {
                if (!warp_wait(acc_full(acc.s), acc.parity, failed)) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            }
            T* out = logits + (size_t)t0 * h.row_stride + v;
#pragma unroll
            for (int i = 0; i < NT_MAX / 32; i++) {
                if (i * 32 >= n) break;
                uint32_t y[32] = {};
                if (active) {
                    const uint32_t from = tmem + ((uint32_t)(quad * 32) << 16) + acc.s * N + i * 32;
                    tmem_load16(from, y);
                    if (i * 32 + 16 < N) tmem_load16(from + 16, y + 16);
                    tmem_wait(y);
                }
#pragma unroll
                for (int j = 0; j < 32; j++) {
                    const uint32_t wj = __shfl_sync(FULL, word[i], j);
                    const float sj = __shfl_sync(FULL, st[i], j);
                    if (i * 32 + j < n && v < h.V)
                        store_f32(out, (wj >> lane) & 1 ? __uint_as_float(y[j]) * sj * sw
                                                        : __uint_as_float(0xFF800000u));
                    out += h.row_stride;
                }
            }
            if (active) {
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    if (PAIR) arrive_at_first(acc_empty(acc.s));
                    else mbar_arrive(acc_empty(acc.s));
                }
                acc.next(2);
            }
        }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (PAIR) cluster_sync();                         // nothing of this block is used by the other any more
    if (warp == 3) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(tmem_cols));
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(tmem_cols));
    }
    if (threadIdx.x == 0 && s_failed) atomicAdd(faults, 1);
}

template <typename T>
psc_status head_mma(const Head& h, T* logits, uint8_t* work, cudaStream_t cs) {
    const Plan p = plan_of(h.T, h.V, h.K);
    int* faults = (int*)work;
    __half* x = (__half*)(work + p.x_at);
    uint8_t* flags = work + p.flags_at;
    CUtensorMap w_map, x_map;
    if (!tensor_map(&w_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, h.w, h.K, h.V, h.w_stride, 128, VT) ||
        !tensor_map(&x_map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, x, p.Kp, h.T, (uint64_t)p.Kp * 2, KB,
                    p.pair ? p.N / 2 : p.N))
        return ops_fail(PSC_ERR_CUDA, "psc_head_logits", "cuTensorMapEncodeTiled failed");
    const int items = p.n_vt * p.n_nt;
    const int x_blocks = (int)(((int64_t)h.T * (p.Kp / 16) + 255) / 256);
    psc_status s = ops_launch(k_head_prep, dim3(x_blocks + (h.bitmask ? (items + 7) / 8 : 0)), 256, 0, 1, cs,
                              "k_head_prep", h, p.Kp, p.N, p.n_vt, p.n_nt, x_blocks, faults, x, flags);
    if (s != PSC_OK) return s;
    const int leave_few = h.T <= 16 && h.bitmask && 16 * (int64_t)((h.K + 15) / 16 * 16) <= ROWS_X_MAX;
    if (leave_few && (s = head_rows<T, 16>(h, logits, work, cs, flags, items)) != PSC_OK) return s;
    const int sides = p.pair ? 2 : 1, wide = (p.n_vt + sides - 1) / sides * p.n_nt;
    return ops_launch(p.pair ? k_head_mma<T, true> : k_head_mma<T, false>,
                      dim3(std::min(wide, current_sms() / sides) * sides), MMA_THREADS, p.smem, sides, cs, "k_head_mma",
                      w_map, x_map, h, logits, p.N, p.n_nt, p.n_vt, p.Kp, p.n_raw, p.n_x, p.x_group, p.tmem, faults,
                      (const uint8_t*)flags, leave_few);
}

// Weights whose rows are not at 16-byte-aligned addresses are packed into the workspace, a slab
// at a time where that is more than 256 MB.  (128,256 x 2047, with 40 MB slabs, which the L2 still
// holds when the products read them, in brackets: 1 token 130 us (143), 256 tokens 187 (325): the
// start and the end of every slab's kernels cost more than its second trip from memory.)
constexpr int64_t SLAB_BYTES = 256 << 20;
int slab_rows(int V, int K) {
    const int64_t pitch = (K + 15) / 16 * 16;
    return (int)std::min<int64_t>((V + VT - 1) / VT * VT, std::max<int64_t>(VT, SLAB_BYTES / pitch / VT * VT));
}
bool is_packed(const int8_t* w, int64_t stride) { return is_aligned(w, stride, 16); }

template <typename T>
psc_status head_aligned(const Head& h, T* logits, uint8_t* work, cudaStream_t cs) {
    // up to 4 tokens, or 8 under a mask (rows of the weights can be left out one by one; up
    // to 16 if it leaves few)
    const int64_t row = (h.K + 15) / 16 * 16;
    if (h.T == 1 && row <= ROWS_X_MAX) return head_rows<T, 1>(h, logits, work, cs);
    if (h.T == 2 && 2 * row <= ROWS_X_MAX) return head_rows<T, 2>(h, logits, work, cs);
    if (h.T <= 4 && 4 * row <= ROWS_X_MAX) return head_rows<T, 4>(h, logits, work, cs);
    if (h.T <= 8 && h.bitmask && 8 * row <= ROWS_X_MAX) return head_rows<T, 8>(h, logits, work, cs);
    return head_mma(h, logits, work, cs);
}

template <typename T>
psc_status head(const Head& h, T* logits, uint8_t* work, cudaStream_t cs) {
    if (is_packed(h.w, h.w_stride)) return head_aligned(h, logits, work, cs);
    const int rows = slab_rows(h.V, h.K), pitch = (h.K + 15) / 16 * 16;
    int8_t* slab = (int8_t*)work + plan_of(h.T, h.V, h.K).bytes;
    const int8_t* end = h.w + (size_t)(h.V - 1) * h.w_stride + h.K;
    for (int v0 = 0; v0 < h.V; v0 += rows) {
        Head part = h;
        part.V = std::min(rows, h.V - v0);
        part.first = v0 == 0;
        psc_status s = ops_launch(k_pack_rows, dim3(std::min((part.V + 7) / 8, current_sms() * 8)), 256, 0, 1, cs,
                                  "k_pack_rows", h.w + (size_t)v0 * h.w_stride, h.w_stride, part.V, h.K, pitch, h.w, end,
                                  slab);
        if (s != PSC_OK) return s;
        part.w = slab;
        part.w_stride = pitch;
        part.w_scale += v0;
        part.W = (part.V + 31) / 32;
        if (part.bitmask) part.bitmask += v0 / 32;
        if ((s = head_aligned(part, logits + v0, work, cs)) != PSC_OK) return s;
    }
    return PSC_OK;
}

}  // namespace

extern "C" {

psc_status psc_quantize_rows(const void* d_x, psc_dtype dtype, int64_t row_stride, int32_t T, int32_t K, int8_t* d_q,
                             int64_t q_stride, float* d_scale, void* stream) {
    const char* me = "psc_quantize_rows";
    if (T < 0 || K <= 0 || row_stride < K || q_stride < K || !is_dtype(dtype) || (T && (!d_x || !d_q || !d_scale)))
        return ops_fail(PSC_ERR_ARG, me, "bad arguments");
    if (K > MAX_QUANTIZE_K) return ops_fail(PSC_ERR_LIMIT, me, "K over 2^30");
    if (T == 0) return PSC_OK;
    cudaStream_t cs = (cudaStream_t)stream;
    if (dtype == PSC_BF16)
        return ops_launch(k_quantize_rows<__nv_bfloat16>, dim3(T), 256, 0, 1, cs, "k_quantize_rows",
                          (const __nv_bfloat16*)d_x, row_stride, K, d_q, q_stride, d_scale);
    return ops_launch(k_quantize_rows<float>, dim3(T), 256, 0, 1, cs, "k_quantize_rows", (const float*)d_x, row_stride,
                      K, d_q, q_stride, d_scale);
}

int64_t psc_head_work_bytes(int32_t T, int32_t V, int32_t K, int32_t aligned) {
    if (T <= 0 || V <= 0 || K <= 0 || T > MAX_T || V > MAX_V || K > MAX_K) return 256;
    return plan_of(T, V, K).bytes + (aligned ? 0 : (int64_t)slab_rows(V, K) * ((K + 15) / 16 * 16));
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
    if (T > MAX_T || V > MAX_V || (int64_t)((T + NT_MAX - 1) / NT_MAX) * ((V + VT - 1) / VT) > 0x7fffffff)
        return ops_fail(PSC_ERR_LIMIT, me, "too many rows");
    if (T == 0) return PSC_OK;
    if (!d_work || (uintptr_t)d_work % 256 || work_bytes < psc_head_work_bytes(T, V, K, is_packed(d_w, w_stride)))
        return ops_fail(PSC_ERR_ARG, me, "workspace missing, unaligned or too small");
    const int W = (V + 31) / 32;
    const Head h{d_q, q_stride, d_scale, T, d_w, w_stride, d_w_scale, V, K, d_bitmask, W, W, row_stride, 1};
    if (dtype == PSC_BF16) return head(h, (__nv_bfloat16*)d_logits, (uint8_t*)d_work, (cudaStream_t)stream);
    return head(h, (float*)d_logits, (uint8_t*)d_work, (cudaStream_t)stream);
}

}  // extern "C"
