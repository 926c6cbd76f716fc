// psc_head_logits_mx4: the vocabulary projection in microscaled 4-bit floating point, under the
// grammar's mask.
#include <algorithm>

#include "mx4.cuh"
#include "tcgen05.cuh"

namespace {

constexpr int MAX_K = 131072;
constexpr int MAX_V = 1 << 30, MAX_T = 1 << 24;     // and numbers of rows, rounded up to tiles, in 32 bits

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

// ------------------------------------------------------------ the tensor-core path
//
// k_mx4_mma: a persistent block per SM over tiles of 128 vocabulary rows (the tensor core's M) by
// up to 192 tokens (its N).  Both operands stay in 4 bits all the way; the tensor core takes their
// blocks' powers of two from TMEM.  A stage is 256 columns of K:
//   warps 0, 2-4  TMA, a part of each stage by each: 128 x 128 bytes of weights; N x 128 bytes of
//                 tokens; both sides' exponents (512 bytes for 128 rows by 128 columns, as they lie in memory)
//   warp 1        tcgen05.cp of the exponents into TMEM, then four tcgen05.mma of 128 x N x 64 into
//                 one of two accumulators
//   warps 8-15    the other accumulator: scales, mask, logits (a lane per vocabulary row, two warps
//                 for 32 of them)
// Beyond 128 tokens blocks pair up (PAIR): 256 vocabulary rows, 128 in each, by the same tokens, half of
// their codes in each (tcgen05's cta_group::2; all of their exponents in both).  An SM takes in 64
// bytes a cycle, and 192 tokens by 128 rows need 43 KB for a stage's 384 cycles of products; in a
// pair it is 31 KB, and where a tile's weights fit shared memory (K up to 2048), they stay there
// for all tiles of tokens (`stay`), which leaves 14 KB.
constexpr int VT = 128;                       // vocabulary rows of a tile
constexpr int NT = 192;                       // tokens of a tile at most; tiles start at multiples of 64
constexpr int KS = 256;                       // columns of K of a stage (128 bytes of codes)
constexpr int A_CODES = VT * KS / 2;
constexpr int SF = 512;                       // a tile of exponents: 128 rows by 128 columns
constexpr int A_BYTES = A_CODES + 2 * SF;
constexpr int MAX_A = 12, MAX_B = 11;         // slots of the rings: weights, tokens
constexpr int PARTS = 2, EPILOGUE = 4 * PARTS;  // warps for the same 32 vocabulary rows, of the epilogue in all
constexpr int GROUPS = NT / 32 / PARTS;       // a warp's groups of 32 tokens
constexpr int SMEM_OWN = 2048 + NT * 32;      // beside the rings: alignment, barriers, the epilogue's tokens
constexpr int FIRST = 8;                      // of the epilogue's warps
constexpr int MMA_THREADS = 32 * (FIRST + EPILOGUE);

struct Plan {
    int N, n_nt, n_vt;                        // tokens per tile, tiles of tokens and of vocabulary rows
    bool pair, stay;
    int n_k;                                  // stages of K
    int n_a, n_b, b_codes, b_bytes;           // slots of the rings, a slot's bytes of tokens (in a block)
    int acc, sf_cols;                         // TMEM columns of an accumulator, of a stage's exponents
    int items;                                // tiles (of pairs: two by two)
    size_t smem;
    int64_t flags_at, bytes;                  // in the workspace: the fault word, the tiles' flags
};

Plan plan_of(int T, int V, int K) {
    Plan p;
    p.n_nt = (T + NT - 1) / NT;
    p.N = p.n_nt > 1 ? NT : (T + 15) / 16 * 16;
    p.n_vt = (V + VT - 1) / VT;
    p.pair = p.N > 128;
    if (p.pair) p.N = (p.N + 31) / 32 * 32;
    p.n_k = (K + KS - 1) / KS;
    p.b_codes = (p.pair ? p.N / 2 : p.N) * KS / 2;
    p.b_bytes = p.b_codes + 2 * SF * (p.pair ? 2 : 1);
    p.acc = (p.N + 31) / 32 * 32;
    p.sf_cols = p.pair ? 24 : 16;
    // a stage's exponents have TMEM columns of their own, free when the tokens' slot is
    const int room = SMEM_MAX - SMEM_OWN, most = std::min(MAX_B, (512 - 2 * p.acc) / p.sf_cols);
    p.n_b = std::min(most, room / (A_BYTES + p.b_bytes));
    p.n_a = p.n_b;
    p.stay = p.n_nt > 1 && p.n_k <= MAX_A && p.n_k * A_BYTES + 4 * p.b_bytes <= room;
    if (p.stay) {
        p.n_b = std::min(most, (room - p.n_k * A_BYTES) / p.b_bytes);
        p.n_a = std::min(MAX_A, (room - p.n_b * p.b_bytes) / A_BYTES);
    }
    const int64_t items = (int64_t)(p.pair ? (p.n_vt + 1) / 2 : p.n_vt) * p.n_nt;
    p.items = (int)std::min<int64_t>(items, 0x7fffffff);
    p.smem = 1024 + (size_t)p.n_a * A_BYTES + (size_t)p.n_b * p.b_bytes;
    p.flags_at = 256;
    p.bytes = p.flags_at + ((int64_t)p.n_vt * p.n_nt + 255) / 256 * 256;
    return p;
}

// Descriptors by their low words (addresses in units of 16 bytes).  Exponents' tiles: 32 rows of 16
// bytes, 8 rows every 128 bytes, no swizzle; operands: operand_desc's.
__device__ __forceinline__ uint64_t exponent_desc(uint32_t lo) {
    return (uint64_t)(8u | (1u << 14)) << 32 | (lo | (8u << 16));
}
__device__ __forceinline__ uint64_t codes_desc(uint32_t lo) {
    return (uint64_t)(64u | (1u << 14) | (2u << 29)) << 32 | (lo | (1u << 16));
}
// 512 bytes to four TMEM columns, the same in all four quarters of the lanes (of both blocks of a pair,
// from their own shared memory).
template <bool PAIR>
__device__ __forceinline__ void copy_exponents(uint32_t to, uint32_t lo) {
    if (PAIR)
        asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(to), "l"(exponent_desc(lo)) : "memory");
    else
        asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(to), "l"(exponent_desc(lo)) : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void mma_mx4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                        uint32_t add) {
    if (PAIR)
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.u32 p, %6, 0;\n"
            " tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(add)
            : "memory");
    else
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.u32 p, %6, 0;\n"
            " tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(add)
            : "memory");
}
// A tile into this block's shared memory; of a pair, the barrier is the first block's.
template <bool PAIR>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    if (PAIR)
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
            " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(bar)
            : "memory");
    else
        tma_2d(dst, map, x, y, bar);
}
// The address of the first block's barrier in the pair's shared memory.
__device__ __forceinline__ uint32_t at_first(uint32_t bar) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(bar));
    return r;
}
// A stage's copies and products: exponents of CHUNKS times 128 columns (those of the weights, then those
// of the tokens, 128 or, of a pair, 256 rows), each of which two products of 64 columns use.  a, b: the
// slots of both sides, ea, eb: their exponents, in units of 16 bytes; sf: the stage's TMEM columns;
// shift: where the tile's tokens begin in theirs.
template <bool PAIR, int CHUNKS>
__device__ __forceinline__ void issue_stage(uint32_t a, uint32_t ea, uint32_t b, uint32_t eb, uint32_t sf,
                                            uint32_t shift, uint32_t d, uint32_t idesc, uint32_t add) {
    constexpr int B = PAIR ? 2 : 1;
#pragma unroll
    for (int c = 0; c < CHUNKS; c++) {
        copy_exponents<PAIR>(sf + 4 * c, ea + 32 * c);
#pragma unroll
        for (int j = 0; j < B; j++) copy_exponents<PAIR>(sf + 8 + 4 * B * c + 4 * j, eb + 64 * j + 32 * c);
    }
#pragma unroll
    for (int c = 0; c < CHUNKS; c++)
#pragma unroll
        for (int i = 0; i < 2; i++)               // the first or the second two of a word's four exponents
            mma_mx4<PAIR>(d, codes_desc(a + 4 * c + 2 * i), codes_desc(b + 4 * c + 2 * i),
                          idesc | (2u * i << 29) | (2u * i << 4), sf + 4 * c, sf + 8 + 4 * B * c + shift, add | c | i);
}

// How many rows of each tile some token allows, and the fault word.
__global__ void __launch_bounds__(256) k_mx4_flags(Head h, int N, int n_vt, int n_nt, int* faults, uint8_t* flags) {
    dep_wait();
    dep_launch();
    if (blockIdx.x == 0 && threadIdx.x == 0) *faults = 0;
    const int item = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (item >= n_vt * n_nt) return;
    const int vt = item / n_nt, t0 = (item - vt * n_nt) * N, t1 = min(h.T, t0 + N);
    uint32_t any = 0;
    // a lane per word of a token's four, eight tokens at a time
    for (int t = t0 + (lane >> 2); t < t1; t += 8) {
        const int wi = vt * 4 + (lane & 3);
        if (wi < h.W) any |= h.bitmask[(size_t)t * h.W + wi];
    }
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) any |= __shfl_xor_sync(FULL, any, o);
    const int rows = __reduce_add_sync(FULL, lane < 4 ? __popc(any) : 0);
    if (lane == 0) flags[item] = (uint8_t)rows;
}

// What the epilogue knows of a token: its scale, and the mask's word for the warp's 32 vocabulary rows.
struct __align__(8) Token {
    float scale;
    uint32_t word;
};

// Products of a lane's vocabulary row (the lanes' are neighbours) with 32 tokens, as logits: out is
// the first token's, `left` how many rows there are from the lane's on.  Two bf16 logits of a token
// go out in one store: lanes pair up, the even one takes the first of two tokens, the odd one the
// second (4-byte aligned where `even` says so).
template <bool MASKED>
__device__ __forceinline__ float logit(uint32_t y, float scale, uint32_t word, float sw, uint32_t bit) {
    const float x = __uint_as_float(y) * scale * sw;
    return !MASKED || (word & bit) ? x : __uint_as_float(0xFF800000u);
}
template <bool MASKED, typename T>
__device__ __forceinline__ void store_group(T* out, int64_t stride, const uint32_t y[32], const Token* tokens, float sw,
                                            int n, int left, bool even) {
    const int lane = threadIdx.x & 31;
    const uint32_t bit = 1u << lane;
    const float4* pairs = reinterpret_cast<const float4*>(tokens);          // of two tokens each
    const bool whole = n == 32 && __all_sync(FULL, left > 0);
    if (sizeof(T) == 2 && whole && even) {
        const bool odd = lane & 1;
        const uint32_t pick = odd ? 0x3276u : 0x5410u;
        T* at = out + (odd ? stride - 1 : 0);
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
            const float4 p = pairs[j / 2];
            const uint32_t u = pack_bf16(logit<MASKED>(y[j], p.x, __float_as_uint(p.y), sw, bit),
                                         logit<MASKED>(y[j + 1], p.z, __float_as_uint(p.w), sw, bit));
            *reinterpret_cast<uint32_t*>(at) = __byte_perm(u, __shfl_xor_sync(FULL, u, 1), pick);
            at += 2 * stride;
        }
    } else if (whole) {
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
            const float4 p = pairs[j / 2];
            store_f32(out, logit<MASKED>(y[j], p.x, __float_as_uint(p.y), sw, bit));
            store_f32(out + stride, logit<MASKED>(y[j + 1], p.z, __float_as_uint(p.w), sw, bit));
            out += 2 * stride;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 32; j++) {
            if (j < n && left > 0) store_f32(out, logit<MASKED>(y[j], tokens[j].scale, tokens[j].word, sw, bit));
            out += stride;
        }
    }
}

template <typename T, bool PAIR, bool MASKED>
__global__ void __launch_bounds__(MMA_THREADS, 1) k_mx4_mma(const __grid_constant__ CUtensorMap w_map,
                                                            const __grid_constant__ CUtensorMap x_map,
                                                            const __grid_constant__ CUtensorMap w_blocks_map,
                                                            const __grid_constant__ CUtensorMap x_blocks_map, Head h,
                                                            T* logits, Plan p, int* faults, const uint8_t* flags,
                                                            bool even) {
    extern __shared__ uint8_t dyn[];
    __shared__ __align__(8) uint64_t s_bars[2 * (MAX_A + MAX_B) + 5];
    __shared__ __align__(16) Token s_tokens[EPILOGUE][GROUPS * 32];
    __shared__ uint32_t s_tmem;
    __shared__ int s_failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int SIDES = PAIR ? 2 : 1;
    const int side = PAIR ? (int)cluster_rank() : 0;
    const uint32_t base = (smem_addr(dyn) + 1023) & ~1023u;
    // slots start at multiples of 1024 bytes: codes, then exponents
    auto a_at = [&](int s) { return base + s * A_BYTES; };
    auto b_at = [&](int s) { return base + p.n_a * A_BYTES + s * p.b_bytes; };
    const uint32_t bars = smem_addr(s_bars);
    auto a_full = [&](int s) { return bars + 8 * s; };
    auto a_empty = [&](int s) { return bars + 8 * (MAX_A + s); };
    auto b_full = [&](int s) { return bars + 8 * (2 * MAX_A + s); };
    auto b_empty = [&](int s) { return bars + 8 * (2 * MAX_A + MAX_B + s); };
    constexpr int LAST = 2 * (MAX_A + MAX_B);
    auto acc_full = [&](int s) { return bars + 8 * (LAST + s); };
    auto acc_empty = [&](int s) { return bars + 8 * (LAST + 2 + s); };
    const uint32_t drained = bars + 8 * (LAST + 4);

    if (threadIdx.x == 0) {
        s_failed = 0;
        for (int s = 0; s < p.n_a; s++) mbar_init(a_full(s), 2), mbar_init(a_empty(s), 1);
        for (int s = 0; s < p.n_b; s++) mbar_init(b_full(s), 2), mbar_init(b_empty(s), 1);
        for (int s = 0; s < 2; s++) mbar_init(acc_full(s), 1), mbar_init(acc_empty(s), EPILOGUE * SIDES);
        mbar_init(drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (PAIR) cluster_sync();
    if (warp == 1) {
        if (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&s_tmem))
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&s_tmem))
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
    const int n_tiles = (h.K + 127) / 128, n_k = p.n_k;
    dep_wait();
    dep_launch();
    // A block that fails has polled for a good part of a second before it counts itself.
    if (!MASKED && blockIdx.x == 0 && threadIdx.x == 0) *faults = 0;
    // This block's (pair's) items, all tiles of tokens of a tile of vocabulary rows after each other.
    const int me = blockIdx.x / SIDES, all = gridDim.x / SIDES;
    const int begin = (int)((int64_t)p.items * me / all), end = (int)((int64_t)p.items * (me + 1) / all);
    // whether an item (its vocabulary tile and tile of tokens) has an allowed token, in either block
    auto is_active = [&](int vt, int nt) {
        if (!MASKED) return true;
        const int at = vt * SIDES * p.n_nt + nt;
        return flags[at] != 0 || (PAIR && vt * 2 + 1 < p.n_vt && flags[at + p.n_nt] != 0);
    };
    // of a tile of tokens: how many the products take (both halves of a pair's in whole eights)
    auto tokens_of = [&](int t0) {
        const int n = min(p.N, h.T - t0);
        return PAIR ? (n + 31) / 32 * 32 : (n + 15) / 16 * 16;
    };

    // Loads one part of every stage: a box at (x, y), x + step, ... of a map into its place in the slots of
    // a ring.  origin: (x, y) of a vocabulary tile and a tile of tokens; once: weights that stay.
    auto load_part = [&](const CUtensorMap* map, int step, uint32_t to0, int slot_bytes, int slots, uint32_t full0,
                         uint32_t empty0, int bytes, bool once, auto row_of) {
        const uint32_t there0 = PAIR ? at_first(full0) : full0;
        const bool counts = !PAIR || side == 0;
        Place at;
        int c = 0;
        bool fresh = true;                            // the tile's weights are not there yet
        for (int item = begin, vt = begin / p.n_nt, nt = begin % p.n_nt; item < end && !*failed; item++) {
            if (is_active(vt, nt) && (fresh || !once)) {
                fresh = false;
                const int y = row_of(vt, nt);
                int x = 0;
                for (int k = 0; k < n_k; k++, x += step, at.next(slots)) {
                    if (!mbar_wait(empty0 + 8 * at.s, at.parity ^ 1, failed)) break;
                    if (counts) mbar_arrive_tx(full0 + 8 * at.s, bytes);
                    load_tile<PAIR>(to0 + at.s * slot_bytes, map, x, y, there0 + 8 * at.s);
                    c++;
                }
            }
            if (++nt == p.n_nt) nt = 0, vt++, fresh = true;
        }
        // let the copies in flight land (of a pair, the first block sees both blocks', and the second does
        // not end before it)
        if (*failed && counts)
            for (int i = max(0, c - slots); i < c; i++)
                for (int it = 0; it < (1 << 20) && !mbar_try(full0 + 8 * (i % slots), (i / slots) & 1); it++) {}
    };

    if (warp == 0 && lane == 0) {
        load_part(&w_map, 128, a_at(0), A_BYTES, p.n_a, a_full(0), a_empty(0), SIDES * A_CODES, p.stay,
                  [&](int vt, int) { return (vt * SIDES + side) * VT; });
    } else if (warp == 2 && lane == 0) {
        load_part(&x_map, 128, b_at(0), p.b_bytes, p.n_b, b_full(0), b_empty(0), SIDES * p.b_codes, false,
                  [&](int, int nt) { return nt * p.N + side * (tokens_of(nt * p.N) / 2); });
    } else if (warp == 3 && lane == 0) {
        load_part(&x_blocks_map, 256, b_at(0) + p.b_codes, p.b_bytes, p.n_b, b_full(0), b_empty(0),
                  SIDES * (p.b_bytes - p.b_codes), false, [&](int, int nt) { return nt * p.N / 128; });
    } else if (warp == 4 && lane == 0) {
        load_part(&w_blocks_map, 256, a_at(0) + A_CODES, A_BYTES, p.n_a, a_full(0), a_empty(0), SIDES * 2 * SF, p.stay,
                  [&](int vt, int) { return vt * SIDES + side; });
    } else if (warp == 1 && side == 0) {
        // The whole warp waits, so that addresses and descriptors stay in uniform registers; one lane
        // issues (of a pair, for both blocks).
        const bool issuer = elect_one();
        Place unit, at_b, acc;                        // unit: the first slot of the tile's weights
        bool ok = true, fresh = true;
        for (int item = begin, vt = begin / p.n_nt, nt = begin % p.n_nt; item < end && ok; item++) {
            if (is_active(vt, nt)) {
                // whether the weights have to be waited for, and whether nothing of them is used after this item
                const bool first = fresh || !p.stay;
                bool last = true;
                if (p.stay)
                    for (int i = item + 1, j = nt + 1; last && i < end && j < p.n_nt; i++, j++) last = !is_active(vt, j);
                fresh = false;
                const int t0 = nt * p.N;
                // D f32; A and B of E2M1, both along K; exponents alone as scales; N and M
                const uint32_t idesc = (1u << 7) | (1u << 10) | ((uint32_t)(tokens_of(t0) >> 3) << 17) | (1u << 23) |
                                       ((uint32_t)(VT * SIDES >> 4) << 24);
                const uint32_t d = tmem + acc.s * p.acc, shift = t0 % 128 / 32;
                if (!(ok = warp_wait(acc_empty(acc.s), acc.parity ^ 1, failed))) break;
                Place at_a = unit;
                for (int k = 0; k < n_k; k++, at_a.next(p.n_a), at_b.next(p.n_b)) {
                    const uint32_t a = (a_at(at_a.s) & 0x3FFFF) >> 4, b = (b_at(at_b.s) & 0x3FFFF) >> 4;
                    const uint32_t ea = a + A_CODES / 16, eb = b + p.b_codes / 16, sf = tmem + 2 * p.acc + at_b.s * p.sf_cols;
                    if (!(ok = first ? warp_wait2(a_full(at_a.s), at_a.parity, b_full(at_b.s), at_b.parity, failed)
                                     : warp_wait(b_full(at_b.s), at_b.parity, failed)))
                        break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    if (issuer) {
                        if (2 * k + 2 <= n_tiles) issue_stage<PAIR, 2>(a, ea, b, eb, sf, shift, d, idesc, k);
                        else issue_stage<PAIR, 1>(a, ea, b, eb, sf, shift, d, idesc, k);
                        mma_commit<PAIR>(b_empty(at_b.s));
                        if (last) mma_commit<PAIR>(a_empty(at_a.s));
                        if (k + 1 == n_k) mma_commit<PAIR>(acc_full(acc.s));
                    }
                }
                if (last) unit = at_a;
                acc.next(2);
            }
            if (++nt == p.n_nt) nt = 0, vt++, fresh = true;
        }
        if (!ok && issuer) {                          // let the products in flight finish
            mma_commit<PAIR>(drained);
            for (int it = 0; it < (1 << 20) && !mbar_try(drained, 0); it++) {}
        }
    } else if (warp >= FIRST) {
        const int quad = warp & 3, part = (warp - FIRST) >> 2;      // of every PARTS groups of 32 tokens, this warp's
        Token* tokens = s_tokens[warp - FIRST];
        Place acc;
        for (int item = begin, pt = begin / p.n_nt, nt = begin % p.n_nt; item < end; item++) {
            const bool active = is_active(pt, nt);
            const int vt = pt * SIDES + side, t0 = nt * p.N, n = min(p.N, h.T - t0);
            const int v = vt * VT + quad * 32 + lane, wi = vt * 4 + quad;
            if (++nt == p.n_nt) nt = 0, pt++;
            // the tile's scales and mask words, read while its products run
            const float sw = v < h.V && h.w_scale ? h.w_scale[v] : 1.f;
            __syncwarp();
#pragma unroll
            for (int i = 0; i < GROUPS; i++) {
                const int t = (PARTS * i + part) * 32 + lane;
                if (t >= n) continue;
                tokens[i * 32 + lane] = {
                    h.scale ? h.scale[t0 + t] : 1.f,
                    !MASKED ? FULL : active && wi < h.W ? h.bitmask[(size_t)(t0 + t) * h.W + wi] : 0u};
            }
            __syncwarp();
            if (active) {
                if (!warp_wait(acc_full(acc.s), acc.parity, failed)) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            }
#pragma unroll 1
            for (int i = 0; i < GROUPS; i++) {
                const int g = PARTS * i + part;
                if (g * 32 >= n) break;
                uint32_t y[32] = {};
                if (active) {
                    const uint32_t from = tmem + ((uint32_t)(quad * 32) << 16) + acc.s * p.acc + g * 32;
                    tmem_load16(from, y);
                    tmem_load16(from + 16, y + 16);
                    tmem_wait(y);
                }
                store_group<MASKED>(logits + (size_t)(t0 + g * 32) * h.row_stride + v, h.row_stride, y, tokens + i * 32,
                                    sw, min(32, n - g * 32), h.V - v, even);
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
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
    if (threadIdx.x == 0 && s_failed) atomicAdd(faults, 1);
}

template <typename T>
psc_status head_mma(const Head& h, T* logits, uint8_t* work, cudaStream_t cs) {
    const char* me = "psc_head_logits_mx4";
    const Plan p = plan_of(h.T, h.V, h.K);
    int* faults = (int*)work;
    uint8_t* flags = work + p.flags_at;
    CUtensorMap w_map, x_map;
    CUtensorMap w_blocks_map, x_blocks_map;
    const uint64_t row = (h.K + 31) / 32 * 16, n_tiles = (h.K + 127) / 128;
    if (!tensor_map(&w_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, h.w, row, h.V, h.w_stride, 128, VT) ||
        !tensor_map(&x_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, h.q, row, h.T, h.q_stride, 128,
                    p.pair ? p.N / 2 : p.N) ||
        !tensor_map(&w_blocks_map, CU_TENSOR_MAP_DATA_TYPE_UINT32, h.w_blocks, n_tiles * SF / 4, p.n_vt, n_tiles * SF,
                    256, 1, CU_TENSOR_MAP_SWIZZLE_NONE) ||
        !tensor_map(&x_blocks_map, CU_TENSOR_MAP_DATA_TYPE_UINT32, h.q_blocks, n_tiles * SF / 4, (h.T + 127) / 128,
                    n_tiles * SF, 256, p.pair ? 2 : 1, CU_TENSOR_MAP_SWIZZLE_NONE))
        return ops_fail(PSC_ERR_CUDA, me, "cuTensorMapEncodeTiled failed");
    const int items = p.n_vt * p.n_nt;
    if (h.bitmask) {
        psc_status s = ops_launch(k_mx4_flags, dim3((items + 7) / 8), 256, 0, 1, cs, "k_mx4_flags", h, p.N, p.n_vt,
                                  p.n_nt, faults, flags);
        if (s != PSC_OK) return s;
    }
    auto kernel = h.bitmask ? (p.pair ? k_mx4_mma<T, true, true> : k_mx4_mma<T, false, true>)
                            : (p.pair ? k_mx4_mma<T, true, false> : k_mx4_mma<T, false, false>);
    const bool even = is_aligned(logits, h.row_stride * (int64_t)sizeof(T), 4);
    const int sides = p.pair ? 2 : 1;
    return ops_launch(kernel, dim3(std::min(p.items, current_sms() / sides) * sides), MMA_THREADS, p.smem, sides, cs,
                      "k_mx4_mma", w_map, x_map, w_blocks_map, x_blocks_map, h, logits, p, faults,
                      (const uint8_t*)flags, even);
}

template <typename T>
psc_status head(const Head& h, T* logits, uint8_t* work, cudaStream_t cs) {
    return head_mma(h, logits, work, cs);
}

}  // namespace

extern "C" {

int64_t psc_head_mx4_work_bytes(int32_t T, int32_t V, int32_t K) {
    if (T <= 0 || V <= 0 || K <= 0 || T > MAX_T || V > MAX_V || K > MAX_K) return 256;
    return plan_of(T, V, K).bytes;
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
    if (T > MAX_T || V > MAX_V || (int64_t)((T + NT - 1) / NT) * ((V + VT - 1) / VT) > 0x7fffffff)
        return ops_fail(PSC_ERR_LIMIT, me, "too many rows");
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
