// psc_head_logits_mx4: the vocabulary projection in microscaled 4-bit floating point, under the
// grammar's mask.
#include <algorithm>
#include <mutex>

#include "mx4.cuh"
#include "tcgen05.cuh"

namespace {

const char* const ME = "psc_head_logits_mx4";

constexpr int MAX_K = 131072;
constexpr int MAX_V = 1 << 30, MAX_T = 1 << 24;     // and numbers of rows, rounded up to tiles, in 32 bits

// Blocks in which a bounded wait gave up; what a reset takes off it is what it has reported, so that none is lost that
// another stream adds meanwhile.
__device__ int g_faults;
std::mutex g_faults_read;                   // a report with its reset at a time

__global__ void k_take_faults(int reported) {
    dep_wait();
    dep_launch();
    atomicSub(&g_faults, reported);
}

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
    int polls;                          // CHECK: looks after which a wait gives up
};

// ------------------------------------------------------------ the tensor-core path
//
// Both operands stay in 4 bits all the way; the tensor core takes their blocks' powers of two from
// TMEM.  A stage is 256 columns of K (128 bytes of codes a row): tcgen05.cp of its exponents, then four
// tcgen05.mma of 64 columns each.  Threads load by TMA, each one part of every stage, into rings of
// slots, and other warps take the other one of two accumulators to the logits meanwhile.
constexpr int KS = 256;                       // columns of K of a stage
constexpr int SF = 512;                       // a tile of exponents: 128 rows by 128 columns, as it lies in memory
constexpr int EPILOGUE = 8, FIRST = 8;        // warps of the epilogue, the first of them
constexpr int MMA_THREADS = 32 * (FIRST + EPILOGUE);

// Descriptors by their low words (addresses in units of 16 bytes).  Exponents' tiles: 32 rows of 16
// bytes, 8 rows every 128 bytes, no swizzle; operands: operand_desc's.
__device__ __forceinline__ uint64_t exponent_desc(uint32_t lo) {
    return (uint64_t)(8u | (1u << 14)) << 32 | (lo | (8u << 16));
}
__device__ __forceinline__ uint64_t codes_desc(uint32_t lo) {
    return (uint64_t)(64u | (1u << 14) | (2u << 29)) << 32 | (lo | (1u << 16));
}
// D f32; A and B of E2M1, both along K; exponents alone as scales; N and M.
__device__ __forceinline__ uint32_t instruction(int m, int n) {
    return (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(m >> 4) << 24);
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
// A stage's exponents (two tiles a row) to TMEM from column sf on: four columns each of side A's 128
// rows, then of side B's B_TILES times 128; a, b: where they are, in units of 16 bytes.
template <bool PAIR, int B_TILES>
__device__ __forceinline__ void copy_stage(uint32_t a, uint32_t b, uint32_t sf) {
#pragma unroll
    for (int c = 0; c < 2; c++) {
        copy_exponents<PAIR>(sf + 4 * c, a + 32 * c);
#pragma unroll
        for (int j = 0; j < B_TILES; j++) copy_exponents<PAIR>(sf + 8 + 4 * B_TILES * c + 4 * j, b + 64 * j + 32 * c);
    }
}
// A stage's products; a, b: the operands' slots in units of 16 bytes; shift: where B's exponents begin.
// Past K codes and exponents are zeros, as the TMA fills them in.
template <bool PAIR, int B_TILES>
__device__ __forceinline__ void mma_stage(uint32_t a, uint32_t b, uint32_t sf, uint32_t shift, uint32_t d, uint32_t idesc,
                                          uint32_t add) {
#pragma unroll
    for (int c = 0; c < 2; c++)
#pragma unroll
        for (int i = 0; i < 2; i++)               // the first or the second two of a word's four exponents
            mma_mx4<PAIR>(d, codes_desc(a + 4 * c + 2 * i), codes_desc(b + 4 * c + 2 * i),
                          idesc | (2u * i << 29) | (2u * i << 4), sf + 4 * c, sf + 8 + 4 * B_TILES * c + shift, add | c | i);
}
template <bool PAIR>
__device__ __forceinline__ void tmem_alloc(uint32_t* to) {
    if (PAIR) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(to)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(to)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
}
template <bool PAIR>
__device__ __forceinline__ void tmem_free(uint32_t tmem) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}
// A tile on its way to the L2.
__device__ __forceinline__ void prefetch_tile(const CUtensorMap* map, int x, int y) {
    asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(map), "r"(x), "r"(y) : "memory");
}
// A map's own bytes on their way to the TMA.
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
// After a wait that gave up: blocks end only when nothing is under way to their memory any more.  All warps
// have left their loops by then, and some may have loaded stages that others did not come to; those arrive without
// their copies, so that every stage that any warp began completes when its copies have landed.  (A stage begins when
// the one before it in its slot has been used, so it was complete, and no slot has two stages that are not.)
__device__ __forceinline__ void drain(uint32_t full0, int stages, int slots) {
    int left = 1 << 20;
    for (int i = max(0, stages - slots); i < stages; i++)
        while (left > 0 && !mbar_try(full0 + 8 * (i % slots), (i / slots) & 1)) left--;
}
__device__ __forceinline__ void drain_products(uint32_t bar) {
    for (int it = 0; it < (1 << 20) && !mbar_try(bar, 0); it++) {}
}

// -------------------------------------------------------------------- up to 128 tokens
//
// k_mx4_few: a persistent block per SM over tiles of 128 vocabulary rows (the tensor core's M) by all
// tokens (its N): with few tokens the weights' bytes are all that counts, and tensor cores that give
// most of their columns away keep up with them.
// Bound by memory and its beginning and end: 1 token over 128,256 x 2048 takes 23.1 us (140 MB, 6.1 TB/s), 64 tokens
// 24.7; 16 tokens over 151,936 x 1024 under masks that leave a few dozen tokens each 12.1 us, mostly latency (the masks,
// then the first stages) and the -inf of the other tiles.  Device times of calls that follow each other; behind the
// norm, which a step has in front, 27.3 and 15.2 with it.
//   warps 0, 2-4  TMA: the weights' codes (16 KB a stage), the tokens', both sides' exponents
//   warp 1        the exponents' way to TMEM, the products
//   warps 8-15    a lane per vocabulary row, two warps for 32 of them: scales, mask, logits
constexpr int FEW = 128;                      // tokens at most
constexpr int VT = 128;                       // vocabulary rows of a tile
constexpr int W_CODES = VT * KS / 2;
constexpr int MAX_STAGES = 11;
constexpr int GROUPS = FEW / 32 / 2;          // a warp's groups of 32 tokens
constexpr int WARM = 24;                      // stages whose weights are prefetched (1 token over 128,256 x 2048, norm in front: 28.3 us without, 26.5)
constexpr int MAX_TILES = 8192;               // of a block, for which masks are looked at beforehand

struct Few {
    int N, n_vt;                              // tokens, rounded up; tiles of vocabulary rows
    int stages, stage_bytes;
    int acc;                                  // TMEM columns of an accumulator
    size_t smem;
};

Few few_of(int T, int V) {
    Few p;
    p.N = (T + 15) / 16 * 16;
    p.n_vt = (V + VT - 1) / VT;
    p.stage_bytes = W_CODES + p.N * KS / 2 + 4 * SF;
    p.acc = (p.N + 31) / 32 * 32;
    // a stage's exponents have TMEM columns of their own, free when the stage is
    p.stages = std::min({MAX_STAGES, (SMEM_MAX - 7 * 1024) / p.stage_bytes, (512 - 2 * p.acc) / 16});
    p.smem = 1024 + (size_t)p.stages * p.stage_bytes;
    return p;
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
            if (j >= n) break;
            if (left > 0) store_f32(out, logit<MASKED>(y[j], tokens[j].scale, tokens[j].word, sw, bit));
            out += stride;
        }
    }
}

// -inf for `n` neighbouring logits of each of T tokens, by the epilogue's warps.
template <typename T>
__device__ __forceinline__ void forbid_tile(T* out, int64_t stride, int tokens, int n, bool wide) {
    constexpr uint32_t NONE = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
    constexpr int EACH = 16 / sizeof(T);
    const int warp = (threadIdx.x >> 5) - FIRST, lane = threadIdx.x & 31;
    if (wide && n == VT) {
        constexpr int LANES = VT / EACH;              // of a token
        for (int t = warp * (32 / LANES) + lane / LANES; t < tokens; t += EPILOGUE * (32 / LANES))
            *reinterpret_cast<uint4*>(out + (size_t)t * stride + lane % LANES * EACH) = make_uint4(NONE, NONE, NONE, NONE);
    } else {
        for (int t = warp; t < tokens; t += EPILOGUE)
            for (int i = lane; i < n; i += 32) store_f32(out + (size_t)t * stride + i, __uint_as_float(0xFF800000u));
    }
}

// What drain's comment says, by all warps of the block.  (Not inline, so that the kernel's last instructions do not lie
// behind it: 79 tokens over 71,701 x 96, 15.1 us, take 0.1 more with it inline.)
__device__ __noinline__ void settle_few(uint32_t full0, int slots, uint32_t drained, const int* loaded) {
    const int warp = threadIdx.x >> 5;
    const bool issuer = elect_one();                  // the lane that issued (it is the same every time)
    if (warp == 1 && issuer) {
        mma_commit<false>(drained);
        drain_products(drained);
    } else if (warp <= 4 && issuer) {
        const int most = max(max(loaded[0], loaded[1]), max(loaded[2], loaded[3]));
        for (int i = loaded[max(0, warp - 1)]; i < most; i++) mbar_arrive(full0 + 8 * (i % slots));
        drain(full0, most, slots);
    }
    __syncwarp();
}

template <typename T, bool MASKED, bool CHECK>
__global__ void __launch_bounds__(MMA_THREADS, 1) k_mx4_few(const __grid_constant__ CUtensorMap w_map,
                                                            const __grid_constant__ CUtensorMap x_map,
                                                            const __grid_constant__ CUtensorMap w_blocks_map,
                                                            const __grid_constant__ CUtensorMap x_blocks_map, Head h,
                                                            T* logits, Few p, bool even, bool wide) {
    extern __shared__ uint8_t dyn[];
    __shared__ __align__(8) uint64_t s_bars[2 * MAX_STAGES + 5];
    __shared__ __align__(16) Token s_tokens[EPILOGUE][GROUPS * 32];
    __shared__ uint32_t s_active[MASKED ? MAX_TILES / 32 : 1];
    __shared__ uint32_t s_tmem;
    __shared__ int s_failed, s_loaded[4];             // stages that each loading warp has begun
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // stages start at multiples of 1024 bytes: weights, tokens, the weights' exponents, the tokens'
    const uint32_t base = (smem_addr(dyn) + 1023) & ~1023u, x_codes = p.N * KS / 2;
    const uint32_t bars = smem_addr(s_bars);
    auto full = [&](int s) { return bars + 8 * s; };
    auto empty = [&](int s) { return bars + 8 * (MAX_STAGES + s); };
    auto acc_full = [&](int s) { return bars + 8 * (2 * MAX_STAGES + s); };
    auto acc_empty = [&](int s) { return bars + 8 * (2 * MAX_STAGES + 2 + s); };
    const uint32_t drained = bars + 8 * (2 * MAX_STAGES + 4);

    if (warp == 2 && lane < 4)
        prefetch_map(lane == 0 ? &w_map : lane == 1 ? &x_map : lane == 2 ? &w_blocks_map : &x_blocks_map);
    if (threadIdx.x == 0) {
        s_failed = 0;
        for (int s = 0; s < p.stages; s++) mbar_init(full(s), 4), mbar_init(empty(s), 1);
        for (int s = 0; s < 2; s++) mbar_init(acc_full(s), 1), mbar_init(acc_empty(s), EPILOGUE);
        mbar_init(drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc<false>(&s_tmem);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = s_tmem;
    volatile int* failed = &s_failed;
    const int n_k = (h.K + KS - 1) / KS;
    if (!MASKED && warp == 0 && lane == 0)            // the first stages' weights on their way to the L2, while others finish
        for (int i = 0, k = 0, vt = blockIdx.x; i < WARM && vt < p.n_vt; i++) {
            prefetch_tile(&w_map, k * 128, vt * VT);
            if (++k == n_k) k = 0, vt += gridDim.x;
        }
    dep_wait();
    dep_launch();
    // Of this block's tiles, those in which some token is allowed; the others' weights are not read.
    const int mine = (p.n_vt - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;
    if (MASKED) {
        for (int i = threadIdx.x; i < MAX_TILES / 32; i += MMA_THREADS) s_active[i] = mine > MAX_TILES ? FULL : 0u;
        __syncthreads();
        for (int i = warp; i < min(mine, MAX_TILES); i += MMA_THREADS / 32) {
            uint32_t any = 0;
            // a lane per word of a token's four, eight tokens at a time
            const int wi = (blockIdx.x + i * gridDim.x) * 4 + (lane & 3);
            if (wi < h.W)
#pragma unroll 4
                for (int t = lane >> 2; t < h.T; t += 8) any |= h.bitmask[(size_t)t * h.W + wi];
            if (__any_sync(FULL, any) && lane == 0) atomicOr(&s_active[i / 32], 1u << (i & 31));
        }
        __syncthreads();
    }
    auto is_active = [&](int i) { return !MASKED || mine > MAX_TILES || (s_active[i / 32] >> (i & 31) & 1); };
    const int vt0 = blockIdx.x, vt_step = gridDim.x;  // tile i of this block

    // Loads one part of every stage: a box at (x, y), x + step, ... of a map; y_step: from tile to tile.  All lanes
    // leave together, by what the warp's wait said (the flag itself may change between two lanes' looks at it).
    auto load_part = [&](int loader, const CUtensorMap* map, int step, int y_step, int part, int bytes) {
        const bool issuer = elect_one();
        Place at;
        int c = 0;
        bool ok = true;
        for (int i = 0; i < mine && ok; i++) {
            if (!is_active(i)) continue;
            const int vt = vt0 + i * vt_step;
            for (int k = 0; k < n_k; k++, c++, at.next(p.stages)) {
                const uint32_t to = base + at.s * p.stage_bytes + part, bar = full(at.s);
                if (!(ok = warp_wait<CHECK>(empty(at.s), at.parity ^ 1, failed, h.polls))) break;
                if (issuer) {
                    mbar_arrive_tx(bar, bytes);
                    tma_2d(to, map, k * step, vt * y_step, bar);
                }
            }
        }
        if (issuer) s_loaded[loader] = c;
    };

    if (warp == 0) {
        load_part(0, &w_map, 128, VT, 0, W_CODES);
    } else if (warp == 2) {
        load_part(1, &x_map, 128, 0, W_CODES, x_codes);
    } else if (warp == 3) {
        load_part(2, &w_blocks_map, 256, 1, W_CODES + x_codes, 2 * SF);
    } else if (warp == 4) {
        load_part(3, &x_blocks_map, 256, 0, W_CODES + x_codes + 2 * SF, 2 * SF);
    } else if (warp == 1) {
        // The whole warp waits, so that addresses and descriptors stay in uniform registers; one lane issues.
        const bool issuer = elect_one();
        const uint32_t lo = (base & 0x3FFFF) >> 4, step = p.stage_bytes / 16, idesc = instruction(VT, p.N);
        Place at, acc;
        bool ok = true;
        for (int i = 0; i < mine && ok; i++) {
            if (!is_active(i)) continue;
            if (!(ok = warp_wait<CHECK>(acc_empty(acc.s), acc.parity ^ 1, failed, h.polls))) break;
            const uint32_t d = tmem + acc.s * p.acc;
            for (int k = 0; k < n_k; k++, at.next(p.stages)) {
                const uint32_t a = lo + at.s * step, b = a + W_CODES / 16, e = b + x_codes / 16;
                const uint32_t sf = tmem + 2 * p.acc + at.s * 16;
                if (!(ok = warp_wait<CHECK>(full(at.s), at.parity, failed, h.polls))) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (issuer) {
                    copy_stage<false, 1>(e, e + 64, sf);
                    mma_stage<false, 1>(a, b, sf, 0, d, idesc, k);
                    mma_commit<false>(empty(at.s));
                    if (k + 1 == n_k) mma_commit<false>(acc_full(acc.s));
                }
            }
            acc.next(2);
        }
    } else if (warp >= FIRST) {
        const int quad = warp & 3, part = (warp - FIRST) >> 2;      // of every two groups of 32 tokens, this warp's
        Token* tokens = s_tokens[warp - FIRST];
        Place acc;
        for (int it = 0; it < mine; it++) {
            const int vt = vt0 + it * vt_step;
            if (!is_active(it)) {
                forbid_tile(logits + vt * VT, h.row_stride, h.T, min(VT, h.V - vt * VT), wide);
                continue;
            }
            const int v = vt * VT + quad * 32 + lane, wi = vt * 4 + quad;
            // the tile's scales and mask words, read while its products run
            const float sw = v < h.V && h.w_scale ? h.w_scale[v] : 1.f;
            __syncwarp();
#pragma unroll
            for (int i = 0; i < GROUPS; i++) {
                const int t = (2 * i + part) * 32 + lane;
                if (t >= h.T) continue;
                tokens[i * 32 + lane] = {
                    h.scale ? h.scale[t] : 1.f,
                    !MASKED ? FULL : wi < h.W ? h.bitmask[(size_t)t * h.W + wi] : 0u};
            }
            __syncwarp();
            if (!warp_wait<CHECK>(acc_full(acc.s), acc.parity, failed, h.polls)) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
            for (int i = 0; i < GROUPS; i++) {
                const int t = (2 * i + part) * 32;
                if (t >= h.T) break;
                uint32_t y[32];
                const uint32_t from = tmem + ((uint32_t)(quad * 32) << 16) + acc.s * p.acc + t;
                tmem_load16(from, y);
                tmem_load16(from + 16, y + 16);
                tmem_wait(y);
                store_group<MASKED>(logits + (size_t)t * h.row_stride + v, h.row_stride, y, tokens + i * 32, sw,
                                    min(32, h.T - t), h.V - v, even);
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(acc_empty(acc.s));
            acc.next(2);
        }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (*failed) {                                    // nobody writes the flag any more
        settle_few(bars, p.stages, drained, s_loaded);
        if (threadIdx.x == 0) atomicAdd(&g_faults, 1);
        __syncthreads();
    }
    if (warp == 1) tmem_free<false>(tmem);
}

template <typename T, bool CHECK>
psc_status head_few(const Head& h, T* logits, cudaStream_t cs) {
    const Few p = few_of(h.T, h.V);
    CUtensorMap w_map, x_map, w_blocks_map, x_blocks_map;
    const uint64_t row = (h.K + 31) / 32 * 16, n_tiles = (h.K + 127) / 128;
    if (!tensor_map(&w_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, h.w, row, h.V, h.w_stride, 128, VT) ||
        !tensor_map(&x_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, h.q, row, h.T, h.q_stride, 128, p.N) ||
        !tensor_map(&w_blocks_map, CU_TENSOR_MAP_DATA_TYPE_UINT32, h.w_blocks, n_tiles * SF / 4, p.n_vt, n_tiles * SF,
                    256, 1, CU_TENSOR_MAP_SWIZZLE_NONE) ||
        !tensor_map(&x_blocks_map, CU_TENSOR_MAP_DATA_TYPE_UINT32, h.q_blocks, n_tiles * SF / 4, 1, n_tiles * SF, 256, 1,
                    CU_TENSOR_MAP_SWIZZLE_NONE))
        return ops_fail(PSC_ERR_CUDA, ME, "cuTensorMapEncodeTiled failed");
    const int64_t stride = h.row_stride * (int64_t)sizeof(T);
    const bool even = is_aligned(logits, stride, 4), wide = is_aligned(logits, stride, 16);
    return ops_launch(h.bitmask ? k_mx4_few<T, true, CHECK> : k_mx4_few<T, false, CHECK>, dim3(std::min(p.n_vt, current_sms())),
                      MMA_THREADS, p.smem, 1, cs, "k_mx4_few", w_map, x_map, w_blocks_map, x_blocks_map, h, logits, p,
                      even, wide);
}

// ------------------------------------------------------------------------ many tokens
//
// k_mx4_many: pairs of blocks (tcgen05's cta_group::2) over tiles of 256 tokens (the tensor core's M, 128
// in each block) by 192 vocabulary rows (its N; half of their codes in each block, all of their
// exponents in both).  Where a tile's tokens fit shared memory (K up to 2048) they stay there, and
// only the weights are loaded, from memory once and from the L2 for the other tiles of tokens: an SM
// takes in 64 bytes a cycle, and a stage's 384 cycles of products need 14 KB this way, 31 KB where
// the tokens come along.  256 tokens over 128,256 x 4096: 58 us, at the memory's latency (seven slots, 86 KB of
// weights an SM); 1024 over it 192 us, 5.6 PFLOP/s, 1024 over 262,144 x 2048 under mixed masks 183, 6.0 PFLOP/s beside
// 537 MB of logits, at 2.07 GHz: calls that follow each other for milliseconds.  For seconds the GPU's power cap
// takes the clock to 1.75 GHz, and the last of these to 218 us.  (With the norm in front 63 and 206 us.)
// A lane of the epilogue has a token, and 32 neighbouring logits of it with one word of the mask; they go out by
// way of shared memory, 64 bytes of a token at a time.
//   warps 0, 2-4  TMA: the weights' codes and exponents, the tokens' codes and exponents
//   warp 5        the exponents' way to TMEM
//   warp 1        the products
//   warps 8-15    32 tokens by 96 vocabulary rows each
constexpr int MT = 256;                       // tokens of a tile
constexpr int NV = 192;                       // vocabulary rows of a tile
constexpr int TOGETHER = 4;                   // tiles of tokens that are worked on at the same time
constexpr int A_CODES = MT / 2 * KS / 2, A_BYTES = A_CODES + 2 * SF;
constexpr int B_CODES = NV / 2 * KS / 2, B_EXPS = 4 * SF;
constexpr int MAX_A = 8, MAX_B = 16;          // slots for the tokens, for the weights' codes
constexpr int SF_SLOTS = 5;                   // for the weights' exponents, and in TMEM for a stage's
constexpr int SF_COLS = 24;                   // TMEM columns of a stage's exponents
static_assert(2 * NV + SF_SLOTS * SF_COLS <= 512, "TMEM");
constexpr int STAGING = 32 * 64;              // a warp's, in the epilogue
constexpr int SLOTS_BYTES = MAX_A * A_BYTES + 5 * B_CODES;            // for the tokens and the weights' codes
constexpr size_t MANY_SMEM = 1024 + SLOTS_BYTES + SF_SLOTS * B_EXPS + EPILOGUE * STAGING;

// A tile into this block's shared memory; the barrier is the pair's first block's.
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
// The address of the first block's barrier in the pair's shared memory.
__device__ __forceinline__ uint32_t at_first(uint32_t bar) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(bar));
    return r;
}
// A word of the pair's other block; how to set it.
__device__ __forceinline__ int read_other(const int* p, int other) {
    int v;
    asm volatile("{\n .reg .b32 r;\n mapa.shared::cluster.u32 r, %1, %2;\n ld.shared::cluster.s32 %0, [r];\n}"
                 : "=r"(v)
                 : "r"(smem_addr(p)), "r"(other)
                 : "memory");
    return v;
}
__device__ __forceinline__ void set_other(int* p, int other) {
    asm volatile("{\n .reg .b32 r;\n mapa.shared::cluster.u32 r, %0, %1;\n st.shared::cluster.s32 [r], 1;\n}" ::"r"(smem_addr(p)),
                 "r"(other)
                 : "memory");
}
// Takes `bytes` that do not come off what a barrier of this block waits for.
__device__ __forceinline__ void forgo_bytes(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Arrives at this block's barrier when the pair's copies and products so far are done.
__device__ __forceinline__ void commit_here(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Two products at once.
__device__ __forceinline__ void times2(uint32_t& a, uint32_t& b, float x, float y) {
    asm("{\n .reg .b64 u, v;\n mov.b64 u, {%0, %1};\n mov.b64 v, {%2, %3};\n mul.rn.f32x2 u, u, v;\n"
        " mov.b64 {%0, %1}, u;\n}"
        : "+r"(a), "+r"(b)
        : "f"(x), "f"(y));
}

// The top bit of byte i of a, in all bits of the low half, and that of b in the high half.
__device__ __forceinline__ uint32_t both_bytes(uint32_t a, uint32_t b, int i) {
    uint32_t r;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(0xCC88u + 0x1111u * i));
    return r;
}

// What drain's comment says, by all warps of both blocks (not inline, as settle_few).
__device__ __noinline__ void settle_many(uint32_t a_full0, int a_slots, uint32_t b_full0, int b_slots, uint32_t e_full0,
                                         uint32_t drained, const int* loaded) {
    const int warp = threadIdx.x >> 5, side = (int)cluster_rank();
    const bool issuer = elect_one();                  // the lane that issued (it is the same every time)
    if (side == 0 && (warp == 1 || warp == 5) && issuer) mma_commit<true>(drained);
    if (warp == 1 && issuer) drain_products(drained);
    // both blocks' copies are counted at the first's barriers: there a stage takes an arrival with the bytes of
    // both, of each of its loaders
    auto finish = [&](int loader, uint32_t full0, int slots, int bytes, int most) {
        const int own = loaded[loader], theirs = read_other(&loaded[loader], 1);
        for (int i = own; i < most; i++) {
            if (i < theirs) mbar_arrive_tx(full0 + 8 * (i % slots), bytes);
            else mbar_arrive(full0 + 8 * (i % slots));
        }
        for (int i = theirs; i < own; i++) forgo_bytes(full0 + 8 * (i % slots), bytes);
        drain(full0, most, slots);
    };
    auto begun = [&](int loader) { return max(loaded[loader], read_other(&loaded[loader], 1)); };
    if (side == 0 && issuer) {
        if (warp == 0) finish(0, b_full0, b_slots, B_CODES, begun(0));
        if (warp == 2) finish(1, e_full0, SF_SLOTS, B_EXPS, begun(1));
        if (warp == 3) finish(2, a_full0, a_slots, A_CODES, max(begun(2), begun(3)));
        if (warp == 4) finish(3, a_full0, a_slots, 2 * SF, max(begun(2), begun(3)));
    }
    __syncwarp();
}

template <typename T, bool MASKED, bool CHECK>
__global__ void __launch_bounds__(MMA_THREADS, 1) k_mx4_many(const __grid_constant__ CUtensorMap w_map,
                                                             const __grid_constant__ CUtensorMap x_map,
                                                             const __grid_constant__ CUtensorMap w_blocks_map,
                                                             const __grid_constant__ CUtensorMap x_blocks_map, Head h,
                                                             T* logits, int n_mt, int n_vt, bool wide) {
    extern __shared__ uint8_t dyn[];
    __shared__ __align__(8) uint64_t s_bars[2 * MAX_A + 2 * MAX_B + 4 * SF_SLOTS + 5];
    __shared__ __align__(16) float s_scale[EPILOGUE][NV / 2];
    __shared__ uint32_t s_tmem;
    __shared__ int s_failed, s_item;                  // how many items' weights have begun to be loaded
    __shared__ int s_other_failed, s_loaded[4];       // stages that each loading warp has begun
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int side = (int)cluster_rank();
    // slots start at multiples of 1024 bytes: the tokens' codes and exponents, the weights' codes, their exponents
    // Tokens that do not stay come from the L2, weights from memory, which takes longer (256 tokens over 128,256 x
    // 4096, norm in front: 64.4 us with 4 slots for the tokens and 10 for the weights, 62.8 with 6 and 7, 64.5 with 7 and 6).
    const int n_k = (h.K + KS - 1) / KS;
    const bool stay = n_k <= MAX_A;
    const int a_slots = stay ? n_k : 6, b_slots = min(MAX_B, (SLOTS_BYTES - a_slots * A_BYTES) / B_CODES);
    const uint32_t base = (smem_addr(dyn) + 1023) & ~1023u, b_base = base + a_slots * A_BYTES;
    const uint32_t e_base = base + SLOTS_BYTES;
    const uint32_t bars = smem_addr(s_bars);
    auto a_full = [&](int s) { return bars + 8 * s; };
    auto a_empty = [&](int s) { return bars + 8 * (MAX_A + s); };
    auto b_full = [&](int s) { return bars + 8 * (2 * MAX_A + s); };
    auto b_empty = [&](int s) { return bars + 8 * (2 * MAX_A + MAX_B + s); };
    constexpr int SF_BARS = 2 * (MAX_A + MAX_B), LAST = SF_BARS + 4 * SF_SLOTS;
    auto e_full = [&](int s) { return bars + 8 * (SF_BARS + s); };
    auto e_empty = [&](int s) { return bars + 8 * (SF_BARS + SF_SLOTS + s); };
    auto sf_full = [&](int s) { return bars + 8 * (SF_BARS + 2 * SF_SLOTS + s); };
    auto sf_empty = [&](int s) { return bars + 8 * (SF_BARS + 3 * SF_SLOTS + s); };
    auto acc_full = [&](int s) { return bars + 8 * (LAST + s); };
    auto acc_empty = [&](int s) { return bars + 8 * (LAST + 2 + s); };
    const uint32_t drained = bars + 8 * (LAST + 4);

    if (warp == 2 && lane < 4)
        prefetch_map(lane == 0 ? &w_map : lane == 1 ? &x_map : lane == 2 ? &w_blocks_map : &x_blocks_map);
    if (threadIdx.x == 0) {
        s_failed = 0, s_item = 0, s_other_failed = 0;
        for (int s = 0; s < a_slots; s++) mbar_init(a_full(s), 2), mbar_init(a_empty(s), 1);
        for (int s = 0; s < b_slots; s++) mbar_init(b_full(s), 1), mbar_init(b_empty(s), 1);
        for (int s = 0; s < SF_SLOTS; s++) {
            mbar_init(e_full(s), 1), mbar_init(e_empty(s), 1);
            mbar_init(sf_full(s), 1), mbar_init(sf_empty(s), 1);
        }
        for (int s = 0; s < 2; s++) mbar_init(acc_full(s), 1), mbar_init(acc_empty(s), EPILOGUE * 2);
        mbar_init(drained, 2);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    cluster_sync();
    if (warp == 1) tmem_alloc<true>(&s_tmem);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = s_tmem;
    volatile int* failed = &s_failed;
    dep_wait();
    dep_launch();
    // This pair's items, in order: up to TOGETHER tiles of tokens at a time, a pair staying with one of
    // them; pairs that share a tile of vocabulary rows come to it at the same time.  f(tile of tokens, of
    // vocabulary rows, whether its tokens are new, whether they are not used after it) says whether to go on.
    const int me = blockIdx.x / 2, all = gridDim.x / 2;
    auto each = [&](auto f) {
        for (int m0 = 0; m0 < n_mt; m0 += TOGETHER) {
            const int c = min(min(TOGETHER, n_mt - m0), all), per = all / c, g = me / c;
            if (g >= per) continue;
            for (int m = m0 + me % c; m < min(m0 + TOGETHER, n_mt); m += c)
                for (int vt = g; vt < n_vt; vt += per)
                    if (!f(m, vt, vt == g || !stay, vt + per >= n_vt || !stay)) return;
        }
    };
    // vocabulary rows of a tile that the products take: both halves in whole sixteens
    auto rows_of = [&](int vt) { return (min(NV, h.V - vt * NV) + 31) / 32 * 32; };

    // Loads one part of every stage (of tokens that stay, of the first item with them).  All lanes leave together,
    // by what the warp's wait said.
    auto load_part = [&](int loader, const CUtensorMap* map, int step, uint32_t to0, int slot_bytes, int slots, uint32_t full0,
                         uint32_t empty0, int bytes, bool tokens, auto row_of) {
        const uint32_t there0 = at_first(full0);
        const bool issuer = elect_one();
        Place at;
        int c = 0;
        each([&](int mt, int vt, bool fresh, bool) {
            if (tokens && !fresh) return true;
            const int y = row_of(mt, vt);
            int x = 0;
            for (int k = 0; k < n_k; k++, c++, x += step, at.next(slots)) {
                const uint32_t to = to0 + at.s * slot_bytes, own = full0 + 8 * at.s, bar = there0 + 8 * at.s;
                if (!warp_wait<CHECK>(empty0 + 8 * at.s, at.parity ^ 1, failed, h.polls)) return false;
                if (issuer) {
                    if (side == 0) mbar_arrive_tx(own, 2 * bytes);
                    load_tile(to, map, x, y, bar);
                }
            }
            return true;
        });
        if (issuer) s_loaded[loader] = c;
    };

    auto codes_row = [&](int, int vt) { return vt * NV + side * (rows_of(vt) / 2); };
    if (warp == 0) {
        load_part(0, &w_map, 128, b_base, B_CODES, b_slots, b_full(0), b_empty(0), B_CODES, false, codes_row);
    } else if (warp == 2) {
        load_part(1, &w_blocks_map, 256, e_base, B_EXPS, SF_SLOTS, e_full(0), e_empty(0), B_EXPS, false, [&](int, int vt) {
            *const_cast<volatile int*>(&s_item) = s_item + 1;
            return vt * NV / 128;
        });
    } else if (warp == 6 && lane == 0) {
        // Brings the next item's weights to the L2 when an item's are loaded: the slots cover the L2's latency, not
        // the memory's.  Pairs that come to a tile together share its stages out.
        int item = 0;
        each([&](int mt, int vt, bool, bool) {
            const int c = min(min(TOGETHER, n_mt - mt / TOGETHER * TOGETHER), all), next = vt + all / c;
            item++;
            if (c == 1 || next >= n_vt) return true;
            for (int i = 0; i < (1 << 16) && *const_cast<volatile int*>(&s_item) < item && !*failed; i++) __nanosleep(100);
            for (int k = me % c; k < n_k; k += c) prefetch_tile(&w_map, k * 128, codes_row(0, next));
            return !*failed;
        });
    } else if (warp == 3) {
        load_part(2, &x_map, 128, base, A_BYTES, a_slots, a_full(0), a_empty(0), A_CODES, true,
                  [&](int mt, int) { return mt * MT + side * (MT / 2); });
    } else if (warp == 4) {
        load_part(3, &x_blocks_map, 256, base + A_CODES, A_BYTES, a_slots, a_full(0), a_empty(0), 2 * SF, true,
                  [&](int mt, int) { return mt * 2 + side; });
    } else if (warp == 5 && side == 0) {
        // The whole warp waits, so that addresses and descriptors stay in uniform registers; one lane
        // issues, for both blocks.  Exponents go to TMEM as soon as the products of SF_SLOTS stages before are
        // done with theirs, while the codes that take those products' place are still on their way.
        const bool issuer = elect_one();
        const uint32_t a_lo = ((base + A_CODES) & 0x3FFFF) >> 4, e_lo = (e_base & 0x3FFFF) >> 4;
        Place unit, at;                               // unit: the first slot of the tile's tokens
        each([&](int, int, bool fresh, bool last) {
            Place at_a = unit;
            for (int k = 0; k < n_k; k++, at_a.next(a_slots), at.next(SF_SLOTS)) {
                const uint32_t a = a_lo + at_a.s * (A_BYTES / 16), e = e_lo + at.s * (B_EXPS / 16);
                const uint32_t sf = tmem + 2 * NV + at.s * SF_COLS;
                if (!warp_wait2<CHECK>(e_full(at.s), at.parity, sf_empty(at.s), at.parity ^ 1, failed, h.polls) ||
                    (fresh && !warp_wait<CHECK>(a_full(at_a.s), at_a.parity, failed, h.polls)))
                    return false;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (issuer) {
                    copy_stage<true, 2>(a, e, sf);
                    commit_here(sf_full(at.s));
                    mma_commit<true>(e_empty(at.s));
                }
            }
            if (last) unit = at_a;
            return true;
        });
    } else if (warp == 1 && side == 0) {
        const bool issuer = elect_one();
        const uint32_t a_lo = (base & 0x3FFFF) >> 4, b_lo = (b_base & 0x3FFFF) >> 4;
        Place unit, at_b, at_e, acc;
        each([&](int, int vt, bool fresh, bool last) {
            const uint32_t idesc = instruction(MT, rows_of(vt)), d = tmem + acc.s * NV, shift = vt * NV % 128 / 32;
            Place at_a = unit;
            if (!warp_wait<CHECK>(acc_empty(acc.s), acc.parity ^ 1, failed, h.polls)) return false;
            for (int k = 0; k < n_k; k++, at_a.next(a_slots), at_b.next(b_slots), at_e.next(SF_SLOTS)) {
                const uint32_t a = a_lo + at_a.s * (A_BYTES / 16), b = b_lo + at_b.s * (B_CODES / 16);
                const uint32_t sf = tmem + 2 * NV + at_e.s * SF_COLS;
                if (!warp_wait2<CHECK>(sf_full(at_e.s), at_e.parity, b_full(at_b.s), at_b.parity, failed, h.polls) ||
                    (fresh && !warp_wait<CHECK>(a_full(at_a.s), at_a.parity, failed, h.polls)))
                    return false;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (issuer) {
                    mma_stage<true, 2>(a, b, sf, shift, d, idesc, k);
                    mma_commit<true>(b_empty(at_b.s));
                    commit_here(sf_empty(at_e.s));
                    if (last) mma_commit<true>(a_empty(at_a.s));
                    if (k + 1 == n_k) mma_commit<true>(acc_full(acc.s));
                }
            }
            if (last) unit = at_a;
            acc.next(2);
            return true;
        });
    } else if (warp >= FIRST) {
        constexpr int COLS = 64 / sizeof(T);          // logits of a token that go out together
        const int quad = warp & 3, part = (warp - FIRST) >> 2;
        const uint32_t staging = e_base + SF_SLOTS * B_EXPS + (warp - FIRST) * STAGING;
        const uint32_t own = staging + lane * 64, own_swap = (lane >> 1) & 3;       // 16-byte pieces change places by rows
        float* scales = s_scale[warp - FIRST];
        Place acc;
        each([&](int mt, int vt, bool, bool) {
            const int t0 = mt * MT + side * (MT / 2) + quad * 32, t = t0 + lane;
            const int v0 = vt * NV + part * (NV / 2);
            // scales and mask words, read while the products run
            const float st = t < h.T && h.scale ? h.scale[t] : 1.f;
            uint32_t words[3];
#pragma unroll
            for (int i = 0; i < 3; i++) {
                const int wi = v0 / 32 + i;
                words[i] = !MASKED ? FULL : t < h.T && wi < h.W ? h.bitmask[(size_t)t * h.W + wi] : 0u;
            }
            if (h.w_scale) {
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 3; i++)
                    if (v0 + i * 32 + lane < h.V) scales[i * 32 + lane] = h.w_scale[v0 + i * 32 + lane];
                __syncwarp();
            }
            if (!warp_wait<CHECK>(acc_full(acc.s), acc.parity, failed, h.polls)) return false;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            T* rows = logits + (size_t)(t0 + (lane >> 2)) * h.row_stride + v0 + (lane & 3) * (COLS / 4);
#pragma unroll
            for (int i = 0; i < 3; i++) {
                const int n = min(32, h.V - v0 - i * 32);             // vocabulary rows that there are
                uint32_t y[32];
                if (t0 < h.T && n > 0) {
                    const uint32_t from = tmem + ((uint32_t)(quad * 32) << 16) + acc.s * NV + part * (NV / 2) + i * 32;
                    tmem_load16(from, y);
                    tmem_load16(from + 16, y + 16);
                    tmem_wait(y);
                }
                if (i == 2) {                         // the accumulator is free
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) arrive_at_first(acc_empty(acc.s));
                }
                if (t0 >= h.T || n <= 0) continue;
#pragma unroll
                for (int j = 0; j < 32; j += 2) times2(y[j], y[j + 1], st, st);
                if (h.w_scale) {
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        const float4 s = *reinterpret_cast<const float4*>(scales + i * 32 + j);
                        times2(y[j], y[j + 1], s.x, s.y);
                        times2(y[j + 2], y[j + 3], s.z, s.w);
                    }
                }
                if (MASKED && sizeof(T) == 4) {
#pragma unroll
                    for (int j = 0; j < 32; j++)
                        if (!((words[i] >> j) & 1)) y[j] = 0xFF800000u;
                }
                uint32_t spread[8];                   // bit b of the word as the top bit of byte b / 8 of spread[b % 8]
#pragma unroll
                for (int j = 0; j < 8; j++) spread[j] = words[i] << (7 - j);
#pragma unroll
                for (int half = 0; half < (int)sizeof(T) / 2; half++) {       // 64 bytes a token
                    uint32_t u[16];
#pragma unroll
                    for (int j = 0; j < 16; j++) {
                        u[j] = sizeof(T) == 2 ? pack_bf16(__uint_as_float(y[2 * j]), __uint_as_float(y[2 * j + 1]))
                                              : y[half * 16 + j];
                        if (MASKED && sizeof(T) == 2) {
                            const uint32_t keep = both_bytes(spread[2 * j % 8], spread[2 * j % 8 + 1], j / 4);
                            u[j] = (u[j] & keep) | (0xFF80FF80u & ~keep);
                        }
                    }
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 4; j++)
                        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(own + ((j ^ own_swap) << 4)),
                                     "r"(u[4 * j]), "r"(u[4 * j + 1]), "r"(u[4 * j + 2]), "r"(u[4 * j + 3])
                                     : "memory");
                    __syncwarp();
                    const int c0 = i * 32 + half * 16;
                    if (wide && n == 32) {            // four lanes a token, eight tokens at a time
#pragma unroll
                        for (int j = 0; j < 4; j++) {
                            const int r = j * 8 + (lane >> 2);
                            uint4 x;
                            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                                         : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w)
                                         : "r"(staging + r * 64 + (((lane & 3) ^ ((r >> 1) & 3)) << 4)));
                            if (t0 + r < h.T) *reinterpret_cast<uint4*>(rows + (size_t)(j * 8) * h.row_stride + c0) = x;
                        }
                    } else {                          // a lane a logit
                        for (int r = 0; r < 32 && t0 + r < h.T; r++) {
                            const uint32_t at = staging + r * 64 + (((lane * 4 / COLS) ^ ((r >> 1) & 3)) << 4) +
                                                (lane % (COLS / 4)) * (int)sizeof(T);
                            if (lane < COLS && half * 16 + lane < n) {
                                T* out = logits + (size_t)(t0 + r) * h.row_stride + v0 + c0 + lane;
                                if (sizeof(T) == 2) {
                                    uint16_t x;
                                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(at));
                                    *reinterpret_cast<uint16_t*>(out) = x;
                                } else {
                                    uint32_t x;
                                    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(at));
                                    *reinterpret_cast<uint32_t*>(out) = x;
                                }
                            }
                        }
                    }
                }
            }
            acc.next(2);
            return true;
        });
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0 && *failed) set_other(&s_other_failed, side ^ 1);
    cluster_sync();                                   // nothing of this block is used by the other any more, unless
    if (*failed || *const_cast<volatile int*>(&s_other_failed)) {     // both blocks come here or neither
        settle_many(a_full(0), a_slots, b_full(0), b_slots, e_full(0), drained, s_loaded);
        if (threadIdx.x == 0 && *failed) atomicAdd(&g_faults, 1);
        cluster_sync();
    }
    if (warp == 1) tmem_free<true>(tmem);
}

template <typename T, bool CHECK>
psc_status head_many(const Head& h, T* logits, cudaStream_t cs) {
    CUtensorMap w_map, x_map, w_blocks_map, x_blocks_map;
    const uint64_t row = (h.K + 31) / 32 * 16, n_tiles = (h.K + 127) / 128;
    if (!tensor_map(&w_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, h.w, row, h.V, h.w_stride, 128, NV / 2) ||
        !tensor_map(&x_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, h.q, row, h.T, h.q_stride, 128, MT / 2) ||
        !tensor_map(&w_blocks_map, CU_TENSOR_MAP_DATA_TYPE_UINT32, h.w_blocks, n_tiles * SF / 4, (h.V + 127) / 128,
                    n_tiles * SF, 256, 2, CU_TENSOR_MAP_SWIZZLE_NONE) ||
        !tensor_map(&x_blocks_map, CU_TENSOR_MAP_DATA_TYPE_UINT32, h.q_blocks, n_tiles * SF / 4, (h.T + 127) / 128,
                    n_tiles * SF, 256, 1, CU_TENSOR_MAP_SWIZZLE_NONE))
        return ops_fail(PSC_ERR_CUDA, ME, "cuTensorMapEncodeTiled failed");
    const int n_mt = (h.T + MT - 1) / MT, n_vt = (h.V + NV - 1) / NV;
    const bool wide = is_aligned(logits, h.row_stride * (int64_t)sizeof(T), 16);
    const int pairs = (int)std::min<int64_t>((int64_t)n_mt * n_vt, std::max(1, current_sms() / 2));
    return ops_launch(h.bitmask ? k_mx4_many<T, true, CHECK> : k_mx4_many<T, false, CHECK>, dim3(2 * pairs), MMA_THREADS, MANY_SMEM, 2,
                      cs, "k_mx4_many", w_map, x_map, w_blocks_map, x_blocks_map, h, logits, n_mt, n_vt, wide);
}

template <typename T, bool CHECK>
psc_status head(const Head& h, T* logits, cudaStream_t cs) {
    return h.T <= FEW ? head_few<T, CHECK>(h, logits, cs) : head_many<T, CHECK>(h, logits, cs);
}

// CHECK: the kernels that psc_mx4_check_wait runs, the same but for when their waits give up; f32 only.
template <bool CHECK>
psc_status head_entry(const char* me, Head h, void* logits, psc_dtype dtype, void* stream) {
    if (h.T < 0 || h.V <= 0 || h.K <= 0 || h.row_stride < h.V || !is_dtype(dtype) || !h.w || !h.w_blocks ||
        (h.T && (!h.q || !h.q_blocks || !logits)))
        return ops_fail(PSC_ERR_ARG, me, "bad arguments");
    if (h.K > MAX_K) return ops_fail(PSC_ERR_LIMIT, me, "K over 131,072");
    if (h.T > MAX_T || h.V > MAX_V) return ops_fail(PSC_ERR_LIMIT, me, "too many rows");
    if (!is_mx4(h.w, h.w_stride, h.w_blocks, h.K) || (h.T && !is_mx4(h.q, h.q_stride, h.q_blocks, h.K)))
        return ops_fail(PSC_ERR_ARG, me, "codes or blocks with a bad stride or alignment");
    if (!is_whole(logits, dtype) || (uintptr_t)h.scale % 4 || (uintptr_t)h.w_scale % 4 || (uintptr_t)h.bitmask % 4)
        return ops_fail(PSC_ERR_ARG, me, "an address that is no multiple of its elements' size");
    if (h.T == 0) return PSC_OK;
    h.W = (h.V + 31) / 32;
    if constexpr (!CHECK) {
        if (dtype == PSC_BF16) return head<__nv_bfloat16, CHECK>(h, (__nv_bfloat16*)logits, (cudaStream_t)stream);
    }
    return head<float, CHECK>(h, (float*)logits, (cudaStream_t)stream);
}

}  // namespace

extern "C" {

psc_status psc_head_logits_mx4(const uint8_t* d_q, int64_t q_stride, const uint8_t* d_q_blocks, const float* d_scale,
                               int32_t T, const uint8_t* d_w, int64_t w_stride, const uint8_t* d_w_blocks,
                               const float* d_w_scale, int32_t V, int32_t K, const uint32_t* d_bitmask, void* d_logits,
                               psc_dtype dtype, int64_t row_stride, void* stream) {
    return head_entry<false>(ME, Head{d_q, q_stride, d_q_blocks, d_scale, T, d_w, w_stride, d_w_blocks, d_w_scale, V, K, d_bitmask,
                                      0, row_stride, 0},
                             d_logits, dtype, stream);
}

psc_status psc_mx4_check_wait(const uint8_t* d_q, int64_t q_stride, const uint8_t* d_q_blocks, const float* d_scale,
                              int32_t T, const uint8_t* d_w, int64_t w_stride, const uint8_t* d_w_blocks,
                              const float* d_w_scale, int32_t V, int32_t K, const uint32_t* d_bitmask, void* d_logits,
                              psc_dtype dtype, int64_t row_stride, int32_t limit, void* stream) {
    const char* me = "psc_mx4_check_wait";
    if (limit < 0 || limit > WAIT_POLLS || dtype != PSC_F32) return ops_fail(PSC_ERR_ARG, me, "bad arguments");
    return head_entry<true>(me, Head{d_q, q_stride, d_q_blocks, d_scale, T, d_w, w_stride, d_w_blocks, d_w_scale, V, K, d_bitmask,
                                     0, row_stride, limit},
                            d_logits, dtype, stream);
}

psc_status psc_mx4_faults(int32_t* h_faults, int32_t reset, void* stream) {
    const char* me = "psc_mx4_faults";
    if (!h_faults) return ops_fail(PSC_ERR_ARG, me, "bad arguments");
    cudaStream_t cs = (cudaStream_t)stream;
    std::unique_lock<std::mutex> alone(g_faults_read, std::defer_lock);
    if (reset) alone.lock();
    psc_status s = ops_check(cudaMemcpyFromSymbolAsync(h_faults, g_faults, 4, 0, cudaMemcpyDeviceToHost, cs), me);
    if (s == PSC_OK) s = ops_check(cudaStreamSynchronize(cs), me);
    if (s == PSC_OK && reset && *h_faults) {
        s = ops_launch(k_take_faults, dim3(1), 1, 0, 1, cs, me, *h_faults);
        if (s == PSC_OK) s = ops_check(cudaStreamSynchronize(cs), me);
    }
    return s;
}

}  // extern "C"
