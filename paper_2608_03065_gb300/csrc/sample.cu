// psc_sample: one token per row among the allowed ones, by temperature, top-k,
// top-p and min-p.
//
// Every filter keeps the tokens whose logit is at least some value: the k-th
// largest; the smallest whose strictly larger ones hold less than p of the
// weight; the one where e^z reaches min_p.  So a row is filtered by one
// threshold, found digit by digit of the logits' order (a histogram per 8-bit
// digit, of counts for top-k, of weights for top-p), and the draw is the same
// search by index.  Weights are whole numbers of 2^-40 of the largest: integer
// sums are the same in any order, so neither the atomics nor the split of a row
// over blocks can change a draw.  41 bits hold every f32 e^z over 2^-17 exactly;
// what is rounded away of a row is below V * 2^-41 of its largest weight.
#include <cooperative_groups.h>

#include <algorithm>

#include "ops_common.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int NT = 512;                 // threads of a block
constexpr int NW = NT / 32;
constexpr int CHUNK = 256;              // tokens a warp takes at a time: 8 neighbours a lane
constexpr int MAX_CLUSTER = 8;
constexpr int MAX_V = 1 << 22;
constexpr float NEG_INF = -__builtin_huge_valf();
constexpr float FLT_BIG = 3.402823466e+38f;

typedef unsigned long long u64;

// Order of f32 values as unsigned numbers.
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t u = __float_as_uint(x);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

struct Row {
    const void* logits;
    const uint8_t* mask;    // its packed mask, byte by byte (8 tokens each), or NULL
    int V, lo, hi;          // this block's tokens, lo a multiple of CHUNK
};

// The 8 tokens of piece v0..v0+7: their logits, -inf where masked, NaN, or past the end.
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const Row& r, int v0, float x[8]) {
    const T* p = static_cast<const T*>(r.logits) + v0;
    const int n = r.hi - v0;
    uint32_t bits = n <= 0 ? 0u : r.mask ? r.mask[v0 >> 3] : 0xffu;
    if (n < 8 && n > 0) bits &= (1u << n) - 1;
    if (VEC && n >= 8 && bits) {
        if (sizeof(T) == 2) {
            const uint4 q = *reinterpret_cast<const uint4*>(p);
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int i = 0; i < 4; i++) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        } else {
            const float4 a = reinterpret_cast<const float4*>(p)[0], c = reinterpret_cast<const float4*>(p)[1];
            x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = c.x, x[5] = c.y, x[6] = c.z, x[7] = c.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = (bits >> i) & 1 ? load_f32(p + i) : NEG_INF;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = ((bits >> i) & 1) && x[i] > NEG_INF ? fminf(x[i], FLT_BIG) : NEG_INF;
}

// What a row's weights are computed from; the arithmetic is the header's, step by step.
struct Weigh {
    float m, inv, tau, min_e;
    __device__ __forceinline__ float z(float x) const { return __fmul_rn(__fsub_rn(x, m), inv); }
    // weight of x before the filters
    __device__ __forceinline__ u64 raw(float x) const { return __float2ull_rn(expf(z(x)) * 0x1p40f); }
    // weight after them
    __device__ __forceinline__ u64 kept(float x) const {
        const float e = expf(z(x));
        return x >= tau && e >= min_e ? __float2ull_rn(e * 0x1p40f) : 0ull;
    }
};

struct Shared {
    uint32_t cnt[2][256], hi[2][256];   // a histogram's counts, or its weights as two words
    u64 part[8];                        // this block's share of what the cluster combines, a slot per use
    u64 warp[NW];
    u64 found[2];
    int at;
};

__device__ __forceinline__ u64 warp_sum(u64 v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
    return v;
}

// Sum over the block's threads of v before this thread; *total: over all of them.
__device__ __forceinline__ u64 block_before(Shared& s, u64 v, u64* total) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    u64 in = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const u64 y = __shfl_up_sync(FULL, in, o);
        if (lane >= o) in += y;
    }
    __syncthreads();
    if (lane == 31) s.warp[warp] = in;
    __syncthreads();
    u64 before = 0, all = 0;
    for (int w = 0; w < NW; w++) {
        if (w < warp) before += s.warp[w];
        all += s.warp[w];
    }
    *total = all;
    return before + in - v;
}

// One digit of a search from the largest value down: the cluster's histogram of
// the tokens whose order starts with `prefix`, then the first digit, from the top,
// at which the running sum reaches `need`.  Returns the digit; need becomes what is
// left to reach inside it.
template <bool MASS>
__device__ int pick_digit(cg::cluster_group& cl, Shared& s, int buf, u64* need) {
    cl.sync();                              // every block's histogram is whole
    u64 v = 0;
    const int bin = 255 - (int)threadIdx.x;
    if (threadIdx.x < 256) {
        for (unsigned r = 0; r < cl.num_blocks(); r++) {
            const Shared* p = cl.map_shared_rank(&s, r);
            v += MASS ? ((u64)p->hi[buf][bin] << 32) + p->cnt[buf][bin] : (u64)p->cnt[buf][bin];
        }
    }
    u64 total;
    const u64 before = block_before(s, v, &total);
    if (threadIdx.x < 256 && before < *need && before + v >= *need) {
        s.at = bin;
        s.found[0] = *need - before;
    }
    __syncthreads();
    *need = s.found[0];
    return s.at;
}

struct Settings {
    const float* uniform;
    const float* temperature;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
};

// A cluster of blocks per row, each with a contiguous part of the vocabulary.
template <typename T, bool VEC>
__global__ void __launch_bounds__(NT) k_sample(const T* logits, int64_t stride, int V, int per_block,
                                               const uint32_t* bitmask, int W, Settings S, int32_t* tokens,
                                               float* logprobs) {
    extern __shared__ u64 chunk_sum[];
    __shared__ Shared s;
    cg::cluster_group cl = cg::this_cluster();
    const int rank = (int)cl.block_rank(), n_blocks = (int)cl.num_blocks();
    const int b = blockIdx.x / n_blocks;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    dep_wait();
    dep_launch();

    Row r{logits + (size_t)b * stride, bitmask ? reinterpret_cast<const uint8_t*>(bitmask + (size_t)b * W) : nullptr, V,
          min(V, rank * per_block), min(V, (rank + 1) * per_block)};
    const int n_chunks = (r.hi - r.lo + CHUNK - 1) / CHUNK;
    float x[8];

    auto combine_max = [&](u64 v, int slot) {   // over the cluster
#pragma unroll
        for (int o = 16; o; o >>= 1) v = max(v, __shfl_xor_sync(FULL, v, o));
        if (lane == 0) s.warp[warp] = v;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < NW; w++) v = max(v, s.warp[w]);
            s.part[slot] = v;
        }
        cl.sync();
        v = 0;
        for (int q = 0; q < n_blocks; q++) v = max(v, cl.map_shared_rank(&s, q)->part[slot]);
        return v;
    };

    // the largest candidate
    float mx = NEG_INF;
    for (int c = warp; c < n_chunks; c += NW) {
        load8<T, VEC>(r, r.lo + c * CHUNK + lane * 8, x);
#pragma unroll
        for (int i = 0; i < 8; i++) mx = fmaxf(mx, x[i]);
    }
    const float m = unordered((uint32_t)combine_max(ordered(mx), 0));
    if (m == NEG_INF) {                         // nothing to choose from
        if (rank == 0 && threadIdx.x == 0) {
            tokens[b] = -1;
            if (logprobs) logprobs[b] = NEG_INF;
        }
        cl.sync();
        return;
    }
    const float temp = S.temperature ? S.temperature[b] : 1.f;
    if (!(temp >= 1e-6f)) {                     // greedy
        uint32_t first = 0;                     // V - index, so that the largest is the lowest index
        for (int c = warp; c < n_chunks; c += NW) {
            const int v0 = r.lo + c * CHUNK + lane * 8;
            load8<T, VEC>(r, v0, x);
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (x[i] == m) first = max(first, (uint32_t)(V - v0 - i));
        }
        const uint32_t all = (uint32_t)combine_max(first, 1);
        if (rank == 0 && threadIdx.x == 0) {
            tokens[b] = V - (int)all;
            if (logprobs) logprobs[b] = 0.f;
        }
        cl.sync();
        return;
    }

    Weigh g{m, __fdiv_rn(1.f, temp), NEG_INF, 0.f};
    // the threshold of top_k, then of top_p, a digit at a time
    int buf = 0;
    auto search = [&](auto mass, u64 need, auto limit) -> float {
        constexpr bool MASS = decltype(mass)::value;
        uint32_t prefix = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = threadIdx.x; i < 256; i += NT) s.cnt[buf][i] = s.hi[buf][i] = 0;
            __syncthreads();
            for (int c = warp; c < n_chunks; c += NW) {
                load8<T, VEC>(r, r.lo + c * CHUNK + lane * 8, x);
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const uint32_t k = ordered(x[i]);
                    if (x[i] == NEG_INF || x[i] < g.tau || (shift < 24 && (k >> (shift + 8)) != prefix)) continue;
                    const int bin = (k >> shift) & 255;
                    if (!MASS) {
                        atomicAdd(&s.cnt[buf][bin], 1u);
                    } else {
                        const u64 w = g.raw(x[i]);
                        const uint32_t lo = (uint32_t)w, old = atomicAdd(&s.cnt[buf][bin], lo);
                        const uint32_t up = (uint32_t)(w >> 32) + (old + lo < old);
                        if (up) atomicAdd(&s.hi[buf][bin], up);
                    }
                }
            }
            if (shift == 24) need = limit(buf);
            prefix = (prefix << 8) | (uint32_t)pick_digit<MASS>(cl, s, buf, &need);
            buf ^= 1;
        }
        return unordered(prefix);
    };
    // sum of the cluster's histogram
    auto hist_total = [&](int at) {
        cl.sync();
        u64 v = 0;
        if (threadIdx.x < 256)
            for (int q = 0; q < n_blocks; q++) {
                const Shared* p = cl.map_shared_rank(&s, q);
                v += ((u64)p->hi[at][threadIdx.x] << 32) + p->cnt[at][threadIdx.x];
            }
        u64 total;
        block_before(s, v, &total);
        return total;
    };
    const int k = S.top_k ? S.top_k[b] : 0;
    if (k > 0 && k < V) {
        // fewer candidates than k: all stay
        const float t = search(std::false_type{}, 0, [&](int at) { return min((u64)k, hist_total(at)); });
        g.tau = t;
    }
    const float p = S.top_p ? S.top_p[b] : 1.f;
    if (p < 1.f) {
        const u64 p24 = (u64)__float2ll_rn(fmaxf(p, 0.f) * 0x1p24f);
        const float t = search(std::true_type{}, 0, [&](int at) {
            const u64 total = hist_total(at);
            return max((u64)1, p24 * (total >> 24) + ((p24 * (total & 0xffffff)) >> 24));
        });
        g.tau = t;
    }
    if (S.min_p && S.min_p[b] > 0.f) g.min_e = fminf(S.min_p[b], 1.f);

    // the draw: weights by chunk, then the block, the chunk and the token that hold the target
    u64 mine = 0;
    for (int c = warp; c < n_chunks; c += NW) {
        load8<T, VEC>(r, r.lo + c * CHUNK + lane * 8, x);
        u64 w = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) w += g.kept(x[i]);
        w = warp_sum(w);
        if (lane == 0) chunk_sum[c] = w;
    }
    __syncthreads();
    const int per = (n_chunks + NT - 1) / NT, c0 = min(n_chunks, (int)threadIdx.x * per), c1 = min(n_chunks, c0 + per);
    for (int c = c0; c < c1; c++) mine += chunk_sum[c];
    u64 total;
    u64 before = block_before(s, mine, &total);
    if (threadIdx.x == 0) s.part[2] = total;
    cl.sync();
    u64 lower = 0, sum = 0;
    for (int q = 0; q < n_blocks; q++) {
        const u64 w = cl.map_shared_rank(&s, q)->part[2];
        if (q < rank) lower += w;
        sum += w;
    }
    const float uf = S.uniform[b];
    const u64 u = uf > 0.f ? min((u64)0xffffff, (u64)__float2ull_rz(fminf(uf, 1.f) * 0x1p24f)) : 0ull;
    const u64 target = u * (sum >> 24) + ((u * (sum & 0xffffff)) >> 24);
    if (target >= lower && target < lower + total) {
        const u64 t = target - lower;
        if (t >= before && t < before + mine) {
            int c = c0;
            while (before + chunk_sum[c] <= t) before += chunk_sum[c++];
            s.at = c;
            s.found[1] = t - before;
        }
        __syncthreads();
        if (warp == 0) {
            const int v0 = r.lo + s.at * CHUNK + lane * 8;
            u64 t2 = s.found[1], w = 0;
            load8<T, VEC>(r, v0, x);
#pragma unroll
            for (int i = 0; i < 8; i++) w += g.kept(x[i]);
            u64 in = w;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const u64 y = __shfl_up_sync(FULL, in, o);
                if (lane >= o) in += y;
            }
            if (t2 >= in - w && t2 < in) {
                t2 -= in - w;
                for (int i = 0; i < 8; i++) {
                    const u64 wi = g.kept(x[i]);
                    if (t2 < wi) {
                        tokens[b] = v0 + i;
                        if (logprobs) logprobs[b] = g.z(x[i]) - logf((float)sum * 0x1p-40f);
                        break;
                    }
                    t2 -= wi;
                }
            }
        }
    }
    cl.sync();                                  // peers may still read this block's shared memory
}

template <typename T>
psc_status sample(const T* logits, int64_t stride, int B, int V, const uint32_t* bitmask, const Settings& S,
                  int32_t* tokens, float* logprobs, cudaStream_t cs) {
    const int cluster = V > 524288 ? MAX_CLUSTER : 1;
    const int per = ((V + cluster - 1) / cluster + CHUNK - 1) / CHUNK * CHUNK;
    const size_t smem = (size_t)(per / CHUNK) * 8;
    const bool vec = is_aligned(logits, stride * sizeof(T), 16);
    return ops_launch(vec ? k_sample<T, true> : k_sample<T, false>, dim3((unsigned)B * cluster), NT, smem, cluster, cs,
                      "k_sample", logits, stride, V, per, bitmask, (V + 31) / 32, S, tokens, logprobs);
}

}  // namespace

extern "C" psc_status psc_sample(const void* d_logits, psc_dtype dtype, int64_t row_stride, int32_t B, int32_t V,
                                 const uint32_t* d_bitmask, const float* d_uniform, const float* d_temperature,
                                 const int32_t* d_top_k, const float* d_top_p, const float* d_min_p,
                                 int32_t* d_tokens, float* d_logprobs, void* stream) {
    const char* me = "psc_sample";
    if (B < 0 || V <= 0 || row_stride < V || !is_dtype(dtype) || (B && (!d_logits || !d_uniform || !d_tokens)))
        return ops_fail(PSC_ERR_ARG, me, "bad arguments");
    if (V > MAX_V) return ops_fail(PSC_ERR_LIMIT, me, "vocabulary over 4,194,304 tokens");
    if (B > 0x7fffffff / MAX_CLUSTER) return ops_fail(PSC_ERR_LIMIT, me, "batch too large");
    if (B == 0) return PSC_OK;
    const Settings S{d_uniform, d_temperature, d_top_k, d_top_p, d_min_p};
    if (dtype == PSC_BF16)
        return sample((const __nv_bfloat16*)d_logits, row_stride, B, V, d_bitmask, S, d_tokens, d_logprobs,
                      (cudaStream_t)stream);
    return sample((const float*)d_logits, row_stride, B, V, d_bitmask, S, d_tokens, d_logprobs, (cudaStream_t)stream);
}
