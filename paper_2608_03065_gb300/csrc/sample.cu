// psc_sample: one token per row among the allowed ones, by temperature, top-k,
// top-p and min-p.
//
// Every filter keeps the tokens whose logit is at least some value: the k-th
// largest; the smallest whose strictly larger ones hold less than p of the
// weight; the one where e^z reaches min_p.  So a row is filtered by one
// threshold, found digit by digit of the logits' order (a histogram per 8-bit
// digit, of counts for top-k, of weights for top-p), and the draw is the same
// search by token.  Weights are whole numbers of 2^-40 of the largest: integer
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
constexpr int CHUNK = 256;              // tokens a warp takes at a time: a piece of 8 neighbours a lane
constexpr int UNROLL = 4;               // chunks in flight per warp
constexpr int LIST = 2048;              // candidates that a block holds
constexpr int BINS = NT;                // of the histogram of the groups' maxima
constexpr int NUCLEUS_GROUPS = 640;     // maxima above the bound from which a nucleus is looked for
constexpr int PAIRS = 256;              // candidates that are compared pair by pair
constexpr float Z_END = -29.f;          // below it a weight is 0: 2^40 e^-29 < 1/2
constexpr int MAX_CLUSTER = 8;
constexpr int MAX_V = 1 << 22;
constexpr float NEG_INF = -__builtin_huge_valf();
constexpr float FLT_BIG = 3.402823466e+38f;

typedef unsigned long long u64;

// Order of f32 values as unsigned numbers (0 and -0 are one value).
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t u = __float_as_uint(__fadd_rn(x, 0.f));
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
// NaN as -inf, +inf as the largest finite value.
__device__ __forceinline__ float clean(float x) { return fminf(fmaxf(x, NEG_INF), FLT_BIG); }

struct Row {
    const void* logits;
    const uint8_t* mask;    // its packed mask, byte by byte (8 tokens each), or NULL
    int V, lo, hi;          // this block's tokens, lo a multiple of CHUNK
};

// Eight neighbouring tokens, -inf where they are masked or past the end.
template <typename T>
struct Piece;
template <>
struct Piece<__nv_bfloat16> {
    uint32_t w[4];
    __device__ __forceinline__ void read(const __nv_bfloat16* p) {
        const uint4 q = *reinterpret_cast<const uint4*>(p);
        w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
    }
    __device__ __forceinline__ void set(int i, const __nv_bfloat16* p) {
        const uint32_t h = *reinterpret_cast<const uint16_t*>(p);
        w[i >> 1] = i & 1 ? (w[i >> 1] & 0xffffu) | h << 16 : (w[i >> 1] & 0xffff0000u) | h;
    }
    __device__ __forceinline__ void keep(const uint4& m) {      // m: ones where allowed
        const uint32_t k[4] = {m.x, m.y, m.z, m.w};
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = (w[i] & k[i]) | (0xFF80FF80u & ~k[i]);
    }
    __device__ __forceinline__ float max8() const {             // NaN only if all are
        __nv_bfloat162 h[4];
#pragma unroll
        for (int i = 0; i < 4; i++) h[i] = *reinterpret_cast<const __nv_bfloat162*>(&w[i]);
        const __nv_bfloat162 a = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
        return fmaxf(__low2float(a), __high2float(a));
    }
    __device__ __forceinline__ float get(int i) const {
        return clean(__uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16));
    }
};
template <>
struct Piece<float> {
    float x[8];
    __device__ __forceinline__ void read(const float* p) {
        const float4 a = reinterpret_cast<const float4*>(p)[0], c = reinterpret_cast<const float4*>(p)[1];
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = c.x, x[5] = c.y, x[6] = c.z, x[7] = c.w;
    }
    __device__ __forceinline__ void set(int i, const float* p) { x[i] = *p; }
    __device__ __forceinline__ void keep(uint32_t bits) {
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = (bits >> i) & 1 ? x[i] : NEG_INF;
    }
    __device__ __forceinline__ float max8() const {
        float m = fmaxf(x[0], x[1]);
#pragma unroll
        for (int i = 2; i < 8; i++) m = fmaxf(m, x[i]);
        return m;
    }
    __device__ __forceinline__ float get(int i) const { return clean(x[i]); }
};

// Calls f(piece, first token, chunk, u, any) for every piece of the block's part of the
// row, UNROLL chunks in flight per warp (u: which of them).
// Whole warps call it; `any` is false where a lane's piece holds nothing.
template <typename T, bool VEC, typename F>
__device__ __forceinline__ void for_pieces(const Row& r, const uint4* lut, F&& f) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n_chunks = (r.hi - r.lo + CHUNK - 1) / CHUNK;
    for (int c0 = warp; c0 < n_chunks; c0 += UNROLL * NW) {
        Piece<T> p[UNROLL];
        uint32_t bits[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; u++) {
            const int v0 = r.lo + (c0 + u * NW) * CHUNK + lane * 8, n = r.hi - v0;
            bits[u] = n <= 0 ? 0u : r.mask ? r.mask[v0 >> 3] : 0xffu;
            if (n > 0 && n < 8) bits[u] &= (1u << n) - 1;
        }
#pragma unroll
        for (int u = 0; u < UNROLL; u++) {
            const int v0 = r.lo + (c0 + u * NW) * CHUNK + lane * 8;
            const T* at = static_cast<const T*>(r.logits) + v0;
            if (!bits[u]) continue;
            if (VEC && r.hi - v0 >= 8) {
                p[u].read(at);
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++)
                    if ((bits[u] >> i) & 1) p[u].set(i, at + i);
            }
        }
#pragma unroll
        for (int u = 0; u < UNROLL; u++) {
            const int c = c0 + u * NW;
            if (c >= n_chunks) break;
            if constexpr (sizeof(T) == 2) p[u].keep(lut[bits[u]]);
            else p[u].keep(bits[u]);
            f(p[u], r.lo + c * CHUNK + lane * 8, c, u, bits[u] != 0);
        }
    }
}

// Calls f(value, token) for the tokens of the thread's own groups whose maximum reaches `bound`.
template <typename T, bool VEC, typename F>
__device__ __forceinline__ void for_groups(const Row& r, const uint4* lut, const float (&group)[UNROLL], float bound,
                                           F&& f) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n_chunks = (r.hi - r.lo + CHUNK - 1) / CHUNK;
    for (int u = 0; u < UNROLL; u++) {
        float top = group[0];
#pragma unroll
        for (int j = 1; j < UNROLL; j++) top = u == j ? group[j] : top;
        if (!(top >= bound)) continue;
#pragma unroll 4
        for (int c = warp + u * NW; c < n_chunks; c += UNROLL * NW) {
            const int v0 = r.lo + c * CHUNK + lane * 8, n = r.hi - v0;
            uint32_t bits = n <= 0 ? 0u : r.mask ? r.mask[v0 >> 3] : 0xffu;
            if (n > 0 && n < 8) bits &= (1u << n) - 1;
            if (!bits) continue;
            const T* at = static_cast<const T*>(r.logits) + v0;
            Piece<T> p;
            if (VEC && n >= 8) {
                p.read(at);
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++)
                    if ((bits >> i) & 1) p.set(i, at + i);
            }
            if constexpr (sizeof(T) == 2) p.keep(lut[bits]);
            else p.keep(bits);
            if (!(p.max8() >= bound)) continue;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float x = p.get(i);
                if (x >= bound) f(x, v0 + i);
            }
        }
    }
}

// What a row's weights are computed from; the arithmetic is the header's, step by step.
struct Weigh {
    float m, inv, tau, min_e;
    __device__ __forceinline__ float z(float x) const { return __fmul_rn(__fsub_rn(x, m), inv); }
    __device__ __forceinline__ float e(float x) const { return expf(z(x)); }
    // weight of x before the filters
    __device__ __forceinline__ u64 raw(float x) const { return __float2ull_rn(e(x) * 0x1p40f); }
    // weight after them
    __device__ __forceinline__ u64 kept(float x) const {
        const float y = e(x);
        return x >= tau && y >= min_e ? __float2ull_rn(y * 0x1p40f) : 0ull;
    }
};
// A sum of weights as two 32-bit sums: of 2^20 e, its whole part and its fraction in units
// of 2^-20, each taken from the low bits of a sum with 2^23 (rounded down, then to nearest
// even; together rint(2^40 e), since the whole part is an even number of units).  Good for
// 2048 weights.
struct WeightSum {
    uint32_t hi = 0, lo = 0;
    __device__ __forceinline__ void add(float e, WeightSum* also = nullptr, bool too = false) {
        const float a = __fmaf_rz(e, 0x1p20f, 0x1p23f);
        const float c = __fmaf_rn(__fmaf_rn(e, 0x1p20f, 0x1p23f - a), 0x1p20f, 0x1p23f);
        const uint32_t h = __float_as_uint(a) - 0x4B000000u, l = __float_as_uint(c) - 0x4B000000u;
        hi += h, lo += l;
        if (also && too) also->hi += h, also->lo += l;
    }
    __device__ __forceinline__ u64 value() const { return ((u64)hi << 20) + lo; }
};

struct Shared {
    uint32_t cnt[2][256], hi[2][256];   // a histogram's counts, or its weights as two words
    uint32_t bins[BINS], bins_hi[BINS];
    u64 part[12];                       // this block's share of what the cluster combines, a slot per use
    u64 warp[NW];
    u64 found[2];
    int at, n, from, to;
    uint4 lut[256];                     // mask byte -> ones where it allows (bf16 pairs)
    uint32_t key[LIST];                 // candidates: order of the value, token, weight
    uint32_t token[LIST];
    u64 weight[LIST];
};

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
#pragma unroll
    for (int w = 0; w < NW; w++) {
        if (w < warp) before += s.warp[w];
        all += s.warp[w];
    }
    *total = all;
    return before + in - v;
}

// One digit of a search from the largest key down: the histogram of the keys that start
// with the digits found so far (over the cluster, or this block's alone), then the first
// digit, from the top, at which the running sum reaches `need`.  Returns the digit; need
// becomes what is left to reach inside it.
template <bool MASS>
__device__ int pick_digit(cg::cluster_group& cl, int n_blocks, Shared& s, int buf, u64* need) {
    if (n_blocks > 1) cl.sync();            // every block's histogram is whole
    else __syncthreads();
    u64 v = 0;
    const int bin = 255 - (int)threadIdx.x;
    if (threadIdx.x < 256) {
        for (int r = 0; r < n_blocks; r++) {
            const Shared* p = n_blocks > 1 ? cl.map_shared_rank(&s, r) : &s;
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
template <bool MASS>
__device__ __forceinline__ void count_in(Shared& s, int buf, int bin, u64 w) {
    if (!MASS) {
        atomicAdd(&s.cnt[buf][bin], 1u);
    } else {
        const uint32_t lo = (uint32_t)w, old = atomicAdd(&s.cnt[buf][bin], lo);
        const uint32_t up = (uint32_t)(w >> 32) + (old + lo < old);
        if (up) atomicAdd(&s.hi[buf][bin], up);
    }
}

// floor(total * u24 / 2^24)
__device__ __forceinline__ u64 part_of(u64 total, u64 u24) {
    return u24 * (total >> 24) + ((u24 * (total & 0xffffff)) >> 24);
}

// The search among the block's n listed candidates, by value (TOKEN false: the largest
// first) or by token (the lowest first), of those for which `in` holds.
template <bool MASS, bool TOKEN, typename In>
__device__ uint32_t list_search(cg::cluster_group& cl, Shared& s, int n, u64 need, In&& in) {
    uint32_t prefix = 0;
    for (int shift = TOKEN ? 16 : 24; shift >= 0; shift -= 8) {
        for (int i = threadIdx.x; i < 256; i += NT) s.cnt[0][i] = s.hi[0][i] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += NT) {
            const uint32_t k = TOKEN ? ~s.token[i] & 0xffffff : s.key[i];
            if (!in(i) || (shift < (TOKEN ? 16 : 24) && (k >> (shift + 8)) != prefix)) continue;
            count_in<MASS>(s, 0, (k >> shift) & 255, MASS ? s.weight[i] : 1);
        }
        prefix = (prefix << 8) | (uint32_t)pick_digit<MASS>(cl, 1, s, 0, &need);
        __syncthreads();
    }
    return TOKEN ? ~prefix & 0xffffff : prefix;
}

// The cluster's lists behind the first block's own; their length (over LIST: not gathered).
__device__ int gather(cg::cluster_group& cl, Shared& s, int n_blocks) {
    int n = s.n;
    for (int q = 1; q < n_blocks; q++) {
        const Shared* o = cl.map_shared_rank(&s, q);
        const int more = o->n;
        if (n + more <= LIST)
            for (int i = threadIdx.x; i < more; i += NT) s.key[n + i] = o->key[i], s.token[n + i] = o->token[i];
        n += more;
    }
    __syncthreads();
    return n;
}

// Filters and draws among the block's n listed candidates, of which the weights sum to
// `listed`: k (0: off), then a nucleus of `limit` (0: limit_of what top-k leaves, ~0: off),
// then min_e.  The calling thread that holds the drawn one gets its place, others -1;
// *kept: the weight of what stays.
template <typename Limit>
__device__ int settle(cg::cluster_group& cl, Shared& s, const Weigh& g, int n, int k, u64 listed, u64 limit,
                      Limit&& limit_of, u64 u24, u64* kept) {
    const int tid = threadIdx.x;
    if (n <= PAIRS) {
        // Pair by pair, `per` threads to a candidate: how many are larger, and their weight;
        // then the weight that stays at lower tokens.
        int per = 2;
        while (per < 32 && 2 * per * n <= NT) per *= 2;
        const int i = tid / per, j0 = tid & (per - 1);
        const bool mine = i < n;
        const uint32_t key = mine ? s.key[i] : 0, token = mine ? s.token[i] : 0;
        u64 w = mine ? s.weight[i] : 0, over = 0;
        int larger = 0;
        if (mine)
            for (int j = j0; j < n; j += per)
                if (s.key[j] > key) larger++, over += s.weight[j];
        for (int o = per >> 1; o; o >>= 1) {
            larger += __shfl_xor_sync(FULL, larger, o);
            over += __shfl_xor_sync(FULL, over, o);
        }
        bool stays = mine && (!k || larger < k);
        if (!limit) {
            block_before(s, stays && !j0 ? w : 0, &listed);
            limit = limit_of(listed);
        }
        stays = stays && over < limit && g.e(unordered(key)) >= g.min_e;
        if (!stays) w = 0;
        __syncthreads();
        if (mine && !j0) s.weight[i] = w;
        block_before(s, j0 ? 0 : w, kept);      // and every weight is written
        const u64 target = part_of(*kept, u24);
        u64 before = 0;
        if (mine)
            for (int j = j0; j < n; j += per)
                if (s.token[j] < token) before += s.weight[j];
        for (int o = per >> 1; o; o >>= 1) before += __shfl_xor_sync(FULL, before, o);
        return mine && !j0 && before <= target && target < before + w ? i : -1;
    }
    uint32_t tau = 0;
    if (k && k < n) {
        tau = list_search<false, false>(cl, s, n, k, [](int) { return true; });
        u64 w = 0;
        for (int i = tid; i < n; i += NT) w += s.key[i] >= tau ? s.weight[i] : 0ull;
        block_before(s, w, &listed);
    }
    if (!limit) limit = limit_of(listed);
    if (limit != ~0ull) {
        const uint32_t low = tau;
        tau = list_search<true, false>(cl, s, n, limit, [&](int i) { return s.key[i] >= low; });
    }
    auto in = [&](int i) { return s.key[i] >= tau && g.e(unordered(s.key[i])) >= g.min_e; };
    u64 w = 0;
    for (int i = tid; i < n; i += NT) w += in(i) ? s.weight[i] : 0ull;
    block_before(s, w, kept);
    const uint32_t token = list_search<true, true>(cl, s, n, part_of(*kept, u24) + 1, in);
    for (int i = tid; i < n; i += NT)
        if (s.token[i] == token) return i;
    return -1;
}

// f(value) for the tokens of a row of one chunk, by one warp.
template <typename T, bool VEC, typename F>
__device__ __forceinline__ void one_chunk(const Row& r, const uint4* lut, F&& f) {
    const int v0 = r.lo + (threadIdx.x & 31) * 8, n = r.hi - v0;
    uint32_t bits = n <= 0 ? 0u : r.mask ? r.mask[v0 >> 3] : 0xffu;
    if (n > 0 && n < 8) bits &= (1u << n) - 1;
    if (!bits) return;
    const T* at = static_cast<const T*>(r.logits) + v0;
    for (int i = 0; i < 8; i++)
        if ((bits >> i) & 1) f(clean(load_f32(at + i)));
}

// The search over the whole row, digit by digit of the values' order: of the candidates
// that reach g.tau, the value at which the running count or weight from the largest
// down reaches need_of(their sum).
template <bool MASS, typename T, bool VEC, typename Need>
__device__ __noinline__ float row_search(cg::cluster_group& cl, Shared& s, const Row& r, const Weigh& g, int n_blocks,
                                         Need need_of) {
    uint32_t prefix = 0;
    u64 need = 0;
    int buf = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = threadIdx.x; i < 256; i += NT) s.cnt[buf][i] = s.hi[buf][i] = 0;
        __syncthreads();
        for_pieces<T, VEC>(r, s.lut, [&](const Piece<T>& q, int, int, int, bool any) {
            if (!any) return;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float x = q.get(i);
                const uint32_t key = ordered(x);
                if (x == NEG_INF || x < g.tau || (shift < 24 && (key >> (shift + 8)) != prefix)) continue;
                count_in<MASS>(s, buf, (key >> shift) & 255, MASS ? g.raw(x) : 1);
            }
        });
        if (shift == 24) {
            if (n_blocks > 1) cl.sync();
            else __syncthreads();
            u64 h = 0, all;
            if (threadIdx.x < 256)
                for (int q = 0; q < n_blocks; q++) {
                    const Shared* o = n_blocks > 1 ? cl.map_shared_rank(&s, q) : &s;
                    h += (MASS ? (u64)o->hi[buf][threadIdx.x] << 32 : 0) + o->cnt[buf][threadIdx.x];
                }
            block_before(s, h, &all);
            need = need_of(all);
        }
        prefix = (prefix << 8) | (uint32_t)pick_digit<MASS>(cl, n_blocks, s, buf, &need);
        buf ^= 1;
    }
    return unordered(prefix);
}

struct Settings {
    const float* uniform;
    const float* temperature;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
};

// A cluster of blocks per row, each with a contiguous part of the vocabulary.
//
// A pass from memory finds the largest candidate and the maxima of a few thousand groups
// of tokens.  At least k tokens lie at or above the k-th largest of those maxima, and not
// many more; the groups that reach it are read again, their tokens listed, and top-k, top-p
// and the draw are searches in that list by the cluster's first block.  Without top-k the
// weights have to be summed in a second pass (from L2): the nucleus is sought in the list
// of the tokens at or above the NUCLEUS_GROUPS-th maximum or, where a sample of the row
// says that it ends below, in the stretch of z around the sample's estimate: its weights
// go to bins, and the bin in which the nucleus ends is listed by a third pass.  The
// estimate decides only what is looked at: whatever it misses is searched digit by digit
// over the whole row.  What no list holds is drawn from sums by chunk.
template <typename T, bool VEC>
__global__ void __launch_bounds__(NT, 2) k_sample(const T* logits, int64_t stride, int V, int per_block,
                                                  const uint32_t* bitmask, int W, Settings S, int32_t* tokens,
                                                  float* logprobs) {
    extern __shared__ __align__(16) uint8_t dyn[];
    Shared& s = *reinterpret_cast<Shared*>(dyn);
    u64* chunk_sum = reinterpret_cast<u64*>(dyn + sizeof(Shared));
    cg::cluster_group cl = cg::this_cluster();
    const int rank = (int)cl.block_rank(), n_blocks = (int)cl.num_blocks();
    const int b = blockIdx.x / n_blocks;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x < 256) {
        auto pair = [&](int i) {
            return ((threadIdx.x >> i) & 1) * 0x0000ffffu + ((threadIdx.x >> (i + 1)) & 1) * 0xffff0000u;
        };
        s.lut[threadIdx.x] = make_uint4(pair(0), pair(2), pair(4), pair(6));
    }
    s.bins[threadIdx.x] = 0;
    if (threadIdx.x == 0) s.n = 0;
    dep_wait();
    dep_launch();
    __syncthreads();

    Row r{logits + (size_t)b * stride, bitmask ? reinterpret_cast<const uint8_t*>(bitmask + (size_t)b * W) : nullptr, V,
          min(V, rank * per_block), min(V, (rank + 1) * per_block)};
    const int n_chunks = (r.hi - r.lo + CHUNK - 1) / CHUNK;
    auto sync = [&]() {
        if (n_blocks > 1) cl.sync();
        else __syncthreads();
    };
    auto peer = [&](int q) -> const Shared* { return n_blocks > 1 ? cl.map_shared_rank(&s, q) : &s; };
    // the largest v over the cluster
    auto combine_max = [&](u64 v, int slot) {
#pragma unroll
        for (int o = 16; o; o >>= 1) v = max(v, __shfl_xor_sync(FULL, v, o));
        if (lane == 0) s.warp[warp] = v;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < NW; w++) v = max(v, s.warp[w]);
            s.part[slot] = v;
        }
        sync();
        v = 0;
        for (int q = 0; q < n_blocks; q++) v = max(v, peer(q)->part[slot]);
        return v;
    };
    // sum of v over the cluster, and over the blocks before this one
    auto combine_sum = [&](u64 v, int slot, u64* lower) {
        u64 total;
        block_before(s, v, &total);
        if (threadIdx.x == 0) s.part[slot] = total;
        sync();
        u64 sum = 0;
        *lower = 0;
        for (int q = 0; q < n_blocks; q++) {
            const u64 w = peer(q)->part[slot];
            if (q < rank) *lower += w;
            sum += w;
        }
        return sum;
    };
    auto finish = [&](int token, float lp) {
        tokens[b] = token;
        if (logprobs) logprobs[b] = lp;
    };

    // pass 1
    float group[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; u++) group[u] = NEG_INF;
    for_pieces<T, VEC>(r, s.lut, [&](const Piece<T>& p, int, int, int u, bool) { group[u] = fmaxf(group[u], p.max8()); });
    uint32_t top = 0, low = 0;              // low: ~order, so that the largest is the lowest maximum
#pragma unroll
    for (int u = 0; u < UNROLL; u++) {
        group[u] = clean(group[u]);
        top = max(top, ordered(group[u]));
        if (group[u] > NEG_INF) low = max(low, ~ordered(group[u]));
    }
    const uint32_t top_all = (uint32_t)combine_max(top, 0);
    const float m = unordered(top_all);
    if (m == NEG_INF) {                     // nothing to choose from
        if (rank == 0 && threadIdx.x == 0) finish(-1, NEG_INF);
        sync();
        return;
    }
    const float temp = S.temperature ? S.temperature[b] : 1.f;
    if (!(temp >= 1e-6f)) {                 // greedy
        uint32_t first = 0;                 // V - token, so that the largest is the lowest token
        for_groups<T, VEC>(r, s.lut, group, m, [&](float, int v) { first = max(first, (uint32_t)(V - v)); });
        const uint32_t all = (uint32_t)combine_max(first, 1);
        if (rank == 0 && threadIdx.x == 0) finish(V - (int)all, 0.f);
        sync();                             // peers may still read this block's shared memory
        return;
    }

    Weigh g{m, __fdiv_rn(1.f, temp), NEG_INF, 0.f};
    const int k = S.top_k && S.top_k[b] > 0 && S.top_k[b] < V ? S.top_k[b] : 0;
    const float p = S.top_p ? S.top_p[b] : 1.f;
    const bool nucleus = p < 1.f;
    const u64 p24 = nucleus ? (u64)__float2ll_rn(fmaxf(p, 0.f) * 0x1p24f) : 0ull;
    if (S.min_p && S.min_p[b] > 0.f) g.min_e = fminf(S.min_p[b], 1.f);
    const float uf = S.uniform[b];
    const u64 u24 = uf > 0.f ? min((u64)0xffffff, (u64)__float2ull_rz(fminf(uf, 1.f) * 0x1p24f)) : 0ull;
    auto limit_of = [&](u64 total) { return max((u64)1, part_of(total, p24)); };

    if (k || nucleus || g.min_e > 0.f) {
        float bound;
        if (k || nucleus) {
            // a bound that at least `want` groups reach, or no bound when there are fewer groups
            const uint32_t low_all = (uint32_t)combine_max(low, 2);
            const float range = m - unordered(~low_all), scale = BINS / range;
#pragma unroll
            for (int u = 0; u < UNROLL; u++)
                if (group[u] > NEG_INF) atomicAdd(&s.bins[min(BINS - 1, (int)fmaxf(0.f, (m - group[u]) * scale))], 1u);
            sync();
            u64 v = 0, groups;
            for (int q = 0; q < n_blocks; q++) v += peer(q)->bins[threadIdx.x];
            const u64 before = block_before(s, v, &groups), want = k ? k : NUCLEUS_GROUPS;
            if (groups < want) {
                if (threadIdx.x == 0) s.at = BINS;
            } else if (before < want && before + v >= want) {
                s.at = threadIdx.x;
            }
            __syncthreads();
            // a little below the bin's lower edge: the bins' own arithmetic is rounded
            bound = s.at == BINS ? -FLT_BIG : m - (s.at + 1) * (range / BINS) * 1.001f - fabsf(m) * 0x1p-20f;
        } else {
            // a little below the value at which e^z is min_e
            bound = m + (logf(g.min_e) * 1.0001f - 1e-4f) * temp - fabsf(m) * 0x1p-20f;
        }
        bound = fmaxf(bound, -FLT_BIG);     // not NaN, not -inf
        for_groups<T, VEC>(r, s.lut, group, bound, [&](float x, int v) {
            const int at = atomicAdd(&s.n, 1);
            if (at < LIST) s.key[at] = ordered(x), s.token[at] = v;
        });
        sync();
        // the first block gathers the lists and weighs what is listed
        u64 listed = 0;
        int n = 0;
        if (rank == 0) {
            n = gather(cl, s, n_blocks);
            u64 w = 0;
            if (n <= LIST) {
                for (int i = threadIdx.x; i < n; i += NT) w += s.weight[i] = g.raw(unordered(s.key[i]));
                block_before(s, w, &listed);
            }
        }
        if (k || !nucleus) {                // the list holds all that is needed
            if (rank == 0) {
                if (n <= LIST) {
                    u64 kept;
                    const int i = settle(cl, s, g, n, k, listed, nucleus ? 0 : ~0ull, limit_of, u24, &kept);
                    if (i >= 0) finish((int)s.token[i], g.z(unordered(s.key[i])) - logf((float)kept * 0x1p-40f));
                }
                if (threadIdx.x == 0) s.part[4] = n <= LIST;
            }
            sync();
            if (peer(0)->part[4]) {
                sync();
                return;
            }
            if (k) {                        // too many for the list: digit by digit (fewer than k candidates: all stay)
                g.tau = row_search<false, T, VEC>(cl, s, r, g, n_blocks, [&](u64 all) { return min((u64)k, all); });
                if (nucleus) g.tau = row_search<true, T, VEC>(cl, s, r, g, n_blocks, limit_of);
            }
        } else {
            // Where the list ends and the nucleus may not, from a sample of the row: the
            // weights below the bound in BINS bins of z, in units of the bound's weight / 2^16.
            if (rank == 0 && threadIdx.x == 0) s.part[4] = n <= LIST ? listed : 0;
            s.bins[threadIdx.x] = 0;
            sync();
            const u64 in_list = peer(0)->part[4];
            const float unit = 65536.f / fmaxf(g.e(bound), 1e-37f), top_z = fmaxf(g.z(bound), Z_END + 1.f);
            const float to_bin = BINS / (top_z - Z_END);
            const int n_sample = min(n_chunks, UNROLL * NW);
            for (int j = warp; j < n_sample; j += NW) {
                Row one = r;
                one.lo = r.lo + (int)((int64_t)j * n_chunks / n_sample) * CHUNK;
                one.hi = min(r.hi, one.lo + CHUNK);
                one_chunk<T, VEC>(one, s.lut, [&](float x) {
                    if (x >= bound) return;
                    const float z = g.z(x);
                    if (z > Z_END)
                        atomicAdd(&s.bins[min(BINS - 1, (int)((top_z - z) * to_bin))],
                                  (uint32_t)fminf(g.e(x) * unit, 65536.f));
                });
            }
            sync();
            u64 v = 0, rest;
            for (int q = 0; q < n_blocks; q++) v += peer(q)->bins[threadIdx.x];
            const u64 upto = block_before(s, v, &rest) + v;
            // sample units -> weights; the same in all blocks, also where the last one's part is short
            const int full = per_block / CHUNK;
            const float ratio = (float)full / min(full, UNROLL * NW) * 0x1p40f / unit;
            const float est = (float)rest * ratio, need = p * ((float)in_list + est) - (float)in_list;
            const float slack = 0.04f * est + 0.002f * (float)in_list;
            const bool in_doubt = need + slack > 0.f;
            // the stretch of z in which the nucleus ends, to be looked at closely
            if (threadIdx.x == 0) s.from = 0, s.to = BINS;
            __syncthreads();
            const float mine = (float)upto * ratio, prior = (float)(upto - v) * ratio;
            if (mine >= need - slack && prior < need - slack) s.from = threadIdx.x;
            if (mine >= need + slack && prior < need + slack) s.to = threadIdx.x + 1;
            __syncthreads();
            const float z_from = !in_doubt || s.from == 0 ? 1.f : top_z - s.from / to_bin;
            const float z_to = !in_doubt ? 1.f : s.to >= BINS ? Z_END : top_z - s.to / to_bin;
            const float fine_top = fminf(z_from, 0.f), fine = BINS / fmaxf(fine_top - z_to, 1e-3f);
            auto fine_bin = [&](float z) { return min(BINS - 1, (int)((fine_top - z) * fine)); };
            sync();                         // every block has read the bins
            s.bins[threadIdx.x] = s.bins_hi[threadIdx.x] = 0;
            __syncthreads();
            // all weights; those above the stretch; those inside it by bins
            WeightSum all, above;
            for_pieces<T, VEC>(r, s.lut, [&](const Piece<T>& q, int, int, int, bool any) {
                if (!any) return;
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float z = g.z(q.get(i)), e = expf(z);
                    all.add(e, &above, z >= z_from);
                    if (z >= z_to && z < z_from) {
                        const uint64_t w = __float2ull_rn(e * 0x1p40f);
                        const int at = fine_bin(z);
                        const uint32_t lo = (uint32_t)w, old = atomicAdd(&s.bins[at], lo);
                        const uint32_t up = (uint32_t)(w >> 32) + (old + lo < old);
                        if (up) atomicAdd(&s.bins_hi[at], up);
                    }
                }
            });
            u64 lower;
            const u64 total = combine_sum(all.value(), 5, &lower), limit = limit_of(total);
            if (!in_doubt) {                // expected inside the list
                if (rank == 0) {
                    const bool good = n <= LIST && limit <= listed;
                    if (good) {
                        u64 kept;
                        const int i = settle(cl, s, g, n, 0, listed, limit, limit_of, u24, &kept);
                        if (i >= 0) finish((int)s.token[i], g.z(unordered(s.key[i])) - logf((float)kept * 0x1p-40f));
                    }
                    if (threadIdx.x == 0) s.part[6] = good;
                }
                sync();
                if (peer(0)->part[6]) {
                    sync();
                    return;
                }
                g.tau = row_search<true, T, VEC>(cl, s, r, g, n_blocks, limit_of);
            } else {
                const u64 over = combine_sum(above.value(), 7, &lower);
                u64 w = 0, inside;
                for (int q = 0; q < n_blocks; q++)
                    w += ((u64)peer(q)->bins_hi[threadIdx.x] << 32) + peer(q)->bins[threadIdx.x];
                const u64 till = over + block_before(s, w, &inside);
                const bool hit = limit > over && limit <= over + inside;
                if (till < limit && limit <= till + w) s.at = threadIdx.x, s.found[0] = limit - till;
                if (threadIdx.x == 0) s.n = 0;
                __syncthreads();
                const int bin = s.at;
                const u64 left = s.found[0];
                __syncthreads();
                if (hit) {                  // the same in all blocks: the bin's tokens, and the value among them
                    for_pieces<T, VEC>(r, s.lut, [&](const Piece<T>& q, int v0, int, int, bool any) {
                        if (!any) return;
#pragma unroll
                        for (int i = 0; i < 8; i++) {
                            const float x = q.get(i), z = g.z(x);
                            if (z >= z_to && z < z_from && fine_bin(z) == bin) {
                                const int at = atomicAdd(&s.n, 1);
                                if (at < LIST) s.key[at] = ordered(x), s.token[at] = v0 + i;
                            }
                        }
                    });
                }
                sync();
                if (rank == 0) {
                    uint32_t tau = 0;
                    if (hit && (n = gather(cl, s, n_blocks)) <= LIST) {
                        for (int i = threadIdx.x; i < n; i += NT) s.weight[i] = g.raw(unordered(s.key[i]));
                        __syncthreads();
                        tau = list_search<true, false>(cl, s, n, left, [](int) { return true; });
                    }
                    if (threadIdx.x == 0) s.part[8] = tau;
                }
                sync();
                const uint32_t tau = (uint32_t)peer(0)->part[8];
                if (tau) g.tau = unordered(tau);
                else g.tau = row_search<true, T, VEC>(cl, s, r, g, n_blocks, limit_of);
            }
        }
    }

    // the draw: weights by chunk, then the block, the chunk and the token that hold the target
    for_pieces<T, VEC>(r, s.lut, [&](const Piece<T>& q, int, int c, int, bool any) {
        WeightSum sum;
        if (any) {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float x = q.get(i), e = g.e(x);
                sum.add(x >= g.tau && e >= g.min_e ? e : 0.f);
            }
        }
        const uint32_t hi = __reduce_add_sync(FULL, sum.hi), lo = __reduce_add_sync(FULL, sum.lo);
        if (lane == 0) chunk_sum[c] = ((u64)hi << 20) + lo;
    });
    __syncthreads();
    const int per = (n_chunks + NT - 1) / NT, c0 = min(n_chunks, (int)threadIdx.x * per), c1 = min(n_chunks, c0 + per);
    u64 mine = 0, total, lower;
    for (int c = c0; c < c1; c++) mine += chunk_sum[c];
    u64 before = block_before(s, mine, &total);
    const u64 sum = combine_sum(mine, 9, &lower);
    const u64 target = part_of(sum, u24);
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
            Row one = r;                    // the chunk alone
            one.lo = r.lo + s.at * CHUNK;
            one.hi = min(r.hi, one.lo + CHUNK);
            u64 t2 = s.found[1];
            for_pieces<T, VEC>(one, s.lut, [&](const Piece<T>& q, int v0, int, int, bool) {
                u64 w = 0;
#pragma unroll
                for (int i = 0; i < 8; i++) w += g.kept(q.get(i));
                u64 in = w;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const u64 y = __shfl_up_sync(FULL, in, o);
                    if (lane >= o) in += y;
                }
                if (t2 >= in - w && t2 < in) {
                    t2 -= in - w;
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        const u64 wi = g.kept(q.get(i));
                        if (t2 < wi) {
                            finish(v0 + i, g.z(q.get(i)) - logf((float)sum * 0x1p-40f));
                            break;
                        }
                        t2 -= wi;
                    }
                }
            });
        }
    }
    sync();                                 // peers may still read this block's shared memory
}

template <typename T>
psc_status sample(const T* logits, int64_t stride, int B, int V, const uint32_t* bitmask, const Settings& S,
                  int32_t* tokens, float* logprobs, cudaStream_t cs) {
    // Enough blocks for four to an SM, each with 4096 tokens at least and 2^20 at most.
    const int want = 4 * current_sms();
    int cluster = 1;
    while (cluster < MAX_CLUSTER && ((int64_t)B * cluster < want || V / cluster > 1 << 20) && V / (2 * cluster) >= 4096)
        cluster *= 2;
    const int per = ((V + cluster - 1) / cluster + CHUNK - 1) / CHUNK * CHUNK;
    const size_t smem = sizeof(Shared) + (size_t)(per / CHUNK) * 8;
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
