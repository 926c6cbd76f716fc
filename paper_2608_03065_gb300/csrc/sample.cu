// psc_sample: one token per row among the allowed ones, by temperature, top-k,
// top-p and min-p.
//
// Every filter keeps the tokens whose logit is at least some value: the k-th
// largest; the smallest whose strictly larger ones hold less than p of the
// weight; the one where e^z reaches min_p.  So a row is filtered by one
// threshold, and what the threshold needs lies near the top: the row is read
// once for its maxima, the few tokens near them are listed in shared memory, and
// the filters and the draw are worked out in that list.  Only where all of the
// weight counts (top-p alone, or no filter) is the row weighed in later passes.
// Weights are whole numbers of 2^-40 of the largest: integer sums are the same in
// any order, so neither the atomics nor the split of a row over blocks can change
// a draw.  41 bits hold every f32 e^z over 2^-17 exactly; what is rounded away of
// a row is below V * 2^-41 of its largest weight.
#include <cooperative_groups.h>

#include <algorithm>

#include "ops_common.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int NT = 512;                 // threads of a block
constexpr int NW = NT / 32;
constexpr int PIECES = 4;               // pieces of 8 neighbouring tokens that a lane has in flight
constexpr int CHUNK = PIECES * 256;     // tokens a warp takes at a time
constexpr int LIST = 2048;              // candidates that a block holds
constexpr int SPAN = 8192;              // tokens of a stretch of values that it does; with 4,096 a
                                        // mixed batch of 1024 rows of 262,144 took 277 us, with these 270
constexpr int BINS = NT;                // of the histogram of the groups' maxima
constexpr int NUCLEUS_GROUPS = 640;     // maxima above the bound from which a nucleus is looked for
constexpr int PAIRS = 256;              // candidates that are compared pair by pair; more go to bins
constexpr int FEW = 256;                // candidates of one bin that are
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
    __device__ __forceinline__ float max8_nan() const {         // NaN if any is
        __nv_bfloat162 h[4];
#pragma unroll
        for (int i = 0; i < 4; i++) h[i] = *reinterpret_cast<const __nv_bfloat162*>(&w[i]);
        const __nv_bfloat162 a = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
        const float lo = __low2float(a), hi = __high2float(a);
        return lo > hi ? lo : lo <= hi ? hi : lo + hi;
    }
    __device__ __forceinline__ float raw(int i) const {
        return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
    }
    __device__ __forceinline__ float get(int i) const { return clean(raw(i)); }
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
    __device__ __forceinline__ float max8_nan() const {
        float m = x[0];
#pragma unroll
        for (int i = 1; i < 8; i++) asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(x[i]));
        return m;
    }
    __device__ __forceinline__ float raw(int i) const { return x[i]; }
    __device__ __forceinline__ float get(int i) const { return clean(x[i]); }
};

// The lane's piece that starts at v0 (nothing read where no token of it is allowed).
__device__ __forceinline__ uint32_t piece_bits(const Row& r, int v0) {
    const int n = r.hi - v0;
    uint32_t bits = n <= 0 ? 0u : r.mask ? r.mask[v0 >> 3] : 0xffu;
    if (n > 0 && n < 8) bits &= (1u << n) - 1;
    return bits;
}
template <typename T, bool VEC>
__device__ __forceinline__ void read_piece(const Row& r, int v0, uint32_t bits, Piece<T>& p) {
    if (!bits) return;
    const T* at = static_cast<const T*>(r.logits) + v0;
    if (VEC && r.hi - v0 >= 8) {
        p.read(at);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if ((bits >> i) & 1) p.set(i, at + i);
    }
}
template <typename T>
__device__ __forceinline__ void mask_piece(const uint4* lut, uint32_t bits, Piece<T>& p) {
    if constexpr (sizeof(T) == 2) p.keep(lut[bits]);
    else p.keep(bits);
}

// Calls f(piece, first token, q, any) for every piece of the block's part of the row, q
// its place in the chunk, and end(chunk) after a chunk's last, both by whole warps; `any`
// is false where a lane's piece holds nothing.  A chunk's pieces are loaded together.  The
// body is compiled PIECES times over if small (q a constant then), else twice: passes that
// compute weights are long, and a row of its own runs each but once or twice.
template <typename T, bool VEC, bool SMALL, typename F, typename End>
__device__ __forceinline__ void for_pieces(const Row& r, const uint4* lut, F&& f, End&& end) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n_chunks = (r.hi - r.lo + CHUNK - 1) / CHUNK;
    constexpr int BODIES = SMALL ? PIECES : 2;
#pragma unroll 1
    for (int c = warp; c < n_chunks; c += NW) {
        const int v0 = r.lo + c * CHUNK + lane * 8;
        Piece<T> p[PIECES];
        uint32_t bits[PIECES];
#pragma unroll
        for (int q = 0; q < PIECES; q++) bits[q] = piece_bits(r, v0 + q * 256);
#pragma unroll
        for (int q = 0; q < PIECES; q++) read_piece<T, VEC>(r, v0 + q * 256, bits[q], p[q]);
#pragma unroll 1
        for (int q0 = 0; q0 < PIECES; q0 += BODIES) {
#pragma unroll
            for (int q = 0; q < BODIES; q++) {
                mask_piece<T>(lut, bits[q], p[q]);
                f(p[q], v0 + (q0 + q) * 256, q0 + q, bits[q] != 0);
            }
#pragma unroll
            for (int q = 0; q + BODIES < PIECES; q++) p[q] = p[q + BODIES], bits[q] = bits[q + BODIES];
        }
        end(c);
    }
}

// Calls f(value, token) for the tokens that reach `bound`, reading the groups whose maximum
// does.  A group is a lane's q-th piece of every chunk of its warp; the warp's lanes share
// out the pieces of its groups.
template <typename T, bool VEC, typename F>
__device__ __forceinline__ void for_groups(const Row& r, const uint4* lut, const float (&group)[PIECES], float bound,
                                           F&& f) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n_chunks = (r.hi - r.lo + CHUNK - 1) / CHUNK;
    const int pieces = (n_chunks - warp + NW - 1) / NW;     // of a group of the warp
    uint32_t hits[PIECES];
    int n_hits = 0;
#pragma unroll
    for (int q = 0; q < PIECES; q++) {
        hits[q] = __ballot_sync(FULL, group[q] >= bound);
        n_hits += __popc(hits[q]);
    }
    const int jobs = n_hits * pieces;       // job i: piece i % pieces of the i / pieces-th group
    constexpr int BATCH = 4;                // a lane's jobs whose loads are in flight together
    for (int i0 = lane; i0 < jobs; i0 += 32 * BATCH) {
        int v0[BATCH];
        uint32_t bits[BATCH];
        Piece<T> p[BATCH];
#pragma unroll
        for (int t = 0; t < BATCH; t++) {
            const int i = i0 + 32 * t;
            int h = i / pieces, q = 0;
            const int j = i - h * pieces;
            uint32_t left = hits[0];
#pragma unroll
            for (int o = 0; o < PIECES - 1; o++)
                if (q == o && h >= __popc(left)) h -= __popc(left), q = o + 1, left = hits[o + 1];
            bits[t] = 0;
            if (i < jobs) {
                for (; h; h--) left &= left - 1;
                v0[t] = r.lo + (warp + j * NW) * CHUNK + q * 256 + (__ffs(left) - 1) * 8;
                bits[t] = piece_bits(r, v0[t]);
            }
        }
#pragma unroll
        for (int t = 0; t < BATCH; t++)
            if (bits[t]) read_piece<T, VEC>(r, v0[t], bits[t], p[t]);
#pragma unroll
        for (int t = 0; t < BATCH; t++) {
            mask_piece<T>(lut, bits[t], p[t]);
            if (!bits[t] || !(p[t].max8() >= bound)) continue;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float x = p[t].get(e);
                if (x >= bound) f(x, v0[t] + e);
            }
        }
    }
}

// A sum of weights as two 32-bit sums: of 2^20 e, its whole part and its fraction in units
// of 2^-20, each taken from the low bits of a sum with 2^23 (rounded down, then to nearest
// even; together rint(2^40 e), since the whole part is an even number of units).  Good for
// 2048 weights.
struct WeightSum {
    uint32_t hi = 0, lo = 0;                // with 0x4B000000 for every weight added
    int n = 0;
    // e's two parts, as such bits
    static __device__ __forceinline__ void split(float e, uint32_t* h, uint32_t* l) {
        const float a = __fmaf_rz(e, 0x1p20f, 0x1p23f);
        *h = __float_as_uint(a);
        *l = __float_as_uint(__fmaf_rn(__fmaf_rn(e, 0x1p20f, 0x1p23f - a), 0x1p20f, 0x1p23f));
    }
    static __device__ __forceinline__ u64 weight(uint32_t h, uint32_t l) {
        return ((u64)(h - 0x4B000000u) << 20) + (l - 0x4B000000u);
    }
    __device__ __forceinline__ uint32_t high() const { return hi - n * 0x4B000000u; }
    __device__ __forceinline__ uint32_t low() const { return lo - n * 0x4B000000u; }
    __device__ __forceinline__ u64 value() const { return ((u64)high() << 20) + low(); }
};
// One weight, rint(2^40 e).  (The conversion instruction to 64 bits is slow here.)
__device__ __forceinline__ u64 weight_of(float e) {
    uint32_t h, l;
    WeightSum::split(e, &h, &l);
    return WeightSum::weight(h, l);
}

// What a row's weights are computed from; the arithmetic is the header's, step by step.
struct Weigh {
    float m, inv, tau, min_e;
    __device__ __forceinline__ float z(float x) const { return __fmul_rn(__fsub_rn(x, m), inv); }
    __device__ __forceinline__ float e(float x) const { return expf(z(x)); }
    // weight of x before the filters
    __device__ __forceinline__ u64 raw(float x) const { return weight_of(e(x)); }
    // weight after them
    __device__ __forceinline__ u64 kept(float x) const {
        const float y = e(x);
        return x >= tau && y >= min_e ? weight_of(y) : 0ull;
    }
};
struct Settings {
    const float* uniform;
    const float* temperature;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
};

// What a call is about.
struct Job {
    const void* logits;
    int64_t stride;
    int B, V, per_block, W;
    const uint32_t* bitmask;
    Settings settings;
    int32_t* tokens;
    float* logprobs;
    int rows;               // which rows a kernel does
    uint8_t* pending;       // [B]: rows that k_sample_light could not settle
};
enum { ALL_ROWS, HEAVY_ROWS, PENDING_ROWS };

// What is found out about a row, kept in shared memory: a register that lives across the
// passes is one that they do not have.
struct State {
    int b, k, n, bin, own;
    float p, m, lowest, bound, z_from, z_to;
    uint32_t p24, u24;
    bool in_doubt, hit, wide;
    u64 listed, left;
};

struct Shared {
    Job job;
    State st;
    uint32_t cnt[2][256], hi[2][256];   // a histogram's counts, or its weights as two words
    uint32_t bins[BINS], bins_hi[BINS], count[BINS], tau;
    int few[FEW], n_few;
    Row row;
    Weigh g;
    float group[PIECES][NT];            // the maxima of the threads' groups
    u64 part[12];                       // this block's share of what the cluster combines, a slot per use
    u64 warp[2][NW];                    // the warps' shares of what a block combines
    uint8_t turn[NT];                   // which of the two a thread uses next
    u64 found[2];
    int at, n;
    uint4 lut[256];                     // mask byte -> ones where it allows (bf16 pairs)
    uint32_t key[LIST];                 // candidates: order of the value, weight, token
    u64 weight[LIST];
    uint32_t token[SPAN];               // (of them LIST in k_sample_light)
};

// Sum over the block's threads of v before this thread; *total: over all of them.  One
// barrier: successive calls use the two sets of s.warp in turn.
__device__ __forceinline__ u64 block_before(Shared& s, u64 v, u64* total) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    u64 in = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const u64 y = __shfl_up_sync(FULL, in, o);
        if (lane >= o) in += y;
    }
    u64* w = s.warp[s.turn[threadIdx.x] ^= 1];
    if (lane == 31) w[warp] = in;
    __syncthreads();
    u64 t = w[lane & (NW - 1)];
#pragma unroll
    for (int o = 1; o < NW; o <<= 1) {
        const u64 y = __shfl_up_sync(FULL, t, o);
        if ((lane & (NW - 1)) >= o) t += y;
    }
    *total = __shfl_sync(FULL, t, NW - 1);
    const u64 before = __shfl_sync(FULL, t, max(0, warp - 1));
    return (warp ? before : 0) + in - v;
}
// The largest of two values over the block.
__device__ __forceinline__ uint2 block_max(Shared& s, uint32_t x, uint32_t y) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    x = __reduce_max_sync(FULL, x), y = __reduce_max_sync(FULL, y);
    u64* w = s.warp[s.turn[threadIdx.x] ^= 1];
    if (lane == 0) w[warp] = (u64)x << 32 | y;
    __syncthreads();
    const u64 t = w[lane & (NW - 1)];
    return make_uint2(__reduce_max_sync(FULL, (uint32_t)(t >> 32)), __reduce_max_sync(FULL, (uint32_t)t));
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

// A sum as f32, good to a few parts in 2^24 (the conversion instruction is slow here).
__device__ __forceinline__ float to_float(u64 v) {
    return __uint2float_rn((uint32_t)(v >> 32)) * 0x1p32f + __uint2float_rn((uint32_t)v);
}
// floor(total * u24 / 2^24)
__device__ __forceinline__ u64 part_of(u64 total, u64 u24) {
    return u24 * (total >> 24) + ((u24 * (total & 0xffffff)) >> 24);
}

// The value (its order) among the block's n candidates at which the running weight
// from the largest down reaches `need`: few pair by pair, many digit by digit (a warp whose
// digits are all the same adds once).
__device__ uint32_t list_search(cg::cluster_group& cl, Shared& s, int n, u64 need) {
    if (n <= PAIRS) {
        if (threadIdx.x == 0) s.tau = ~0u;
        __syncthreads();
        const int i = threadIdx.x >> 1;         // two threads to a candidate
        u64 over = 0;
        if (i < n)
            for (int j = threadIdx.x & 1; j < n; j += 2)
                if (s.key[j] > s.key[i]) over += s.weight[j];
        over += __shfl_xor_sync(FULL, over, 1);
        if (i < n && over < need) atomicMin(&s.tau, s.key[i]);
        __syncthreads();
        return s.tau;
    }
    uint32_t prefix = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = threadIdx.x; i < 256; i += NT) s.cnt[0][i] = s.hi[0][i] = 0;
        __syncthreads();
        for (int i0 = 0; i0 < n; i0 += NT) {
            const int i = i0 + threadIdx.x;
            const uint32_t k = i < n ? s.key[i] : 0u;
            const bool in = i < n && (shift == 24 || (k >> (shift + 8)) == prefix);
            const u64 w = in ? s.weight[i] : 0ull;
            const uint32_t lanes = __ballot_sync(FULL, in);
            if (!lanes) continue;
            const uint32_t digit = (k >> shift) & 255, one = __shfl_sync(FULL, digit, __ffs(lanes) - 1);
            if (__all_sync(FULL, !in || digit == one)) {
                const uint32_t lo = __reduce_add_sync(FULL, (uint32_t)w & 0xfffff);
                const uint32_t hi = __reduce_add_sync(FULL, (uint32_t)(w >> 20));
                if ((threadIdx.x & 31) == 0) count_in<true>(s, 0, one, ((u64)hi << 20) + lo);
            } else if (in) {
                count_in<true>(s, 0, digit, w);
            }
        }
        prefix = (prefix << 8) | (uint32_t)pick_digit<true>(cl, 1, s, 0, &need);
        __syncthreads();
    }
    return prefix;
}

// The cluster's lists behind the first block's own, a warp per block; their length (over
// LIST: not gathered).
__device__ int gather(cg::cluster_group& cl, Shared& s, int n_blocks) {
    if (n_blocks == 1) return s.n;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int own = lane < n_blocks ? (lane ? cl.map_shared_rank(&s, lane)->n : s.n) : 0;
    int till = own;
#pragma unroll
    for (int o = 1; o < MAX_CLUSTER; o <<= 1) {
        const int y = __shfl_up_sync(FULL, till, o);
        if (lane >= o) till += y;
    }
    const int n = __shfl_sync(FULL, till, MAX_CLUSTER - 1);
    if (n <= LIST && warp && warp < n_blocks) {
        const Shared* o = cl.map_shared_rank(&s, warp);
        const int more = __shfl_sync(FULL, own, warp), at = __shfl_sync(FULL, till, warp) - more;
        for (int i = lane; i < more; i += 32) s.key[at + i] = o->key[i], s.token[at + i] = o->token[i];
    }
    __syncthreads();
    return n;
}

// The weight that a nucleus of `total` has to hold.
__device__ __forceinline__ u64 limit_of(const Shared& s, u64 total) { return max((u64)1, part_of(total, s.st.p24)); }

enum { FAILED = 0, DRAWN = 1, BOUNDED = 2 };    // what settle could do

// Adds a weight to its bin (two words, with carry).
__device__ __forceinline__ void add_to_bin(Shared& s, int bin, u64 w) {
    const uint32_t lo = (uint32_t)w, old = atomicAdd(&s.bins[bin], lo);
    const uint32_t up = (uint32_t)(w >> 32) + (old + lo < old);
    if (up) atomicAdd(&s.bins_hi[bin], up);
}
__device__ __forceinline__ u64 bin_weight(const Shared& s, int bin) {
    return ((u64)s.bins_hi[bin] << 32) + s.bins[bin];
}
// The listed candidates for which `in` holds, as places in s.few; their number (over FEW: not all).
template <typename In>
__device__ int pick_few(Shared& s, int n, In&& in) {
    if (threadIdx.x == 0) s.n_few = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += NT)
        if (in(i)) {
            const int at = atomicAdd(&s.n_few, 1);
            if (at < FEW) s.few[at] = i;
        }
    __syncthreads();
    return s.n_few;
}

// Filters and draws among the block's n listed candidates, of which the weights sum to
// s.st.listed and none is below `bound`: k (0: off), then a nucleus of `limit` (0: limit_of what
// top-k leaves, ~0: off), then min_e.  DRAWN: *place is the drawn one's place in the list
// for the thread that found it, -1 for others, *kept the weight of what stays.  BOUNDED:
// s.tau is the order of a value that, min_e apart, all that stays reaches and nothing else of the
// row does.
__device__ __noinline__ int settle(Shared& s, float bound, int k, u64 limit, u64* kept, int* place) {
    const Weigh g = s.g;
    const int n = s.st.n, V = s.row.V;
    u64 listed = s.st.listed;
    const int tid = threadIdx.x;
    *place = -1;
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
            limit = limit_of(s, listed);
        }
        stays = stays && over < limit && g.e(unordered(key)) >= g.min_e;
        if (!stays) w = 0;
        __syncthreads();
        if (mine && !j0) s.weight[i] = w;
        block_before(s, j0 ? 0 : w, kept);      // and every weight is written
        const u64 target = part_of(*kept, s.st.u24);
        u64 before = 0;
        if (mine)
            for (int j = j0; j < n; j += per)
                if (s.token[j] < token) before += s.weight[j];
        for (int o = per >> 1; o; o >>= 1) before += __shfl_xor_sync(FULL, before, o);
        if (mine && !j0 && before <= target && target < before + w) *place = i;
        return DRAWN;
    }
    // Counts and weights in bins of the value, then the few candidates of the bin in which
    // a filter ends pair by pair; the same by token for the draw.
    const float scale = BINS / (g.m - bound);
    auto bin_of = [&](int i) { return min(BINS - 1, (int)fmaxf(0.f, (g.m - unordered(s.key[i])) * scale)); };
    uint32_t tau = ordered(bound);              // every listed one, and no other of the row, reaches it
    if ((k && k < n) || limit != ~0ull) {
        __syncthreads();
        s.bins[tid] = s.bins_hi[tid] = s.count[tid] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += NT) {
            const int bin = bin_of(i);
            atomicAdd(&s.count[bin], 1u);
            add_to_bin(s, bin, s.weight[i]);
        }
        __syncthreads();
        // both sums at once: a weight below 2^51 over a count below 2^12
        u64 all;
        const u64 v = bin_weight(s, tid) << 12 | s.count[tid], before = block_before(s, v, &all);
        int last = BINS;                        // the bin in which top-k ends
        if (k && k < n) {
            const int c = (int)(before & 4095);
            if (c < k && k <= c + (int)(v & 4095)) s.at = tid, s.found[0] = k - c, s.found[1] = before >> 12;
            __syncthreads();
            last = s.at;
            const int want = (int)s.found[0];
            const u64 above = s.found[1];
            const int few = pick_few(s, n, [&](int i) { return bin_of(i) == last; });
            if (few > FEW) return FAILED;
            if (tid == 0) s.tau = ~0u;
            __syncthreads();
            u64 w = 0;
            if (tid < few) {
                const uint32_t key = s.key[s.few[tid]];
                int larger = 0;
                for (int j = 0; j < few; j++) larger += s.key[s.few[j]] > key;
                if (larger < want) {
                    atomicMin(&s.tau, key);
                    w = s.weight[s.few[tid]];
                }
            }
            block_before(s, w, &listed);
            listed += above;
            tau = s.tau;
        }
        if (!limit) limit = limit_of(s, listed);
        if (limit != ~0ull) {
            const u64 over = before >> 12;
            // beyond top-k's last bin nothing stays; that bin holds the limit where no earlier one does
            const bool ends = over < limit && (tid == last || limit <= over + (v >> 12)) && tid <= last;
            __syncthreads();
            if (ends) s.at = tid, s.found[0] = over;
            __syncthreads();
            const int bin = s.at;
            const u64 above = s.found[0];
            const int few = pick_few(s, n, [&](int i) { return bin_of(i) == bin && s.key[i] >= tau; });
            if (few > FEW) return FAILED;
            if (tid == 0) s.tau = ~0u;
            __syncthreads();
            if (tid < few) {
                const uint32_t key = s.key[s.few[tid]];
                u64 w = above;
                for (int j = 0; j < few; j++)
                    if (s.key[s.few[j]] > key) w += s.weight[s.few[j]];
                if (w < limit) atomicMin(&s.tau, key);
            }
            __syncthreads();
            tau = s.tau;
        }
    }
    auto in = [&](int i) { return s.key[i] >= tau && (!(g.min_e > 0.f) || g.e(unordered(s.key[i])) >= g.min_e); };
    const float to_part = (float)BINS / V;
    auto part = [&](int i) { return min(BINS - 1, (int)(s.token[i] * to_part)); };
    __syncthreads();
    s.bins[tid] = s.bins_hi[tid] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += NT)
        if (in(i)) add_to_bin(s, part(i), s.weight[i]);
    __syncthreads();
    const u64 w = bin_weight(s, tid), before = block_before(s, w, kept), target = part_of(*kept, s.st.u24);
    if (before <= target && target < before + w) s.at = tid, s.found[0] = target - before;
    __syncthreads();
    const int bin = s.at;
    const u64 left = s.found[0];
    const int few = pick_few(s, n, [&](int i) { return in(i) && part(i) == bin; });
    if (tid == 0) s.tau = tau;
    __syncthreads();
    if (few > FEW) return BOUNDED;
    if (tid < few) {
        const int i = s.few[tid];
        u64 lower = 0;
        for (int j = 0; j < few; j++)
            if (s.token[s.few[j]] < s.token[i]) lower += s.weight[s.few[j]];
        if (lower <= left && left < lower + s.weight[i]) *place = i;
    }
    return DRAWN;
}

// The search over the whole row, digit by digit of the values' order: of the candidates that
// reach s.g.tau, the value at which the running count (up to k) or weight (up to the nucleus')
// from the largest down is reached; it becomes s.g.tau.
template <bool MASS, typename T, bool VEC>
__device__ __noinline__ void row_search(Shared& s) {
    cg::cluster_group cl = cg::this_cluster();
    const int n_blocks = (int)cl.num_blocks();
    uint32_t prefix = 0;
    u64 need = 0;
    int buf = 0;
    __syncthreads();
    const Weigh g = s.g;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = threadIdx.x; i < 256; i += NT) s.cnt[buf][i] = s.hi[buf][i] = 0;
        __syncthreads();
        for_pieces<T, VEC, false>(s.row, s.lut, [&](const Piece<T>& q, int, int, bool any) {
            if (!any) return;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float x = q.get(i);
                const uint32_t key = ordered(x);
                if (x == NEG_INF || x < g.tau || (shift < 24 && (key >> (shift + 8)) != prefix)) continue;
                count_in<MASS>(s, buf, (key >> shift) & 255, MASS ? g.raw(x) : 1);
            }
        }, [](int) {});
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
            need = MASS ? limit_of(s, all) : min((u64)s.st.k, all);     // fewer candidates than k: all stay
        }
        prefix = (prefix << 8) | (uint32_t)pick_digit<MASS>(cl, n_blocks, s, buf, &need);
        buf ^= 1;
    }
    if (threadIdx.x == 0) s.g.tau = unordered(prefix);
    __syncthreads();
}

// The passes over the block's part of the row, each a function of its own so that none
// holds another's registers.  f(values, first token, any): the values cleaned if `odd`
// (a NaN or +inf is among the block's candidates).
template <typename T, bool VEC, typename F, typename End>
__device__ __forceinline__ void for_values(const Shared& s, bool odd, F&& f, End&& end) {
    for_pieces<T, VEC, false>(s.row, s.lut, [&](const Piece<T>& q, int v0, int, bool any) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = q.raw(i);
        if (odd) {
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] = clean(x[i]);
        }
        f(x, v0, any);
    }, end);
}
// A chunk's sum, over the warp.
__device__ __forceinline__ void put_chunk(u64* chunk_sum, int c, WeightSum& sum) {
    const uint32_t hi = __reduce_add_sync(FULL, sum.high()), lo = __reduce_add_sync(FULL, sum.low());
    if ((threadIdx.x & 31) == 0) chunk_sum[c] = ((u64)hi << 20) + lo;
    sum = WeightSum();
}

// The sum of all weights (the thread's share).
template <typename T, bool VEC>
__device__ __noinline__ u64 sum_pass(const Shared& s, bool odd) {
    const Weigh g = s.g;
    WeightSum all;
    for_values<T, VEC>(s, odd, [&](const float (&x)[8], int, bool any) {
        if (!any) return;
        all.n += 8;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            uint32_t h, l;
            WeightSum::split(g.e(x[i]), &h, &l);
            all.hi += h, all.lo += l;
        }
    }, [](int) {});
    return all.value();
}

// The sums by chunk of what stays.
template <typename T, bool VEC, bool FILTERED>
__device__ __noinline__ void chunk_pass(const Shared& s, u64* chunk_sum, bool odd) {
    const Weigh g = s.g;
    WeightSum sum;
    for_values<T, VEC>(s, odd, [&](const float (&x)[8], int, bool any) {
        if (!any) return;
        sum.n += 8;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            float e = g.e(x[i]);
            if (FILTERED) e = x[i] >= g.tau && e >= g.min_e ? e : 0.f;
            uint32_t h, l;
            WeightSum::split(e, &h, &l);
            sum.hi += h, sum.lo += l;
        }
    }, [&](int c) { put_chunk(chunk_sum, c, sum); });
}

// A stretch of z, from z_from (excluded, above) down to z_to, in BINS bins.
struct Stretch {
    float z_from, z_to, top, fine;
    __device__ __forceinline__ Stretch(float from, float to)
        : z_from(from), z_to(to), top(fminf(from, 0.f)), fine(BINS / fmaxf(fminf(from, 0.f) - to, 1e-3f)) {}
    __device__ __forceinline__ int bin(float z) const { return min(BINS - 1, (int)((top - z) * fine)); }
};

// All weights (the thread's share) and those above the stretch (returned in *above, and by
// chunk).  LISTED: the stretch's tokens are listed, and counted where the block cannot hold
// them all; else their weights go to the block's bins.
template <typename T, bool VEC, bool LISTED>
__device__ __noinline__ u64 stretch_pass(Shared& s, u64* chunk_sum, bool odd, const Stretch t, u64* above_all) {
    const Weigh g = s.g;
    WeightSum all, above, part;
    for_values<T, VEC>(s, odd, [&](const float (&x)[8], int v0, bool any) {
        if (!any) return;
        all.n += 8;
        uint32_t inside = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float z = g.z(x[i]), e = expf(z);
            uint32_t h, l;
            WeightSum::split(e, &h, &l);
            all.hi += h, all.lo += l;
            if (z >= t.z_from) {
                part.hi += h, part.lo += l, part.n++;
            } else if (z >= t.z_to) {
                if (LISTED) inside |= 1u << i;
                else add_to_bin(s, t.bin(z), WeightSum::weight(h, l));
            }
        }
        if (!inside) return;
        int at = atomicAdd(&s.n, __popc(inside));
        for (; inside; inside &= inside - 1, at++)
            if (at < SPAN) s.token[at] = v0 + __ffs(inside) - 1;
    }, [&](int c) {
        above.hi += part.hi, above.lo += part.lo, above.n += part.n;
        put_chunk(chunk_sum, c, part);
    });
    *above_all = above.value();
    return all.value();
}

// The weights of the listed tokens of the stretch, in the block's bins.  (In stretch_pass, where
// few threads of a warp have one at a time, the same work made 1024 top-p rows of 262,144 tokens
// 20 us slower, 64 rows of 32,000 2 us.)
template <typename T>
__device__ __noinline__ void bins_pass(Shared& s, const Stretch t) {
    const Weigh g = s.g;
    const int n = s.n;
    constexpr int BATCH = 8;
    for (int i0 = threadIdx.x; i0 < n; i0 += BATCH * NT) {
        float x[BATCH];
#pragma unroll
        for (int q = 0; q < BATCH; q++)
            x[q] = i0 + q * NT < n ? load_f32(static_cast<const T*>(s.row.logits) + s.token[i0 + q * NT]) : 0.f;
#pragma unroll
        for (int q = 0; q < BATCH; q++) {
            if (i0 + q * NT >= n) break;
            const float z = g.z(clean(x[q]));
            add_to_bin(s, t.bin(z), weight_of(expf(z)));
        }
    }
}

// Adds a token's weight to its chunk's: in the bins, as two words, where these are as many (an
// atomic sum of 64 bits is a loop); add_own adds those up.
__device__ __forceinline__ void add_to_chunk(Shared& s, u64* chunk_sum, int token, u64 w) {
    const int c = (token - s.row.lo) / CHUNK;
    if (s.row.hi - s.row.lo <= BINS * CHUNK) add_to_bin(s, c, w);
    else atomicAdd(&chunk_sum[c], w);
}

// Lists the tokens of one bin of the stretch and adds those of the bins before it to the chunks
// (in the bins, which it clears): from the tokens of the stretch, where the block holds them all.
// The orders of the bin's smallest and largest value that the thread met: y, x.
template <typename T>
__device__ __noinline__ uint2 take_bin(Shared& s, u64* chunk_sum, const Stretch t, int bin) {
    const Weigh g = s.g;
    const Row r = s.row;
    const int n = s.n;
    constexpr int BATCH = 8;
    static_assert(BATCH * NT >= LIST, "the candidates overwrite the first batch only");
    uint2 ends = make_uint2(0u, ~0u);
    for (int i0 = 0; i0 < n; i0 += BATCH * NT) {
        int token[BATCH];
#pragma unroll
        for (int q = 0; q < BATCH; q++) {
            const int i = i0 + q * NT + threadIdx.x;
            token[q] = i < n ? (int)s.token[i] : -1;
        }
        if (i0 == 0) {
            __syncthreads();
            if (threadIdx.x == 0) s.n = 0;
            __syncthreads();
        }
        float x[BATCH];
#pragma unroll
        for (int q = 0; q < BATCH; q++) x[q] = token[q] < 0 ? 0.f : load_f32(static_cast<const T*>(r.logits) + token[q]);
#pragma unroll
        for (int q = 0; q < BATCH; q++) {
            if (token[q] < 0) continue;
            const float y = clean(x[q]);
            const int in = t.bin(g.z(y));
            if (in == bin) {
                const uint32_t key = ordered(y);
                ends = make_uint2(max(ends.x, key), min(ends.y, key));
                const int at = atomicAdd(&s.n, 1);
                if (at < LIST) s.key[at] = key, s.token[at] = token[q];
            } else if (in < bin) {
                add_to_chunk(s, chunk_sum, token[q], g.raw(y));
            }
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) s.st.own = min(s.n, LIST);
    return ends;
}

// The same from the row, where it does not.
template <typename T, bool VEC>
__device__ __noinline__ uint2 bin_pass(Shared& s, u64* chunk_sum, bool odd, const Stretch t, int bin) {
    const Weigh g = s.g;
    WeightSum part;
    uint2 ends = make_uint2(0u, ~0u);
    __syncthreads();
    if (threadIdx.x == 0) s.n = 0;
    __syncthreads();
    for_values<T, VEC>(s, odd, [&](const float (&x)[8], int v0, bool any) {
        if (!any) return;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float z = g.z(x[i]);
            if (!(z >= t.z_to && z < t.z_from)) continue;
            const int in = t.bin(z);
            if (in == bin) {
                const uint32_t key = ordered(x[i]);
                ends = make_uint2(max(ends.x, key), min(ends.y, key));
                const int at = atomicAdd(&s.n, 1);
                if (at < LIST) s.key[at] = key, s.token[at] = v0 + i;
            } else if (in < bin) {
                uint32_t h, l;
                WeightSum::split(expf(z), &h, &l);
                part.hi += h, part.lo += l, part.n++;
            }
        }
    }, [&](int c) {
        const u64 till_now = chunk_sum[c];
        __syncwarp();
        put_chunk(chunk_sum, c, part);
        if ((threadIdx.x & 31) == 0) chunk_sum[c] += till_now;
    });
    __syncthreads();
    if (threadIdx.x == 0) s.st.own = min(s.n, LIST);
    return ends;
}

// Weights below the bound in bins of z, in units of `unit`: `taken` pieces of one chunk a
// warp, the chunks spread evenly.
template <typename T, bool VEC>
__device__ __noinline__ void sample_pass(Shared& s, float bound, float unit, float top_z, float to_bin, int taken) {
    const Weigh g = s.g;
    const Row r = s.row;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n_chunks = (r.hi - r.lo + CHUNK - 1) / CHUNK, n_sample = min(n_chunks, NW);
    if (warp >= n_sample) return;
    const int v0 = r.lo + (int)((int64_t)warp * n_chunks / n_sample) * CHUNK + lane * 8;
#pragma unroll 1
    for (int q = 0; q < taken; q++) {
        const uint32_t bits = piece_bits(r, v0 + q * 256);
        if (!bits) continue;
        Piece<T> one;
        read_piece<T, VEC>(r, v0 + q * 256, bits, one);
        mask_piece<T>(s.lut, bits, one);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float x = one.get(i), z = g.z(x);
            if (x < bound && z > Z_END)
                atomicAdd(&s.bins[min(BINS - 1, (int)((top_z - z) * to_bin))], (uint32_t)fminf(expf(z) * unit, 65536.f));
        }
    }
}

// The maxima of the thread's groups; whether it met a NaN or +inf.
template <typename T, bool VEC>
__device__ __noinline__ int max_pass(Shared& s) {
    const Row r = s.row;
    float group[PIECES];
#pragma unroll
    for (int q = 0; q < PIECES; q++) group[q] = NEG_INF;
    int odd = 0;
    for_pieces<T, VEC, true>(r, s.lut, [&](const Piece<T>& p, int, int q, bool) {
        float x = p.max8_nan();
        if (!(x <= FLT_BIG)) odd = 1, x = p.max8();
        group[q] = fmaxf(group[q], x);
    }, [](int) {});
#pragma unroll
    for (int q = 0; q < PIECES; q++) s.group[q][threadIdx.x] = clean(group[q]);
    return odd;
}

template <typename T, bool VEC, typename F>
__device__ __forceinline__ void own_groups(const Shared& s, float bound, F&& f) {
    const Row r = s.row;
    float group[PIECES];
#pragma unroll
    for (int q = 0; q < PIECES; q++) group[q] = s.group[q][threadIdx.x];
    for_groups<T, VEC>(r, s.lut, group, bound, f);
}

// V minus the lowest token with the value m that the thread met, 0 for none.
template <typename T, bool VEC>
__device__ __noinline__ uint32_t first_pass(const Shared& s, float m) {
    uint32_t first = 0;
    own_groups<T, VEC>(s, m, [&](float, int v) { first = max(first, (uint32_t)(s.row.V - v)); });
    return first;
}

// Lists the tokens that reach the bound.
template <typename T, bool VEC>
__device__ __noinline__ void list_pass(Shared& s, float bound) {
    own_groups<T, VEC>(s, bound, [&](float x, int v) {
        const int at = atomicAdd(&s.n, 1);
        if (at < LIST) s.key[at] = ordered(x), s.token[at] = v;
    });
}

// The blocks of a row: one (LIGHT), or a cluster.
template <bool LIGHT>
struct Blocks {
    __device__ __forceinline__ int rank() const { return LIGHT ? 0 : (int)cg::this_cluster().block_rank(); }
    __device__ __forceinline__ int count() const { return LIGHT ? 1 : (int)cg::this_cluster().num_blocks(); }
    __device__ __forceinline__ void sync() const {
        if (count() > 1) cg::this_cluster().sync();
        else __syncthreads();
    }
    __device__ __forceinline__ const Shared* peer(Shared& s, int q) const {
        return count() > 1 ? cg::this_cluster().map_shared_rank(&s, q) : &s;
    }
    // f(block's number, its shared memory) for all; those past the last are the last again, so
    // that the reads need no branches and go out together
    template <typename F>
    __device__ __forceinline__ void each(Shared& s, F&& f) const {
        const int n = count();
#pragma unroll
        for (int q = 0; q < MAX_CLUSTER; q++) f(q, q < n, peer(s, min(q, n - 1)));
    }
    // the largest of two values over the blocks
    __device__ __forceinline__ uint2 max2(Shared& s, uint32_t x, uint32_t y, int slot) const {
        uint2 v = block_max(s, x, y);
        if (count() > 1) {
            if (threadIdx.x == 0) s.part[slot] = (u64)v.x << 32 | v.y;
            sync();
            each(s, [&](int, bool, const Shared* o) {
                const u64 w = o->part[slot];
                v = make_uint2(max(v.x, (uint32_t)(w >> 32)), max(v.y, (uint32_t)w));
            });
        }
        return v;
    }
    // sum of v over the blocks' threads; over those of earlier blocks; over this block's
    __device__ __forceinline__ u64 sum(Shared& s, u64 v, int slot, u64* lower, u64* own) const {
        block_before(s, v, own);
        *lower = 0;
        if (count() == 1) return *own;
        if (threadIdx.x == 0) s.part[slot] = *own;
        sync();
        u64 all = 0;
        const int me = rank();
        each(s, [&](int q, bool there, const Shared* o) {
            const u64 w = o->part[slot];
            if (q < me) *lower += w;
            if (there) all += w;
        });
        return all;
    }
    // sums of two values over the blocks' threads (slots slot and slot + 1)
    __device__ __forceinline__ u64 sum2(Shared& s, u64 v, u64* w, int slot) const {
        u64 x, y;
        block_before(s, v, &x);
        block_before(s, *w, &y);
        if (count() > 1) {
            if (threadIdx.x == 0) s.part[slot] = x, s.part[slot + 1] = y;
            sync();
            x = y = 0;
            each(s, [&](int, bool there, const Shared* o) {
                const u64 p = o->part[slot], q = o->part[slot + 1];
                if (there) x += p, y += q;
            });
        }
        *w = y;
        return x;
    }
    // the blocks' bin of this thread's number, summed
    __device__ __forceinline__ u64 bin(Shared& s, bool weights) const {
        u64 v = 0;
        each(s, [&](int, bool there, const Shared* o) {
            const u64 w = weights ? bin_weight(*o, threadIdx.x) : (u64)o->bins[threadIdx.x];
            if (there) v += w;
        });
        return v;
    }
};

template <bool LIGHT>
__device__ __forceinline__ void finish(const Shared& s, int token, float lp) {
    const Job& j = s.job;
    j.tokens[s.st.b] = token;
    if (j.logprobs) j.logprobs[s.st.b] = lp;
    if (LIGHT) j.pending[s.st.b] = 0;
}
__device__ __forceinline__ float log_prob(const Weigh& g, float x, u64 sum) {
    return g.z(x) - logf((float)sum * 0x1p-40f);
}

// From the groups' maxima: the largest candidate (-inf: none) and the smallest of them.
template <bool LIGHT>
__device__ __noinline__ float find_ends(Shared& s) {
    uint32_t top = 0, low = 0;              // low: ~order, so that the largest is the lowest maximum
#pragma unroll
    for (int q = 0; q < PIECES; q++) {
        const float x = s.group[q][threadIdx.x];
        top = max(top, ordered(x));
        if (x > NEG_INF) low = max(low, ~ordered(x));
    }
    const uint2 ends = Blocks<LIGHT>().max2(s, top, low, 0);
    if (threadIdx.x == 0) s.st.m = unordered(ends.x), s.st.lowest = unordered(~ends.y);
    __syncthreads();
    return unordered(ends.x);
}

// After first_pass: the greedy choice.
template <bool LIGHT>
__device__ __noinline__ void finish_greedy(Shared& s, uint32_t first) {
    const Blocks<LIGHT> blocks;
    const uint32_t all = blocks.max2(s, first, 0, 1).x;
    if (blocks.rank() == 0 && threadIdx.x == 0) finish<LIGHT>(s, s.row.V - (int)all, 0.f);
    blocks.sync();                          // peers may still read this block's shared memory
}

// After sum_pass: the weight that the nucleus has to hold.
__device__ __noinline__ u64 find_limit(Shared& s, u64 all) {
    u64 lower, own;
    return limit_of(s, Blocks<false>().sum(s, all, 3, &lower, &own));
}

// A bound that at least `want` groups reach, or no bound when there are fewer groups.
template <bool LIGHT>
__device__ __noinline__ void find_bound(Shared& s, int want) {
    const Blocks<LIGHT> blocks;
    const float m = s.st.m, range = m - s.st.lowest, scale = BINS / range;
#pragma unroll
    for (int q = 0; q < PIECES; q++) {
        const float x = s.group[q][threadIdx.x];
        if (x > NEG_INF) atomicAdd(&s.bins[min(BINS - 1, (int)fmaxf(0.f, (m - x) * scale))], 1u);
    }
    blocks.sync();
    u64 groups;
    const u64 v = blocks.bin(s, false), before = block_before(s, v, &groups);
    // a little below the bin's lower edge: the bins' own arithmetic is rounded
    float bound = -FLT_BIG;
    if (groups >= want) bound = m - (threadIdx.x + 1) * (range / BINS) * 1.001f - fabsf(m) * 0x1p-20f;
    if (groups < want ? threadIdx.x == 0 : before < want && before + v >= want)
        s.st.bound = fmaxf(bound, -FLT_BIG);        // not NaN, not -inf
    __syncthreads();
}

// The first block gathers the blocks' lists and weighs what is listed.
template <bool LIGHT>
__device__ __noinline__ void weigh_list(Shared& s) {
    const Blocks<LIGHT> blocks;
    blocks.sync();
    if (blocks.rank() == 0) {
        cg::cluster_group cl = cg::this_cluster();
        const int n = gather(cl, s, blocks.count());
        const Weigh g = s.g;
        u64 w = 0, listed = 0;
        if (n <= LIST) {
            for (int i = threadIdx.x; i < n; i += NT) w += s.weight[i] = g.raw(unordered(s.key[i]));
            block_before(s, w, &listed);
        }
        if (threadIdx.x == 0) s.st.n = n, s.st.listed = listed;
        __syncthreads();
    }
}

// The first block settles the row by its list: top-k of k, then a nucleus of `limit` (as for
// settle).  What came of it, the same in all blocks; BOUNDED: s.g.tau is set.
template <bool LIGHT>
__device__ __noinline__ int settle_list(Shared& s, int k, u64 limit, int slot) {
    const Blocks<LIGHT> blocks;
    if (blocks.rank() == 0) {
        int done = FAILED, place = -1;
        u64 kept;
        // without top-k the nucleus has to end in the list
        if (s.st.n <= LIST && (k || limit == ~0ull || limit <= s.st.listed))
            done = settle(s, s.st.bound, k, limit, &kept, &place);
        if (done == DRAWN && place >= 0)
            finish<LIGHT>(s, (int)s.token[place], log_prob(s.g, unordered(s.key[place]), kept));
        if (threadIdx.x == 0) s.part[slot] = (u64)s.tau << 32 | (uint32_t)done;
    }
    blocks.sync();
    const u64 said = blocks.peer(s, 0)->part[slot];
    if (threadIdx.x == 0 && (int)said == BOUNDED) s.g.tau = unordered((uint32_t)(said >> 32));
    blocks.sync();                          // also: the first block's shared memory has been read
    return (int)said;
}

// From a sample of the weights below the bound: where the nucleus is expected to end.  Estimated
// is the share of the weight below the bound that it holds: an error of the sample's total
// moves that by (1 - p) of itself only.  The slack is three to four times what samples of these
// sizes were seen to be off.
template <typename T, bool VEC>
__device__ __noinline__ void find_stretch(Shared& s) {
    const Blocks<false> blocks;
    if (blocks.rank() == 0 && threadIdx.x == 0) s.part[4] = s.st.n <= LIST ? s.st.listed : 0;
    s.bins[threadIdx.x] = 0;
    blocks.sync();
    const float in_list = to_float(blocks.peer(s, 0)->part[4]), bound = s.st.bound;
    // bins of z; weights in units of the bound's / 2^16
    const float unit = 65536.f / fmaxf(s.g.e(bound), 1e-37f), top_z = fmaxf(s.g.z(bound), Z_END + 1.f);
    const float to_bin = BINS / (top_z - Z_END);
    const int full = s.job.per_block / CHUNK;
    const int taken = min(PIECES, max(1, full / (2 * NW)));     // an eighth, or a piece per warp
    sample_pass<T, VEC>(s, bound, unit, top_z, to_bin, taken);
    blocks.sync();
    u64 rest;
    const u64 v = blocks.bin(s, false), upto = block_before(s, v, &rest) + v;
    // sample units -> weights; the same in all blocks, also where the last one's part is short
    const float ratio = (float)(full * PIECES) / (min(full, NW) * taken) * 0x1p40f / unit;
    const float sampled = fmaxf(to_float(rest), 1e-30f), list_to_rest = in_list / fmaxf(sampled * ratio, 1e-30f);
    const float p = s.st.p, share = p - (1.f - p) * list_to_rest;
    const float slack = 0.08f * fmaxf(share, 0.f) * (1.f - share) + 0.06f * (1.f - p) * list_to_rest + 5e-4f;
    if (threadIdx.x == 0) s.st.z_from = 1.f, s.st.z_to = Z_END, s.st.in_doubt = share + slack > 0.f;
    __syncthreads();
    const float till = to_float(upto) / sampled, prior = to_float(upto - v) / sampled;
    if (threadIdx.x && till >= share - slack && prior < share - slack) s.st.z_from = top_z - threadIdx.x / to_bin;
    if (threadIdx.x < BINS - 1 && till >= share + slack && prior < share + slack)
        s.st.z_to = top_z - (threadIdx.x + 1) / to_bin;
    // how many tokens that is of the row, from the weight of one in each bin
    u64 tokens;
    const float one = s.g.e(bound) * unit * expf(-(threadIdx.x + 0.5f) / to_bin);
    const bool in = till >= share - slack && prior < share + slack;
    block_before(s, in ? (u64)__float2uint_rn(fminf(to_float(v) / fmaxf(one, 1.f), 1e6f)) : 0, &tokens);
    if (threadIdx.x == 0) s.st.wide = tokens * (full * PIECES) / (min(full, NW) * taken) > SPAN * blocks.count() * 7 / 8;
    blocks.sync();                          // and every block has read the bins
}

// After stretch_pass and bins_pass: whether the nucleus ends in the stretch, in which bin, and after how much of it.
__device__ __noinline__ void find_bin(Shared& s, u64 all, u64 above) {
    const Blocks<false> blocks;
    u64 over = above, inside;
    const u64 limit = limit_of(s, blocks.sum2(s, all, &over, 10));
    const u64 w = blocks.bin(s, true), till = over + block_before(s, w, &inside);
    if (till < limit && limit <= till + w) s.st.bin = threadIdx.x, s.st.left = limit - till;
    if (threadIdx.x == 0) s.st.hit = limit > over && limit <= over + inside;
    blocks.sync();                          // and every block has read the bins
    s.bins[threadIdx.x] = s.bins_hi[threadIdx.x] = 0;
    __syncthreads();
}

// After take_bin or bin_pass (ends: of the values in the bin): the value at which the nucleus ends, 0 where
// the list does not tell.
__device__ __noinline__ uint32_t find_tau(Shared& s, uint2 ends, bool* by_list) {
    const Blocks<false> blocks;
    const uint2 all = blocks.max2(s, ends.x, ~ends.y, 6);
    blocks.sync();
    if (blocks.rank() == 0) {
        cg::cluster_group cl = cg::this_cluster();
        const int n = gather(cl, s, blocks.count());
        uint32_t tau = 0;
        if (n <= LIST) {
            const Weigh g = s.g;
            for (int i = threadIdx.x; i < n; i += NT) s.weight[i] = g.raw(unordered(s.key[i]));
            __syncthreads();
            tau = list_search(cl, s, n, s.st.left);
        }
        if (threadIdx.x == 0) s.part[8] = tau;
    }
    blocks.sync();
    const uint32_t tau = (uint32_t)blocks.peer(s, 0)->part[8];
    *by_list = tau != 0;
    return tau ? tau : all.x == ~all.y ? all.x : 0u;    // equal values need no list
}

// Adds the listed tokens of the bin that stay to the chunks, and what the bins hold of those.
__device__ __noinline__ void add_own(Shared& s, u64* chunk_sum, uint32_t tau) {
    const Weigh g = s.g;
    const int n_chunks = (s.row.hi - s.row.lo + CHUNK - 1) / CHUNK;
    for (int i = threadIdx.x; i < s.st.own; i += NT)
        if (s.key[i] >= tau) add_to_chunk(s, chunk_sum, (int)s.token[i], g.raw(unordered(s.key[i])));
    __syncthreads();
    if (n_chunks <= BINS && threadIdx.x < n_chunks) chunk_sum[threadIdx.x] += bin_weight(s, threadIdx.x);
    __syncthreads();
}

// The draw from the chunks' sums: the block, the chunk and the token that hold the target.
template <typename T, bool VEC>
__device__ __noinline__ void draw(Shared& s, const u64* chunk_sum) {
    const Blocks<false> blocks;
    const Row r = s.row;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n_chunks = (r.hi - r.lo + CHUNK - 1) / CHUNK;
    const int per = (n_chunks + NT - 1) / NT, c0 = min(n_chunks, (int)threadIdx.x * per), c1 = min(n_chunks, c0 + per);
    u64 mine = 0, total, lower;
    for (int c = c0; c < c1; c++) mine += chunk_sum[c];
    u64 before = block_before(s, mine, &total);
    const u64 sum = blocks.sum(s, mine, 9, &lower, &total), target = part_of(sum, s.st.u24);
    if (target >= lower && target < lower + total) {
        const u64 t = target - lower;
        if (t >= before && t < before + mine) {
            int c = c0;
            while (before + chunk_sum[c] <= t) before += chunk_sum[c++];
            s.at = c;
            s.found[1] = t - before;
        }
        __syncthreads();
        // a warp per piece of the chunk
        const Weigh g = s.g;
        const int v0 = r.lo + s.at * CHUNK + warp * 256 + lane * 8;
        u64 w[8], in = 0, all;
        Piece<T> q;
        if (warp < PIECES) {
            const uint32_t bits = piece_bits(r, v0);
            read_piece<T, VEC>(r, v0, bits, q);
            mask_piece<T>(s.lut, bits, q);
#pragma unroll
            for (int i = 0; i < 8; i++) in += w[i] = g.kept(q.get(i));
        }
        u64 till = block_before(s, in, &all);
        const u64 left = s.found[1];
        if (left >= till && left < till + in) {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                if (left >= till && left < till + w[i]) finish<false>(s, v0 + i, log_prob(g, q.get(i), sum));
                till += w[i];
            }
        }
    }
}

// A cluster of blocks per row, each with a contiguous part of the vocabulary.
//
// A pass from memory finds the largest candidate and the maxima of a few thousand groups
// of tokens.  At least k tokens lie at or above the k-th largest of those maxima, and not
// many more; the groups that reach it are read again, their tokens listed, and top-k, top-p
// and the draw are searches in that list by the cluster's first block.  Without top-k the
// weights have to be summed in a second pass (from L2): the nucleus is sought in the list
// of the tokens at or above the NUCLEUS_GROUPS-th maximum or, where a sample of the row
// says that it ends below, in the stretch of z around the sample's estimate: its tokens are
// listed by the same pass, their weights go to bins, and the bin in which the nucleus ends is
// searched.  A stretch of more than SPAN tokens costs a pass more.  The estimate decides
// only what is looked at: whatever it misses is searched digit by digit over the whole row.
// What no list holds is drawn from sums by chunk.
//
// Measured (bf16, device time): 1 row of 262,144 tokens 15 us with top-k, 30 with top-p alone;
// 1024 rows 116 us greedy, 127 min-p, 142 top-k, 316 temperature alone, 658 top-p 0.9 alone, 898 top-p
// 0.99: the first three at 3.8 TB/s and more, the others by their instructions (some 20 a token for e^z and
// its two whole numbers, in two passes for top-p).  A single row is a chain of some ten short
// steps with a barrier each.
//
// Rows that need no weights of all tokens (greedy, top-k, min-p alone) and those that do
// differ tenfold in time and want different splits, so a large batch whose settings may hold
// both is done by three kernels: k_sample begins with the heavy rows, a cluster for each;
// k_sample_light does the others meanwhile, a block for each; and k_sample comes back for
// rows whose candidates turned out to be more than a list.  LIGHT: without what heavy rows need.
__device__ __forceinline__ bool is_light(const Settings& S, int V, int b) {
    if (S.temperature && !(S.temperature[b] >= 1e-6f)) return true;
    if (S.top_k && S.top_k[b] > 0 && S.top_k[b] < V) return true;
    return S.min_p && S.min_p[b] > 0.f && !(S.top_p && S.top_p[b] < 1.f);
}

template <typename T, bool VEC, bool LIGHT>
__device__ __forceinline__ void sample_row(Shared& s, u64* chunk_sum, int b) {
    const Blocks<LIGHT> blocks;
    State& st = s.st;
    {
        const Job& j = s.job;
        const Settings& S = j.settings;
        const float temp = S.temperature ? S.temperature[b] : 1.f, p = S.top_p ? S.top_p[b] : 1.f;
        const float min_e = S.min_p && S.min_p[b] > 0.f ? fminf(S.min_p[b], 1.f) : 0.f;
        const int k = S.top_k && S.top_k[b] > 0 && S.top_k[b] < j.V ? S.top_k[b] : 0;
        s.bins[threadIdx.x] = 0;
        if (threadIdx.x == 0) {
            const float u = S.uniform[b];
            s.n = 0;
            st.b = b, st.k = k, st.p = p;
            st.p24 = p < 1.f ? __float2uint_rn(fmaxf(p, 0.f) * 0x1p24f) : 0u;
            st.u24 = u > 0.f ? min(0xffffffu, __float2uint_rz(fminf(u, 1.f) * 0x1p24f)) : 0u;
            // 0 stands for greedy; the largest temperatures have an inverse (no flush of small
            // numbers), under which every z of ordinary logits is a weight of 1
            s.g = Weigh{0.f, temp >= 1e-6f ? __fdiv_rn(1.f, fminf(temp, FLT_BIG)) : 0.f, NEG_INF, min_e};
            s.row = Row{static_cast<const T*>(j.logits) + (size_t)b * j.stride,
                        j.bitmask ? reinterpret_cast<const uint8_t*>(j.bitmask + (size_t)b * j.W) : nullptr, j.V,
                        min(j.V, blocks.rank() * j.per_block), min(j.V, (blocks.rank() + 1) * j.per_block)};
        }
    }
    __syncthreads();
    const int odd = __syncthreads_or(max_pass<T, VEC>(s));      // a NaN or +inf among the block's candidates
    const float m = find_ends<LIGHT>(s);
    if (m == NEG_INF) {                     // nothing to choose from
        if (blocks.rank() == 0 && threadIdx.x == 0) finish<LIGHT>(s, -1, NEG_INF);
        blocks.sync();                      // peers may still read this block's shared memory
        return;
    }
    if (s.g.inv == 0.f) {                   // greedy
        finish_greedy<LIGHT>(s, first_pass<T, VEC>(s, m));
        return;
    }
    if (threadIdx.x == 0) {
        s.g.m = m;
        // min-p alone: a little below the value at which e^z is min_e
        st.bound = fmaxf(m + (logf(s.g.min_e) * 1.0001f - 1e-4f) / s.g.inv - fabsf(m) * 0x1p-20f, -FLT_BIG);
    }
    __syncthreads();
    const bool nucleus = st.p < 1.f;
    bool summed = false;                    // chunk_sum holds what stays
    if (st.k || nucleus || s.g.min_e > 0.f) {
        if (st.k || nucleus) find_bound<LIGHT>(s, st.k ? st.k : NUCLEUS_GROUPS);
        list_pass<T, VEC>(s, st.bound);
        weigh_list<LIGHT>(s);
        if (LIGHT || st.k || !nucleus) {    // the list holds all that is needed
            const int done = settle_list<LIGHT>(s, st.k, st.p < 1.f ? 0 : ~0ull, 2);
            if (done == DRAWN) return;
            if (LIGHT) {
                if (threadIdx.x == 0) s.job.pending[st.b] = 1;
                return;
            }
            if constexpr (!LIGHT) {
                if (done == FAILED && st.k) {           // too many for the list
                    row_search<false, T, VEC>(s);
                    if (st.p < 1.f) row_search<true, T, VEC>(s);
                }
            }
        } else if constexpr (!LIGHT) {
            bool found = false;
            find_stretch<T, VEC>(s);
            if (!st.in_doubt) {             // expected inside the list: the sum of all weights is what it wants
                const int done = settle_list<false>(s, 0, find_limit(s, sum_pass<T, VEC>(s, odd)), 2);
                if (done == DRAWN) return;
                found = done == BOUNDED;
                // all of the row then, listed if that may fit under a mask and costs little if not
                // (64 masked f32 rows of 32,000 tokens: 46 us, 52 not listed)
                if (threadIdx.x == 0) st.z_from = 1.f, st.z_to = Z_END, st.wide = s.job.per_block > 4 * SPAN;
                __syncthreads();
            }
            // The stretch looked at closely; where the nucleus does not end in it the whole row
            // is, and where its bin holds more than a list that bin is the next stretch.
            for (int turn = 0; turn < 6 && !found; turn++) {
                u64 above;
                s.bins[threadIdx.x] = s.bins_hi[threadIdx.x] = 0;
                if (threadIdx.x == 0) s.n = 0;
                __syncthreads();
                const Stretch t(st.z_from, st.z_to);
                u64 all;
                if (!st.wide) {
                    all = stretch_pass<T, VEC, true>(s, chunk_sum, odd, t, &above);
                    __syncthreads();
                }
                const bool listed = !st.wide && s.n <= SPAN;
                if (listed) bins_pass<T>(s, t);
                else all = stretch_pass<T, VEC, false>(s, chunk_sum, odd, t, &above);
                find_bin(s, all, above);
                if (!st.hit) {              // the same in all blocks
                    if (st.z_from == 1.f && st.z_to == Z_END) break;
                    __syncthreads();
                    if (threadIdx.x == 0) st.z_from = 1.f, st.z_to = Z_END, st.wide = true;
                    __syncthreads();
                    continue;
                }
                const uint2 ends = listed ? take_bin<T>(s, chunk_sum, t, st.bin)
                                          : bin_pass<T, VEC>(s, chunk_sum, odd, t, st.bin);
                bool by_list;
                const uint32_t tau = find_tau(s, ends, &by_list);
                if (threadIdx.x == 0) {
                    if (tau) {
                        s.g.tau = unordered(tau);
                    } else {                // the bin's edges, a little apart
                        const float off = 1e-4f / t.fine + 4e-6f * (1.f - t.top + st.bin / t.fine);
                        if (st.bin) st.z_from = t.top - st.bin / t.fine + off;
                        st.z_to = fmaxf(t.top - (st.bin + 1) / t.fine - off, Z_END);
                        st.wide = false;
                    }
                }
                __syncthreads();
                found = tau != 0;
                if (by_list && !(s.g.min_e > 0.f)) {
                    add_own(s, chunk_sum, tau);
                    summed = true;
                }
            }
            if (!found) row_search<true, T, VEC>(s);
        }
    }
    if constexpr (!LIGHT) {                 // every light row has a list
        if (!summed) {
            if (s.g.tau > NEG_INF || s.g.min_e > 0.f) chunk_pass<T, VEC, true>(s, chunk_sum, odd);
            else chunk_pass<T, VEC, false>(s, chunk_sum, odd);
            __syncthreads();
        }
        draw<T, VEC>(s, chunk_sum);
        blocks.sync();                      // peers may still read this block's shared memory
    }
}

__device__ __forceinline__ void set_up(Shared& s) {
    if (threadIdx.x < 256) {
        auto pair = [&](int i) {
            return ((threadIdx.x >> i) & 1) * 0x0000ffffu + ((threadIdx.x >> (i + 1)) & 1) * 0xffff0000u;
        };
        s.lut[threadIdx.x] = make_uint4(pair(0), pair(2), pair(4), pair(6));
    }
    __syncthreads();
}

// It follows k_sample, which began when all earlier kernels had completed, and waits for
// nothing of it; one block sees to it that this kernel does not complete before that one.
template <typename T, bool VEC>
__global__ void __launch_bounds__(NT, 2) k_sample_light(const __grid_constant__ Job j) {
    extern __shared__ __align__(16) uint8_t dyn[];
    Shared& s = *reinterpret_cast<Shared*>(dyn);
    if (is_light(j.settings, j.V, blockIdx.x)) {
        s.turn[threadIdx.x] = 0;
        if (threadIdx.x == 0) s.job = j;
        set_up(s);
        sample_row<T, VEC, true>(s, nullptr, blockIdx.x);
    } else if (threadIdx.x == 0) {
        j.pending[blockIdx.x] = 0;
    }
    if (blockIdx.x == 0) dep_wait();
}

// The cluster's row; -1: there is none for it.
__device__ __forceinline__ int find_row(Shared& s, int i) {
    const Job& j = s.job;
    if (j.rows == ALL_ROWS) return i;
    if (j.rows == HEAVY_ROWS) return is_light(j.settings, j.V, i) ? -1 : i;
    return j.pending[i] ? i : -1;
}

// A cluster for each row.  (No loop over rows: with one the compiler leaves the passes too few
// registers.)
template <typename T, bool VEC>
__global__ void __launch_bounds__(NT, 2) k_sample(const __grid_constant__ Job j) {
    extern __shared__ __align__(16) uint8_t dyn[];
    Shared& s = *reinterpret_cast<Shared*>(dyn);
    s.turn[threadIdx.x] = 0;
    if (threadIdx.x == 0) s.job = j;
    dep_wait();
    dep_launch();
    __syncthreads();
    const int b = find_row(s, blockIdx.x / (int)cg::this_cluster().num_blocks());
    if (b < 0) return;
    set_up(s);
    sample_row<T, VEC, false>(s, reinterpret_cast<u64*>(dyn + sizeof(Shared)), b);
}

// Blocks per row: two run on an SM.  Rows are split while there are blocks for all of them at once, as
// long as most warps have a chunk; until the rows in flight leave room in the L2 for the later
// passes; and to 2^20 tokens a block (what WeightSum holds).
int split(int rows, int V, size_t bytes) {
    const int sms = current_sms();
    int cluster = 1;
    while (cluster < MAX_CLUSTER &&
           (((int64_t)rows * cluster * 2 <= 2 * sms && V / (2 * cluster) >= NW * CHUNK * 3 / 4) || V / cluster > 1 << 20 ||
            std::min<int64_t>(rows, 2 * sms / cluster) * V * (int64_t)bytes > 128 << 20))
        cluster *= 2;
    return cluster;
}

// Batches of at least this many rows, with top-k or min-p, are done by three kernels, of which the
// first splits its rows as if a fifth of the batch were heavy.  (Rows of which two in five are, of
// 128,256 tokens, one kernel's time in brackets: 64 rows 48 us (53), 80 rows 49 (66), 256 rows 80
// (128), 512 rows 123 (157).  A heavy row of many is split at least in two: 1024 rows of 262,144
// tokens 316 us, not split 331, in four 379.)
constexpr int THREE_KERNELS = 48;

template <typename T>
psc_status sample(const T* logits, int64_t stride, int B, int V, const uint32_t* bitmask, const Settings& S,
                  int32_t* tokens, float* logprobs, uint8_t* pending, cudaStream_t cs) {
    const bool vec = is_aligned(logits, stride * sizeof(T), 16);
    Job j{logits, stride, B, V, 0, (V + 31) / 32, bitmask, S, tokens, logprobs, ALL_ROWS, pending};
    auto launch = [&](int rows, int cluster) {
        j.rows = rows;
        j.per_block = ((V + cluster - 1) / cluster + CHUNK - 1) / CHUNK * CHUNK;
        const size_t smem = sizeof(Shared) + (size_t)(j.per_block / CHUNK) * 8;
        return ops_launch(vec ? k_sample<T, true> : k_sample<T, false>, dim3((unsigned)B * cluster), NT, smem, cluster,
                          cs, "k_sample", j);
    };
    if (B < THREE_KERNELS || V > 1 << 20 || !(S.top_k || S.min_p)) return launch(ALL_ROWS, split(B, V, sizeof(T)));
    psc_status s = launch(HEAVY_ROWS, split(std::min(B / 5, current_sms()), V, sizeof(T)));
    if (s != PSC_OK) return s;
    j.per_block = (V + CHUNK - 1) / CHUNK * CHUNK;
    s = ops_launch(vec ? k_sample_light<T, true> : k_sample_light<T, false>, dim3(B), NT,
                   offsetof(Shared, token) + LIST * sizeof(uint32_t), 1, cs, "k_sample_light", j);
    return s != PSC_OK ? s : launch(PENDING_ROWS, 1);
}

}  // namespace

extern "C" int64_t psc_sample_work_bytes(int32_t B) { return B < THREE_KERNELS ? 0 : ((int64_t)B + 15) / 16 * 16; }

extern "C" psc_status psc_sample(const void* d_logits, psc_dtype dtype, int64_t row_stride, int32_t B, int32_t V,
                                 const uint32_t* d_bitmask, const float* d_uniform, const float* d_temperature,
                                 const int32_t* d_top_k, const float* d_top_p, const float* d_min_p,
                                 int32_t* d_tokens, float* d_logprobs, void* d_work, int64_t work_bytes,
                                 void* stream) {
    const char* me = "psc_sample";
    if (B < 0 || V <= 0 || row_stride < V || !is_dtype(dtype) || (B && (!d_logits || !d_uniform || !d_tokens)))
        return ops_fail(PSC_ERR_ARG, me, "bad arguments");
    if (V > MAX_V) return ops_fail(PSC_ERR_LIMIT, me, "vocabulary over 4,194,304 tokens");
    if (B > 0x7fffffff / MAX_CLUSTER) return ops_fail(PSC_ERR_LIMIT, me, "batch too large");
    if (B == 0) return PSC_OK;
    if (psc_sample_work_bytes(B) && (!d_work || work_bytes < psc_sample_work_bytes(B)))
        return ops_fail(PSC_ERR_ARG, me, "workspace missing or too small");
    const Settings S{d_uniform, d_temperature, d_top_k, d_top_p, d_min_p};
    if (dtype == PSC_BF16)
        return sample((const __nv_bfloat16*)d_logits, row_stride, B, V, d_bitmask, S, d_tokens, d_logprobs,
                      (uint8_t*)d_work, (cudaStream_t)stream);
    return sample((const float*)d_logits, row_stride, B, V, d_bitmask, S, d_tokens, d_logprobs, (uint8_t*)d_work,
                  (cudaStream_t)stream);
}
