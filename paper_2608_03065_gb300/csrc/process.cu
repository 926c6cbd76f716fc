// psc_process_logits: penalties for repeated tokens, biases and the grammar mask.
//
// Of a row's V logits the penalties and biases change only the tokens that its
// history and biases name, so they cost what the history is long and not what
// the vocabulary is wide: k_mask_copy streams the row through the mask (a copy
// at memory speed, left out when nothing has to be copied or masked), and
// k_penalize counts the row's history in a shared-memory table and rewrites the
// few tokens that it names.
#include <algorithm>

#include "ops_common.cuh"

namespace {

constexpr int MAX_V = 1 << 30;
constexpr int MAX_BIAS = 4096;
constexpr int MAX_HISTORY = (1 << 24) - 1;      // a count fits 24 bits
constexpr uint32_t SEEN = 1u << 30;             // the token is in the prompt
constexpr uint32_t COUNT = (1u << 24) - 1;      // times in the output
constexpr uint32_t EMPTY = 0xffffffffu;

constexpr int HASH_SLOTS = 8192;                // most slots of a hashed table: see TableKind
constexpr int TABLE_BYTES = 192 * 1024;         // of a direct table at most

template <typename T>
struct Ninf;
template <>
struct Ninf<__nv_bfloat16> {
    static constexpr uint32_t word = 0xFF80FF80u;
};
template <>
struct Ninf<float> {
    static constexpr uint32_t word = 0xFF800000u;
};

// A 16-byte piece with -inf where `bits` (8 of bf16, 4 of f32) is 0.
template <typename T>
__device__ __forceinline__ uint4 mask_piece(uint4 v, uint32_t bits) {
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; i++) {
        uint32_t m;
        if (sizeof(T) == 2) m = ((bits >> (2 * i)) & 1) * 0x0000FFFFu + ((bits >> (2 * i + 1)) & 1) * 0xFFFF0000u;
        else m = ((bits >> i) & 1) * 0xFFFFFFFFu;
        w[i] = (w[i] & m) | (Ninf<T>::word & ~m);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// out = mask ? logits : -inf, a warp per 1024 columns.
template <typename T>
__global__ void __launch_bounds__(256, 4) k_mask_copy(const T* logits, int64_t stride, T* out, int64_t out_stride,
                                                      int B, int V, const uint32_t* bitmask, int W, int vec) {
    constexpr int E = 16 / sizeof(T), PASSES = 1024 / (32 * E);
    const int lane = threadIdx.x & 31;
    const int cpr = (V + 1023) >> 10;
    const long total = (long)B * cpr, nw = ((long)gridDim.x * blockDim.x) >> 5;
    dep_wait();
    dep_launch();
    for (long c = ((long)blockIdx.x * blockDim.x + threadIdx.x) >> 5; c < total; c += nw) {
        const int b = (int)(c / cpr), j = (int)(c - (long)b * cpr), col0 = j << 10;
        const int wi = j * 32 + lane;
        const uint32_t word = !bitmask ? FULL : wi < W ? bitmask[(size_t)b * W + wi] : 0u;
        const T* src = logits + (size_t)b * stride + col0;
        T* dst = out + (size_t)b * out_stride + col0;
        if (vec && col0 + 1024 <= V) {
            uint32_t bits[PASSES];
            uint4 v[PASSES];
#pragma unroll
            for (int k = 0; k < PASSES; k++) {
                const int col = (k * 32 + lane) * E;
                bits[k] = (__shfl_sync(FULL, word, col >> 5) >> (col & 31)) & ((1u << E) - 1);
                v[k] = make_uint4(0, 0, 0, 0);
                if (bits[k]) v[k] = *reinterpret_cast<const uint4*>(src + col);
            }
#pragma unroll
            for (int k = 0; k < PASSES; k++)
                *reinterpret_cast<uint4*>(dst + (k * 32 + lane) * E) = mask_piece<T>(v[k], bits[k]);
        } else {
            const int n = min(1024, V - col0);
            for (int e = 0; e < 32; e++) {
                const int col = e * 32 + lane;
                const uint32_t w = __shfl_sync(FULL, word, e);
                if (col < n) {
                    if ((w >> lane) & 1) dst[col] = src[col];
                    else store_f32(dst + col, __uint_as_float(0xFF800000u));
                }
            }
        }
    }
}

struct Penalties {
    const int32_t* history;
    int64_t history_stride;
    int H;
    const int32_t* history_len;
    const int32_t* prompt_len;
    const float* repetition;
    const float* frequency;
    const float* presence;
    const int32_t* bias_ids;
    const float* bias;
    int n_bias;
};

// The tokens that a row's history and biases name, counted in shared memory, then
// rewritten one by one.  HASH: one block per row, an open-addressed table keyed by
// token with at least twice as many slots as history entries.  Otherwise, for any history
// length, 2^shares blocks per row, each with a table indexed by token for every 2^shares-th
// token (neighbours apart, because the frequent ones often have neighbouring ids).  A table
// word holds the output count and the prompt bit.  The biases have a hashed table of their
// own, of the last position of each id, so that the order of threads does not matter.
// What takes the time is latency, not bytes: a thread loads LOADS ids, and rewrites BATCH
// tokens, at a time.  (Measured on 20,000 ids of 151,936 tokens in 201 rows, with the copy:
// tables of 16,384 neighbouring tokens 353 us, LOADS at a time 100 us; a table spread over a
// cluster of 8 blocks, each id read once and counted in its owner's memory, 106 us.)
constexpr int LOADS = 8;

// The slot of token v in an open-addressed table of `cap` keys (never more than half full).
__device__ __forceinline__ int hash_slot(uint32_t* key, int cap, int shift, uint32_t v) {
    uint32_t i = (v * 2654435761u) >> shift;
    for (int it = 0; it < cap; it++) {
        const uint32_t k = atomicCAS(&key[i], EMPTY, v);
        if (k == EMPTY || k == v) break;
        i = (i + 1) & (cap - 1);
    }
    return (int)i;
}
// The slot that holds v, or -1.
__device__ __forceinline__ int hash_find(const uint32_t* key, int cap, int shift, uint32_t v) {
    uint32_t i = (v * 2654435761u) >> shift;
    for (int it = 0; it < cap; it++) {
        if (key[i] == v) return (int)i;
        if (key[i] == EMPTY) break;
        i = (i + 1) & (cap - 1);
    }
    return -1;
}
__host__ __device__ inline int hash_cap(int entries) {
    int cap = 32;
    while (cap < 2 * entries) cap <<= 1;
    return cap;
}

// A direct table's words are 16 bits while no count can pass 15 (SHORT), 32 otherwise.  Hashed
// tables, for up to 4,096 ids (64 rows of 151,936 tokens: 25 us, direct 23; 201 rows: 55, direct
// 67; 64 rows of 8,192 ids: 35, direct 25), are worked by 1024 threads (WIDE); by 256 where
// there are rows for every SM and under 2,048 ids in each: four blocks of an SM hide each other's
// latency (201 rows of 151,936 tokens: 1,024 ids 38 us, with 1024 threads 41; 4,096 ids 79 and
// 55; 64 rows of 2,047 ids of 32,000 tokens 24 and 13).
enum TableKind { HASHED, WIDE, SHORT, LONG };
constexpr int SHORT_HISTORY = 32767;
constexpr int WIDE_HISTORY = 2048;
__host__ __device__ constexpr int table_threads(TableKind k) { return k == HASHED ? 256 : 1024; }

template <typename T, TableKind KIND>
__global__ void __launch_bounds__(table_threads(KIND), KIND == HASHED ? 4 : 1)
    k_penalize(const T* logits, int64_t stride, T* out, int64_t out_stride, int V, Penalties P,
               const uint32_t* bitmask, int W, int shares, int early) {
    constexpr bool HASH = KIND == HASHED || KIND == WIDE;
    constexpr int NT = table_threads(KIND);
    extern __shared__ uint32_t tab[];
    // After k_mask_copy, which began once every earlier kernel had completed, the table is
    // built while that copy still runs; otherwise the history may be an earlier kernel's.
    if (!early) dep_wait();
    const int b = HASH ? blockIdx.x : blockIdx.x >> shares, share = blockIdx.x & ((1 << shares) - 1);
    const int places = HASH ? 0 : (V - share + (1 << shares) - 1) >> shares;
    const int len = !P.H ? 0 : P.history_len ? min(max(P.history_len[b], 0), P.H) : P.H;
    const int plen = P.prompt_len ? P.prompt_len[b] : 0;
    const int cap = HASH ? hash_cap(len) : places, shift = HASH ? __clz(cap) + 1 : 0;    // 32 - log2(cap)
    const int bias_cap = P.n_bias ? hash_cap(P.n_bias) : 0, bias_shift = P.n_bias ? __clz(bias_cap) + 1 : 0;
    uint32_t* bias_key = tab;
    uint32_t* bias_pos = bias_key + bias_cap;
    uint32_t* cnt = bias_pos + bias_cap;
    uint32_t* key = cnt + cap;                  // HASH only
    for (int i = threadIdx.x; i < bias_cap; i += NT) bias_key[i] = EMPTY, bias_pos[i] = 0;
    for (int i = threadIdx.x; i < (KIND == SHORT ? (cap + 1) / 2 : cap); i += NT) {
        cnt[i] = 0;
        if (HASH) key[i] = EMPTY;
    }
    // a place's count and prompt bit; and nothing left of it
    auto count_at = [&](int i) -> uint32_t {
        if (KIND != SHORT) return cnt[i];
        const uint32_t c = reinterpret_cast<const uint16_t*>(cnt)[i];
        return (c & 0x7fff) | (c >> 15 ? SEEN : 0u);
    };
    auto clear = [&](int i) {
        if (KIND == SHORT) reinterpret_cast<uint16_t*>(cnt)[i] = 0;
        else cnt[i] = 0;
    };
    __syncthreads();

    const int32_t* hist = P.history + (size_t)b * P.history_stride;
    for (int i0 = threadIdx.x; i0 < len; i0 += LOADS * NT) {
        int v[LOADS];
#pragma unroll
        for (int k = 0; k < LOADS; k++) v[k] = i0 + k * NT < len ? hist[i0 + k * NT] : -1;
#pragma unroll
        for (int k = 0; k < LOADS; k++) {
            uint32_t *word, one = 1, seen = SEEN;
            if (v[k] < 0 || v[k] >= V) continue;
            if (HASH) {
                word = &cnt[hash_slot(key, cap, shift, v[k])];
            } else {
                if ((v[k] & ((1 << shares) - 1)) != share) continue;
                const int place = v[k] >> shares;
                word = cnt + (KIND == SHORT ? place / 2 : place);
                if (KIND == SHORT) one = place & 1 ? 0x10000u : 1u, seen = one << 15;
            }
            if (i0 + k * NT < plen) atomicOr(word, seen);
            else atomicAdd(word, one);
        }
    }
    for (int j = threadIdx.x; j < P.n_bias; j += NT) {
        const int v = P.bias_ids[(size_t)b * P.n_bias + j];
        if (v < 0 || v >= V) continue;
        if (!HASH && (v & ((1 << shares) - 1)) != share) continue;
        atomicMax(&bias_pos[hash_slot(bias_key, bias_cap, bias_shift, v)], (uint32_t)j + 1);
    }
    __syncthreads();
    if (early) dep_wait();                      // the masked copy is complete
    dep_launch();

    const uint32_t* mask = bitmask ? bitmask + (size_t)b * W : nullptr;
    const T* src = logits + (size_t)b * stride;
    T* dst = out + (size_t)b * out_stride;
    const float rep = P.repetition ? P.repetition[b] : 1.f;
    const float freq = P.frequency ? P.frequency[b] : 0.f;
    const float pres = P.presence ? P.presence[b] : 0.f;
    // a thread's tokens are fetched together (logit and mask word at once), then rewritten
    constexpr int BATCH = 4;
    auto rewrite = [&](int from, int n, auto&& pick, int by = table_threads(KIND)) {
        for (int i0 = from; i0 < n; i0 += BATCH * by) {
            int v[BATCH];
            uint32_t c[BATCH], word[BATCH];
            float bias[BATCH], y[BATCH];
#pragma unroll
            for (int k = 0; k < BATCH; k++) {
                const int i = i0 + k * by;
                v[k] = -1;
                if (i < n) pick(i, &v[k], &c[k], &bias[k]);
            }
#pragma unroll
            for (int k = 0; k < BATCH; k++) {
                if (v[k] < 0) continue;
                y[k] = load_f32(src + v[k]);
                word[k] = mask ? mask[v[k] >> 5] : FULL;
            }
#pragma unroll
            for (int k = 0; k < BATCH; k++) {
                if (v[k] < 0 || !((word[k] >> (v[k] & 31)) & 1)) continue;
                float z = y[k];
                if (c[k]) z = z > 0.f ? z / rep : z * rep;
                if (c[k] & COUNT) z = z - freq * (float)(c[k] & COUNT) - pres;
                store_f32(dst + v[k], z + bias[k]);
            }
        }
    };
    // biased tokens, with what the history says of them; then the history's others
    if (P.n_bias) {
        rewrite(threadIdx.x, bias_cap, [&](int i, int* v, uint32_t* c, float* bias) {
            if (bias_key[i] == EMPTY) return;
            *v = (int)bias_key[i];
            const int s = HASH ? hash_find(key, cap, shift, *v) : *v >> shares;
            *c = s >= 0 ? count_at(s) : 0u;
            if (s >= 0) clear(s);
            *bias = P.bias[(size_t)b * P.n_bias + bias_pos[i] - 1];
        });
        __syncthreads();
    }
    auto named = [&](int i, int* v, uint32_t* c, float* bias) {
        *c = count_at(i);
        if (*c) *v = HASH ? (int)key[i] : i << shares | share;
        *bias = 0.f;
    };
    // of a direct table few words are named: a thread's next 32 as bits, then those
    if constexpr (HASH) rewrite(threadIdx.x, cap, named);
    else for (int i0 = 0; i0 < cap; i0 += 32 * NT) {
        uint32_t bits = 0;
#pragma unroll 8
        for (int k = 0; k < 32; k++) {
            const int i = i0 + k * NT + threadIdx.x;
            if (i < cap && count_at(i)) bits |= 1u << k;
        }
        while (bits) {
            int place[BATCH];
#pragma unroll
            for (int k = 0; k < BATCH; k++) {
                place[k] = bits ? i0 + (__ffs(bits) - 1) * NT + (int)threadIdx.x : -1;
                bits &= bits - 1;
            }
            rewrite(0, BATCH, [&](int k, int* v, uint32_t* c, float* bias) {
#pragma unroll
                for (int j = 0; j < BATCH; j++)
                    if (j == k && place[j] >= 0) named(place[j], v, c, bias);
            }, 1);
        }
    }
}

template <typename T>
psc_status process(const T* logits, int64_t stride, T* out, int64_t out_stride, int B, int V, const Penalties& P,
                   const uint32_t* bitmask, psc_dtype dtype, cudaStream_t cs) {
    const int W = (V + 31) / 32;
    psc_status s = PSC_OK;
    const int early = out != logits;
    if (out != logits) {
        const int vec = is_aligned(logits, stride * sizeof(T), 16) && is_aligned(out, out_stride * sizeof(T), 16);
        const long chunks = (long)B * ((V + 1023) / 1024);
        const int blocks = (int)std::min<long>((chunks + 7) / 8, (long)current_sms() * 4);
        s = ops_launch(k_mask_copy<T>, dim3(blocks), 256, 0, 1, cs, "k_mask_copy", logits, stride, out, out_stride, B,
                       V, bitmask, W, vec);
    } else if (bitmask) {
        s = psc_apply_mask(out, dtype, out_stride, bitmask, B, V, cs);
    }
    if (s != PSC_OK || (!P.H && !P.n_bias)) return s;
    const size_t bias_bytes = P.n_bias ? (size_t)hash_cap(P.n_bias) * 8 : 0;
    if (2 * P.H <= HASH_SLOTS) {
        const bool wide = B <= current_sms() || P.H >= WIDE_HISTORY;
        return ops_launch(wide ? k_penalize<T, WIDE> : k_penalize<T, HASHED>, dim3(B),
                          table_threads(wide ? WIDE : HASHED), bias_bytes + (size_t)hash_cap(P.H) * 8, 1, cs,
                          "k_penalize", logits, stride, out, out_stride, V, P, bitmask, W, 0, early);
    }
    const bool narrow = P.H <= SHORT_HISTORY;
    const int word = narrow ? 2 : 4;
    int shares = 0;
    while (((((int64_t)V - 1) >> shares) + 1) * word > TABLE_BYTES - (int64_t)bias_bytes / 2) shares++;
    return ops_launch(narrow ? k_penalize<T, SHORT> : k_penalize<T, LONG>, dim3((unsigned)B << shares),
                      table_threads(LONG), bias_bytes + (((V - 1) >> shares) + 2) / 2 * 2 * (size_t)word, 1, cs,
                      "k_penalize", logits, stride, out, out_stride, V, P, bitmask, W, shares, early);
}

}  // namespace

extern "C" psc_status psc_process_logits(const void* d_logits, psc_dtype dtype, int64_t row_stride, void* d_out,
                                         int64_t out_stride, int32_t B, int32_t V, const int32_t* d_history,
                                         int64_t history_stride, int32_t H, const int32_t* d_history_len,
                                         const int32_t* d_prompt_len, const float* d_repetition,
                                         const float* d_frequency, const float* d_presence, const int32_t* d_bias_ids,
                                         const float* d_bias, int32_t n_bias, const uint32_t* d_bitmask,
                                         void* stream) {
    const char* me = "psc_process_logits";
    if (B < 0 || V <= 0 || row_stride < V || out_stride < V || !is_dtype(dtype) || (B && (!d_logits || !d_out)))
        return ops_fail(PSC_ERR_ARG, me, "bad arguments");
    if (H < 0 || n_bias < 0 || (H && history_stride < H) ||
        (B && ((H && !d_history) || (n_bias && (!d_bias_ids || !d_bias)))))
        return ops_fail(PSC_ERR_ARG, me, "bad history or biases");
    if (V > MAX_V) return ops_fail(PSC_ERR_LIMIT, me, "vocabulary over 2^30 tokens");
    if (H > MAX_HISTORY) return ops_fail(PSC_ERR_LIMIT, me, "history over 16,777,215 tokens");
    if (n_bias > MAX_BIAS) return ops_fail(PSC_ERR_LIMIT, me, "more than 4,096 biases a row");
    if (B == 0) return PSC_OK;
    if ((int64_t)B * (V / 16384 + 1) > 0x7fffffff) return ops_fail(PSC_ERR_LIMIT, me, "batch too large");
    const size_t e = dtype == PSC_BF16 ? 2 : 4;
    if (d_logits == d_out) {
        if (row_stride != out_stride) return ops_fail(PSC_ERR_ARG, me, "in place with two row strides");
    } else {
        const uintptr_t a0 = (uintptr_t)d_logits, a1 = a0 + ((size_t)(B - 1) * row_stride + V) * e;
        const uintptr_t b0 = (uintptr_t)d_out, b1 = b0 + ((size_t)(B - 1) * out_stride + V) * e;
        // rows that alternate in one buffer are apart although their ranges are not
        const int64_t step = row_stride * (int64_t)e, off = ((int64_t)(b0 - a0) % step + step) % step;
        const bool apart = row_stride == out_stride && off >= V * (int64_t)e && step - off >= V * (int64_t)e;
        if (a0 < b1 && b0 < a1 && !apart) return ops_fail(PSC_ERR_ARG, me, "logits and out overlap");
    }
    const Penalties P{d_history,   history_stride, H,          d_history_len, d_prompt_len, d_repetition,
                      d_frequency, d_presence,     d_bias_ids, d_bias,        n_bias};
    cudaStream_t cs = (cudaStream_t)stream;
    if (dtype == PSC_BF16)
        return process((const __nv_bfloat16*)d_logits, row_stride, (__nv_bfloat16*)d_out, out_stride, B, V, P,
                       d_bitmask, dtype, cs);
    return process((const float*)d_logits, row_stride, (float*)d_out, out_stride, B, V, P, d_bitmask, dtype, cs);
}
