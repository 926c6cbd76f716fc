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

constexpr int MAX_BIAS = 4096;
constexpr int MAX_HISTORY = (1 << 24) - 1;      // a count fits 24 bits
constexpr uint32_t SEEN = 1u << 30;             // the token is in the prompt
constexpr uint32_t COUNT = (1u << 24) - 1;      // times in the output
constexpr uint32_t EMPTY = 0xffffffffu;

constexpr int HASH_SLOTS = 16384;               // most slots of a hashed table
constexpr int PART = 16384;                     // tokens of the vocabulary per direct table

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
__global__ void __launch_bounds__(256) k_mask_copy(const T* logits, int64_t stride, T* out, int64_t out_stride, int B,
                                                   int V, const uint32_t* bitmask, int W, int vec) {
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
// token with at least twice as many slots as entries.  Otherwise a block per row
// and PART tokens of the vocabulary, a table indexed by token: any history length.
// Each table word holds the output count and the prompt bit; a second table the
// last position among the biases, so that the order of threads does not matter.
template <typename T, bool HASH>
__global__ void __launch_bounds__(512) k_penalize(const T* logits, int64_t stride, T* out, int64_t out_stride, int V,
                                                  Penalties P, const uint32_t* bitmask, int W, int parts, int early) {
    extern __shared__ uint32_t tab[];
    // After k_mask_copy, which began once every earlier kernel had completed, the table is
    // built while that copy still runs; otherwise the history may be an earlier kernel's.
    if (!early) dep_wait();
    const int b = blockIdx.x / parts, v0 = (blockIdx.x - b * parts) * PART;
    const int n_tok = HASH ? V : min(PART, V - v0);
    const int len = !P.H ? 0 : P.history_len ? min(max(P.history_len[b], 0), P.H) : P.H;
    const int plen = P.prompt_len ? P.prompt_len[b] : 0;
    int cap = n_tok, shift = 0;
    if (HASH) {
        const int need = 2 * (len + P.n_bias);
        cap = 32;
        while (cap < need) cap <<= 1;
        shift = __clz(cap) + 1;                 // 32 - log2(cap)
    }
    uint32_t* cnt = tab;
    uint32_t* pos = tab + cap;                  // used with biases only
    uint32_t* key = HASH ? pos + (P.n_bias ? cap : 0) : nullptr;
    for (int i = threadIdx.x; i < cap; i += blockDim.x) {
        cnt[i] = 0;
        if (P.n_bias) pos[i] = 0;
        if (HASH) key[i] = EMPTY;
    }
    __syncthreads();

    auto slot_of = [&](uint32_t v) -> int {
        if (!HASH) return (int)v - v0;
        uint32_t i = (v * 2654435761u) >> shift;
        for (int it = 0; it < cap; it++) {
            const uint32_t k = atomicCAS(&key[i], EMPTY, v);
            if (k == EMPTY || k == v) break;
            i = (i + 1) & (cap - 1);
        }
        return (int)i;
    };
    const int32_t* hist = P.history + (size_t)b * P.history_stride;
    for (int i = threadIdx.x; i < len; i += blockDim.x) {
        const int v = hist[i];
        if (v < v0 || v >= v0 + n_tok) continue;
        const int s = slot_of(v);
        if (i < plen) atomicOr(&cnt[s], SEEN);
        else atomicAdd(&cnt[s], 1u);
    }
    for (int j = threadIdx.x; j < P.n_bias; j += blockDim.x) {
        const int v = P.bias_ids[(size_t)b * P.n_bias + j];
        if (v < v0 || v >= v0 + n_tok) continue;
        atomicMax(&pos[slot_of(v)], (uint32_t)j + 1);
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
    for (int i = threadIdx.x; i < cap; i += blockDim.x) {
        const uint32_t c = cnt[i], j = P.n_bias ? pos[i] : 0u;
        if (!c && !j) continue;
        const int v = HASH ? (int)key[i] : v0 + i;
        if (!allows(mask, v)) continue;
        float y = load_f32(src + v);
        if (c) y = y > 0.f ? y / rep : y * rep;
        if (c & COUNT) y = y - freq * (float)(c & COUNT) - pres;
        if (j) y += P.bias[(size_t)b * P.n_bias + j - 1];
        store_f32(dst + v, y);
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
        const int blocks = (int)std::min<long>((chunks + 7) / 8, (long)current_sms() * 8);
        s = ops_launch(k_mask_copy<T>, dim3(blocks), 256, 0, 1, cs, "k_mask_copy", logits, stride, out, out_stride, B,
                       V, bitmask, W, vec);
    } else if (bitmask) {
        s = psc_apply_mask(out, dtype, out_stride, bitmask, B, V, cs);
    }
    if (s != PSC_OK || (!P.H && !P.n_bias)) return s;
    const int words = P.n_bias ? 2 : 1;
    const int64_t entries = (int64_t)P.H + P.n_bias;
    if (2 * entries <= HASH_SLOTS) {
        int cap = 32;
        while (cap < 2 * entries) cap <<= 1;
        return ops_launch(k_penalize<T, true>, dim3(B), 512, (size_t)cap * (words + 1) * 4, 1, cs, "k_penalize", logits,
                          stride, out, out_stride, V, P, bitmask, W, 1, early);
    }
    const int parts = (V + PART - 1) / PART;
    return ops_launch(k_penalize<T, false>, dim3(B * parts), 512, (size_t)std::min(V, PART) * words * 4, 1, cs,
                      "k_penalize", logits, stride, out, out_stride, V, P, bitmask, W, parts,
                      early);
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
    if (H > MAX_HISTORY) return ops_fail(PSC_ERR_LIMIT, me, "history over 16,777,215 tokens");
    if (n_bias > MAX_BIAS) return ops_fail(PSC_ERR_LIMIT, me, "more than 4,096 biases a row");
    if (B == 0) return PSC_OK;
    if ((int64_t)B * ((V + PART - 1) / PART) > 0x7fffffff) return ops_fail(PSC_ERR_LIMIT, me, "batch too large");
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
