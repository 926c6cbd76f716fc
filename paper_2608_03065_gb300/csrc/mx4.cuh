// The microscaled 4-bit format (psc_mx4.h) on the device: eight columns at a time in a thread,
// four neighbouring threads a block of 32 columns, sixteen a row's piece of a tile of exponents.
#pragma once

#include <type_traits>

#include "../../include/psc_mx4.h"
#include "ops_common.cuh"

namespace {

constexpr int MAX_QUANTIZE_K = 1 << 30;

// Eight neighbouring columns (a chunk) of a row go in and out by accesses of 16 or 32 bytes.  Where a row starts
// elsewhere than at a multiple of those, or does not end with a chunk, they still do (WIDE false), but
// for its ends: what is loaded at aligned addresses is shifted into place, and stores take over the end
// of the previous lane's chunk.  (Element by element: 16,384 rows of 4,095 bf16 columns through the
// norm into 8 bits 379 us; 16,384 x 4,096 at aligned addresses 111.)
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
}
// A chunk's words as values and back.
__device__ __forceinline__ void unpack8(const uint32_t (&w)[8], float v[8], const float*) {
#pragma unroll
    for (int j = 0; j < 8; j++) v[j] = __uint_as_float(w[j]);
}
__device__ __forceinline__ void unpack8(const uint32_t (&w)[4], float v[8], const __nv_bfloat16*) {
#pragma unroll
    for (int j = 0; j < 4; j++) {
        v[2 * j] = __uint_as_float(w[j] << 16);
        v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
}
__device__ __forceinline__ void pack8(const float v[8], uint32_t (&w)[8], const float*) {
#pragma unroll
    for (int j = 0; j < 8; j++) w[j] = __float_as_uint(v[j]);
}
__device__ __forceinline__ void pack8(const float v[8], uint32_t (&w)[4], const __nv_bfloat16*) {
#pragma unroll
    for (int j = 0; j < 4; j++) w[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
}
// A whole, aligned chunk: eight f32 are a sector of the L2, and go in one access (two of 16 bytes each write half of
// every sector: 151,936 x 1,024 f32 into 4 bits and back 241 us, 214 this way).
__device__ __forceinline__ void load_chunk(const float* from, uint32_t (&w)[8]) {
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(from));
}
__device__ __forceinline__ void load_chunk(const __nv_bfloat16* from, uint32_t (&w)[4]) {
    const uint4 x = *reinterpret_cast<const uint4*>(from);
    w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
}
__device__ __forceinline__ void store_chunk(float* to, const uint32_t (&w)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                 "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
}
__device__ __forceinline__ void store_chunk(__nv_bfloat16* to, const uint32_t (&w)[4]) {
    *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
}

// f(std::integral_constant) of a number from 0 to 3 (words' places have to be known to the compiler).
template <typename F>
__device__ __forceinline__ void with_place(int i, F f) {
    if (i == 0) f(std::integral_constant<int, 0>());
    else if (i == 1) f(std::integral_constant<int, 1>());
    else if (i == 2) f(std::integral_constant<int, 2>());
    else f(std::integral_constant<int, 3>());
}

// Columns k to k + 7 of a row, zeros past K.
template <bool WIDE, typename T>
__device__ __forceinline__ void load8(const T* row, int k, int K, float v[8]) {
    constexpr int N = sizeof(T) * 2;                    // words of a chunk
    const int off = WIDE ? 0 : (int)((uintptr_t)(row + k) & 15);
    const uint4* at = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(row + k) - off);
    uint32_t w[N];
    if (WIDE) {
        load_chunk(row + k, w);
    } else if (off == 0 && k + 8 <= K) {
#pragma unroll
        for (int i = 0; i < N / 4; i++) {
            const uint4 x = at[i];
            w[4 * i] = x.x, w[4 * i + 1] = x.y, w[4 * i + 2] = x.z, w[4 * i + 3] = x.w;
        }
    } else if ((const void*)at >= (const void*)row && (const void*)(at + N / 4 + 1) <= (const void*)(row + K)) {
        uint32_t x[N + 4];
#pragma unroll
        for (int i = 0; i <= N / 4; i++) {
            const uint4 y = at[i];
            x[4 * i] = y.x, x[4 * i + 1] = y.y, x[4 * i + 2] = y.z, x[4 * i + 3] = y.w;
        }
        with_place(off >> 2, [&](auto known) {
            constexpr int place = decltype(known)::value;
#pragma unroll
            for (int i = 0; i < N; i++)
                w[i] = sizeof(T) == 2 ? __funnelshift_r(x[i + place], x[i + place + 1], (off & 2) * 8) : x[i + place];
        });
    } else {
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] = k + j < K ? load_f32(row + k + j) : 0.f;
        return;
    }
    unpack8(w, v, (const T*)nullptr);
}

// A chunk of N words to `to`, of which the first `valid` elements (of ES bytes) are there, in pieces of 16 bytes.
// All lanes of a warp call it; follows: the lane's chunk lies behind the lane's before it.
template <int N, int ES>
__device__ __forceinline__ void store_shifted(uint8_t* to, const uint32_t (&w)[N], int valid, bool follows) {
    constexpr int ELEMENTS = 4 * N / ES, P = 4;
    const int lane = threadIdx.x & 31, off = (int)((uintptr_t)to & (4 * P - 1));
    const bool whole = valid >= ELEMENTS;
    const bool joins = __shfl_up_sync(FULL, whole, 1) && whole && follows && lane > 0;      // the lane before, to this one
    const bool joined = __shfl_down_sync(FULL, joins, 1) && lane < 31;
    uint32_t x[P + 1 + N];                              // the last words before the chunk (and one for shifts), the chunk
#pragma unroll
    for (int i = 0; i < P; i++) x[1 + i] = __shfl_up_sync(FULL, w[N - P + i], 1);
    x[0] = 0;
#pragma unroll
    for (int i = 0; i < N; i++) x[P + 1 + i] = w[i];
    auto element = [&](int e) {
        if (ES == 4) reinterpret_cast<uint32_t*>(to)[e] = w[e];
        else reinterpret_cast<uint16_t*>(to)[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
    };
    // the elements one by one: all of a partial chunk, else those in pieces that are not all this lane's to store
    const int head = off == 0 || joins ? 0 : (4 * P - off) / ES, tail = off == 0 || joined ? 0 : off / ES;
    if (!whole || head || tail)
#pragma unroll
        for (int e = 0; e < ELEMENTS; e++)
            if (whole ? e < head || e >= ELEMENTS - tail : e < valid) element(e);
    if (!whole) return;
    with_place(off >> 2, [&](auto known) {
        constexpr int from = P + 1 - decltype(known)::value;
#pragma unroll
        for (int q = 0; q < N / P; q++) {
            if (q == 0 && off != 0 && !joins) continue;
            uint32_t y[P];
#pragma unroll
            for (int i = 0; i < P; i++) {               // words from off / 4 before the chunk on, the bits in front from the word before
                y[i] = ES == 4 ? x[q * P + i + from] : __funnelshift_l(x[q * P + i + from - 1], x[q * P + i + from], (off & 3) * 8);
            }
            *reinterpret_cast<uint4*>(to - off + q * 4 * P) = make_uint4(y[0], y[1], y[2], y[3]);
        }
    });
}

// Columns k to k + 7 of a row, up to K.  WIDE false: all lanes of a warp call it, `there` or not.
template <bool WIDE, typename T>
__device__ __forceinline__ void store8(T* row, int k, int K, const float v[8], bool there, bool follows) {
    constexpr int N = sizeof(T) * 2;
    uint32_t w[N];
    pack8(v, w, (const T*)nullptr);
    if (WIDE) {
        if (there) store_chunk(row + k, w);
    } else {
        store_shifted<N, sizeof(T)>(reinterpret_cast<uint8_t*>(row + k), w, there ? min(8, K - k) : 0, follows);
    }
}
// Where rows start at no multiple of 16 bytes, but all that a chunk takes part in starts alike (tensors of one
// shape do), chunks may start there instead, at column 8 c - shift: all are then whole and aligned but a row's
// first and last.  These take any columns k to k + 7, of which some may lie outside of the row, `in_place`
// where the whole chunk is at an aligned address.
template <typename T>
__device__ __forceinline__ int row_shift(const T* row) {
    return (int)((uintptr_t)row / sizeof(T) & 7);
}
template <typename T>
__device__ __forceinline__ void load8_at(const T* row, int k, int K, bool in_place, float v[8]) {
    if (in_place && k >= 0 && k + 8 <= K) return load8<true>(row, k, K, v);
#pragma unroll
    for (int j = 0; j < 8; j++) v[j] = k + j >= 0 && k + j < K ? load_f32(row + k + j) : 0.f;
}
template <typename T>
__device__ __forceinline__ void store8_at(T* row, int k, int K, bool in_place, const float v[8]) {
    if (in_place && k >= 0 && k + 8 <= K) return store8<true>(row, k, K, v, true, false);
#pragma unroll
    for (int j = 0; j < 8; j++)
        if (k + j >= 0 && k + j < K) store_f32(row + k + j, v[j]);
}
// Whether rows of these elements (none at all, too) are whole chunks at multiples of a chunk's size.
template <typename T>
inline bool wide_rows(const void* p, int64_t stride, int K) {
    return !p || (K % 8 == 0 && is_aligned(p, stride * (int64_t)sizeof(T), 8 * sizeof(T)));
}

// The largest of |a|, |b| and |c|; NaN if one is.  As bit patterns magnitudes order as they do as numbers, with
// infinities and then NaN above all.
__device__ __forceinline__ float largest(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float largest8(const float v[8], float top) {
#pragma unroll
    for (int j = 0; j < 8; j += 2) top = largest(top, v[j], v[j + 1]);
    return top;
}
constexpr uint32_t INF_BITS = 0x7f800000u;

// Where the exponent of row r's block b is; n_tiles = ceil(K / 128).
__host__ __device__ __forceinline__ int64_t block_at(int r, int b, int n_tiles) {
    return 512 * ((int64_t)(r / 128) * n_tiles + b / 4) + 16 * (r % 32) + 4 * (r % 128 / 32) + b % 4;
}

// Of a block whose largest magnitude has these bits: the byte e + 127, and 2^-e.  The largest
// magnitude lies in [4, 8) 2^e (below where e is -127), so x 2^-e is exact and codes reach 4 or 6.
__device__ __forceinline__ uint32_t block_byte(uint32_t top) {
    return top >= INF_BITS ? 255u : (uint32_t)max((int)(top >> 23) - 2, 0);
}
__device__ __forceinline__ float block_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
// 2^e, NaN for a NaN block.
__device__ __forceinline__ float block_value(uint32_t byte) {
    return __uint_as_float(byte == 255 ? 0x7fc00000u : byte ? byte << 23 : 1u << 22);
}

// Eight values as codes, the first in the lowest bits (ties to even, 6 at most).
__device__ __forceinline__ uint32_t codes8(const float v[8], float inverse) {
    uint32_t out;
    asm("{\n .reg .b8 a, b, c, d;\n"
        " cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
        " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n"
        " mov.b32 %0, {a, b, c, d};\n}"
        : "=r"(out)
        : "f"(v[0] * inverse), "f"(v[1] * inverse), "f"(v[2] * inverse), "f"(v[3] * inverse), "f"(v[4] * inverse),
          "f"(v[5] * inverse), "f"(v[6] * inverse), "f"(v[7] * inverse));
    return out;
}

// A thread's eight columns from 8 c on of a row, to codes and exponents; `top` the largest magnitude of
// them.  All 32 lanes of a warp call it for neighbouring chunks c (or 16 of one row and 16 of another), lane
// 0's a multiple of 16; what lies past the row's last tile stores nothing.  row_blocks: where the row's first
// block's exponent is.  INSIDE: all chunks lie in the row, which is whole tiles.  Returns whether the block is NaN.
template <bool INSIDE = false>
__device__ __forceinline__ bool quantize8(const float v[8], float top, int c, int K, uint8_t* q_row,
                                          uint8_t* row_blocks) {
    const int lane = threadIdx.x & 31;
    uint32_t bits = __float_as_uint(top) & 0x7fffffffu;
    bits = max(bits, __shfl_xor_sync(FULL, bits, 1));
    bits = max(bits, __shfl_xor_sync(FULL, bits, 2));
    const uint32_t byte = block_byte(bits);
    if (INSIDE || c < (K + 31) / 32 * 4)
        *reinterpret_cast<uint32_t*>(q_row + c * 4) = byte == 255 ? 0u : codes8(v, block_inverse(byte));
    // the four blocks of a tile's row, by one of its sixteen lanes
    uint32_t word = byte << (8 * ((lane >> 2) & 3));
    word |= __shfl_xor_sync(FULL, word, 4);
    word |= __shfl_xor_sync(FULL, word, 8);
    if (!(lane & 15) && (INSIDE || c < (K + 127) / 128 * 16)) *reinterpret_cast<uint32_t*>(row_blocks + (int64_t)c * 32) = word;
    return byte == 255;
}
inline bool is_mx4(const void* q, int64_t stride, const void* blocks, int K) {
    return is_aligned(q, stride, 16) && (uintptr_t)blocks % 16 == 0 && stride >= ((int64_t)K + 31) / 32 * 16;
}

}  // namespace
