// Rows of the paged cache as the pages hold them: bf16, or 8-bit codes with a power of two per row.
//
// A row x of D values (one token, one KV head) is held as codes c and a byte e + 127,
//   e = the least integer with max|x| <= M 2^e,   c = x / 2^e to nearest, ties to even,
// on the grid of the kind: e4m3 (M = 448) or whole numbers (M = 127).  The power of two makes every step
// exact but the one rounding: x / 2^e has x's digits, and c 2^e, at most 4 or 7 significant bits, is a bf16,
// so attention over 8-bit pages does the arithmetic of attention over bf16 pages that hold the same values.
// e4m3 loses nothing to it (a float's relative step does not depend on the scale); whole numbers lose up to
// one bit of eight against a scale of max|x| / 127 and are still the finer kind for rows without outliers.
// e is at least -100, so no value a code stands for is below the normal range.  A row with an infinity or
// a NaN has the byte 255 and codes 0: 0 times 2^128 = inf reads as NaN, and only where the row is read.
#pragma once

#include "tgvkv_device.h"
#include "tgvkv_shape.h"

namespace tgvkv {

constexpr int kCacheBf16 = 0, kCacheFp8 = 1, kCacheInt8 = 2;
constexpr int kMinExpByte = 27;  // e = -100

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Bytes of one element in the pages.
constexpr int code_bytes(int kind) { return kind == kCacheBf16 ? 2 : 1; }

// The row's exponent byte from the largest |x| as 15 bits of bf16 (the exponent field is biased by 127 too):
// 448 = 1.75 2^8 and 127 = 1.984375 2^6, and the added constant carries where the mantissa is above that.
template <int KIND>
__device__ __forceinline__ uint32_t exp_byte(uint32_t amax_bits) {
    static_assert(KIND == kCacheFp8 || KIND == kCacheInt8, "8-bit kinds");
    const int e = KIND == kCacheFp8 ? (int)((amax_bits + 31u) >> 7) - 8 : (int)((amax_bits + 1u) >> 7) - 6;
    return amax_bits >= 0x7F80u ? 255u : (uint32_t)max(e, kMinExpByte);
}

// 2^e of an exponent byte (255: inf), and 2^-e.
__device__ __forceinline__ float exp_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ float exp_inverse(uint32_t byte) { return __uint_as_float((254u - min(byte, 254u)) << 23); }

// The larger |x| of 8 bf16, as 15 bits.
__device__ __forceinline__ uint32_t amax8(u32x4 r) {
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) a = max(a, max(r[i] & 0x7FFFu, (r[i] >> 16) & 0x7FFFu));
    return a;
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_read_u32(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xF, 0xF, true);
}

// Maximum over each aligned group of W = 8 or 16 lanes, as group_sum.
template <int W>
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
    static_assert(W == 8 || W == 16, "group width");
    x = max(x, dpp_read_u32<0xB1>(x));
    x = max(x, dpp_read_u32<0x4E>(x));
    x = max(x, dpp_read_u32<0x141>(x));
    if (W == 16) x = max(x, dpp_read_u32<0x140>(x));
    return x;
}

// 8 bf16 of a row as 8 codes, given the row's exponent byte.
template <int KIND>
__device__ __forceinline__ u32x2 encode8(u32x4 r, uint32_t byte) {
    const float inv = byte == 255u ? 0.f : exp_inverse(byte);
    float y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // a row with non-finite values has codes 0 (inf * 0 would be a NaN)
        y[2 * i] = byte == 255u ? 0.f : __uint_as_float(r[i] << 16) * inv;
        y[2 * i + 1] = byte == 255u ? 0.f : __uint_as_float(r[i] & 0xFFFF0000u) * inv;
    }
    u32x2 c;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (KIND == kCacheFp8) {
            int w = 0;
            w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], w, false);
            w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], w, true);
            c[i] = (uint32_t)w;
        } else {
            uint32_t w = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) w |= ((uint32_t)(int)__builtin_rintf(y[4 * i + j]) & 0xFFu) << (8 * j);
            c[i] = w;
        }
    }
    return c;
}

// 4 codes (one register) as 4 bf16 in two registers, without the row's power of two: exact.
template <int KIND>
__device__ __forceinline__ u32x2 decode4(uint32_t w) {
    if constexpr (KIND == kCacheFp8) {
        return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true))};
    } else {
        float f[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = (float)(int8_t)(w >> (8 * j));
        // the upper halves of two floats that are bf16 already
        return u32x2{__builtin_amdgcn_perm(__float_as_uint(f[1]), __float_as_uint(f[0]), 0x07060302u),
                     __builtin_amdgcn_perm(__float_as_uint(f[3]), __float_as_uint(f[2]), 0x07060302u)};
    }
}

// 8 codes as 8 bf16, without the row's power of two.
template <int KIND>
__device__ __forceinline__ u32x4 decode8(u32x2 c) {
    const u32x2 a = decode4<KIND>(c[0]), b = decode4<KIND>(c[1]);
    return u32x4{a[0], a[1], b[0], b[1]};
}

// 8 codes as the 8 bf16 that they stand for, s = 2^e of their row: exact.  (Byte 255: s is inf and the values NaN, by
// 0 * inf, or by the conversion's own rule for that exponent.)
template <int KIND>
__device__ __forceinline__ u32x4 values8(u32x2 c, float s) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if constexpr (KIND == kCacheFp8) {
            r[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[i], s, false));
            r[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[i], s, true));
        } else {
            float f[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = (float)(int8_t)(c[i] >> (8 * j)) * s;
            r[2 * i] = __builtin_amdgcn_perm(__float_as_uint(f[1]), __float_as_uint(f[0]), 0x07060302u);
            r[2 * i + 1] = __builtin_amdgcn_perm(__float_as_uint(f[3]), __float_as_uint(f[2]), 0x07060302u);
        }
    }
    return r;
}

// Row `n` of segment bl: the pool's row index of KV head kvh (an id outside the pool is clamped into it).
__device__ __forceinline__ size_t pool_row(const Pages& pg, int hkv, int kvh, int page, int n) {
    const size_t p = (size_t)min(max(page, 0), pg.n_pages - 1);
    return ((p * hkv + kvh) << pg.shift) | (size_t)(n & ((1 << pg.shift) - 1));
}
__device__ __forceinline__ int table_page(const Pages& pg, int bl, int n) {
    return pg.table[(size_t)bl * pg.max_pages + min(n >> pg.shift, pg.max_pages - 1)];
}

// Rows of a segment's pages: the first pool row of every page of rows [n0, n1), in LDS.  A pool's rows are
// numbered in 32 bits (2^32 of the smallest rows, in two pools, are more memory than the GPU has).
struct PageRows {
    const uint32_t* base;
    int p0, shift;
    template <int THREADS>
    __device__ __forceinline__ void init(const Shape& s, const Pages& pg, int bl, int kvh, int n0, int n1, uint32_t* lds) {
        shift = pg.shift;
        p0 = n0 >> shift;
        base = lds;
        const int p1 = n1 > n0 ? ((n1 - 1) >> shift) + 1 : p0;
        for (int i = p0 + (int)threadIdx.x; i < p1; i += THREADS)
            lds[i - p0] = (uint32_t)pool_row(pg, s.Hkv, kvh, pg.table[(size_t)bl * pg.max_pages + i], 0);
    }
    // row() of a row that is the same in every lane of the wave, as a scalar.
    __device__ __forceinline__ size_t uniform_row(int n) const {
        return (uint32_t)__builtin_amdgcn_readfirstlane((int)base[(n >> shift) - p0]) + (uint32_t)(n & ((1 << shift) - 1));
    }
    __device__ __forceinline__ size_t row(int n) const { return base[(n >> shift) - p0] + (uint32_t)(n & ((1 << shift) - 1)); }
};

inline size_t lds_pages_bytes(const Pages& pg) { return sizeof(uint32_t) * (size_t)pg.max_pages; }

}  // namespace tgvkv
