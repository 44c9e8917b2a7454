// Device-side helpers of the operators around attention (rotary positions, layer norm, 8-bit checkpoints): eight bf16 channels
// a lane, sums and maxima over groups of lanes, and the 8-bit format.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/varlen_attn.h"
#include "va_device.h"

namespace va {

// ---- groups of lanes ------------------------------------------------------------------------------------------------
// Butterflies over aligned groups of G lanes, every lane ends with the same bits: within 16 lanes by DPP (a mirrored group adds
// what the other half holds, once the halves agree), over 32 and 64 by the row swaps of gfx950.  All lanes must be active.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}
constexpr int kDppSwap1 = 0xB1, kDppSwap2 = 0x4E, kDppHalfMirror = 0x141, kDppMirror = 0x140;

template <int G, typename Op>
__device__ __forceinline__ uint32_t lanes_reduce(uint32_t x, Op op) {
    static_assert(G == 8 || G == 16 || G == 32 || G == 64, "group of lanes");
    x = op(x, dpp<kDppSwap1>(x));
    x = op(x, dpp<kDppSwap2>(x));
    x = op(x, dpp<kDppHalfMirror>(x));
    if (G >= 16) x = op(x, dpp<kDppMirror>(x));
    if (G >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        x = op(r[0], r[1]);
    }
    if (G >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        x = op(r[0], r[1]);
    }
    return x;
}
template <int G>
__device__ __forceinline__ float lanes_sum(float x) {
    return __uint_as_float(lanes_reduce<G>(__float_as_uint(x), [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }));
}
// Sum of x over the wave's groups of G lanes, lane i of each: every group ends with the same bits.
template <int G>
__device__ __forceinline__ float groups_sum(float x) {
    if (G <= 8) x += __uint_as_float(dpp<0x128>(__float_as_uint(x)));  // rotated by 8 within 16 lanes
    if (G <= 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (G <= 32) x = xhalf_sum(x);
    return x;
}
template <int G>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
    return lanes_reduce<G>(x, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

// ---- eight channels of a row ----------------------------------------------------------------------------------------
// n > 0 of the eight exist; the others read as zero and are not written.  Eight are moved by one 16-byte access (8-byte, of codes),
// whatever their alignment: the memory system takes one at any address, and the type says so to the compiler.  The rows' shape:
//   RAGGED  the last run of a row may be shorter than eight, and is moved element by element
//   WIDE    every run has eight (n >= 8 or n <= 0)
//   STREAM  and they go past the caches, which will not hold them until they are used again.  For rows of whole 128-byte lines only: where
//           a line is written by two instructions it pays twice (rotary heads of 64 channels 426 -> 535 us).
enum RowMode { RAGGED, WIDE, STREAM };
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef u32x2 u32x2_any __attribute__((aligned(1)));
template <int MODE>
__device__ __forceinline__ u32x4 load8(const uint16_t* p, int n) {
    u32x4 w = {0, 0, 0, 0};
    if (MODE != RAGGED ? n > 0 : n >= 8) {
        w = MODE == STREAM ? __builtin_nontemporal_load((const u32x4_any*)p) : *(const u32x4_any*)p;
    } else if (MODE == RAGGED && n > 0) {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) w[e >> 1] |= (uint32_t)p[e] << (16 * (e & 1));
    }
    return w;
}
template <int MODE>
__device__ __forceinline__ void store8(uint16_t* p, const u32x4& w, int n) {
    if (MODE != RAGGED ? n > 0 : n >= 8) {
        if (MODE == STREAM) __builtin_nontemporal_store(w, (u32x4_any*)p);
        else *(u32x4_any*)p = w;
    } else if (MODE == RAGGED && n > 0) {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) p[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
    }
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ void to_float8(const u32x4& w, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
}
// Rounds to nearest even: the one rounding a result of these operators goes through on its way to bf16.
__device__ __forceinline__ u32x4 to_bf16x8(const float* x) {
    bf16x8 v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (__bf16)x[e];
    return __builtin_bit_cast(u32x4, v);
}

// Row `row` of [tokens, rows_per_token, channels] with a stride between tokens starts at this element.  A division only where the
// tokens do not lie side by side, in 32 bits where the rows' number allows: in 64 it is 100 instructions, on 8 channels a lane.
__device__ __forceinline__ int64_t strided_row(int64_t row, int64_t rows, int rows_per_token, int channels, int64_t stride) {
    if (stride == (int64_t)rows_per_token * channels) return row * channels;
    if (rows_per_token == 1) return row * stride;
    if (rows <= INT32_MAX) {
        const uint32_t r = (uint32_t)row, t = r / (uint32_t)rows_per_token;
        return t * stride + (int64_t)(r - t * (uint32_t)rows_per_token) * channels;
    }
    return row / rows_per_token * stride + row % rows_per_token * channels;
}

// ---- the 8-bit format -----------------------------------------------------------------------------------------------
// A block is up to 128 consecutive channels of a row.  scale = max(amax * fl(1 / M), 2^-126), M the largest code (127, or 448 in
// e4m3), code = the format's nearest to x * fl(1 / scale), ties to even; it stands for code * scale.  The floor keeps scale and its
// inverse ordinary numbers; a block that small is off by less than 2^-126.  A block that holds an infinity or a NaN gets scale
// NaN, so that all of it comes back as NaN instead of as numbers that nobody can tell from good ones.
// The bf16 values' magnitudes compare as integers: amax costs one packed 16-bit maximum per two channels and sees NaN.
constexpr int kAct8Block = VA_ACT8_BLOCK;
__device__ __forceinline__ float act8_most(int format) { return format == VA_ACT8_INT8 ? 1.f / 127.f : 1.f / 448.f; }

__device__ __forceinline__ uint32_t magnitude8(const u32x4& w) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    u16x2 m = __builtin_bit_cast(u16x2, w[0] & 0x7fff7fffu);
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
    return m[0] > m[1] ? m[0] : m[1];
}
// Largest magnitude (bf16 bits) of a block -> its scale.
__device__ __forceinline__ float act8_scale(uint32_t magnitude, int format) {
    const float s = fmaxf(__uint_as_float(magnitude << 16) * act8_most(format), 0x1p-126f);
    return magnitude >= 0x7f80u ? __uint_as_float(0x7fc00000u) : s;
}
__device__ __forceinline__ u32x2 act8_encode(const float* x, float scale, int format) {
#pragma clang fp contract(off)  // (the product with inv is rounded by itself: that is the format's definition)
    const float inv = 1.f / scale;
    u32x2 w = {0, 0};
    if (format == VA_ACT8_INT8) {
        // adding 1.5 * 2^23 rounds to an integer, to nearest even, and leaves it in the lowest bits
        uint32_t u[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = __float_as_uint(x[e] * inv + 0x1.8p23f);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            w[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(u[4 * i + 3], u[4 * i + 2], 0x0c0c0400),
                                         __builtin_amdgcn_perm(u[4 * i + 1], u[4 * i], 0x0c0c0400), 0x05040100);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int v = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * inv, x[4 * i + 1] * inv, 0, false);
            w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * inv, x[4 * i + 3] * inv, v, true);
        }
    }
    return w;
}
// code * scale - off (off = 0: with the one rounding that the format's value has).  The product is formed from the signed code, never
// from code + 128: 128 * scale is beyond fp32 where a block holds one of bf16's two largest numbers.
__device__ __forceinline__ void act8_decode(const u32x2& w, float scale, int format, float* x, float off = 0.f) {
    if (format == VA_ACT8_INT8) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = fmaf((float)(int8_t)(w[e >> 2] >> (8 * (e & 3))), scale, -off);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
            x[4 * i] = fmaf(lo[0], scale, -off); x[4 * i + 1] = fmaf(lo[1], scale, -off);
            x[4 * i + 2] = fmaf(hi[0], scale, -off); x[4 * i + 3] = fmaf(hi[1], scale, -off);
        }
    }
}
template <int MODE>
__device__ __forceinline__ u32x2 load_codes(const uint8_t* p, int n) {
    u32x2 w = {0, 0};
    if (MODE != RAGGED ? n > 0 : n >= 8) {
        w = MODE == STREAM ? __builtin_nontemporal_load((const u32x2_any*)p) : *(const u32x2_any*)p;
    } else if (MODE == RAGGED && n > 0) {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) w[e >> 2] |= (uint32_t)p[e] << (8 * (e & 3));
    }
    return w;
}
template <int MODE>
__device__ __forceinline__ void store_codes(uint8_t* p, const u32x2& w, int n) {
    if (MODE != RAGGED ? n > 0 : n >= 8) {
        if (MODE == STREAM) __builtin_nontemporal_store(w, (u32x2_any*)p);
        else *(u32x2_any*)p = w;
    } else if (MODE == RAGGED && n > 0) {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) p[e] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
    }
}

}  // namespace va
