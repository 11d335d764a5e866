// Cache rows of 4-bit blocks (S3_MXFP4) on gfx950: the open microscaling format of e2m1 codes (1 sign, 2 exponent bits with
// bias 1, 1 fraction bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6) in blocks of 32 consecutive elements of a head under one power of two,
// 2^(byte - 127).  In the arena a row's codes ([H][D/2] bytes, element 2i in the low half of byte i) and its scales ([H][D/32]
// bytes, zeros up to a multiple of 16) lie in planes of their own: with both in one row, rows began anywhere in a cache line, every head's
// wave fetched the line of the row's scales for itself, and half of what was fetched was not used.
//
// Rounding a block: the scale is the least power of two under which the largest magnitude is below 7, where the nearest code
// is 6 at the most, so no element is off by more than half the distance between its neighbours (the next value would be 8).
// It is at most 2^125, for 16-bit floats 2^13, so that every code stands for a finite number of the type of the new rows.
// Codes are the nearest, ties to even.  A block with an infinity or a NaN has scale byte 255 and reads as NaN.
#pragma once
#include "s3kv_device.h"

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

__host__ __device__ __forceinline__ int fp4_code_bytes(int heads, int d) { return heads * (d / 2); }
__host__ __device__ __forceinline__ int fp4_scale_bytes(int heads, int d) { return (heads * (d / 32) + 15) & ~15; }

// Two numbers, rounded to bf16 by the conversion instruction (to the nearest, ties to even; NaN stays NaN).
__device__ __forceinline__ unsigned round_bf16x2(const float x0, const float x1) {
    const bf16x2 h = {(__bf16)x0, (__bf16)x1};
    return __builtin_bit_cast(unsigned, h);
}

// Scale byte of a block whose largest magnitude is `most`: its exponent, one more from 1.75 * 2^k up, less 2.
template <int ACT>
__device__ __forceinline__ unsigned fp4_scale_byte(const float most) {
    const unsigned bits = __builtin_bit_cast(unsigned, most);
    if (bits >= 0x7F800000u) return 255u;
    const int byte = (int)((bits + 0x200000u) >> 23) - 2;
    return (unsigned)min(max(byte, 1), ACT == S3_F16 ? 140 : 252);
}

// max(|x|, so far) that keeps infinities and NaN (as an infinity): magnitudes compare as their bits do.
__device__ __forceinline__ unsigned fp4_magnitude(const float x, const unsigned most) {
    return max(most, min(__builtin_bit_cast(unsigned, x) & 0x7FFFFFFFu, 0x7F800000u));
}

// Eight consecutive elements -> their codes in element order (v_cvt_scalef32_pk_fp4_f32 rounds to the nearest, ties to even,
// and takes what is beyond 6 as 6; a block that is not finite has zeros under its scale byte 255).
__device__ __forceinline__ unsigned fp4_codes8(const float (&x)[8], const unsigned byte) {
    const unsigned sb = byte << 23;
    const float scale = __builtin_bit_cast(float, sb);
    unsigned w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
    return byte == 255u ? 0u : w;
}

// Largest of a value over the lanes of groups of 2 or 4 neighbours.
template <int LANES>
__device__ __forceinline__ unsigned group_max(unsigned v) {
    v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));  // quad_perm [1,0,3,2]
    if (LANES >= 4) v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));  // quad_perm [2,3,0,1]
    return v;
}

// Eight 16-bit elements of type ACT -> fp32.
template <int ACT>
__device__ __forceinline__ void widen8(const u32x4 v, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const unsigned w = v[i];
        x[2 * i] = widen16<ACT>((unsigned short)(w & 0xFFFFu));
        x[2 * i + 1] = widen16<ACT>((unsigned short)(w >> 16));
    }
}

// The scale that v_cvt_scalef32_* take: they read its exponent only (byte 255 makes every value NaN, byte 0 is 2^-127).
__device__ __forceinline__ float fp4_scale(const unsigned byte) {
    const unsigned bits = byte << 23;
    return __builtin_bit_cast(float, bits);
}

// Codes 2*SEL and 2*SEL+1 of a word, widened exactly.
template <int SEL>
__device__ __forceinline__ bf16x2 fp4_widen2(const unsigned w, const float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL);
}
