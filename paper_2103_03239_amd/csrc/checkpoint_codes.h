// The 8-bit form of a saved activation row, for gfx950.  32 consecutive elements of a row (fewer at its end)
// share a power of two, 2^e: e is the smallest whole number from -126 to 121 with which every code
//   q = x / 2^e, rounded to the nearest whole number, ties to even,
// lies within -127 .. 127.  The scale byte is e + 127.  Elements that reach 127.5 * 2^121 (3.39e38, the largest finite ones) get
// the code +-127 of e = 121: a rounded one would stand for 2^128, an infinity.  A group that holds an infinity or a NaN has the
// scale byte 255 and restores as NaN throughout, so that an overflow is not lost.
//
// A power of two and not the largest element / 127: x / 2^e is exact, so a code is the same whoever computes it,
// and q * 2^e is exact in bfloat16 (7 bits of q, 8 of a significand), so the matrix instructions take it as it
// is.  The price is a step of up to twice the finest one: the largest code is 64 .. 127.
#pragma once

#include "row_elems.h"

namespace moshpit {

constexpr uint32_t kScaleNaN = 255, kScaleTop = 121 + 127;

// The scale byte of a group from the largest of its elements' bits without their signs.
__device__ __forceinline__ uint32_t scale_byte(uint32_t most)
{
    if (most >= 0x7f800000u) return kScaleNaN;
    // 64 .. 127.5 - 2^-18 times 2^e is within 127 after rounding; from 127.5 on (a significand of 255 / 128 or more) it is not
    const int e = static_cast<int>(most >> 23) - 127 - 6 + ((most & 0x7fffffu) >= 0x7f0000u ? 1 : 0);
    return static_cast<uint32_t>((e < -126 ? -126 : e > 121 ? 121 : e) + 127);
}

// 2^-e and 2^e of a scale byte, 1 .. kScaleTop; NaN for 255
__device__ __forceinline__ float to_code_factor(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
__device__ __forceinline__ float to_value_factor(uint32_t byte)
{
    return __uint_as_float(byte == kScaleNaN ? 0x7fc00000u : byte << 23);
}

// Four codes in the bytes of a word, lowest first.  Adding 1.5 * 2^23 rounds to whole numbers, ties to even, and leaves the
// code, as a signed byte, in the sum's lowest bits.
__device__ __forceinline__ uint32_t pack_codes(const float *x, float factor)
{
    uint32_t u[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) u[k] = __float_as_uint(fmaf(x[k], factor, 12582912.f));
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(u[3], u[2], 0x00000400), __builtin_amdgcn_perm(u[1], u[0], 0x00000400), 0x05040100);
}

// Elements of a group with the scale byte kScaleTop, kept from rounding to 128.
template <int C> __device__ __forceinline__ void keep_finite(float (&x)[C])
{
    const float most = __uint_as_float(0x7f7e0000u);                 // 127 * 2^121
#pragma unroll
    for (int k = 0; k < C; ++k) x[k] = fminf(fmaxf(x[k], -most), most);
}

__device__ __forceinline__ float code_of(uint32_t w, int k) { return static_cast<float>(static_cast<int>(w << (24 - 8 * k)) >> 24); }

}  // namespace moshpit
