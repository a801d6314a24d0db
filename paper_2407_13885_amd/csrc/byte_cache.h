// Shared by the kernels of a paged cache that holds a byte an element.
//
// An element is an e4m3 number (3 bits of mantissa, 448 at most, no infinities, 0x7f and 0xff NaN) times a power of 2 that the slots of a block share, for a kv head, keys
// and values apart.  Powers of 2: bf16 holds every element exactly, so that attention multiplies what is cached without rounding it again, and a
// block whose scale grows while it fills has its older rows moved down by whole binades, which changes only what becomes smaller than 2^-6 of the scale.
#pragma once

#include "paged_common.h"

namespace attnw {
namespace {

constexpr int kLeastScale = -117, kMostScale = 119;   // exponents: 2^-9 of the least scale and 448 of the greatest are normal fp32 numbers

// A scale's byte as a number (255, which nothing here writes, as 254)
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(min(byte, 254u) << 23); }

// The least e with |x| <= 448 2^e, x as the bits of a finite number without its sign.
__device__ __forceinline__ int exponent_for(uint32_t x)
{
    return max(kLeastScale, min((int)(x >> 23) - 127 - 8 + ((x & 0x7fffffu) > 0x600000u ? 1 : 0), kMostScale));
}

// To nearest even; numbers beyond 448 (where the scale is the greatest there is) as 448, infinities as NaN.
__device__ __forceinline__ float in_reach(float x)
{
    return (__float_as_uint(x) & 0x7fffffffu) < 0x7f800000u ? __builtin_amdgcn_fmed3f(x, -448.0f, 448.0f) : __builtin_nanf("");
}
template <bool HIGH> __device__ __forceinline__ uint32_t pack_e4m3(float lo, float hi, uint32_t old)
{
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(in_reach(lo), in_reach(hi), (int)old, HIGH);
}
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) { return pack_e4m3<true>(c, d, pack_e4m3<false>(a, b, 0)); }

}  // namespace
}  // namespace attnw
