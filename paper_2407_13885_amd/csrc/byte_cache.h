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

// A scale's byte as a number.  (Nothing here writes others than 10 to 246; from there on 448 times it would be no bf16 number.)
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(max(1u, min(byte, 127u + kMostScale)) << 23); }

// Of four elements, whether one is NaN: flags in the signs' places.
__device__ __forceinline__ uint32_t any_nan(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// The least e with |x| <= 448 2^e, x as the bits of a finite number without its sign.
__device__ __forceinline__ int exponent_for(uint32_t x)
{
    return max(kLeastScale, min((int)(x >> 23) - 127 - 8 + ((x & 0x7fffffu) > 0x600000u ? 1 : 0), kMostScale));
}

// Numbers in units of a power of 2, to nearest even; what is infinite or beyond 464 of them as NaN.
template <bool HIGH> __device__ __forceinline__ uint32_t pack_e4m3(float lo, float hi, uint32_t old, float scale)
{
#if defined(__HIP_DEVICE_COMPILE__)
    typedef short s16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(__builtin_bit_cast(s16x2, old), lo, hi, scale, HIGH));
#else
    (void)lo;
    (void)hi;
    (void)scale;
    return old;
#endif
}
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d, float scale) { return pack_e4m3<true>(c, d, pack_e4m3<false>(a, b, 0, scale), scale); }

// Four elements as bf16, times a power of 2; eight of them, the operand of a matrix instruction.
__device__ __forceinline__ u32x2 bf16_of(uint32_t w, float scale)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true))};
#else
    (void)w;
    (void)scale;
    return u32x2{0u, 0u};
#endif
}
__device__ __forceinline__ u32x4 bf16_of(uint32_t a, uint32_t b, float scale) { return u32x4_of(bf16_of(a, scale), bf16_of(b, scale)); }

// 8 numbers as bf16: as they are, or their three parts
template <int PARTS> struct Parts { u32x4 of[PARTS]; };
template <int PARTS> __device__ __forceinline__ Parts<PARTS> parts_of(const float (&y)[8])
{
    Parts<PARTS> r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a = y[2 * i], b = y[2 * i + 1];
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            const uint32_t w = pack_bf16x2(a, b);
            r.of[p][i] = w;
            a -= bf16_lo_to_f32(w);
            b -= bf16_hi_to_f32(w);
        }
    }
    return r;
}
// (the smallest part first)
template <int PARTS> __device__ __forceinline__ void multiply_parts(f32x4& acc, const u32x4& x, const Parts<PARTS>& y)
{
#pragma unroll
    for (int p = PARTS - 1; p >= 0; --p) mma16(acc, x, y.of[p]);
}

// Where the keys of a place of 2^grain lie, and the bytes of their scales in the upper 16 bits.
__device__ __forceinline__ int64_t slot_place(const CacheView& c, const ScalesView& s, const int32_t* pages_of, int kv_head, int j)
{
    const uint32_t p = quotient((uint32_t)j, c.page);
    const int32_t id = max(0, min(pages_of[p], c.pages - 1)), row = j - (int)(p * c.page.d);
    const int64_t scale = ((int64_t)id * c.kv_heads + kv_head) * s.per_page + quotient(row, s.block);
    const uint64_t at = (uint64_t)(uint32_t)id * c.page_bytes + (uint32_t)kv_head * c.head_bytes + (uint32_t)row * (uint32_t)c.row_bytes;
    return (int64_t)(at | (uint64_t)s.K[scale] << 48 | (uint64_t)s.V[scale] << 56);
}
__device__ __forceinline__ int64_t place_offset(int64_t place) { return place & (((int64_t)1 << 48) - 1); }
__device__ __forceinline__ float key_scale(uint32_t high) { return scale_of(high >> 16 & 255); }
__device__ __forceinline__ float value_scale(uint32_t high) { return scale_of(high >> 24); }
// 2^grain slots lie in one page and share their scales
inline int key_grain(const CacheView& c, const ScalesView& s)
{
    CacheView of = c;
    of.page = s.block;                            // (it divides the page)
    return key_grain(of);
}

}  // namespace
}  // namespace attnw
