// Elements and scales of the key/value caches: bf16, or 8 and 4 bits with a power of two per 32 elements.
#pragma once

#include "moe_internal.h"

namespace moe {

constexpr int kScaleBlock = 32;                              // elements that share a scale

template <int KIND> struct CacheKind;
template <> struct CacheKind<MOE_CACHE_BF16> { static constexpr int bits = 16; };
template <> struct CacheKind<MOE_CACHE_FP8> { static constexpr int bits = 8; };
template <> struct CacheKind<MOE_CACHE_FP4> { static constexpr int bits = 4; };

typedef __bf16 bf16x2_vec __attribute__((ext_vector_type(2)));

// 2^(byte - 127); byte 255 is an infinity, with which the converters below give NaN for every element
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte << 23); }

// Two elements of 8 bits, the lower or the upper half of w, as bf16: exact, the scale is applied by the converter
template <bool UPPER> __device__ __forceinline__ uint32_t fp8_pair(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, UPPER));
}
// Two elements of 4 bits, byte B of w
template <int B> __device__ __forceinline__ uint32_t fp4_pair(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
}

// The scale byte of a block whose largest magnitude has the bf16 bits `top`: the smallest exponent e >= -100 with
// top <= 448 2^e = 1.75 2^(e + 8), or 6 2^e = 1.5 2^(e + 2), where top is at most kLargest; 255 for a block with an infinity or NaN.  From 2^-100 on,
// whatever is stored is a normal bf16 number, and what is too small for bf16's normal numbers rounds to 0.
// (kLargest, bf16 bits of 1.75 2^127 and 1.5 2^127: beyond it a value could round to 2^128)
template <int KIND> constexpr uint32_t kLargest = KIND == MOE_CACHE_FP8 ? 0x7f60 : 0x7f40;
template <int KIND> __device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    if (top >= 0x7f80u) return 255;
    constexpr int power = KIND == MOE_CACHE_FP8 ? 8 : 2;
    constexpr uint32_t most = KIND == MOE_CACHE_FP8 ? 0x60 : 0x40;     // mantissa bits of 1.75 and 1.5
    const int e = (int)(top >> 7) - 127 - power + ((top & 0x7fu) > most ? 1 : 0);
    return (uint32_t)(max(e, -100) + 127);
}

}  // namespace moe
