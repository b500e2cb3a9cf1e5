// Layout and numbers of the cache held in 4 bits (tbn_kv4_pages.hip, tbn_kv4_attention.hip); what they mean: include/tbn.h.
#pragma once
#include <type_traits>

#include "tbn_kv.h"

namespace tbn {

constexpr int8_t kNoNumber = -128;   // exponent of a key and value that are not numbers

inline int exponent_bytes(int dim) { return dim <= 128 ? 4 : 8; }   // of a key of one head

// calls f with dim / 32 as a constant
template <typename F>
inline void kv4_by_groups(int dim, F f) {
    switch (dim / 32) {
        case 1: return f(std::integral_constant<int, 1>());
        case 2: return f(std::integral_constant<int, 2>());
        case 3: return f(std::integral_constant<int, 3>());
        case 4: return f(std::integral_constant<int, 4>());
        case 5: return f(std::integral_constant<int, 5>());
        case 6: return f(std::integral_constant<int, 6>());
        case 7: return f(std::integral_constant<int, 7>());
        default: return f(std::integral_constant<int, 8>());
    }
}

#if defined(__HIPCC__)

// Least x with a <= 6 * 2^x, -100 .. 125.  6 * 2^x is 1.5 * 2^(x + 2).
__device__ __forceinline__ int kv4_exponent(float a) {
    const uint32_t u = __float_as_uint(a);
    return min(max(static_cast<int>(u >> 23) - 129 + ((u & 0x7fffffu) > 0x400000u ? 1 : 0), -100), 125);
}

// 2^x of the byte x of a word of exponents, as the conversions take it: they look at the exponent alone, and all ones (of kNoNumber) give not-a-number
template <typename W>
__device__ __forceinline__ float kv4_scale(W exps, int byte) {
    const int x = static_cast<int8_t>(exps >> (8 * byte));
    return __uint_as_float(static_cast<uint32_t>(x + 127) << 23);
}

// eight codes to bfloat16, times the scale: exact
typedef __bf16 kv4_pair_t __attribute__((ext_vector_type(2)));
typedef uint32_t kv4_eight_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ kv4_eight_t kv4_values(uint32_t codes, float scale) {
    return kv4_eight_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                       __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                       __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                       __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
}

// eight numbers to codes: divided by the scale, rounded to nearest even, at most 6 in magnitude, the sign kept
__device__ __forceinline__ uint32_t kv4_codes(const float (&f)[8], float scale) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[0], f[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[2], f[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[4], f[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[6], f[7], scale, 3);
}

// the low halves of eight bytes, as one word (high halves may hold anything: nobody wrote bytes of keys that are not there)
__device__ __forceinline__ uint32_t kv4_pack(uint2 bytes) {
    bytes.x &= 0x0f0f0f0fu;
    bytes.y &= 0x0f0f0f0fu;
    const uint32_t a = bytes.x | bytes.x >> 4, b = bytes.y | bytes.y >> 4;
    return __builtin_amdgcn_perm(b, a, 0x06040200u);
}

// word of values: octet of keys `g` of a block of 32, channel d; NF = dim / 16
__device__ __forceinline__ int kv4_value_word(int g, int d, int NF) { return (g * 16 + (d & 15)) * NF + (d >> 4); }

#endif
}  // namespace tbn
