// What the kernels of the 4-bit cache share: its layout, and a row's values as fp16.
//
//   codes  [B * Hkv][T][d / 2]         byte j: channel 2j (low half), 2j + 1 (high half)
//   params [B * Hkv][d / group][T][2]  fp16 scale s, minimum m
//   value  = fp16(s * code + m)
#pragma once
#include "csr_internal.h"

namespace csr {
namespace q4 {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

__device__ __forceinline__ half2v as_half2(uint32_t v) { return __builtin_bit_cast(half2v, v); }
__device__ __forceinline__ uint32_t as_u32(half2v v) { return __builtin_bit_cast(uint32_t, v); }
__device__ __forceinline__ half2v fma2(half2v a, half2v b, half2v c) { return __builtin_elementwise_fma(a, b, c); }
__device__ __forceinline__ half2v splat2(float v) { return half2v{(_Float16)v, (_Float16)v}; }

// (v & mask) | bits in one instruction: the mask in a scalar register, the bits in a vector one.  The compiler makes two of it,
// with a literal each.
__device__ __forceinline__ uint32_t and_or(uint32_t v, uint32_t mask, uint32_t bits)
{
    uint32_t r;
    asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(r) : "v"(v), "s"(mask), "v"(bits));
    return r;
}

// Nibbles K and K + 4 of w as fp16 whole numbers.  A nibble in the lowest bits of an fp16 with the exponent of 1024 reads as
// 1024 + code, four bits higher as 1024 + 16 code; either way one packed operation leaves the code, exactly.
template <int K> __device__ __forceinline__ half2v nibble_pair(uint32_t w)
{
    const uint32_t v = K >= 2 ? w >> 8 : w;
    if constexpr (K % 2 == 0)
        return as_half2(and_or(v, 0x000f000fu, 0x64006400u)) - splat2(1024.0f);
    else
        return fma2(as_half2(and_or(v, 0x00f000f0u, 0x64006400u)), splat2(0.0625f), splat2(-64.0f));
}

// The low (high) halves of two words side by side
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// Whether the scale or the minimum of a parameter word is no finite number
__device__ __forceinline__ bool not_finite(uint32_t sm)
{
    return (sm & 0x7c00u) == 0x7c00u || (sm & 0x7c000000u) == 0x7c000000u;
}

__device__ __forceinline__ uint16_t float_to_bf16(float f)   // to nearest, halves to even; a NaN stays one
{
    const uint32_t u = __float_as_uint(f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return (uint16_t)((u >> 16) | 0x40u);
    return (uint16_t)((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}

// Unsigned division by a number that the host knows: x / d = (x * mul) >> (32 + shift) for x below 2^31
struct FastDiv {
    uint32_t mul, shift, div;
};
inline FastDiv fast_div(uint32_t d)
{
    FastDiv f{0, 0, d};
    if (d == 1) return f;
    while ((1ull << f.shift) < d) ++f.shift;   // ceil(log2 d): mul < 2^32, and the error stays below 1 / d for x < 2^31
    --f.shift;
    f.mul = (uint32_t)(((1ull << (32 + f.shift)) + d - 1) / d);
    return f;
}
__device__ __forceinline__ uint32_t quotient(uint32_t x, const FastDiv &f)
{
    return f.div == 1 ? x : __umulhi(x, f.mul) >> f.shift;
}

}  // namespace q4
}  // namespace csr
