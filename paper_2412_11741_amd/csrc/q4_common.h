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

// Eight codes as whole numbers.  The bytes of `evens` hold channels 0, 2, 4, 6, those of `odds` 1, 3, 5, 7; a byte 0000cccc read as
// an 8-bit float with four bits of exponent and three of fraction is c * 2^-9, among the subnormals and in the first binade
// alike, so that one conversion with a factor of 2^9 turns two bytes into two fp16, at the rate of any other instruction
// (measured), without the difference that a bias in an fp16's fraction would need.
__device__ __forceinline__ uint32_t evens(uint32_t w) { return w & 0x0f0f0f0fu; }
__device__ __forceinline__ uint32_t odds(uint32_t w) { return (w >> 4) & 0x0f0f0f0fu; }
template <bool HIGH> __device__ __forceinline__ half2v whole2(uint32_t bytes)   // of bytes 0, 1 (2, 3)
{
    return __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(bytes, 512.0f, HIGH));
}

// The low (high) halves of two words side by side
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// Bytes 0 and 1 (2 and 3) of two words by turns: a0 b0 a1 b1
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05010400u); }
__device__ __forceinline__ uint32_t high_bytes(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07030602u); }

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
