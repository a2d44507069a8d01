// What the two attention kernels over the 4-bit cache share: the queries a workgroup has and what they see, their conversion to
// fp16, the output.
#pragma once
#include <cfloat>
#include <cmath>

#include "q4_common.h"

namespace csr {
namespace q4 {

constexpr float kShift = 12.0f;         // p = 2^(score - maximum + kShift), as two fp16
constexpr float kShiftOne = 8.0f;       // as one
constexpr float kMostHalf = 65504.0f;   // the largest fp16
// Maxima are those of the products as the matrix cores give them, before the row's unit: none is beyond 128 * 65504^2 in size, so
// that a maximum before any token is below every one that a token may have, whatever the unit.
constexpr float kNone = -0x1p40f;
constexpr int kPromptTile = 64;    // tokens of a turn of the kernel for many rows
constexpr int kPromptWaves = 8;    // of a workgroup of the kernel for many rows, 32 rows each

struct AttnKernelArgs {
    Q4AttnArgs a;
    int32_t splits, row_blocks, rows;
    int32_t log_group_k, log_group_v;
    FastDiv by_splits, by_group;
    float *acc, *ml;
};

// Tokens that the queries of a block see: [0, end) by some, [0, all) by all
struct Sight {
    int len, qn, end, all;
};
__device__ __forceinline__ Sight sight_of(const AttnKernelArgs &ka, int len, int qn, int row0, int row_end)
{
    Sight s;
    s.len = max(0, min(len, (int)ka.a.T));
    s.qn = max(0, min(qn, ka.a.Tq));
    const int first = quotient(row0, ka.by_group), last = quotient(row_end - 1, ka.by_group);
    if (first >= s.qn) { s.end = s.all = 0; return s; }
    s.end = ka.a.causal ? max(0, s.len - s.qn + min(last, s.qn - 1) + 1) : s.len;
    s.all = last >= s.qn ? 0 : ka.a.causal ? max(0, s.len - s.qn + first + 1) : s.len;
    return s;
}
// The last token that query token i sees, -1 for none
__device__ __forceinline__ int limit_of(const AttnKernelArgs &ka, const Sight &s, int i)
{
    if (i >= s.qn) return -1;
    return ka.a.causal ? s.len - s.qn + i : s.len - 1;
}

// Four neighbouring channels of the output
__device__ __forceinline__ void store_out4(const Q4AttnArgs &a, int64_t at, float4v v)
{
    if (a.out_dtype == CSR_F32) {
        *reinterpret_cast<float4v *>(static_cast<float *>(a.out) + at) = v;
    } else if (a.out_dtype == CSR_F16) {
        *reinterpret_cast<uint2v *>(static_cast<_Float16 *>(a.out) + at) =
            uint2v{as_u32(half2v{(_Float16)v[0], (_Float16)v[1]}), as_u32(half2v{(_Float16)v[2], (_Float16)v[3]})};
    } else {
        *reinterpret_cast<uint2v *>(static_cast<uint16_t *>(a.out) + at) =
            uint2v{(uint32_t)float_to_bf16(v[0]) | (uint32_t)float_to_bf16(v[1]) << 16, (uint32_t)float_to_bf16(v[2]) | (uint32_t)float_to_bf16(v[3]) << 16};
    }
}

// Eight channels of a query row, as they are stored
template <int QMODE> struct Stored8 {
    uint4v w[QMODE == CSR_F32 ? 2 : 1];
};
template <int QMODE> __device__ __forceinline__ void load_q8(Stored8<QMODE> &s, const void *q, int64_t at)
{
    const uint4v *p = reinterpret_cast<const uint4v *>(static_cast<const uint8_t *>(q) + at * (QMODE == CSR_F32 ? 4 : 2));
    s.w[0] = p[0];
    if constexpr (QMODE == CSR_F32) s.w[1] = p[1];
}
template <int QMODE> __device__ __forceinline__ float channel_of(const Stored8<QMODE> &s, int k)
{
    if constexpr (QMODE == CSR_F32) return __uint_as_float(s.w[k / 4][k % 4]);
    else if constexpr (QMODE == CSR_F16) return (float)as_half2(s.w[0][k / 2])[k % 2];
    else return __uint_as_float(k % 2 ? s.w[0][k / 2] & 0xffff0000u : s.w[0][k / 2] << 16);
}

__device__ __forceinline__ half8v join(half2v a, half2v b, half2v c, half2v d) { return half8v{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]}; }
// sum + p[0] + p[1]
__device__ __forceinline__ float dot2(half2v p, float sum) { return __builtin_amdgcn_fdot2(p, half2v{(_Float16)1.0f, (_Float16)1.0f}, sum, false); }

// The factor of a row's scores, in powers of two, and the power of two that its channels are multiplied by before they become
// fp16: none for fp16, else what brings the largest to 2^14 .. 2^15.
struct RowUnit {
    float unit;
    int up;
};
__device__ __forceinline__ RowUnit unit_of(float scale, bool shifted, float most)
{
    RowUnit u{scale, 0};
    if (shifted) {
        u.up = most > 0.0f && most < INFINITY ? 14 - ilogbf(most) : 0;
        u.unit = ldexpf(scale, -u.up);
    }
    u.unit *= 1.44269504088896340736f;   // (last: a scale next to the largest float is within range by then)
    // An unseen token's score, minus infinity, times 0 would be no number; and kNone times the unit is one.  (Products that differ do
    // so by 2^-48 and more: at a unit of 2^87 already nothing but the largest has a probability.)
    u.unit = fminf(fmaxf(u.unit, FLT_MIN), 0x1p87f);
    return u;
}

// Probabilities are 2^(product * unit + (shift - maximum * unit)), one fused operation.  Where the maximum is far from zero the sum in
// brackets is rounded by powers of two and more, and the largest probability would be anything from nothing to an infinity: there the
// maximum is subtracted from the products, at every turn.  (At 2^20 a float's step is 2^-3.)
__device__ __forceinline__ bool is_far(float top, float unit) { return fabsf(top * unit) >= 0x1p20f && top != kNone; }

// The channels of a word in the order that evens() and odds() give them
__device__ __forceinline__ constexpr int word_order(int j) { return 2 * (j & 3) + (j >> 2); }

}  // namespace q4

hipError_t launch_q4_prompt(const q4::AttnKernelArgs &ka);  // many query rows per KV head (q4_prompt.hip)

}  // namespace csr
