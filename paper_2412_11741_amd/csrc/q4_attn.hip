// Attention over the 4-bit cache: a few query rows per KV head.
//
// A query row is a (query token, query head) of the KV head; row r is query token r / G, head r % G of the group.  The cache is
// read once per block of rows and bounds the time, so everything else is arranged around wide requests in flight: a wave
// streams tokens, 32 at a time, straight into registers, with the next 32 requested before these are used, and shares nothing
// with other waves until the end.
//
// For 32 tokens: S^T = K q^T and O^T += V^T p^T on the matrix cores (16x16x32, fp16 in, fp32 out).  With the tokens as rows of
// S^T and channels as rows of O^T a query row stays in the same 16th of the lanes throughout: its maximum, sum and
// probabilities never cross lanes but for the maximum.  Which of the instruction's 32 contraction places means which channel
// (S^T) or which token (O^T) is free as long as both operands agree, so
//   - lane (m, kg) takes the channels 32 kg .. of token m's key (d / 4 of them: one or two words, one group of the scale);
//   - a lane's four scores of either half of the 32 tokens are tokens 8 kg .. 8 kg + 7 and go into the next product as they are;
//   - lane (m, kg) takes channels (d / 16) m .. of the values of tokens 8 kg .. 8 kg + 7: two tokens' words are cut into halves and
//     joined, and every pair of codes is then one channel of two tokens.
// Probabilities are 2^12 times their ratio to the running maximum's, which is moved when a lane's eight add up to more than an
// fp16 holds: as two fp16 - the value and what it lacks - they keep 22 bits down to 2^-14 of the largest, where what they lack meets
// fp16's smallest step: below, steps of 2^-36 of the largest.  As one (bf16 queries; more than 16 rows a workgroup) they keep 11 bits, and
// the sum is that of the rounded ones; 2^8 times leaves more room above the maximum, 11 bits down to 2^-22 of the largest and steps of
// 2^-32 of it below.
//   One row of 4 x 32 x 32768 tokens (671 MB): 126 us with the join, 5.3 TB/s; 8 x 8 sequences of up to 131072 tokens, four rows
// (944 MB): 178 us, 5.3 TB/s (a kernel that does nothing but read reaches 6.1).  Twenty rows of 16 x 8 x 8192 tokens: 35 to 38 us with the join's 5:
// vector and matrix instructions, which do not overlap between a SIMD's waves here, are 77 % of its cycles (counted), the rest is
// its two waves waiting.
#include <type_traits>

#include "q4_attn_common.h"

namespace csr {
namespace {

using namespace q4;

constexpr int kStep = 32;          // tokens of a wave's turn

__device__ __forceinline__ float4v mfma(half8v a, half8v b, float4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// p less the fp16 in the low (high) half of a word, exactly
__device__ __forceinline__ float less_low(float p, uint32_t h)
{
    float r;
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(r) : "v"(h), "v"(p));
    return r;
}
__device__ __forceinline__ float less_high(float p, uint32_t h)
{
    float r;
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(r) : "v"(h), "v"(p));
    return r;
}

// The codes and parameters of a wave's 32 tokens, as requested
template <int D> struct Raw {
    uint32_t kc[2][D / 32], kp[2], vc[8], vp[8];
};

// A (sequence, KV head) block of the caches, and where a lane's codes and parameters lie, as bytes behind those of a wave's first
// token
struct Base {
    const uint8_t *kc, *kp, *vc, *vp;
    int T;
};
struct Lane {
    uint32_t kc, kp, vc, vp;
};

typedef uint4v uint4a __attribute__((aligned(4)));

// WHOLE: all 32 tokens are rows of the cache.  Else rows behind the last one are requested as the last one.
template <int D, bool WHOLE> __device__ __forceinline__ void request_keys(Raw<D> &r, const Base &base, const Lane &at, int tb, int m)
{
    const uint8_t *kc = base.kc + (uint32_t)tb * (D / 2), *kp = base.kp + (uint32_t)tb * 4;
    const int last = base.T - 1 - tb;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int mine = 8 * (m >> 2) + (m & 3) + 4 * u, back = WHOLE ? 0 : max(0, mine - last);
        const uint32_t c = at.kc + 4 * u * (D / 2) - back * (D / 2);
        if constexpr (D == 128) {
            const uint4v w = *reinterpret_cast<const uint4v *>(kc + c);
#pragma unroll
            for (int k = 0; k < 4; ++k) r.kc[u][k] = w[k];
        } else {
            const uint2v w = *reinterpret_cast<const uint2v *>(kc + c);
            r.kc[u][0] = w[0];
            r.kc[u][1] = w[1];
        }
        r.kp[u] = *reinterpret_cast<const uint32_t *>(kp + (at.kp + 16 * u - back * 4));
    }
}
template <int D, bool WHOLE> __device__ __forceinline__ void request_values(Raw<D> &r, const Base &base, const Lane &at, int tb, int kg)
{
    const uint8_t *vc = base.vc + (uint32_t)tb * (D / 2), *vp = base.vp + (uint32_t)tb * 4;
    const int last = base.T - 1 - tb;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int back = WHOLE ? 0 : max(0, 8 * kg + j - last);
        const uint32_t c = at.vc + j * (D / 2) - back * (D / 2);
        if constexpr (D == 128) r.vc[j] = *reinterpret_cast<const uint32_t *>(vc + c);
        else r.vc[j] = *reinterpret_cast<const uint16_t *>(vc + c);
        if constexpr (!WHOLE) r.vp[j] = *reinterpret_cast<const uint32_t *>(vp + (at.vp + 4 * j - back * 4));
    }
    if constexpr (WHOLE) {
        const uint4v w0 = *reinterpret_cast<const uint4a *>(vp + at.vp), w1 = *reinterpret_cast<const uint4a *>(vp + (at.vp + 16));
#pragma unroll
        for (int j = 0; j < 4; ++j) { r.vp[j] = w0[j]; r.vp[4 + j] = w1[j]; }
    }
}
template <int D> __device__ __forceinline__ void request_keys(Raw<D> &r, const Base &base, const Lane &at, int tb, int m)
{
    if (tb + kStep <= base.T) request_keys<D, true>(r, base, at, tb, m);
    else request_keys<D, false>(r, base, at, tb, m);
}
template <int D> __device__ __forceinline__ void request_values(Raw<D> &r, const Base &base, const Lane &at, int tb, int kg)
{
    if (tb + kStep <= base.T) request_values<D, true>(r, base, at, tb, kg);
    else request_values<D, false>(r, base, at, tb, kg);
}
template <int D> __device__ __forceinline__ void request(Raw<D> &r, const Base &base, const Lane &at, int tb, int m, int kg)
{
    request_keys<D>(r, base, at, tb, m);
    request_values<D>(r, base, at, tb, kg);
}

// QMODE: csr_dtype of q.  NR: tiles of 16 query rows.  W: waves.
template <int D, int QMODE, int NR, int W>
__global__ __launch_bounds__(64 * W, NR == 1 && QMODE != CSR_F32 && W == 4 ? 3 : 2) void q4_stream_kernel(AttnKernelArgs ka)
{
    constexpr int KM = D / 32;   // matrix instructions along a key's channels
    constexpr int UC = D / 16;   // channels of a lane's values
    constexpr bool kTwo = QMODE == CSR_F32;
    constexpr bool kMany = NR == 4;        // queries wait in LDS
    // probabilities are one fp16, where the second would be a third of the matrix instructions or the queries are rounded to 2^-8 (bf16, one
    // row: 64 x 8 x 2048 tokens 28.1 us, with the second 29.7; 8 x 8 of up to 131072 179 and 189; heads of 64, 8 x 8 x 16384, 20.4 and 23.7)
    constexpr bool kOneP = !kTwo && (NR > 1 || QMODE == CSR_BF16);
    constexpr bool kOneSet = kMany || (kTwo && NR == 2);   // of registers for requests: two do not fit
    static_assert(!kMany || (W == 4 && !kTwo), "a wave converts one tile of queries");
    const Q4AttnArgs &a = ka.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, kg = lane >> 4;
    const int b = blockIdx.z, h = blockIdx.y, bh = b * a.Hkv + h;
    const int rb = quotient(blockIdx.x, ka.by_splits), split = blockIdx.x - rb * ka.splits;
    const int row0 = rb * 16 * NR, row_end = min(row0 + 16 * NR, ka.rows);
    const int len = a.seq_lens ? a.seq_lens[b] : (int)a.T, qn = a.q_lens ? a.q_lens[b] : a.Tq;

    constexpr int NC = kMany ? 1 : NR;   // tiles of queries that a wave converts
    Stored8<QMODE> stored[NC][KM];
#pragma unroll
    for (int t = 0; t < NC; ++t) {
        const int r = min(row0 + 16 * (kMany ? wave : t) + m, ka.rows - 1), i = quotient(r, ka.by_group);
        const int64_t from = (int64_t)b * a.q_stride[0] + (int64_t)(h * a.G + r - i * a.G) * a.q_stride[1] + (int64_t)i * a.q_stride[2] + kg * (D / 4);
#pragma unroll
        for (int k = 0; k < KM; ++k) load_q8<QMODE>(stored[t][k], a.q, from + 8 * k);
    }

    const Sight s = sight_of(ka, len, qn, row0, row_end);
    const uint32_t per = (quotient(s.end + ka.splits - 1, ka.by_splits) + kStep * W - 1) / (kStep * W) * (kStep * W);
    const int begin = min((int)(split * per), s.end), end = min(begin + (int)per, s.end);
    const size_t block = (size_t)bh * a.T;
    const Base cache{static_cast<const uint8_t *>(a.codesK) + block * (D / 2), static_cast<const uint8_t *>(a.paramsK) + (block * D >> ka.log_group_k) * 4,
                     static_cast<const uint8_t *>(a.codesV) + block * (D / 2), static_cast<const uint8_t *>(a.paramsV) + (block * D >> ka.log_group_v) * 4, (int)a.T};
    const uint32_t T = (uint32_t)a.T, token = 8 * (m >> 2) + (m & 3);
    const Lane at{token * (D / 2) + kg * (D / 8), ((uint32_t)(kg * (D / 4)) >> ka.log_group_k) * T * 4 + token * 4,
                  (uint32_t)(8 * kg * (D / 2) + m * (D / 32)), ((uint32_t)(m * UC) >> ka.log_group_v) * T * 4 + 32 * kg};
    Raw<D> even, odd;
    int tb = begin + wave * kStep;
    if (tb < end) request<D>(even, cache, at, tb, m, kg);

    // the queries: fp16, and what that lacks; in units that leave no loss to bf16
    __shared__ half8v waiting[kMany ? NR * KM * 64 : 1];
    __shared__ float waiting_unit[kMany ? NR * 16 : 1];
    half8v qh[NC][KM], ql[kTwo ? NC : 1][KM];
    float unit[NR];
    int limit[NR];
#pragma unroll
    for (int t = 0; t < NC; ++t) {
        float most = 0.0f;
        if constexpr (QMODE != CSR_F16) {
#pragma unroll
            for (int k = 0; k < KM; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(channel_of<QMODE>(stored[t][k], j)));
            most = fmaxf(most, __shfl_xor(most, 16, 64));
            most = fmaxf(most, __shfl_xor(most, 32, 64));
        }
        const RowUnit ru = unit_of(a.scale, QMODE != CSR_F16, most);
        unit[t] = ru.unit;
#pragma unroll
        for (int k = 0; k < KM; ++k) {
            half8v hi, lo;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float f = channel_of<QMODE>(stored[t][k], word_order(j));
                if constexpr (QMODE != CSR_F16) f = ldexpf(f, ru.up);
                hi[j] = (_Float16)f;
                lo[j] = (_Float16)(f - (float)hi[j]);
            }
            qh[t][k] = hi;
            if constexpr (kTwo) ql[t][k] = lo;
            if constexpr (kMany) waiting[(wave * KM + k) * 64 + lane] = hi;
        }
    }
    if constexpr (kMany) {
        if (kg == 0) waiting_unit[16 * wave + m] = unit[0];
        __syncthreads();
#pragma unroll
        for (int t = 0; t < NR; ++t) unit[t] = waiting_unit[16 * t + m];
    }
#pragma unroll
    for (int t = 0; t < NR; ++t) {
        const int r = row0 + 16 * t + m;
        limit[t] = r < ka.rows ? limit_of(ka, s, quotient(r, ka.by_group)) : -1;
    }

    float4v o[NR][UC] = {};
    float top[NR], sum[NR];
#pragma unroll
    for (int t = 0; t < NR; ++t) { top[t] = kNone; sum[t] = 0.0f; }

    int look = 2;   // at the maxima whatever the sums: 2 in the first turn, 1 if a row's is far from zero (one number: two flags cost scalar registers)
    const auto turn = [&](Raw<D> &r) __attribute__((always_inline)) {
        half8v k8[2][KM];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const half2v ks = as_half2(low_halves(r.kp[u], r.kp[u])), km = as_half2(high_halves(r.kp[u], r.kp[u]));
#pragma unroll
            for (int k = 0; k < KM; ++k)
                k8[u][k] = join(fma2(whole2<false>(evens(r.kc[u][k])), ks, km), fma2(whole2<true>(evens(r.kc[u][k])), ks, km),
                                fma2(whole2<false>(odds(r.kc[u][k])), ks, km), fma2(whole2<true>(odds(r.kc[u][k])), ks, km));
        }
        float score[NR][8];
        int from = lane;   // (the queries are read every turn: held back, they would push other values out of the registers)
        asm volatile("" : "+v"(from));
#pragma unroll
        for (int t = 0; t < NR; ++t) {
            float4v c[2] = {};
#pragma unroll
            for (int k = 0; k < KM; ++k) {
                const half8v q = kMany ? waiting[(t * KM + k) * 64 + from] : qh[kMany ? 0 : t][k];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    c[u] = mfma(k8[u][k], q, c[u]);
                    if constexpr (kTwo) c[u] = mfma(k8[u][k], ql[t][k], c[u]);
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) score[t][j] = c[j / 4][j % 4];
        }
        if constexpr (kOneSet)
            if (tb + kStep * W < end) request_keys<D>(r, cache, at, tb + kStep * W, m);
        // tokens that some row does not see: out of its scores, and values that are no finite numbers out of the product - the
        // rows that do see them get NaN
        if (tb + kStep > s.all) {
            bool any_bad = false;
            half8v bad;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const half2v sm = as_half2(r.vp[j]);
                const half2v ends = half2v{__builtin_elementwise_fma((_Float16)15.0f, sm[0], sm[1]), sm[1]};
                const bool bj = not_finite(as_u32(ends));
                any_bad |= bj;
                bad[j] = bj ? (_Float16)1.0f : (_Float16)0.0f;
                if (bj) r.vp[j] = 0;
            }
            const bool poisoned = __any(any_bad);
#pragma unroll
            for (int t = 0; t < NR; ++t) {
                half8v seen;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool sees = tb + 8 * kg + j <= limit[t];
                    if (!sees) score[t][j] = -INFINITY;
                    seen[j] = sees ? (_Float16)1.0f : (_Float16)0.0f;
                }
                if (poisoned) {
                    const float4v n = mfma(bad, seen, float4v{});
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int c = 0; c < UC; ++c) o[t][c][j] = n[j] > 0.0f ? NAN : o[t][c][j];
                }
            }
        }
        // Probabilities against the maxima as they are.  A lane's sum of eight tells whether one of them may have left fp16's range; the
        // maxima are moved first then, and in a wave's first turn, and for rows whose maximum is far from zero.
        half8v ph[NR], pl[kOneP ? 1 : NR];
        float part_sum[NR] = {};
        const auto weigh = [&](int t, float less) __attribute__((always_inline)) {
            const float lift = fmaf(-(top[t] - less), unit[t], kOneP ? kShiftOne : kShift);
            half2v p2[4], rest[4];
            part_sum[t] = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p0 = __builtin_amdgcn_exp2f(fmaf(score[t][2 * j] - less, unit[t], lift));
                const float p1 = __builtin_amdgcn_exp2f(fmaf(score[t][2 * j + 1] - less, unit[t], lift));
                p2[j] = half2v{(_Float16)p0, (_Float16)p1};
                if constexpr (kOneP) {
                    part_sum[t] = dot2(p2[j], part_sum[t]);
                } else {
                    part_sum[t] += p0 + p1;
                    rest[j] = half2v{(_Float16)less_low(p0, as_u32(p2[j])), (_Float16)less_high(p1, as_u32(p2[j]))};
                }
            }
            ph[t] = join(p2[0], p2[1], p2[2], p2[3]);
            if constexpr (!kOneP) pl[t] = join(rest[0], rest[1], rest[2], rest[3]);
        };
        bool moved = true;
        if (look < 2) {
            float largest = 0.0f;
#pragma unroll
            for (int t = 0; t < NR; ++t) {
                weigh(t, 0.0f);
                largest = fmaxf(largest, part_sum[t]);
            }
            moved = (look | __any(largest > kMostHalf)) != 0;
        }
        if (moved) {   // only those rows' that need it: what others see changes no bit of a row
            int far = 0;
#pragma unroll
            for (int t = 0; t < NR; ++t) {
                int mine = look > 1 || part_sum[t] > kMostHalf || is_far(top[t], unit[t]);
                mine |= __shfl_xor(mine, 16, 64);
                mine |= __shfl_xor(mine, 32, 64);
                float best = score[t][0];
#pragma unroll
                for (int j = 1; j < 8; ++j) best = fmaxf(best, score[t][j]);
                best = fmaxf(best, __shfl_xor(best, 16, 64));
                best = fmaxf(best, __shfl_xor(best, 32, 64));
                best = mine ? fmaxf(best, top[t]) : top[t];
                const float fade = __builtin_amdgcn_exp2f((top[t] - best) * unit[t]);
                top[t] = best;
                sum[t] *= fade;
#pragma unroll
                for (int c = 0; c < UC; ++c) o[t][c] *= fade;
                const bool apart = is_far(best, unit[t]);
                far |= __builtin_amdgcn_readfirstlane(__any(apart));
                weigh(t, apart ? best : 0.0f);
            }
            look = far != 0;
        }
#pragma unroll
        for (int t = 0; t < NR; ++t) sum[t] += part_sum[t];
        half2v vs[4], vm[4];
        uint32_t low[4], high[4];   // channels 0 .. 3 and 4 .. 7 of two tokens
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            vs[j] = as_half2(low_halves(r.vp[2 * j], r.vp[2 * j + 1]));
            vm[j] = as_half2(high_halves(r.vp[2 * j], r.vp[2 * j + 1]));
            low[j] = low_bytes(r.vc[2 * j], r.vc[2 * j + 1]);
            high[j] = high_bytes(r.vc[2 * j], r.vc[2 * j + 1]);
        }
        const auto channel = [&](auto c) {
            constexpr int C = decltype(c)::value;
            constexpr bool UPPER = (C & 2) != 0;
            half2v v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t w = C < 4 ? low[j] : high[j];
                v[j] = fma2(whole2<UPPER>(C & 1 ? odds(w) : evens(w)), vs[j], vm[j]);
            }
            const half8v v8 = join(v[0], v[1], v[2], v[3]);
#pragma unroll
            for (int t = 0; t < NR; ++t) {
                o[t][C] = mfma(v8, ph[t], o[t][C]);
                if constexpr (!kOneP) o[t][C] = mfma(v8, pl[t], o[t][C]);
            }
        };
        channel(std::integral_constant<int, 0>{});
        channel(std::integral_constant<int, 1>{});
        channel(std::integral_constant<int, 2>{});
        channel(std::integral_constant<int, 3>{});
        if constexpr (UC == 8) {
            channel(std::integral_constant<int, 4>{});
            channel(std::integral_constant<int, 5>{});
            channel(std::integral_constant<int, 6>{});
            channel(std::integral_constant<int, 7>{});
        }
    };
    if constexpr (kOneSet) {   // one set of registers, filled again as soon as it has been read
        for (; tb < end; tb += kStep * W) {
            turn(even);
            if (tb + kStep * W < end) request_values<D>(even, cache, at, tb + kStep * W, kg);
        }
    } else {
        while (tb < end) {   // two sets in turn: one is used while the other is filled
            if (tb + kStep * W < end) request<D>(odd, cache, at, tb + kStep * W, m, kg);
            turn(even);
            tb += kStep * W;
            if (tb >= end) break;
            if (tb + kStep * W < end) request<D>(even, cache, at, tb + kStep * W, m, kg);
            turn(odd);
            tb += kStep * W;
        }
    }

    // the waves' parts of a row tile, one tile after the other
    __shared__ float part[W][16][D + 4], parts_top[W][16], parts_sum[W][16];
#pragma unroll
    for (int t = 0; t < NR; ++t) {
        float l = sum[t];
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        if (t > 0) __syncthreads();
        if (kg == 0) {
            parts_top[wave][m] = top[t] * unit[t];
            parts_sum[wave][m] = l;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int c = 0; c < UC; c += 4)
                *reinterpret_cast<float4v *>(&part[wave][m][(4 * kg + j) * UC + c]) = float4v{o[t][c][j], o[t][c + 1][j], o[t][c + 2][j], o[t][c + 3][j]};
        __syncthreads();
        for (int e = threadIdx.x; e < 16 * D / 4; e += 64 * W) {
            const int n = e / (D / 4), ch = 4 * (e % (D / 4)), r = row0 + 16 * t + n;
            if (r >= row_end) break;   // (rows ascend with e)
            float best = -FLT_MAX, all = 0.0f;
            float4v value = {};
#pragma unroll
            for (int w = 0; w < W; ++w) best = fmaxf(best, parts_top[w][n]);
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float fade = __builtin_amdgcn_exp2f(parts_top[w][n] - best);
                all = fmaf(parts_sum[w][n], fade, all);
                value += *reinterpret_cast<const float4v *>(&part[w][n][ch]) * fade;
            }
            if (ka.splits == 1) {
                const int i = quotient(r, ka.by_group), hq = h * a.G + r - i * a.G;
                store_out4(a, (int64_t)b * a.out_stride[0] + (int64_t)hq * a.out_stride[1] + (int64_t)i * a.out_stride[2] + ch,
                           all == 0.0f ? float4v{} : value / all);
            } else {
                const size_t to = ((size_t)bh * ka.splits + split) * ka.rows + r;
                *reinterpret_cast<float4v *>(ka.acc + to * D + ch) = value;
                if (ch == 0) {
                    ka.ml[2 * to] = best;
                    ka.ml[2 * to + 1] = all;
                }
            }
        }
    }
}

// Joins the parts of the token axis: a wave per query row, all its parts' requests ahead of their use
template <int D, int DEEP>   // DEEP: requests ahead
__global__ __launch_bounds__(256) void q4_join_kernel(AttnKernelArgs ka)
{
    constexpr int LANES = D / 4, SIDE = 64 / LANES;   // of a part's row; parts side by side
    const Q4AttnArgs &a = ka.a;
    const int lane = threadIdx.x & 63, b = blockIdx.z, h = blockIdx.y, bh = b * a.Hkv + h;
    const int r = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (r >= ka.rows) return;
    const int side = lane / LANES, ch = 4 * (lane % LANES);
    const size_t first = (size_t)bh * ka.splits * ka.rows + r;
    float all = 0.0f, best = -FLT_MAX;
    float4v value = {};
    float4v part[DEEP];
    float top[DEEP], sum[DEEP];
    const auto request = [&](int k0) {
#pragma unroll
        for (int k = 0; k < DEEP; ++k) {
            const size_t from = first + (size_t)min(k0 + SIDE * k, ka.splits - 1) * ka.rows;
            part[k] = *reinterpret_cast<const float4v *>(ka.acc + from * D + ch);
            const float2 ml = *reinterpret_cast<const float2 *>(ka.ml + 2 * from);
            top[k] = ml.x;
            sum[k] = ml.y;
        }
    };
    request(side);   // (ahead of the maxima: they come with it)
    for (int k = lane; k < ka.splits; k += 64) best = fmaxf(best, ka.ml[2 * (first + (size_t)k * ka.rows)]);
#pragma unroll
    for (int w = 32; w >= 1; w >>= 1) best = fmaxf(best, __shfl_xor(best, w, 64));
    for (int k0 = side; k0 < ka.splits; k0 += SIDE * DEEP) {
        if (k0 != side) request(k0);
#pragma unroll
        for (int k = 0; k < DEEP; ++k) {
            if (k0 + SIDE * k >= ka.splits) break;
            const float fade = __builtin_amdgcn_exp2f(top[k] - best);
            all = fmaf(sum[k], fade, all);
            value += part[k] * fade;
        }
    }
#pragma unroll
    for (int w = LANES; w < 64; w <<= 1) {
        all += __shfl_xor(all, w, 64);
#pragma unroll
        for (int c = 0; c < 4; ++c) value[c] += __shfl_xor(value[c], w, 64);
    }
    if (side != 0) return;
    const int i = quotient(r, ka.by_group), hq = h * a.G + r - i * a.G;
    store_out4(a, (int64_t)b * a.out_stride[0] + (int64_t)hq * a.out_stride[1] + (int64_t)i * a.out_stride[2] + ch, all == 0.0f ? float4v{} : value / all);
}

constexpr int kWaves = 4, kAloneWaves = 8;   // of a workgroup; of one that has a CU to itself

template <int D, int QMODE, int NR, int W = kWaves> hipError_t run(const AttnKernelArgs &ka)
{
    hipLaunchKernelGGL((q4_stream_kernel<D, QMODE, NR, W>), dim3(ka.splits * ka.row_blocks, ka.a.Hkv, ka.a.B), dim3(64 * W), 0, ka.a.stream, ka);
    return hipGetLastError();
}
template <int D> hipError_t join_parts(const AttnKernelArgs &ka)
{
    const dim3 groups((ka.rows + 3) / 4, ka.a.Hkv, ka.a.B);
    if (ka.splits * (D / 4) <= 128) hipLaunchKernelGGL((q4_join_kernel<D, 2>), groups, dim3(256), 0, ka.a.stream, ka);
    else if (ka.splits * (D / 4) <= 256) hipLaunchKernelGGL((q4_join_kernel<D, 4>), groups, dim3(256), 0, ka.a.stream, ka);
    else hipLaunchKernelGGL((q4_join_kernel<D, 8>), groups, dim3(256), 0, ka.a.stream, ka);
    return hipGetLastError();
}
template <int D, int QMODE> hipError_t run(const AttnKernelArgs &ka, int row_tiles, bool alone)
{
    if (alone) return run<D, QMODE, 1, kAloneWaves>(ka);
    if constexpr (QMODE != CSR_F32)
        if (row_tiles == 4) return run<D, QMODE, 4>(ka);
    return row_tiles == 1 ? run<D, QMODE, 1>(ka) : run<D, QMODE, 2>(ka);
}
template <int D> hipError_t run(const AttnKernelArgs &ka, int row_tiles, bool alone)
{
    switch (ka.a.q_dtype) {
        case CSR_F32: return run<D, CSR_F32>(ka, row_tiles, alone);
        case CSR_F16: return run<D, CSR_F16>(ka, row_tiles, alone);
        default: return run<D, CSR_BF16>(ka, row_tiles, alone);
    }
}

}  // namespace

// The kernel for a call's query rows, and the parts of its token axis.  In three kernels the waves of a workgroup share the rows, 16, 32
// or 64 of them, and divide the tokens; in the one for many rows (fp16 and bf16 queries) they share the tokens and divide 256 rows.
// Sharing makes codes cheaper and workgroups fewer.  What a call takes is close to (us; size: of a turn, 1, 1.36, 2.45 and 0.75 to 2.2,
// with heads of 64 channels 0.6 of that)
//   turns * (0.2 + 0.8 c) * size   turns: of 128 tokens per workgroup, c: workgroups per CU
//   turns * c * size               turns of 64 tokens, for the many rows
//   + 0, 1.5, 3, 5                 by the rows of a workgroup
//   + 3.6 in one part; in more 6.7, 0.08 for every part beyond 16 and the parts' bytes at 4 TB/s, out and in
// and what is least is taken, fewer rows a workgroup if 3 % less.  (70 shapes, each with all kernels and 1 to 64 parts timed: 1 % slower than
// the fastest on the average, 20 % at most.)  Timed were fp16 and bf16 queries, and sequences as long as their cache; the host knows the
// cache's rows only, and shorter ones pay for parts without tokens: one sequence of 517 tokens takes 6.9 us in 517 rows and 14.8 in 131072,
// 64 of 2048 tokens 29.7 and 62.3.  Measured, us, with 16, 32, 64 and 256 rows at their best numbers of parts: 5 KV heads of 131
// rows, 425 tokens 7.4 (eight waves), 9.8, 12.5, 13.8; 8 of 1200 rows, 300 tokens 10.6, 12.7, 15.8, 18.9; 32 of 512, 512 tokens 17.0,
// 15.5, 17.7, 25.4; 512 of 64, 2048 tokens 99, 67, 57; 128 of 64, 700 tokens 15.6, 13.4, 20.3; 8 of 8192, 10240 tokens 625, 463, 402, 322.
// Parts measured at 8 pairs of 517 tokens: 8.0 us in one, 7.8 in three, 7.0 in one of eight waves; of 8192: 56.4 in one, 13.5 in
// eight, 10.1 in 16, 10.6 in 24; 512 pairs of 2048: 29.8 in one, 32.1 in two.
void plan_q4_attn(const Q4AttnArgs &a, Q4AttnPlan *p)
{
    const int64_t rows = (int64_t)a.G * a.Tq, blocks = (int64_t)a.B * a.Hkv;
    const uint32_t T = (uint32_t)a.T;
    const bool fp32 = a.q_dtype == CSR_F32;
    const int32_t most_tiles = rows <= 16 ? 1 : rows <= 32 || fp32 ? 2 : rows <= 64 ? 4 : 2 * kPromptWaves;
    const float width = a.d == 64 ? 0.6f : 1.0f, part_bytes = (float)(blocks * rows) * (float)(a.d * 8);
    float to_beat = INFINITY;
    for (const int32_t tiles : {2 * kPromptWaves, 4, 2, 1}) {
        if (tiles > most_tiles) continue;
        const bool many = tiles > 4;
        const int64_t block_rows = 16 * tiles, row_blocks = (rows + block_rows - 1) / block_rows, groups = many ? row_blocks * blocks : row_blocks;   // along x
        if (tiles < most_tiles && groups > 1 << 22) break;   // (2^32 threads are the runtime's limit)
        const uint32_t step = many ? kPromptTile : kStep * kWaves;
        const float busy = (float)(rows < block_rows ? rows : block_rows) / (float)block_rows;
        const float size = width * (many ? 0.75f + 1.45f * busy : tiles == 1 ? 1.0f : tiles == 2 ? 1.36f : 2.45f);
        const float more = many ? 5.0f : tiles == 1 ? 0.0f : tiles == 2 ? 1.5f : 3.0f;
        float least = INFINITY;
        int32_t best = 1;
        for (const uint32_t splits : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128, 192, 256}) {
            if (splits > 1 && (splits > (T + 127) / 128 || groups * splits > 1 << 22)) break;
            const float turns = (float)((T + step * splits - 1) / (step * splits)), c = (float)((blocks * row_blocks * splits + kCus - 1) / kCus);
            const float join = splits == 1 ? 3.6f : 6.7f + 0.08f * (float)(splits > 16 ? splits - 16 : 0) + part_bytes * (float)splits / 4e6f;
            const float cost = turns * (many ? c : 0.2f + 0.8f * c) * size + join + more;
            if (cost < least) {
                least = cost;
                best = (int32_t)splits;
            }
        }
        // Short contexts of few pairs: eight waves, two of them to a SIMD, go through 256 tokens in 1.45 where four take 1.0 for 128.
        const float alone = tiles == 1 && blocks * row_blocks <= kCus ? 4.25f + fmaxf(1.0f, (float)((T + 31) / 32) / kAloneWaves) * 1.45f * width : INFINITY;
        if (fminf(least, alone) >= to_beat) continue;
        to_beat = 0.97f * fminf(least, alone);
        p->row_tiles = tiles;
        p->row_blocks = (int32_t)row_blocks;
        p->alone = alone < least;
        p->splits = p->alone ? 1 : best;
    }
    const size_t parts = (size_t)blocks * (size_t)rows * (size_t)p->splits;
    p->off_ml = p->splits > 1 ? (parts * a.d * 4 + 255) / 256 * 256 : 0;
    p->total_bytes = p->splits > 1 ? p->off_ml + (parts * 8 + 255) / 256 * 256 : 0;
}

hipError_t launch_q4_attn(const Q4AttnArgs &a, const Q4AttnPlan &p)
{
    AttnKernelArgs ka{};
    const auto log2_of = [](int32_t group) { return group == 32 ? 5 : group == 64 ? 6 : 7; };
    ka.a = a;
    ka.splits = p.splits; ka.row_blocks = p.row_blocks; ka.rows = a.G * a.Tq;
    ka.log_group_k = log2_of(a.group_k); ka.log_group_v = log2_of(a.group_v);
    ka.by_splits = fast_div((uint32_t)p.splits); ka.by_group = fast_div((uint32_t)a.G);
    ka.acc = static_cast<float *>(a.workspace);
    ka.ml = reinterpret_cast<float *>(static_cast<char *>(a.workspace) + p.off_ml);
    const hipError_t e = p.row_tiles > 4 ? launch_q4_prompt(ka) : a.d == 128 ? run<128>(ka, p.row_tiles, p.alone) : run<64>(ka, p.row_tiles, p.alone);
    if (e != hipSuccess || p.splits == 1) return e;
    return a.d == 128 ? join_parts<128>(ka) : join_parts<64>(ka);
}

}  // namespace csr
