// Attention over the 4-bit cache: many query rows per KV head (a prompt's chunk).
//
// The products bound this shape, and with them the vector ALU, which shares the issue with the matrix cores: turning codes into
// fp16 has to be spread over as many rows as possible.  A workgroup has 32 query rows a wave and goes through the tokens 64 at a
// time: its threads turn the 64 keys and values into fp16 in LDS, each once, while the tile before is multiplied (two buffers, one
// barrier a tile; the next codes are requested a tile ahead).
//
// Per wave and 32 tokens: S^T = K q^T and O^T += V^T p^T in 32x32x16 instructions.  As in the kernel for few rows a query row stays in
// its lanes (row = lane % 32): a lane's 16 scores become the next product's operand as they are, its two 8-byte runs of tokens
// 8 i + 4 (lane / 32) .. + 3 side by side.  Keys and values lie row by row; values are read with the transposing LDS read, four
// tokens of a channel a lane.  Rows are swizzled, keys by 16 bytes, values by 64, so that every read and write touches all banks.
// Channels lie in the order their codes are converted in (0, 2, 4, 6, 1, 3, 5, 7 of a word): the queries are put in the same
// order, the output's lanes exchange halves.
//   8192 rows over 10240 tokens, eight KV heads (309 GFLOP): 320 to 350 us, 880 to 970 TFLOP/s as the clock allows, where a large library product
// reaches 1100 to 1320 by box (1540 with its second operand transposed); heads of 64 channels (155 GFLOP) 196 us, 790 TFLOP/s: half the
// products to every exponential.  Vector and matrix instructions together, which hardly overlap between a SIMD's waves, are 90 % of its cycles
// (counted), at the clock that the chip's power leaves; two or four waves a workgroup are slower (less sharing), the order of the
// instructions is worth 1 %.
#include <type_traits>

#include "q4_attn_common.h"

namespace csr {
namespace {

using namespace q4;

typedef float float16v __attribute__((ext_vector_type(16)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4v lds_short4v;

constexpr int kTile = kPromptTile;
constexpr int kRows = 32;    // query rows of a wave
constexpr int kParts = 8;    // threads that share a token's key (value)

__device__ __forceinline__ float16v mfma32(half8v a, half8v b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

// Where 16 bytes (eight channels) of a token's row lie in a tile, in bytes
template <int D> __device__ __forceinline__ int key_at(int token, int chunk)
{
    return token * D * 2 + 16 * (chunk ^ (D == 128 ? token & 15 : (token >> 1) & 7));
}
template <int D> __device__ __forceinline__ int value_at(int token, int chunk)
{
    return token * D * 2 + 64 * ((chunk >> 2) ^ (D == 128 ? token & 3 : (token >> 1) & 1)) + 16 * (chunk & 3);
}

// A thread's codes of a tile, as requested: WORDS words of each of its TOKENS keys and values
template <int WORDS, int TOKENS> struct RawTile {
    uint32_t kc[TOKENS][WORDS], vc[TOKENS][WORDS], kp[TOKENS], vp[TOKENS];
};

template <int D, int QMODE, int W>
__global__ __launch_bounds__(64 * W, D == 64 ? 4 : 2) void q4_prompt_kernel(AttnKernelArgs ka, int total)
{
    constexpr int KS = D / 16;          // steps of the products along channels
    constexpr int CT = D / 32;          // tiles of output channels
    constexpr int WORDS = D / 8 / kParts, TOKENS = kTile * kParts / (64 * W);
    constexpr int BYTES = kTile * D * 2;
    __shared__ __align__(16) uint8_t tiles[4 * BYTES];   // keys, keys, values, values
    __shared__ __align__(8) uint8_t bad[2][kTile][kParts];   // whose parameters are no finite numbers; of tiles that not all rows see
    const Q4AttnArgs &a = ka.a;
    // the workgroups of an XCD are neighbours: they read the same caches
    const int per_xcd = (total + 7) / 8, id = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if (id >= total) return;
    const int sets = ka.row_blocks * ka.splits, bh = id / sets, b = bh / a.Hkv, h = bh - b * a.Hkv;
    const int rb = (id - bh * sets) / ka.splits, split = id - bh * sets - rb * ka.splits;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, hh = lane >> 5;
    const int len = a.seq_lens ? a.seq_lens[b] : (int)a.T, qn = a.q_lens ? a.q_lens[b] : a.Tq;
    const int row0 = rb * kRows * W, row_end = min(row0 + kRows * W, ka.rows);
    const Sight s = sight_of(ka, len, qn, row0, row_end);
    const int per = (quotient(s.end + ka.splits - 1, ka.by_splits) + kTile - 1) / kTile * kTile;
    const int begin = min(split * per, s.end), end = min(begin + per, s.end);

    // this thread's share of a tile: words part * WORDS .. of tokens mine, mine + 8 W, ...
    const int part = threadIdx.x % kParts, mine = threadIdx.x / kParts;
    const size_t block = (size_t)bh * a.T;
    const uint8_t *const kc = static_cast<const uint8_t *>(a.codesK) + block * (D / 2), *const vc = static_cast<const uint8_t *>(a.codesV) + block * (D / 2);
    const uint8_t *const kp = static_cast<const uint8_t *>(a.paramsK) + (block * D >> ka.log_group_k) * 4;
    const uint8_t *const vp = static_cast<const uint8_t *>(a.paramsV) + (block * D >> ka.log_group_v) * 4;
    const uint32_t kg = ((uint32_t)(part * (D / kParts)) >> ka.log_group_k) * (uint32_t)a.T, vg = ((uint32_t)(part * (D / kParts)) >> ka.log_group_v) * (uint32_t)a.T;
    typedef RawTile<WORDS, TOKENS> Raw;
    Raw raw;
    const auto request = [&](int tb) {
#pragma unroll
        for (int i = 0; i < TOKENS; ++i) {
            const uint32_t t = min(tb + mine + i * (64 * W / kParts), (int)a.T - 1), at = t * (D / 2) + part * (WORDS * 4);
            if constexpr (WORDS == 2) {
                const uint2v k = *reinterpret_cast<const uint2v *>(kc + at), v = *reinterpret_cast<const uint2v *>(vc + at);
                raw.kc[i][0] = k[0]; raw.kc[i][1] = k[1];
                raw.vc[i][0] = v[0]; raw.vc[i][1] = v[1];
            } else {
                raw.kc[i][0] = *reinterpret_cast<const uint32_t *>(kc + at);
                raw.vc[i][0] = *reinterpret_cast<const uint32_t *>(vc + at);
            }
            raw.kp[i] = *reinterpret_cast<const uint32_t *>(kp + (kg + t) * 4);
            raw.vp[i] = *reinterpret_cast<const uint32_t *>(vp + (vg + t) * 4);
        }
    };
    const auto convert = [&](int tb, int buffer) {
#pragma unroll
        for (int i = 0; i < TOKENS; ++i) {
            const int t = mine + i * (64 * W / kParts);
            if (tb + kTile > s.all) {   // (the same for all threads)
                const half2v sm = as_half2(raw.vp[i]);
                const half2v ends = half2v{__builtin_elementwise_fma((_Float16)15.0f, sm[0], sm[1]), sm[1]};
                const bool b = not_finite(as_u32(ends));
                bad[buffer][t][part] = b;
                if (b) raw.vp[i] = 0;
            }
            const half2v ks = as_half2(low_halves(raw.kp[i], raw.kp[i])), km = as_half2(high_halves(raw.kp[i], raw.kp[i]));
            const half2v vs = as_half2(low_halves(raw.vp[i], raw.vp[i])), vm = as_half2(high_halves(raw.vp[i], raw.vp[i]));
#pragma unroll
            for (int w = 0; w < WORDS; ++w) {
                const auto put = [](uint8_t *to, uint32_t c, half2v sc, half2v m) {
                    *reinterpret_cast<uint4v *>(to) = uint4v{as_u32(fma2(whole2<false>(evens(c)), sc, m)), as_u32(fma2(whole2<true>(evens(c)), sc, m)),
                                                            as_u32(fma2(whole2<false>(odds(c)), sc, m)), as_u32(fma2(whole2<true>(odds(c)), sc, m))};
                };
                put(&tiles[buffer * BYTES + key_at<D>(t, part * WORDS + w)], raw.kc[i][w], ks, km);
                put(&tiles[(2 + buffer) * BYTES + value_at<D>(t, part * WORDS + w)], raw.vc[i][w], vs, vm);
            }
        }
    };

    // a lane's query: 16-byte runs 2 k + hh
    const int first_row = row0 + kRows * wave, row = first_row + n;
    const int r = min(row, ka.rows - 1), query = quotient(r, ka.by_group), hq = h * a.G + r - query * a.G;
    Stored8<QMODE> stored[KS];
    const int64_t q_at = (int64_t)b * a.q_stride[0] + (int64_t)hq * a.q_stride[1] + (int64_t)query * a.q_stride[2] + 8 * hh;
#pragma unroll
    for (int k = 0; k < KS; ++k) load_q8<QMODE>(stored[k], a.q, q_at + 16 * k);
    if (begin < end) request(begin);
    float most = 0.0f;
    if constexpr (QMODE != CSR_F16) {
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(channel_of<QMODE>(stored[k], j)));
        most = fmaxf(most, __shfl_xor(most, 32, 64));
    }
    const RowUnit ru = unit_of(a.scale, QMODE != CSR_F16, most);
    const float unit = ru.unit;
    half8v q[KS];
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float f = channel_of<QMODE>(stored[k], word_order(j));
            q[k][j] = (_Float16)(QMODE != CSR_F16 ? ldexpf(f, ru.up) : f);
        }
    const int limit = row < ka.rows ? limit_of(ka, s, query) : -1;
    const bool busy = first_row < row_end;   // waves without rows only convert

    float16v o[CT] = {};
    float top = kNone, sum = 0.0f;
    bool far = false;   // some row's maximum
    uint32_t poison = 0;   // parts of the channels that a token that is no number has reached

    // where a lane reads: of token n channels 16 k + 8 hh .., and for the transposing read, where lane 16 e + 4 i + f reads channels
    // 16 (e % 2) + 4 f .. of token 4 (e / 2) + i and gets four tokens of channel lane % 32.  What tokens, halves and steps add is
    // constant: swizzles repeat after 16 tokens.  A tile's other buffer is one bit away.
    static_assert((BYTES & (BYTES - 1)) == 0, "a power of two");
    uint32_t key_from[KS], value_from[CT];
#pragma unroll
    for (int k = 0; k < KS; ++k) key_from[k] = key_at<D>(n, 2 * k + hh);
#pragma unroll
    for (int t = 0; t < CT; ++t)
        value_from[t] = 2 * BYTES + value_at<D>(4 * hh + ((lane >> 2) & 3), 4 * t + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) + 8 * (lane & 1);

    if (begin < end) {
        convert(begin, 0);
        if (begin + kTile < end) request(begin + kTile);
    }
    __syncthreads();
    int buffer = 0;
    for (int tb = begin; tb < end; tb += kTile, buffer ^= 1) {
        if (tb + kTile < end) {
            convert(tb + kTile, buffer ^ 1);
            if (tb + 2 * kTile < end) request(tb + 2 * kTile);
        }
        if (busy) {
            const bool some = tb + kTile > s.all;
            if (some && __any(*reinterpret_cast<const unsigned long long *>(bad[buffer][lane]) != 0)) {
                for (int t = 0; t < kTile; ++t)
                    if (tb + t <= limit)
                        for (int p = 0; p < kParts; ++p) poison |= (uint32_t)(bad[buffer][t][p] != 0) << p;
            }
            float16v c[2] = {};   // 32 tokens each
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    c[u] = mfma32(*reinterpret_cast<const half8v *>(&tiles[key_from[k] + 32 * u * D * 2]), q[k], c[u]);
            if (some) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (tb + 8 * (j >> 2) + 4 * hh + (j & 3) > limit) c[j >> 4][j & 15] = -INFINITY;
            }
            // probabilities against the maximum as it is; the sum of them as fp16 is infinite where one has left their range, and is
            // held to 32 of 2^13: the maximum is moved first then, and for rows whose maximum is far from zero
            half2v p[16];
            float part_sum;
            const auto weigh = [&](float less) {
                const float lift = fmaf(-(top - less), unit, kShiftOne);
                part_sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float16v &x = c[j >> 3];
                    const int e = 2 * (j & 7);
                    p[j] = half2v{(_Float16)__builtin_amdgcn_exp2f(fmaf(x[e] - less, unit, lift)), (_Float16)__builtin_amdgcn_exp2f(fmaf(x[e + 1] - less, unit, lift))};
                    part_sum = dot2(p[j], part_sum);
                }
            };
            weigh(0.0f);
            if (far | (bool)__any(part_sum > 32.0f * 8192.0f)) {   // (only those rows': what others see changes no bit of a row)
                int mine = part_sum > 32.0f * 8192.0f || is_far(top, unit);
                mine |= __shfl_xor(mine, 32, 64);
                float best = c[0][0];
#pragma unroll
                for (int j = 1; j < 32; ++j) best = fmaxf(best, c[j >> 4][j & 15]);
                best = fmaxf(fmaxf(best, __shfl_xor(best, 32, 64)), top);
                if (!mine) best = top;
                const float fade = __builtin_amdgcn_exp2f((top - best) * unit);
                top = best;
                sum *= fade;
#pragma unroll
                for (int t = 0; t < CT; ++t) o[t] *= fade;
                const bool apart = is_far(top, unit);
                far = __any(apart);
                weigh(apart ? top : 0.0f);
            }
            sum += part_sum;
#pragma unroll
            for (int k = 0; k < 4; ++k)   // 16 tokens each
#pragma unroll
                for (int t = 0; t < CT; ++t) {
                    union {
                        short4v s[2];
                        half8v h;
                    } v;
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        v.s[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v *)&tiles[value_from[t] + (16 * k + 8 * e) * D * 2]);
                    o[t] = mfma32(v.h, join(p[4 * k], p[4 * k + 1], p[4 * k + 2], p[4 * k + 3]), o[t]);
                }
        }
#pragma unroll
        for (int k = 0; k < KS; ++k) key_from[k] ^= BYTES;
#pragma unroll
        for (int t = 0; t < CT; ++t) value_from[t] ^= BYTES;
        __syncthreads();
    }
    if (!busy) return;

    sum += __shfl_xor(sum, 32, 64);
    const size_t to = ((size_t)bh * ka.splits + split) * ka.rows + row;
    const int64_t out_at = (int64_t)b * a.out_stride[0] + (int64_t)hq * a.out_stride[1] + (int64_t)query * a.out_stride[2];
    const float over = ka.splits == 1 ? (sum == 0.0f ? 0.0f : 1.0f / sum) : 1.0f;
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {   // eight channels: lanes below 32 hold 0, 2, 4, 6, the others 1, 3, 5, 7
            const auto swapped = [](float lower, float upper) {   // the upper lanes of the first for the lower ones of the second
                return __builtin_amdgcn_permlane32_swap(__float_as_uint(lower), __float_as_uint(upper), false, false);
            };
            const auto x = swapped(o[t][4 * e], o[t][4 * e + 2]), y = swapped(o[t][4 * e + 1], o[t][4 * e + 3]);
            const int ch = 32 * t + 8 * e + 4 * hh;
            float4v v = float4v{__uint_as_float(x[0]), __uint_as_float(x[1]), __uint_as_float(y[0]), __uint_as_float(y[1])} * over;
            if (poison >> (ch / (D / kParts)) & 1) v = float4v{NAN, NAN, NAN, NAN};
            if (row >= row_end) continue;
            if (ka.splits == 1) store_out4(a, out_at + ch, v);
            else *reinterpret_cast<float4v *>(ka.acc + to * D + ch) = v;
        }
    if (ka.splits > 1 && hh == 0 && row < row_end) {
        ka.ml[2 * to] = top * unit;
        ka.ml[2 * to + 1] = sum;
    }
}

template <int D, int QMODE> hipError_t run(const AttnKernelArgs &ka)
{
    const int total = ka.a.B * ka.a.Hkv * ka.row_blocks * ka.splits;
    hipLaunchKernelGGL((q4_prompt_kernel<D, QMODE, kPromptWaves>), dim3((total + 7) / 8 * 8), dim3(64 * kPromptWaves), 0, ka.a.stream, ka, total);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_q4_prompt(const q4::AttnKernelArgs &ka)
{
    if (ka.a.d == 128) return ka.a.q_dtype == CSR_F16 ? run<128, CSR_F16>(ka) : run<128, CSR_BF16>(ka);
    return ka.a.q_dtype == CSR_F16 ? run<64, CSR_F16>(ka) : run<64, CSR_BF16>(ka);
}

}  // namespace csr
