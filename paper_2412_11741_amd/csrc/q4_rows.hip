// Rows into and out of the 4-bit cache: quantising as they are written, reading back.
//
// Both move bytes: a head vector of 128 fp16 channels is 256 bytes outside and 68 to 80 in the cache.  A channel costs some
// twenty-six vector instructions on the way in (210 a wave and eight channels, counted), three on the way out.  A thread has
// eight channels of one vector, 16 bytes of fp16 and one word of codes; the 4 to 16 threads of a group of channels are
// neighbours in a row of 16 lanes, so that the group's extremes come from data-parallel-primitive moves.  The threads of a wave
// take consecutive tokens: their codes are 256 consecutive bytes.  Two or four vectors a thread, with their requests ahead, took
// the same time.
//   Written and handed back, 2 x 32 x 4096 vectors of 128 fp16: 27.4 us, 153 MB at 5.6 TB/s.  Read back to fp16, the same
// vectors: 16.0 us, 86 MB at 5.4 TB/s; to fp32, 2 x 4 x 8 x 32768 of 64: 86.8 us, 605 MB at 7.0 TB/s (what is read lies in the
// caches for the most part, stores go past them).
#include "lane_ops.h"
#include "q4_common.h"

namespace csr {
namespace {

using namespace q4;

// Outputs of this size and more go past the L2s: what streams through is not the code that the next call reads.  (Measured when this
// came: 2 x 32 x 4096 vectors of 128 fp16 written and handed back 29.0 us instead of 35.5, read back 17.0 instead of 19.5.)  A
// call that reads the output next finds smaller ones in the L2s.
constexpr int64_t kStreamBytes = 4 << 20;

template <bool PAST, typename V> __device__ __forceinline__ void put(V v, V *p)
{
    if constexpr (PAST) __builtin_nontemporal_store(v, p);
    else *p = v;
}

// Which vectors a workgroup has: any (FLAT), or neighbouring tokens of one sequence and head, with normal stores (NEAR) or stores
// past the L2s (PAST)
enum Mode { FLAT, NEAR, PAST };

constexpr float kLargest = 65504.0f;   // of fp16

struct RowsSide {
    const uint8_t *x;
    uint32_t *codes;   // words of eight channels
    uint32_t *params;  // words of (scale, minimum)
    uint8_t *out;
    int64_t xb, xh, xt, ob, oh, ot;   // strides in bytes
    int32_t log_group;
};
struct RowsKernelArgs {
    RowsSide side[2];
    const int32_t *pos, *counts;
    int64_t pos0;
    FastDiv by_tiles, by_h;   // by_tiles: tokens (FLAT) or workgroups (else) per sequence and head
    uint32_t n, T, total;     // total: vectors of a side in this launch
    uint32_t first_block;     // (sequence, head) of the launch's first
};

template <typename P> __device__ __forceinline__ P uniform(P p)
{
    const uint64_t v = (uint64_t)p;
    return (P)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)v));
}

// Where a thread's vector lies.  A workgroup has neighbouring tokens of one sequence and head, so that all but a 32-bit offset is
// the scalar unit's work; where a sequence has less than half a workgroup's worth, or tokens are very far apart (FLAT), any
// vectors.
struct Place {
    const uint8_t *x;
    uint8_t *out;
    uint32_t *codes, *params;       // of the (sequence, head)
    uint32_t x_more, out_more, t;   // bytes from x and out to the vector, its token
    uint32_t b;
};
template <int MODE, int LOGW, int LOGC> __device__ __forceinline__ bool place_of(const RowsKernelArgs &a, const RowsSide &s, Place &p)
{
    constexpr uint32_t PER = 256u >> LOGW;
    const uint32_t mine = threadIdx.x >> LOGW, v = MODE == FLAT ? blockIdx.x * PER + mine : blockIdx.x;
    if (MODE == FLAT && v >= a.total) return false;
    const uint32_t nth = quotient(v, a.by_tiles), first = MODE == FLAT ? v - nth * a.by_tiles.div : (v - nth * a.by_tiles.div) * PER;
    const uint32_t bh = a.first_block + nth;
    const uint32_t h = bh - quotient(bh, a.by_h) * a.by_h.div;
    p.b = quotient(bh, a.by_h);
    p.t = MODE == FLAT ? first : first + mine;
    if (MODE != FLAT && p.t >= a.n) return false;
    p.x = s.x + ((int64_t)p.b * s.xb + (int64_t)h * s.xh + (int64_t)first * s.xt);
    p.out = s.out + ((int64_t)p.b * s.ob + (int64_t)h * s.oh + (int64_t)first * s.ot);
    p.codes = s.codes + (((int64_t)bh * a.T) << LOGC);
    p.params = s.params + (int64_t)bh * ((8u << LOGC) >> s.log_group) * a.T;
    p.x_more = p.out_more = 0;
    if constexpr (MODE != FLAT) {
        p.x = uniform(p.x); p.out = uniform(p.out); p.codes = uniform(p.codes); p.params = uniform(p.params);
        p.x_more = mine * (uint32_t)s.xt;
        p.out_more = mine * (uint32_t)s.ot;
    }
    return true;
}
// Its row of the cache; false for none.  (A first row beyond 32 bits is out of reach of 2^26 tokens and 2^20 rows.)
__device__ __forceinline__ bool row_of(const RowsKernelArgs &a, const Place &p, uint32_t &row)
{
    const int64_t row0 = a.pos0 + (a.pos ? (int64_t)a.pos[p.b] : 0);
    const int32_t low = (int32_t)row0, first = (int32_t)(row0 >> 32) == low >> 31 ? low : 1 << 30;
    row = (uint32_t)first + p.t;
    return row < a.T && (!a.counts || (int)p.t < a.counts[p.b]);
}

// Eight channels as they are stored
template <int DT> struct Stored8 {
    uint4v w[DT == CSR_F32 ? 2 : 1];
};
template <int DT> __device__ __forceinline__ void load8(Stored8<DT> &r, const uint8_t *p)
{
    const uint4v *from = reinterpret_cast<const uint4v *>(p);
    r.w[0] = from[0];
    if constexpr (DT == CSR_F32) r.w[1] = from[1];
}
template <int DT> __device__ __forceinline__ void widen8(const Stored8<DT> &r, float (&v)[8])
{
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        if constexpr (DT == CSR_F32) v[k] = __uint_as_float(r.w[k / 4][k % 4]);
        else if constexpr (DT == CSR_F16) v[k] = (float)as_half2(r.w[0][k / 2])[k % 2];
        else v[k] = __uint_as_float(k % 2 ? r.w[0][k / 2] & 0xffff0000u : r.w[0][k / 2] << 16);
    }
}

// Channels 0..7 from pairs (0, 2), (4, 6), (1, 3), (5, 7)
template <int DT, int MODE> __device__ __forceinline__ void store8(uint8_t *p, const half2v (&pair)[4])
{
    if constexpr (DT == CSR_F32) {
        const float4v v[2] = {float4v{(float)pair[0][0], (float)pair[2][0], (float)pair[0][1], (float)pair[2][1]},
                              float4v{(float)pair[1][0], (float)pair[3][0], (float)pair[1][1], (float)pair[3][1]}};
        if constexpr (MODE == PAST) {
            // past the L2s a store has to fill its 64 bytes: the four lanes of a quad, 128 bytes, put the lower half and then the
            // upper one together (with halves of theirs each, reading back 4 x 8 x 32768 vectors took 204 us instead of 141)
            const int l = threadIdx.x & 3;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float4v mine;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float low = half ? lane::dpp_mov<0xFA>(v[0][c]) : lane::dpp_mov<0x50>(v[0][c]);   // quad_perm [2,2,3,3], [0,0,1,1]
                    const float high = half ? lane::dpp_mov<0xFA>(v[1][c]) : lane::dpp_mov<0x50>(v[1][c]);
                    mine[c] = l & 1 ? high : low;
                }
                __builtin_nontemporal_store(mine, reinterpret_cast<float4v *>(p - 32 * l + 64 * half + 16 * l));
            }
        } else {
            reinterpret_cast<float4v *>(p)[0] = v[0];
            reinterpret_cast<float4v *>(p)[1] = v[1];
        }
    } else {
        uint4v w;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if constexpr (DT == CSR_F16) {
                w[2 * k] = low_halves(as_u32(pair[k]), as_u32(pair[2 + k]));
                w[2 * k + 1] = high_halves(as_u32(pair[k]), as_u32(pair[2 + k]));
            } else {
                w[2 * k] = (uint32_t)float_to_bf16((float)pair[k][0]) | (uint32_t)float_to_bf16((float)pair[2 + k][0]) << 16;
                w[2 * k + 1] = (uint32_t)float_to_bf16((float)pair[k][1]) | (uint32_t)float_to_bf16((float)pair[2 + k][1]) << 16;
            }
        }
        put<MODE == PAST>(w, reinterpret_cast<uint4v *>(p));
    }
}

// fp16(s * code + m) of a word's eight channels, as pairs (0, 2), (4, 6), (1, 3), (5, 7)
__device__ __forceinline__ void word_values(uint32_t w, uint32_t sm, half2v (&pair)[4])
{
    const half2v s = as_half2(low_halves(sm, sm)), m = as_half2(high_halves(sm, sm));
    pair[0] = fma2(whole2<false>(evens(w)), s, m);
    pair[1] = fma2(whole2<true>(evens(w)), s, m);
    pair[2] = fma2(whole2<false>(odds(w)), s, m);
    pair[3] = fma2(whole2<true>(odds(w)), s, m);
}

// Of three, without the quieting of signalling NaNs that fminf and fmaxf put before each operand
__device__ __forceinline__ float min3(float a, float b, float c)
{
    float r;
    asm("v_min3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
struct OpMin { __device__ __forceinline__ float operator()(float a, float b) const { return min3(a, b, b); } };
struct OpMax { __device__ __forceinline__ float operator()(float a, float b) const { return max3(a, b, b); } };

template <typename T, typename Op> __device__ __forceinline__ T group_reduce(T v, int log_group, Op op)
{
    v = lane::row_reduce<4>(v, op);
    if (log_group > 5) v = op(v, lane::dpp_mov<0x141>(v));
    if (log_group > 6) v = op(v, lane::dpp_mov<0x140>(v));
    return v;
}

// x - m as a rounded difference and what that lacks
struct Difference {
    float rounded, rest;
};
__device__ __forceinline__ Difference difference(float x, float m)
{
    const float t = x - m, back = x - t;
    return {t, (x - (t + back)) + (back - m)};
}

// Scale and minimum of a group from its extremes, as exact arithmetic gives them: m = fp16(lo), s the largest fp16 with
// 15 s <= hi - m.  The factor is 1/15 and a little, so that the quotient comes out no smaller than the exact one; as an fp16 it is
// then that s or the next above it (15 s and its difference to the span next to it are exact).
__device__ __forceinline__ uint32_t group_params(float lo, float hi)
{
    const _Float16 m = (_Float16)lo;
    const Difference span = difference(hi, (float)m);
    if (!(span.rounded > 0.0f)) return (uint32_t)__builtin_bit_cast(uint16_t, m) << 16;
    const _Float16 q = (_Float16)(span.rounded * 0x1.111116p-4f);
    uint16_t s = __builtin_bit_cast(uint16_t, q);
    if (fmaf(15.0f, (float)q, -span.rounded) > span.rest) --s;   // (never below zero: 15 * 0 is not above a span)
    return (uint32_t)s | (uint32_t)__builtin_bit_cast(uint16_t, m) << 16;
}

// The whole number next to (x - m) / s, halves to even, from one that is off by one at most.  The rounded difference's distance to
// the middle between two codes is exact where it is small (the middle is 16 bits), and compared with what the difference lacks:
// added to it, the lacking part would be rounded away, and a value next to a middle would pass for one on it.
__device__ __forceinline__ float decided(float x, float m, float s, float r)
{
    const Difference t = difference(x, m);
    const float above = fmaf(-(r + 0.5f), s, t.rounded), below = fmaf(-(r - 0.5f), s, t.rounded);
    const bool odd = ((int)r & 1) != 0;
    if (above > -t.rest || (above == -t.rest && odd)) r += 1.0f;
    else if (below < -t.rest || (below == -t.rest && odd)) r -= 1.0f;
    return r;
}

// The codes of eight channels, as a word.  Adding 1.5 * 2^23 leaves the nearest whole number of (x - m) * (1 / s) in the lowest
// bits of the sum.  The product is off by a few units in its last place: where some channel's lies that near to a half, all
// eight are decided anew.
__device__ __forceinline__ uint32_t codes_of(const float (&x)[8], float m, float s)
{
    constexpr float kWhole = 12582912.0f;
    constexpr uint32_t kBits = 0x4b400000u, kAll = kBits + (kBits << 4) + (kBits << 8) + (kBits << 12);   // (higher ones shift out)
    const float inv = s > 0.0f ? __builtin_amdgcn_rcpf(s) : 0.0f;
    float y[8], off[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float t = x[k] - m;
        y[k] = fmaf(t, inv, kWhole);
        off[k] = fabsf(fmaf(t, inv, kWhole - y[k]));
    }
    const float far = max3(max3(max3(off[0], off[1], off[2]), off[3], off[4]), max3(off[5], off[6], off[7]), 0.0f);
    if (far > 0.49999f) {
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = decided(x[k], m, s, y[k] - kWhole) + kWhole;
    }
    uint32_t w = 0;
#pragma unroll
    for (int k = 7; k >= 0; --k) w = (w << 4) + __float_as_uint(__builtin_amdgcn_fmed3f(y[k], kWhole, kWhole + 15.0f));
    return w - kAll;
}

template <int DT, int OUT, int LOGW, int MODE>   // OUT: csr_dtype of out, -1 without; 2^LOGW threads per vector
__global__ __launch_bounds__(256) void q4_write_kernel(RowsKernelArgs a)
{
    const RowsSide &s = a.side[blockIdx.y];
    const uint32_t o = threadIdx.x & ((1u << LOGW) - 1u);
    Place p;
    if (!place_of<MODE, LOGW, LOGW>(a, s, p)) return;   // (a vector's threads all leave)
    Stored8<DT> stored;
    load8<DT>(stored, p.x + (p.x_more + o * (DT == CSR_F32 ? 32 : 16)));
    uint32_t row;
    if (!row_of(a, p, row)) {
        if constexpr (OUT >= 0) {
            const half2v none[4] = {};
            store8<OUT, MODE>(p.out + (p.out_more + o * (OUT == CSR_F32 ? 32 : 16)), none);
        }
        return;
    }
    float x[8], lo, hi, sum = 0.0f;
    widen8<DT>(stored, x);
#pragma unroll
    for (int k = 0; k < 8; ++k) sum = fmaf(x[k], 0.0f, sum);   // 0, or NaN if one is no finite number
    if constexpr (DT != CSR_F16) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = __builtin_amdgcn_fmed3f(x[k], -kLargest, kLargest);
    }
    lo = min3(min3(min3(x[0], x[1], x[2]), x[3], x[4]), min3(x[5], x[6], x[7]), x[7]);
    hi = max3(max3(max3(x[0], x[1], x[2]), x[3], x[4]), max3(x[5], x[6], x[7]), x[7]);
    lo = group_reduce(lo, s.log_group, OpMin());
    hi = group_reduce(hi, s.log_group, OpMax());
    sum = group_reduce(sum, s.log_group, lane::OpAdd());
    uint32_t sm = group_params(lo, hi);
    uint32_t w = codes_of(x, (float)as_half2(sm)[1], (float)as_half2(sm)[0]);
    if (sum != 0.0f) { sm = 0x7e007e00u; w = 0; }
    p.codes[(row << LOGW) + o] = w;
    if (((8 * o) & ((1u << s.log_group) - 1u)) == 0) p.params[((8 * o) >> s.log_group) * a.T + row] = sm;
    if constexpr (OUT >= 0) {
        half2v pair[4];
        word_values(w, sm, pair);
        store8<OUT, MODE>(p.out + (p.out_more + o * (OUT == CSR_F32 ? 32 : 16)), pair);
    }
}

// A thread stores 16 bytes: eight channels, or four as fp32.  2^LOGW threads per vector.
template <int OUT, int LOGW, int MODE>
__global__ __launch_bounds__(256) void q4_read_kernel(RowsKernelArgs a)
{
    constexpr bool kHalf = OUT == CSR_F32;
    constexpr int LOGC = kHalf ? LOGW - 1 : LOGW;   // words of codes per vector
    const RowsSide &s = a.side[0];
    const uint32_t o = threadIdx.x & ((1u << LOGW) - 1u);
    Place p;
    if (!place_of<MODE, LOGW, LOGC>(a, s, p)) return;
    uint8_t *to = p.out + (p.out_more + o * 16);
    uint32_t row, w = 0, sm = 0;   // (zeros stand for zeros)
    const bool held = row_of(a, p, row);
    if constexpr (kHalf) {
        if (held) {
            w = reinterpret_cast<const uint16_t *>(p.codes)[(row << LOGW) + o];
            sm = p.params[((4 * o) >> s.log_group) * a.T + row];
        }
        const half2v scale = as_half2(low_halves(sm, sm)), least = as_half2(high_halves(sm, sm));
        const half2v even = fma2(whole2<false>(evens(w)), scale, least), odd = fma2(whole2<false>(odds(w)), scale, least);
        put<MODE == PAST>(float4v{(float)even[0], (float)odd[0], (float)even[1], (float)odd[1]}, reinterpret_cast<float4v *>(to));
    } else {
        if (held) {
            w = p.codes[(row << LOGW) + o];
            sm = p.params[((8 * o) >> s.log_group) * a.T + row];
        }
        half2v pair[4];
        word_values(w, sm, pair);
        store8<OUT, MODE>(to, pair);
    }
}

// A workgroup of one sequence and head from half a workgroup's vectors on; fewer share one.
// A launch takes 2^20 workgroups' worth of (sequence, head) blocks (the runtime's limit is 2^32 threads).
constexpr uint32_t kMostGroups = 1u << 20;

template <typename K> hipError_t launch(const Q4RowsArgs &r, int sides, int log_threads, K flat, K near, K past)
{
    RowsKernelArgs a{};
    const uint32_t per = 256u >> log_threads, blocks = (uint32_t)r.B * (uint32_t)r.Hkv;
    const int64_t xe = r.x_dtype == CSR_F32 ? 4 : 2, oe = r.out_dtype == CSR_F32 ? 4 : 2;
    bool any = r.n < per / 2;
    for (int k = 0; k < sides; ++k) {
        const Q4RowsSide &s = r.side[k];
        a.side[k] = {static_cast<const uint8_t *>(s.x), static_cast<uint32_t *>(s.codes), static_cast<uint32_t *>(s.params), static_cast<uint8_t *>(s.out),
                     s.x_stride[0] * xe, s.x_stride[1] * xe, s.x_stride[2] * xe, s.out_stride[0] * oe, s.out_stride[1] * oe, s.out_stride[2] * oe,
                     s.group == 32 ? 5 : s.group == 64 ? 6 : 7};
        if (a.side[k].xt > (1 << 26) || a.side[k].ot > (1 << 26)) any = true;   // (31 of them are 2^31 bytes)
    }
    const bool stream = a.side[0].out && (int64_t)sides * blocks * r.n * r.d * oe >= kStreamBytes;
    const K kernel = any ? flat : stream ? past : near;
    a.pos = r.pos; a.counts = r.counts; a.pos0 = r.pos0;
    a.n = (uint32_t)r.n; a.T = (uint32_t)r.T;
    const uint32_t tiles = any ? a.n : (a.n + per - 1) / per;
    a.by_tiles = fast_div(tiles); a.by_h = fast_div((uint32_t)r.Hkv);
    const uint64_t fit = (uint64_t)kMostGroups * (any ? per : 1) / tiles;
    const uint32_t step = fit < 1 ? 1 : fit < blocks ? (uint32_t)fit : blocks;
    for (uint32_t b = 0; b < blocks; b += step) {
        const uint32_t now = blocks - b < step ? blocks - b : step;
        a.first_block = b;
        a.total = now * a.n;
        hipLaunchKernelGGL(kernel, dim3(any ? (a.total + per - 1) / per : now * tiles, sides), dim3(256), 0, r.stream, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int DT, int OUT> hipError_t write(const Q4RowsArgs &r, int sides)
{
    constexpr int kPast = OUT >= 0 ? PAST : NEAR;
    return r.d == 128 ? launch(r, sides, 4, q4_write_kernel<DT, OUT, 4, FLAT>, q4_write_kernel<DT, OUT, 4, NEAR>, q4_write_kernel<DT, OUT, 4, kPast>)
                      : launch(r, sides, 3, q4_write_kernel<DT, OUT, 3, FLAT>, q4_write_kernel<DT, OUT, 3, NEAR>, q4_write_kernel<DT, OUT, 3, kPast>);
}
template <int DT> hipError_t write(const Q4RowsArgs &r, int sides)
{
    if (!r.side[0].out) return write<DT, -1>(r, sides);
    switch (r.out_dtype) {
        case CSR_F32: return write<DT, CSR_F32>(r, sides);
        case CSR_F16: return write<DT, CSR_F16>(r, sides);
        default: return write<DT, CSR_BF16>(r, sides);
    }
}
template <int OUT> hipError_t read(const Q4RowsArgs &r)
{
    constexpr int W = OUT == CSR_F32 ? 5 : 4;   // log2 of the threads of a vector of 128
    return r.d == 128 ? launch(r, 1, W, q4_read_kernel<OUT, W, FLAT>, q4_read_kernel<OUT, W, NEAR>, q4_read_kernel<OUT, W, PAST>)
                      : launch(r, 1, W - 1, q4_read_kernel<OUT, W - 1, FLAT>, q4_read_kernel<OUT, W - 1, NEAR>, q4_read_kernel<OUT, W - 1, PAST>);
}

}  // namespace

hipError_t launch_q4_write(const Q4RowsArgs &r, int sides)
{
    switch (r.x_dtype) {
        case CSR_F32: return write<CSR_F32>(r, sides);
        case CSR_F16: return write<CSR_F16>(r, sides);
        default: return write<CSR_BF16>(r, sides);
    }
}
hipError_t launch_q4_read(const Q4RowsArgs &r)
{
    switch (r.out_dtype) {
        case CSR_F32: return read<CSR_F32>(r);
        case CSR_F16: return read<CSR_F16>(r);
        default: return read<CSR_BF16>(r);
    }
}

}  // namespace csr
