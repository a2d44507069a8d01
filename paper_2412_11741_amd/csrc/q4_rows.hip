// Rows into and out of the 4-bit cache: quantising as they are written, reading back.
//
// Both move bytes: a head vector of 128 fp16 channels is 256 bytes outside and 68 to 80 in the cache, and a channel costs some
// twenty vector instructions on the way in, six on the way out.  A thread has eight channels of one vector, 16 bytes of fp16
// and one word of codes; the 4 to 16 threads of a group of channels are neighbours in a row of 16 lanes, so that the group's
// extremes come from data-parallel-primitive moves.  The threads of a wave take consecutive tokens: their codes are 256
// consecutive bytes.
#include "lane_ops.h"
#include "q4_common.h"

namespace csr {
namespace {

using namespace q4;

constexpr float kLargest = 65504.0f;   // of fp16

struct RowsSide {
    const void *x;
    uint32_t *codes;   // words of eight channels
    uint32_t *params;  // words of (scale, minimum)
    void *out;
    int64_t xb, xh, xt, ob, oh, ot;   // strides in elements
    int32_t log_group;
};
struct RowsKernelArgs {
    RowsSide side[2];
    const int32_t *pos, *counts;
    int64_t pos0;
    uint32_t total;    // vectors, both sides together
    FastDiv by_n, by_h, by_b;
    uint32_t n, T, B;
    uint32_t words;    // words of codes per vector: d / 8
};

template <int DT> __device__ __forceinline__ void load8(const void *p, int64_t at, float *v)
{
    if constexpr (DT == CSR_F32) {
        const float4v *f = reinterpret_cast<const float4v *>(static_cast<const float *>(p) + at);
        const float4v a = f[0], b = f[1];
#pragma unroll
        for (int k = 0; k < 4; ++k) { v[k] = a[k]; v[4 + k] = b[k]; }
    } else {
        const uint4v w = *reinterpret_cast<const uint4v *>(static_cast<const uint16_t *>(p) + at);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (DT == CSR_F16) {
                const half2v h = as_half2(w[k]);
                v[2 * k] = (float)h[0];
                v[2 * k + 1] = (float)h[1];
            } else {
                v[2 * k] = __uint_as_float(w[k] << 16);
                v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
            }
        }
    }
}

// Channels 0..7 from pairs (k, k + 4)
template <int DT> __device__ __forceinline__ void store8(void *p, int64_t at, const half2v (&pair)[4])
{
    if constexpr (DT == CSR_F32) {
        float4v *f = reinterpret_cast<float4v *>(static_cast<float *>(p) + at);
        f[0] = float4v{(float)pair[0][0], (float)pair[1][0], (float)pair[2][0], (float)pair[3][0]};
        f[1] = float4v{(float)pair[0][1], (float)pair[1][1], (float)pair[2][1], (float)pair[3][1]};
    } else {
        uint4v w;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if constexpr (DT == CSR_F16) {
                w[k] = low_halves(as_u32(pair[2 * k]), as_u32(pair[2 * k + 1]));
                w[2 + k] = high_halves(as_u32(pair[2 * k]), as_u32(pair[2 * k + 1]));
            } else {
                w[k] = (uint32_t)float_to_bf16((float)pair[2 * k][0]) | (uint32_t)float_to_bf16((float)pair[2 * k + 1][0]) << 16;
                w[2 + k] = (uint32_t)float_to_bf16((float)pair[2 * k][1]) | (uint32_t)float_to_bf16((float)pair[2 * k + 1][1]) << 16;
            }
        }
        *reinterpret_cast<uint4v *>(static_cast<uint16_t *>(p) + at) = w;
    }
}

// fp16(s * code + m) of a word's eight channels, as pairs (k, k + 4)
__device__ __forceinline__ void word_values(uint32_t w, uint32_t sm, half2v (&pair)[4])
{
    const half2v s = as_half2(low_halves(sm, sm)), m = as_half2(high_halves(sm, sm));
    pair[0] = fma2(nibble_pair<0>(w), s, m);
    pair[1] = fma2(nibble_pair<1>(w), s, m);
    pair[2] = fma2(nibble_pair<2>(w), s, m);
    pair[3] = fma2(nibble_pair<3>(w), s, m);
}

struct OpMin { __device__ __forceinline__ float operator()(float a, float b) const { return fminf(a, b); } };

template <typename T, typename Op> __device__ __forceinline__ T group_reduce(T v, int log_group, Op op)
{
    v = lane::row_reduce<4>(v, op);
    if (log_group > 5) v = op(v, lane::dpp_mov<0x141>(v));
    if (log_group > 6) v = op(v, lane::dpp_mov<0x140>(v));
    return v;
}

// Scale and minimum of a group from its extremes, and a channel's code - each as exact arithmetic gives it.
//   m = fp16(lo).  s is the largest fp16 with 15 s <= hi - m.  In fp32 the quotient of the rounded span comes out no smaller
// than it is cut to fp16 (15 s is an fp32, and rounding keeps order), so at most one step too large: compared in 64 bits.
__device__ __forceinline__ uint32_t group_params(float lo, float hi)
{
    const _Float16 m = (_Float16)lo;
    const float span = hi - (float)m;
    if (!(span > 0.0f)) return (uint32_t)__builtin_bit_cast(uint16_t, m) << 16;
    const float q = span / 15.0f;
    uint16_t s = __builtin_bit_cast(uint16_t, (_Float16)q);
    const double exact = (double)hi - (double)(float)m;
    if (s && 15.0 * (double)(float)__builtin_bit_cast(_Float16, s) > exact) --s;
    return (uint32_t)s | (uint32_t)__builtin_bit_cast(uint16_t, m) << 16;
}

// Nearest whole number to (x - m) / s.  The quotient by the reciprocal is off by a few units in its last place: where it lies
// that near to a half (`close`), the remainder decides, which is exact with the rounding error of x - m added.
__device__ __forceinline__ float code_of(float x, float m, float s, float inv_s)
{
    const float t = x - m, u = t * inv_s;
    float r = __builtin_rintf(u);
    if (fabsf(u - r) > 0.49999f) {
        const float back = x - t, err = (x - (t + back)) + (back - m);   // x - m = t + err
        const float rest = fmaf(-r, s, t) + err, half = 0.5f * s;
        const bool odd = ((int)r & 1) != 0;
        if (rest > half || (rest == half && odd)) r += 1.0f;
        else if (rest < -half || (rest == -half && odd)) r -= 1.0f;
    }
    return __builtin_amdgcn_fmed3f(r, 0.0f, 15.0f);
}

// Where vector v of the call lies: its side, sequence, head and token, and the cache's row or -1
struct Place {
    uint32_t side, b, h, t;
    int64_t row;
};
__device__ __forceinline__ Place place_of(uint32_t v, const RowsKernelArgs &a)
{
    Place p;
    const uint32_t bh = quotient(v, a.by_n);
    p.t = v - bh * a.n;
    const uint32_t sb = quotient(bh, a.by_h);
    p.h = bh - sb * a.by_h.div;
    p.side = quotient(sb, a.by_b);
    p.b = sb - p.side * a.by_b.div;
    p.row = a.pos0 + (int64_t)p.t + (a.pos ? (int64_t)a.pos[p.b] : 0);
    if ((a.counts && (int64_t)p.t >= (int64_t)a.counts[p.b]) || p.row < 0 || p.row >= (int64_t)a.T) p.row = -1;
    return p;
}

template <int DT, int OUT, int LOGW>   // OUT: csr_dtype of out, -1 without; 2^LOGW threads per vector
__global__ __launch_bounds__(256) void q4_write_kernel(RowsKernelArgs a)
{
    const uint32_t v = blockIdx.x * (256u >> LOGW) + (threadIdx.x >> LOGW), o = threadIdx.x & ((1u << LOGW) - 1u);
    if (v >= a.total) return;   // (a group's threads all leave)
    const Place p = place_of(v, a);
    const RowsSide &s = a.side[p.side];
    const int64_t out_at = (int64_t)p.b * s.ob + (int64_t)p.h * s.oh + (int64_t)p.t * s.ot + 8 * o;
    if (p.row < 0) {
        if constexpr (OUT >= 0) {
            const half2v none[4] = {};
            store8<OUT>(s.out, out_at, none);
        }
        return;
    }
    float x[8], lo, hi, sum = 0.0f;
    load8<DT>(s.x, (int64_t)p.b * s.xb + (int64_t)p.h * s.xh + (int64_t)p.t * s.xt + 8 * o, x);
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += x[k] * 0.0f;   // 0, or NaN if one is no finite number
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = __builtin_amdgcn_fmed3f(x[k], -kLargest, kLargest);
    lo = fminf(fminf(fminf(x[0], x[1]), fminf(x[2], x[3])), fminf(fminf(x[4], x[5]), fminf(x[6], x[7])));
    hi = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    lo = group_reduce(lo, s.log_group, OpMin());
    hi = group_reduce(hi, s.log_group, lane::OpMax());
    sum = group_reduce(sum, s.log_group, lane::OpAdd());
    uint32_t sm = group_params(lo, hi), w = 0;
    const float scale = (float)as_half2(sm)[0], least = (float)as_half2(sm)[1];
    const float inv = scale > 0.0f ? 1.0f / scale : 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) w |= (uint32_t)code_of(x[k], least, scale, inv) << (4 * k);
    if (sum != 0.0f) { sm = 0x7e007e00u; w = 0; }
    const uint32_t block = p.b * a.by_h.div + p.h, g = (8 * o) >> s.log_group, groups = (8u << LOGW) >> s.log_group;
    s.codes[((int64_t)block * a.T + p.row) * (1 << LOGW) + o] = w;
    if (((8 * o) & ((1u << s.log_group) - 1u)) == 0) s.params[((int64_t)block * groups + g) * a.T + p.row] = sm;
    if constexpr (OUT >= 0) {
        half2v pair[4];
        word_values(w, sm, pair);
        store8<OUT>(s.out, out_at, pair);
    }
}

template <int OUT, int LOGW>
__global__ __launch_bounds__(256) void q4_read_kernel(RowsKernelArgs a)
{
    const uint32_t v = blockIdx.x * (256u >> LOGW) + (threadIdx.x >> LOGW), o = threadIdx.x & ((1u << LOGW) - 1u);
    if (v >= a.total) return;
    const Place p = place_of(v, a);
    const RowsSide &s = a.side[0];
    half2v pair[4] = {};
    if (p.row >= 0) {
        const uint32_t block = p.b * a.by_h.div + p.h, g = (8 * o) >> s.log_group, groups = (8u << LOGW) >> s.log_group;
        word_values(s.codes[((int64_t)block * a.T + p.row) * (1 << LOGW) + o], s.params[((int64_t)block * groups + g) * a.T + p.row], pair);
    }
    store8<OUT>(s.out, (int64_t)p.b * s.ob + (int64_t)p.h * s.oh + (int64_t)p.t * s.ot + 8 * o, pair);
}

RowsKernelArgs kernel_args(const Q4RowsArgs &r, int sides)
{
    RowsKernelArgs a{};
    for (int k = 0; k < sides; ++k) {
        const Q4RowsSide &s = r.side[k];
        a.side[k] = {s.x, static_cast<uint32_t *>(s.codes), static_cast<uint32_t *>(s.params), s.out, s.x_stride[0], s.x_stride[1], s.x_stride[2],
                     s.out_stride[0], s.out_stride[1], s.out_stride[2], s.group == 32 ? 5 : s.group == 64 ? 6 : 7};
    }
    a.pos = r.pos; a.counts = r.counts; a.pos0 = r.pos0;
    a.total = (uint32_t)((int64_t)sides * r.B * r.Hkv * r.n);
    a.n = (uint32_t)r.n; a.T = (uint32_t)r.T; a.B = (uint32_t)r.B;
    a.by_n = fast_div((uint32_t)r.n); a.by_h = fast_div((uint32_t)r.Hkv); a.by_b = fast_div((uint32_t)r.B);
    return a;
}

template <int DT, int OUT> hipError_t write(const Q4RowsArgs &r, int sides)
{
    const RowsKernelArgs a = kernel_args(r, sides);
    const unsigned groups = (unsigned)(((uint64_t)a.total * (r.d / 8) + 255) / 256);
    if (r.d == 128) hipLaunchKernelGGL((q4_write_kernel<DT, OUT, 4>), dim3(groups), dim3(256), 0, r.stream, a);
    else hipLaunchKernelGGL((q4_write_kernel<DT, OUT, 3>), dim3(groups), dim3(256), 0, r.stream, a);
    return hipGetLastError();
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
    const RowsKernelArgs a = kernel_args(r, 1);
    const unsigned groups = (unsigned)(((uint64_t)a.total * (r.d / 8) + 255) / 256);
    if (r.d == 128) hipLaunchKernelGGL((q4_read_kernel<OUT, 4>), dim3(groups), dim3(256), 0, r.stream, a);
    else hipLaunchKernelGGL((q4_read_kernel<OUT, 3>), dim3(groups), dim3(256), 0, r.stream, a);
    return hipGetLastError();
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
