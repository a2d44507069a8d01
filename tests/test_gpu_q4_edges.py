"""The 4-bit cache on the GPU where its arithmetic is tightest: values next to the middle of two codes, scores of any size."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2412_11741_amd as csr
from paper_2412_11741_amd import binding
from tests import q4_reference as ref
from tests.q4_plan import plan
from tests.test_gpu_q4 import _bound, _check, _filled, _np, _randn

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def _written(X, group):
    """Codes and parameters of rows X, as the library writes them"""
    c, p = csr.csr_q4_alloc(X.shape[0], X.shape[1], X.shape[2], X.shape[3], group)
    csr.csr_q4_write(X, c, p)
    return c.cpu().numpy(), p.cpu().numpy()


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_middles_moved_by_a_minimum_far_below_a_step(dtype, group):
    # The minimum is 2^-24 to 2^-18, a step 2^-3 to 2^5: a value on the middle of two codes above zero is off the middle by the minimum, less than
    # the difference's rounding holds.  Middles above even codes and above odd ones, either sign of the minimum (bf16, whose 15 steps
    # and a little are too many: below zero).
    n, d = 96, 128
    r = np.random.default_rng(group)
    x = np.zeros((1, 1, n, d))
    for t in range(n):
        for g in range(d // group):
            s, m = 2.0 ** r.integers(-3, 6), r.choice([-1.0, 1.0 if dtype != BF16 else -1.0]) * 2.0 ** r.integers(-24, -17)
            u = r.integers(0, 15, group) + 0.5
            u[0] = 15.0078125 if dtype != BF16 else 15.0         # the scale is s
            x[0, 0, t, g * group:(g + 1) * group] = s * u
            x[0, 0, t, g * group + 1] = m
    X = torch.from_numpy(x).to(dtype)
    want_codes, want_params = ref.quantise(X.double().numpy(), group)
    exact = np.moveaxis(want_params[..., 0], -2, -1).astype(np.float64)       # the scales are powers of two: the quotients are exact in 64 bits
    assert (np.frexp(exact)[0] == 0.5).all()
    codes, params = _written(X.cuda(), group)
    assert (codes == want_codes).all() and (params == want_params).all()


@pytest.mark.parametrize("dtype", [F16, F32])
def test_values_a_step_of_their_type_off_a_middle(dtype):
    # scales of any fraction, minima from none to tens of steps; every value the type's nearest to a middle or one of its neighbours
    n, d, group = 300, 64, 32
    r = np.random.default_rng(11)
    x = np.zeros((1, 1, n, d))
    to = np.float16 if dtype == F16 else np.float32
    for t in range(n):
        for g in range(d // group):
            s = 2.0 ** r.integers(-8, 5) * r.integers(1024, 2048) / 1024
            m = float(np.float16(r.choice([2.0 ** -24, -2.0 ** -20, 2.0 ** -18, s * r.uniform(-20, 20), 0.0])))
            u = to(m + s * (r.integers(0, 15, group) + 0.5))
            for k, way in enumerate(r.integers(-1, 2, group)):
                if way:
                    u[k] = np.nextafter(u[k], to(np.inf * way))
            u[0], u[1] = m, to(m + 15.004 * s)
            x[0, 0, t, g * group:(g + 1) * group] = u
    X = torch.from_numpy(x).to(dtype)
    want_codes, want_params = ref.quantise(X.double().numpy(), group)
    codes, params = _written(X.cuda(), group)
    assert (codes == want_codes).all() and (params == want_params).all()


# ---- attention: scores of any size --------------------------------------------------------------------------------------
# 16s of rows a workgroup, B, Hq, Hkv, T, Tq: a call for each kernel, with one part of the token axis and with several
KERNELS = [(1, 3, 8, 2, 517, 1), (1, 1, 8, 2, 6000, 1), (1, 2, 8, 2, 290, 90), (2, 128, 16, 4, 200, 7), (2, 1, 32, 4, 6000, 12),
           (4, 128, 16, 4, 400, 16), (4, 16, 64, 8, 6000, 5), (16, 128, 2, 2, 200, 150), (16, 2, 64, 8, 6000, 12)]
CALLS = [(shape, dtype) for shape in KERNELS for dtype in (F16, BF16, F32) if dtype != F32 or shape[0] <= 2]


def _against(q, cache, got, where, scale=0.0, size=None):
    """The output of sequences `where` against 64 bits; size: the error of a score that is granted is that of one so large (none for
    None: products and sums that are exact)"""
    k, v = (ref.values(cache[i][where].cpu().numpy(), cache[i + 1][where].cpu().numpy()) for i in (0, 2))
    B, Hq, Tq, d = q[where].shape
    T = k.shape[2]
    want, spread, sizes = ref.attention(_np(q[where]), k, v, [T] * B, [Tq] * B, scale or d ** -0.5, True)
    one_p = q.dtype == BF16 or (Tq * (Hq // k.shape[1]) > 16 and q.dtype != F32)
    off = np.abs(_np(got[where]) - want) / _bound(want, spread, 0 * sizes if size is None else sizes * size, T, d, q.dtype, got.dtype, one_p)
    assert np.isfinite(off).all() and off.max() <= 1, off.max()


@pytest.mark.parametrize("shape,dtype", [c for c in CALLS if c[1] != F16])
def test_rows_whose_scores_are_all_far_below_zero(shape, dtype):
    # Every score is -2^113 / sqrt(128) = -9.2e32, or half of that from a token on: powers of two times the unit, so that products, differences
    # and probabilities are exact.  Rows that see no token of the smaller score average the larger ones.
    tiles, B, Hq, Hkv, T, Tq = shape
    assert plan(B, Hq, Hkv, T, Tq, 128, {F32: 0, BF16: 2}[dtype])[0][0] == tiles
    cache = _filled(500, B, Hkv, T, 128, 32, 64)
    K = torch.full((B, Hkv, T, 128), 8.0, device="cuda")          # groups without spread read back as they are
    q = torch.zeros(B, Hq, Tq, 128, dtype=dtype, device="cuda")
    q[..., 5] = -2.0 ** 110
    where = [0, B - 1] if T < 1000 else [0]
    for first in (T, T - (Tq + 1) // 2, T // 3):
        K[:, :, first:] = 4.0
        csr.csr_q4_write(K, cache[0], cache[1])
        got = csr.csr_q4_attn(q, *cache, out_dtype=F32)
        _against(q, cache, got, where)


@pytest.mark.parametrize("shape,dtype", CALLS)
def test_scores_so_large_that_a_step_of_them_is_many_powers_of_two(shape, dtype):
    # Every token has one key, from a token on half of it: the tokens with the larger score share a row's weight evenly, the others have none.
    # Scores of 2^15 to 2^32 times log2(e), and of 2^116 (which fp16 queries do not reach), either sign; the products round.
    tiles, B, Hq, Hkv, T, Tq = shape
    d = 128
    assert plan(B, Hq, Hkv, T, Tq, d, {F32: 0, F16: 1, BF16: 2}[dtype])[0][0] == tiles
    cache = _filled(510, B, Hkv, T, d, 32, 64)
    v = torch.from_numpy(ref.values(cache[2][:1].cpu().numpy(), cache[3][:1].cpu().numpy())).double()[0].cuda().repeat_interleave(Hq // Hkv, dim=0)
    end = torch.arange(T - Tq + 1, T + 1, device="cuda")          # tokens that each query sees
    before = torch.cat([torch.zeros_like(v[:, :1]), v.cumsum(1)], 1), torch.cat([torch.zeros_like(v[:, :1]), v.abs().cumsum(1)], 1)
    mean = lambda sums, low, high: (sums[:, high] - sums[:, low]) / (high - low).clamp(min=1)[:, None]
    key, query = _randn(511, 1, 1, 1, d, dtype=F32).abs() + 1, _randn(512, B, Hq, Tq, d, dtype=F32).abs() + 1
    one_p = dtype == BF16 or (Tq * (Hq // Hkv) > 16 and dtype != F32)
    for first in (T, T - (Tq + 1) // 2, T // 3):
        for a, b in [(0, 10), (4, 10), (7, 10), (10, 10), (13, 10), (13, 13)] + [(100, 10)] * (dtype != F16):
            K = (key * 2.0 ** b).expand(B, Hkv, T, d).clone()
            K[:, :, first:] *= 0.5
            csr.csr_q4_write(K, cache[0], cache[1])
            for sign in (1.0, -1.0):
                got = csr.csr_q4_attn((query * sign * 2.0 ** a).to(dtype), *cache, out_dtype=F32)[0].double()
                low, high = torch.zeros_like(end), end.clamp(max=first)
                if sign < 0:
                    low, high = torch.where(end > first, first, 0), end
                want, spread = mean(before[0], low, high), mean(before[1], low, high)
                bound = _bound(want.cpu().numpy(), spread.cpu().numpy(), np.zeros(want.shape[:2]), T, d, dtype, F32, one_p)
                off = (got - want).abs().cpu().numpy() / bound
                assert np.isfinite(off).all() and off.max() <= 1, (first, a, b, sign, off.max())


@pytest.mark.parametrize("Tq", [1, 40])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_the_largest_scales(dtype, Tq):
    # queries near the smallest normal float under scales up to the largest: scores of ordinary size
    cache = _filled(520, 1, 2, 200, 128, 64, 64)
    q = _randn(522, 1, 4, Tq, 128, dtype=F32, gain=2.0 ** -124).to(dtype)
    for scale in (1e37, 2.3e38, 2.4e38, 3.4e38):
        scale = float(np.float32(scale))
        _check(q, cache, csr.csr_q4_attn(q, *cache, scale=scale, out_dtype=F32), scale=scale)


@pytest.mark.parametrize("shape,dtype", CALLS)
def test_a_row_far_from_zero_changes_no_bit_of_the_others(shape, dtype):
    # keys of 2^8, queries of 2^-8 but for one head of the last token, whose scores of 2^22 take its wave to the maxima at every turn
    tiles, B, Hq, Hkv, T, Tq = shape
    cache = csr.csr_q4_alloc(B, Hkv, T, 128, 64) + csr.csr_q4_alloc(B, Hkv, T, 128, 64)
    csr.csr_q4_write(_randn(523, B, Hkv, T, 128, dtype=F32, gain=2.0 ** 8), cache[0], cache[1], _randn(524, B, Hkv, T, 128, dtype=F32), cache[2], cache[3])
    q = _randn(528, B, Hq, Tq, 128, dtype=F32, gain=2.0 ** -8).to(dtype)
    want = csr.csr_q4_attn(q, *cache)
    loud = q.clone()
    loud[:, 0, -1] *= 2.0 ** 20
    got = csr.csr_q4_attn(loud, *cache)
    assert torch.isfinite(got).all() and not torch.equal(got[:, 0, -1], want[:, 0, -1])
    got[:, 0, -1] = want[:, 0, -1]
    assert torch.equal(got, want)


@pytest.mark.parametrize("shape,dtype", CALLS)
def test_scales_next_to_nothing(shape, dtype):
    # scales at which the number that stands for no token yet is itself a score of ordinary size: every token weighs nearly the same
    tiles, B, Hq, Hkv, T, Tq = shape
    cache = _filled(525, B, Hkv, T, 128, 32, 64)
    q = _randn(527, B, Hq, Tq, 128, dtype=dtype)
    for scale in (1e-38, 1e-20, 1e-13, 3e-12, 5e-12, 1e-11, 1e-9) if T < 1000 else (3e-12,):
        scale = float(np.float32(scale))
        _against(q, cache, csr.csr_q4_attn(q, *cache, scale=scale, out_dtype=F32), [B - 1], scale=scale, size=1.0)


# ---- what lies side by side ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("d,gk,gv", [(128, 32, 128), (64, 64, 32)])
def test_caches_and_outputs_next_to_each_other(d, gk, gv):
    # keys' and values' codes in one array, their parameters in another, what they stand for by turns in a third
    B, Hkv, n, T = 2, 3, 37, 41
    K, V = _randn(530, B, Hkv, n, d), _randn(531, B, Hkv, n, d)
    codes = torch.zeros(2, B, Hkv, T, d // 2, dtype=torch.uint8, device="cuda")
    params = torch.zeros(B * Hkv * T * 2 * (d // gk + d // gv), dtype=F16, device="cuda")
    cut = B * Hkv * T * 2 * (d // gk)
    pK, pV = params[:cut].view(B, Hkv, d // gk, T, 2), params[cut:].view(B, Hkv, d // gv, T, 2)
    out = torch.zeros(B, n, 2, Hkv, d, dtype=F16, device="cuda")
    csr.csr_q4_write(K, codes[0], pK, V, codes[1], pV, outK=out[:, :, 0].transpose(1, 2), outV=out[:, :, 1].transpose(1, 2))
    for k, (X, p, g) in enumerate(((K, pK, gk), (V, pV, gv))):
        c, p1 = csr.csr_q4_alloc(B, Hkv, T, d, g)
        want = csr.csr_q4_write(X, c, p1, values=True)
        assert torch.equal(codes[k], c) and torch.equal(p, p1) and torch.equal(out[:, :, k].transpose(1, 2), want)
    with pytest.raises(csr.CsrError, match="same cache"):
        csr.csr_q4_write(K, codes[0], pK, V, codes[0], pK)


def test_a_workspace_of_more_elements_than_memory_is_refused():
    cache = _filled(540, 1, 2, 6000, 128, 64, 64)
    q = _randn(542, 1, 8, 128)
    desc = csr.q4_attn_desc(q.unsqueeze(2), cache[0], cache[1], cache[3], torch.empty_like(q).unsqueeze(2))
    need = csr.csr_q4_attn_workspace_bytes(desc)
    assert need > 512
    with pytest.raises(csr.CsrError, match="workspace"):
        csr.csr_q4_attn(q, *cache, workspace=torch.empty(256, dtype=torch.uint8, device="cuda").expand(need, 256))
    half = torch.empty(need // 2 * 4 + 4096, dtype=torch.uint8, device="cuda")[::2]   # every second byte: enough
    assert torch.equal(csr.csr_q4_attn(q, *cache, workspace=half), csr.csr_q4_attn(q, *cache))


def test_strides_that_play_no_part():
    # of X in csr_q4_read, of out in csr_q4_write without one, of dimensions of one: any numbers
    B, Hkv, n, d, wild = 1, 2, 300, 128, (1 << 63) - 1
    X = _randn(550, B, Hkv, n, d)
    c, p = csr.csr_q4_alloc(B, Hkv, n, d, 64)
    want_c, want_p = csr.csr_q4_alloc(B, Hkv, n, d, 64)
    want = csr.csr_q4_write(X, want_c, want_p, values=True)
    desc = binding.Q4RowsDesc(B=B, Hkv=Hkv, n=n, T=n, d=d, group=64, x_dtype=binding.CSR_F16, x_stride_b=wild, x_stride_h=n * d, x_stride_t=d,
                              out_dtype=binding.CSR_F16, out_stride_b=wild, out_stride_h=-wild, out_stride_t=wild, pos0=0, flags=0)
    ptr, L, stream = binding._ptr, csr.lib(), binding._stream()
    assert L.csr_q4_write(ctypes.byref(desc), ptr(X), ptr(c), ptr(p), None, None, None, None, None, None, None, None, stream) == binding.CSR_OK
    assert torch.equal(c, want_c) and torch.equal(p, want_p)
    out = torch.empty_like(X)
    desc.x_dtype, desc.x_stride_b, desc.x_stride_h, desc.x_stride_t = 77, -wild, wild, wild
    desc.out_stride_h, desc.out_stride_t = n * d, d
    assert L.csr_q4_read(ctypes.byref(desc), ptr(c), ptr(p), ptr(out), None, None, stream) == binding.CSR_OK
    assert torch.equal(out, want)


# ---- probabilities: what a kernel keeps of them -------------------------------------------------------------------------
def _kept(one_p):
    """The part of a probability, and of the row's largest one, that its rounding may cost: one fp16 at 2^8 of the maximum (11 bits, and
    half of fp16's smallest step), or two at 2^12"""
    return (2.0 ** -11, 2.0 ** -33) if one_p else (2.0 ** -21, 2.0 ** -37)


# 16s of rows a workgroup, B, Hq, Hkv, T, Tq
TAILS = [((1, 1, 8, 2, 40000, 1), F16), ((1, 1, 8, 2, 40000, 1), BF16), ((1, 1, 8, 2, 40000, 1), F32), ((2, 16, 32, 8, 40000, 5), F16),
         ((2, 16, 32, 8, 40000, 5), BF16), ((2, 1, 32, 4, 40000, 12), F32), ((4, 16, 64, 8, 40000, 5), F16), ((4, 16, 64, 8, 40000, 5), BF16),
         ((16, 2, 64, 8, 40000, 12), F16), ((16, 2, 64, 8, 40000, 12), BF16)]


@pytest.mark.parametrize("shape,dtype", TAILS)
def test_a_long_tail_of_small_probabilities(shape, dtype):
    # One token, whose value is zero, and 40000 others far below it that are all there is in the output: each 2^-13 of the largest probability to
    # 2^-30.  What a kernel leaves out of them, of the products or of the sum, shows whole.
    tiles, B, Hq, Hkv, T, Tq = shape
    d = 128
    assert plan(B, Hq, Hkv, T, Tq, d, {F32: 0, F16: 1, BF16: 2}[dtype])[0][0] == tiles
    cache = csr.csr_q4_alloc(B, Hkv, T, d, 32) + csr.csr_q4_alloc(B, Hkv, T, d, 32)
    one_p = dtype == BF16 or (dtype == F16 and tiles > 1)
    relative, absolute = _kept(one_p)
    end = torch.arange(T - Tq + 1, T + 1, device="cuda")
    q = torch.zeros(B, Hq, Tq, d, dtype=dtype, device="cuda")
    q[..., 0] = 16.0
    for at in (0, T - Tq):                                        # the first token, and one that every query sees last but its own
        V = _randn(560, 1, 1, T, d, dtype=F32) + 1.0
        V[:, :, at] = 0.0
        csr.csr_q4_write(V.expand(B, Hkv, T, d), cache[2], cache[3])
        v = csr.csr_q4_read(cache[2][:1, :1].contiguous(), cache[3][:1, :1].contiguous(), out_dtype=F32)[0, 0].double()
        sums, sizes = v.cumsum(0)[end - 1], v.abs().cumsum(0)[end - 1]
        for bits in (13, 19, 23, 26, 30):
            K = torch.zeros(1, 1, T, d, device="cuda")
            K[:, :, at, 0] = bits * np.log(2.0) * d ** 0.5 / 16.0
            csr.csr_q4_write(K.expand(B, Hkv, T, d), cache[0], cache[1])
            high = float(csr.csr_q4_read(cache[0][:1, :1].contiguous(), cache[1][:1, :1].contiguous(), out_dtype=F32)[0, 0, at, 0])
            score = high * 16.0 * d ** -0.5
            w = np.exp(-score)                                    # of a token of the tail, for 1 of the largest
            all_of = 1.0 + w * (end - 1).double()
            got = csr.csr_q4_attn(q, *cache, out_dtype=F32)[0].double()
            want = w * sums / all_of[:, None]
            spread, total = w * sizes / all_of[:, None], sizes / all_of[:, None]
            error = 2 * (score * (d + 4) * 2.0 ** -24 + 16 * 2.0 ** -24) + relative + (2 * (T / 32 * 8 + 64) + 8) * 2.0 ** -24
            bound = 1.01 * (spread * error + total * absolute + want.abs() * (T * absolute)) + 1e-30
            off = ((got - want).abs() / bound).max().item()
            assert off <= 1, (at, bits, off)


# B, Hq, Hkv, T, Tq, d: several workgroups along a KV head's rows, 16 each, because there are few pairs
SIXTEENS = [(2, 8, 2, 290, 90, 128), (1, 40, 2, 300, 1, 128), (1, 4, 4, 100, 64, 64), (1, 8, 2, 700, 33, 128), (1, 2, 1, 260, 260, 128), (2, 6, 2, 400, 50, 64)]


@pytest.mark.parametrize("shape", SIXTEENS)
def test_sixteen_rows_a_workgroup_keep_two_fp16_of_a_probability(shape):
    B, Hq, Hkv, T, Tq, d = shape
    (tiles, blocks, _, _), _ = plan(B, Hq, Hkv, T, Tq, d, 1)
    assert tiles == 1 and blocks > 1
    cache = _filled(570, B, Hkv, T, d, 32, 32)
    q = _randn(572, B, Hq, Tq, d)
    got = csr.csr_q4_attn(q, *cache, out_dtype=F32)
    k, v = (ref.values(cache[i].cpu().numpy(), cache[i + 1].cpu().numpy()) for i in (0, 2))
    want, spread, size = ref.attention(_np(q), k, v, [T] * B, [Tq] * B, d ** -0.5, True)
    bound = _bound(want, spread, size, T, d, F16, F32, False) + _kept(False)[1] * np.abs(v.astype(np.float64)).sum(axis=2).max()
    off = np.abs(_np(got) - want) / bound
    assert np.isfinite(off).all() and off.max() <= 1, off.max()


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_one_query_for_all_heads_and_tokens(dtype):
    # queries of stride 0, along heads and along tokens
    cache = _filled(580, 2, 2, 150, 128, 32, 64)
    one = _randn(582, 2, 1, 1, 128, dtype=dtype)
    for Hq, Tq in ((8, 1), (4, 9), (2, 70)):
        q = one.expand(2, Hq, Tq, 128)
        assert torch.equal(csr.csr_q4_attn(q, *cache), csr.csr_q4_attn(q.contiguous(), *cache))
