"""The reference of the 4-bit cache against closed forms, and the host side of the calls: refusals before anything is launched."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2412_11741_amd as csr
from paper_2412_11741_amd import binding as B
from tests import q4_reference as ref


def test_whole_numbers_come_back():
    x = np.tile(np.arange(16.0), (3, 8)) * 0.25 - 2.0
    codes, params = ref.quantise(x, 32)
    assert (params[..., 0] == 0.25).all() and (params[..., 1] == -2.0).all()
    assert (ref.values(codes, params) == x).all()
    assert (codes[0, :8] == np.array([0x10, 0x32, 0x54, 0x76, 0x98, 0xba, 0xdc, 0xfe])).all()   # channel 2j low, 2j + 1 high


def test_halves_go_to_the_even_code():
    x = np.zeros((1, 32))
    x[0, :6] = 15.0, 0.5, 1.5, 2.5, 13.5, 14.5                    # s = 1, m = 0
    codes, params = ref.quantise(x, 32)
    assert params[0, 0, 0] == 1.0
    assert ref.values(codes, params)[0, :6].tolist() == [15.0, 0.0, 2.0, 2.0, 14.0, 14.0]


@pytest.mark.parametrize("group", [32, 64, 128])
def test_the_error_is_half_a_step_and_the_cut_of_the_scale(group):
    r = np.random.default_rng(group)
    x = (r.standard_normal((50, 128)) * 10.0 ** r.integers(-3, 4, (50, 1))).astype(np.float16)
    codes, params = ref.quantise(x, group)
    s = np.repeat(np.moveaxis(params[..., 0].astype(np.float64), 0, 1), group, axis=1)
    # the largest values are cut by 15 steps' worth of the scale's rounding (2^-10 of a normal scale); the value itself is an fp16
    limit = 0.5 * s + 15 * np.maximum(s * 2.0 ** -10, 2.0 ** -24) + np.abs(x).max(axis=1, keepdims=True) * 2.0 ** -11
    assert (np.abs(ref.values(codes, params).astype(np.float64) - x) <= limit).all()


def test_the_largest_values_and_no_finite_ones():
    x = np.zeros((4, 64), dtype=np.float32)
    x[0, :2] = 65504, -65504
    x[1, 3], x[2, 40], x[3, 0] = np.nan, np.inf, 1e30
    v = ref.values(*ref.quantise(x, 32))
    assert np.isfinite(v[0]).all() and v[0, 1] == -65504 and v[0, 0] <= 65504
    assert np.isnan(v[1, :32]).all() and np.isnan(v[2, 32:]).all() and (v[1, 32:] == 0).all() and (v[2, :32] == 0).all()
    assert v[3, 0] > 65000 and np.isfinite(v[3]).all()


def test_attention_is_that_of_pytorch():
    r = np.random.default_rng(0)
    q, k, v = (r.standard_normal(s) for s in ((2, 6, 3, 64), (2, 2, 11, 64), (2, 2, 11, 64)))
    out, spread, _ = ref.attention(q, k, v, [11, 7], [3, 2], 0.125, True)
    t = [torch.from_numpy(a) for a in (q, k.repeat(3, 1), v.repeat(3, 1))]
    for b, (n, qn) in enumerate([(11, 3), (7, 2)]):
        mask = torch.ones(qn, n).tril(n - qn).bool()
        want = torch.nn.functional.scaled_dot_product_attention(t[0][b, :, :qn], t[1][b, :, :n], t[2][b, :, :n], attn_mask=mask)
        assert np.allclose(out[b, :, :qn], want.numpy(), rtol=1e-12, atol=1e-13) and (out[b, :, qn:] == 0).all()
    assert (spread >= np.abs(out) - 1e-12).all()


# ---- refusals -----------------------------------------------------------------------------------------------------------
FAKE = ctypes.c_void_p(0x1000)   # never dereferenced


def _rows(**kw):
    base = dict(B=2, Hkv=2, n=5, T=9, d=128, group=64, x_dtype=B.CSR_F16, x_stride_b=1280, x_stride_h=640, x_stride_t=128,
                out_dtype=B.CSR_F16, out_stride_b=1280, out_stride_h=640, out_stride_t=128, pos0=0, flags=0)
    base.update(kw)
    return B.Q4RowsDesc(**base)


BAD_ROWS = [
    (dict(B=-1), B.CSR_ERR_INVALID_ARG), (dict(n=-1), B.CSR_ERR_INVALID_ARG), (dict(T=-1), B.CSR_ERR_INVALID_ARG),
    (dict(Hkv=0), B.CSR_ERR_INVALID_ARG), (dict(flags=1), B.CSR_ERR_INVALID_ARG), (dict(out_dtype=3), B.CSR_ERR_INVALID_ARG),
    (dict(d=96), B.CSR_ERR_UNSUPPORTED), (dict(d=256), B.CSR_ERR_UNSUPPORTED), (dict(group=16), B.CSR_ERR_UNSUPPORTED),
    (dict(d=64, group=128), B.CSR_ERR_UNSUPPORTED), (dict(group=96), B.CSR_ERR_UNSUPPORTED), (dict(T=(1 << 20) + 1), B.CSR_ERR_UNSUPPORTED),
    (dict(pos0=1 << 41), B.CSR_ERR_INVALID_ARG), (dict(n=(1 << 26) + 1), B.CSR_ERR_UNSUPPORTED), (dict(B=1 << 20, Hkv=1 << 11), B.CSR_ERR_UNSUPPORTED),
    (dict(out_stride_t=64), B.CSR_ERR_INVALID_ARG), (dict(out_stride_h=644), B.CSR_ERR_INVALID_ARG), (dict(out_stride_b=-1280), B.CSR_ERR_INVALID_ARG),
    (dict(out_stride_b=1 << 48), B.CSR_ERR_UNSUPPORTED),
]


@pytest.mark.parametrize("kw,status", BAD_ROWS + [
    (dict(x_dtype=3), B.CSR_ERR_INVALID_ARG), (dict(x_stride_t=132), B.CSR_ERR_INVALID_ARG), (dict(x_stride_h=-640), B.CSR_ERR_INVALID_ARG),
    (dict(x_dtype=B.CSR_F32, x_stride_t=130), B.CSR_ERR_INVALID_ARG)])
def test_write_refuses_bad_descriptors(kw, status):
    d = _rows(**kw)
    assert csr.lib().csr_q4_write(ctypes.byref(d), FAKE, FAKE, FAKE, FAKE, None, None, None, None, None, None, None, None) == status
    assert "csr_q4_write" in csr.last_error()


@pytest.mark.parametrize("kw,status", BAD_ROWS)
def test_read_refuses_bad_descriptors(kw, status):
    d = _rows(x_dtype=77, **kw)                                    # X plays no part
    assert csr.lib().csr_q4_read(ctypes.byref(d), FAKE, FAKE, FAKE, None, None, None) == status
    assert "csr_q4_read" in csr.last_error()


def test_write_and_read_refuse_bad_pointers_and_pairs():
    L, d, one = csr.lib(), ctypes.byref(_rows()), ctypes.c_void_p(0x1004)
    odd = ctypes.c_void_p(0x1002)
    none = [None] * 5
    write = lambda *a: L.csr_q4_write(*a)
    for args in ([d, None, FAKE, FAKE, None], [d, FAKE, None, FAKE, None], [d, FAKE, FAKE, None, None], [d, one, FAKE, FAKE, None],
                 [d, FAKE, one, FAKE, None], [d, FAKE, FAKE, odd, None], [d, FAKE, FAKE, FAKE, one], [None, FAKE, FAKE, FAKE, None]):
        assert write(*args, *none, None, None, None) == B.CSR_ERR_INVALID_ARG, args
    assert write(d, FAKE, FAKE, FAKE, None, *none, odd, None, None) == B.CSR_ERR_INVALID_ARG
    for other in (dict(n=4), dict(T=10), dict(x_dtype=B.CSR_BF16), dict(out_dtype=B.CSR_F32), dict(pos0=1), dict(B=1)):
        assert write(d, FAKE, FAKE, FAKE, None, ctypes.byref(_rows(**other)), FAKE, FAKE, FAKE, None, None, None, None) == B.CSR_ERR_INVALID_ARG
    assert write(d, FAKE, FAKE, FAKE, FAKE, d, FAKE, FAKE, FAKE, None, None, None, None) == B.CSR_ERR_INVALID_ARG    # one out of two
    assert write(d, FAKE, FAKE, FAKE, None, None, FAKE, None, None, None, None, None, None) == B.CSR_ERR_INVALID_ARG  # no descriptor
    for args in ([FAKE, FAKE, None], [None, FAKE, FAKE], [FAKE, None, FAKE], [one, FAKE, FAKE], [FAKE, odd, FAKE], [FAKE, FAKE, one]):
        assert L.csr_q4_read(d, *args, None, None, None) == B.CSR_ERR_INVALID_ARG, args
    # nothing to do: nothing is looked at
    for kw in (dict(B=0), dict(n=0)):
        assert write(ctypes.byref(_rows(**kw)), *[None] * 12) == B.CSR_OK
        assert L.csr_q4_read(ctypes.byref(_rows(**kw)), *[None] * 6) == B.CSR_OK


def _attn(**kw):
    base = dict(B=2, Hq=8, Hkv=2, Tq=3, T=1000, d=128, group_k=64, group_v=32, scale=0.0, q_dtype=B.CSR_F16, out_dtype=B.CSR_F16,
                q_stride_b=24 * 128, q_stride_h=384, q_stride_t=128, out_stride_b=24 * 128, out_stride_h=384, out_stride_t=128, flags=0)
    base.update(kw)
    return B.Q4AttnDesc(**base)


@pytest.mark.parametrize("kw,status", [
    (dict(B=-1), B.CSR_ERR_INVALID_ARG), (dict(Tq=-1), B.CSR_ERR_INVALID_ARG), (dict(T=-1), B.CSR_ERR_INVALID_ARG), (dict(Hq=7), B.CSR_ERR_INVALID_ARG),
    (dict(Hkv=0), B.CSR_ERR_INVALID_ARG), (dict(flags=2), B.CSR_ERR_INVALID_ARG), (dict(q_dtype=3), B.CSR_ERR_INVALID_ARG),
    (dict(out_dtype=-1), B.CSR_ERR_INVALID_ARG), (dict(scale=-1.0), B.CSR_ERR_INVALID_ARG), (dict(scale=float("nan")), B.CSR_ERR_INVALID_ARG),
    (dict(scale=float("inf")), B.CSR_ERR_INVALID_ARG), (dict(d=96), B.CSR_ERR_UNSUPPORTED), (dict(group_k=256), B.CSR_ERR_UNSUPPORTED),
    (dict(d=64, group_v=128), B.CSR_ERR_UNSUPPORTED), (dict(T=(1 << 20) + 1), B.CSR_ERR_UNSUPPORTED), (dict(B=65536), B.CSR_ERR_UNSUPPORTED),
    (dict(Tq=1 << 27), B.CSR_ERR_UNSUPPORTED), (dict(q_stride_t=100), B.CSR_ERR_INVALID_ARG), (dict(q_stride_h=-8), B.CSR_ERR_INVALID_ARG),
    (dict(out_stride_t=64), B.CSR_ERR_INVALID_ARG), (dict(out_stride_h=388), B.CSR_ERR_INVALID_ARG)])
def test_attention_refuses_bad_descriptors(kw, status):
    d = ctypes.byref(_attn(**kw))
    assert csr.lib().csr_q4_attn(d, *[FAKE] * 5, None, None, FAKE, None, 0, None) == status
    assert "csr_q4_attn" in csr.last_error()
    assert csr.lib().csr_q4_attn_workspace_bytes(d) == ctypes.c_size_t(-1).value


def test_attention_refuses_bad_pointers_and_small_workspaces():
    L, d = csr.lib(), _attn()
    need = L.csr_q4_attn_workspace_bytes(ctypes.byref(d))
    call = lambda ptrs, lens=None, out=FAKE, ws=FAKE, size=need: L.csr_q4_attn(ctypes.byref(d), *ptrs, lens, None, out, ws, size, None)
    for k in range(5):
        assert call([None if j == k else FAKE for j in range(5)]) == B.CSR_ERR_INVALID_ARG
    for k, p in ((0, 0x1008), (1, 0x1008), (2, 0x1002), (3, 0x1004), (4, 0x1001)):
        assert call([ctypes.c_void_p(p) if j == k else FAKE for j in range(5)]) == B.CSR_ERR_INVALID_ARG
    assert call([FAKE] * 5, out=None) == B.CSR_ERR_INVALID_ARG and call([FAKE] * 5, lens=ctypes.c_void_p(0x1002)) == B.CSR_ERR_INVALID_ARG
    assert need > 0                                                  # 1000 tokens of 4 KV heads are split
    assert call([FAKE] * 5, ws=None) == call([FAKE] * 5, size=need - 1) == call([FAKE] * 5, ws=ctypes.c_void_p(0x1080)) == B.CSR_ERR_WORKSPACE
    for kw in (dict(B=0), dict(Tq=0)):
        assert L.csr_q4_attn(ctypes.byref(_attn(**kw)), *[None] * 9, 0, None) == B.CSR_OK


def test_bytes_per_vector():
    assert csr.csr_q4_bytes(128, 32) == 80 and csr.csr_q4_bytes(128, 64) == 72 and csr.csr_q4_bytes(128, 128) == 68 and csr.csr_q4_bytes(64, 32) == 40
    assert csr.csr_q4_bytes(96, 32) == csr.csr_q4_bytes(64, 128) == csr.csr_q4_bytes(128, 16) == 0


def test_the_calls_take_no_host_tensors():
    codes, params = csr.csr_q4_alloc(1, 1, 4, 64, 32, device="cpu")
    assert codes.shape == (1, 1, 4, 32) and params.shape == (1, 1, 2, 4, 2) and params.dtype == torch.float16
    with pytest.raises(ValueError, match="GPU tensor"):
        csr.csr_q4_read(codes, params)
    with pytest.raises(ValueError, match="GPU tensor"):
        csr.csr_q4_write(torch.zeros(1, 1, 2, 64), codes, params)
    with pytest.raises(ValueError, match="GPU tensor"):
        csr.csr_q4_attn(torch.zeros(1, 1, 64), codes, params, codes, params)
    with pytest.raises(ValueError, match="group"):
        csr.csr_q4_alloc(1, 1, 4, 64, 128, device="cpu")
