"""Calls of the 4-bit cache that would write one place twice are refused, and layouts that only look like it are not: on the host, before
anything is launched."""
import ctypes
import itertools

import numpy as np
import pytest
import torch

import paper_2412_11741_amd as csr
from paper_2412_11741_amd import binding as B
from tests.test_q4_reference import FAKE, _attn, _rows


def _read(desc, out=FAKE):
    """The status of csr_q4_read with an output that is misaligned: where the descriptor passes, that is what is refused"""
    status = csr.lib().csr_q4_read(ctypes.byref(desc), FAKE, FAKE, out, None, None, None)
    return status, csr.last_error()


ODD = ctypes.c_void_p(0x1008)   # 8-byte aligned: refused after the descriptor has been looked at


@pytest.mark.parametrize("b,h,t", [(1280, 128, 128), (1280, 640, 640), (640, 640, 128), (128, 1280, 248), (1272, 640, 128), (1280, 256, 384)])
def test_outputs_whose_rows_overlap_are_refused(b, h, t):
    status, words = _read(_rows(out_stride_b=b, out_stride_h=h, out_stride_t=t))
    assert status == B.CSR_ERR_INVALID_ARG and "overlap" in words
    d = _rows(out_stride_b=b, out_stride_h=h, out_stride_t=t)
    assert csr.lib().csr_q4_write(ctypes.byref(d), FAKE, FAKE, FAKE, FAKE, None, None, None, None, None, None, None, None) == B.CSR_ERR_INVALID_ARG
    assert "overlap" in csr.last_error()
    a = _attn(Hq=2, Tq=5, out_stride_b=b, out_stride_h=h, out_stride_t=t)
    assert csr.lib().csr_q4_attn_workspace_bytes(ctypes.byref(a)) == ctypes.c_size_t(-1).value and "overlap" in csr.last_error()


@pytest.mark.parametrize("order", list(itertools.permutations(range(3))))
@pytest.mark.parametrize("gap", [0, 8, 384])
def test_outputs_of_any_order_and_spacing_are_taken(order, gap):
    size, stride, span = (2, 2, 5), [0, 0, 0], 128
    for k in order:
        stride[k] = span + gap
        span += stride[k] * (size[k] - 1)
    seen = {tuple(np.dot(i, stride) + np.arange(0, 128, 8)) for i in itertools.product(*map(range, size))}
    assert len(set(itertools.chain(*seen))) == 20 * 16            # no place twice
    status, words = _read(_rows(out_stride_b=stride[0], out_stride_h=stride[1], out_stride_t=stride[2]), ODD)
    assert status == B.CSR_ERR_INVALID_ARG and "aligned" in words
    a = _attn(Hq=2, Tq=5, out_stride_b=stride[0], out_stride_h=stride[1], out_stride_t=stride[2])
    assert csr.lib().csr_q4_attn_workspace_bytes(ctypes.byref(a)) != ctypes.c_size_t(-1).value


def test_a_dimension_of_one_has_any_stride():
    status, words = _read(_rows(B=1, n=1, out_stride_b=0, out_stride_h=128, out_stride_t=0), ODD)
    assert status == B.CSR_ERR_INVALID_ARG and "aligned" in words


def _write(codes, params, codes2, params2, out=None, out2=None):
    d, d2 = _rows(), _rows()
    p = lambda at: None if at is None else ctypes.c_void_p(at)
    return csr.lib().csr_q4_write(ctypes.byref(d), FAKE, p(codes), p(params), p(out), ctypes.byref(d2), FAKE, p(codes2), p(params2), p(out2), None, None, None)


CODES, PARAMS = 2 * 2 * 9 * 64, 2 * 2 * 2 * 9 * 4   # bytes of the caches of _rows()


@pytest.mark.parametrize("at", [(0x10000, 0x20000, 0x10000, 0x30000), (0x10000, 0x20000, 0x10000 + CODES - 16, 0x30000),
                                (0x10000, 0x20000, 0x10000 - CODES + 16, 0x30000), (0x10000, 0x20000, 0x40000, 0x20000),
                                (0x10000, 0x20000, 0x40000, 0x20000 + PARAMS - 4), (0x10000, 0x20000, 0x20000, 0x30000), (0x10000, 0x20000, 0x40000, 0x10000)])
def test_keys_and_values_into_one_cache_are_refused(at):
    assert _write(*at) == B.CSR_ERR_INVALID_ARG and "same cache" in csr.last_error()


def test_keys_and_values_into_one_output_are_refused():
    assert _write(0x10000, 0x20000, 0x40000, 0x50000, 0x60000, 0x60000) == B.CSR_ERR_INVALID_ARG and "out2" in csr.last_error()


def test_a_workspace_has_no_more_bytes_than_its_memory():
    byte = lambda n: torch.empty(n, dtype=torch.uint8)
    assert B._room(None) == 0 and B._room(byte(4096)) == 4096 and B._room(torch.empty(64, dtype=torch.float32)) == 256
    assert B._room(byte(256).expand(1 << 20, 256)) == 256 and B._room(byte(4096)[256:].expand(9, 3840)) == 3840
    assert B._room(byte(4096)[1024:2048]) == 1024 and B._room(byte(0)) == 0 and B._room(byte(4096)[::2]) == 2048


def test_a_first_row_that_64_bits_do_not_hold_is_refused():
    desc = lambda pos0: B._q4_rows_desc(None, None, 1, 1, 1, 8, 64, 32, pos0, torch.float16)
    assert desc(5).pos0 == 5 and desc(-(1 << 63)).pos0 == -(1 << 63) and desc(np.int32(7)).pos0 == 7
    for pos0 in (1 << 63, 1 << 64, (1 << 64) + 3, -(1 << 64)):    # (the last three would be rows 0, 3 and 0)
        with pytest.raises(ValueError, match="pos0"):
            desc(pos0)
    with pytest.raises(TypeError):
        desc(2.5)
