"""The 4-bit cache on the GPU where its arithmetic is tightest: values next to the middle of two codes."""
import numpy as np
import pytest
import torch

import paper_2412_11741_amd as csr
from tests import q4_reference as ref

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
