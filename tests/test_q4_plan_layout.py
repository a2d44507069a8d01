"""tests/q4_plan.py asks the library with structures of its own: what it reads has to be what the public call answers."""
import ctypes
import random

import pytest

import paper_2412_11741_amd as csr
from paper_2412_11741_amd import binding as B
from tests.q4_plan import plan


@pytest.mark.parametrize("seed", range(4))
def test_the_plan_that_tests_read_is_the_librarys(seed):
    r = random.Random(seed)
    several = 0
    for _ in range(200):
        b, Hkv, G, d, dtype = r.randint(1, 64), r.choice([1, 2, 8, 32]), r.choice([1, 3, 4, 8]), r.choice([64, 128]), r.choice([0, 1, 2])
        T, Tq = int(2 ** r.uniform(0, 17)), int(2 ** r.uniform(0, 9))
        Hq = Hkv * G
        desc = B.Q4AttnDesc(B=b, Hq=Hq, Hkv=Hkv, Tq=Tq, T=T, d=d, group_k=64, group_v=64, scale=0.0, q_dtype=dtype, out_dtype=dtype, q_stride_b=Hq * Tq * d,
                            q_stride_h=Tq * d, q_stride_t=d, out_stride_b=Hq * Tq * d, out_stride_h=Tq * d, out_stride_t=d, flags=0)
        (tiles, blocks, splits, alone), total = plan(b, Hq, Hkv, T, Tq, d, dtype)
        assert total == csr.csr_q4_attn_workspace_bytes(desc)
        up = lambda n: -(-n // 256) * 256
        parts = b * Hkv * G * Tq * splits
        assert total == (up(parts * d * 4) + up(parts * 8) if splits > 1 else 0)
        assert tiles in (1, 2, 4, 16) and blocks == -(-G * Tq // (16 * tiles)) and alone in (False, True)
        several += splits > 1
    assert 20 < several < 180
