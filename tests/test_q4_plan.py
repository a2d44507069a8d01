"""The rule that gives an attention call over the 4-bit cache its kernel and parts: what it promises whatever its figures are."""
import random

import pytest

from tests.q4_plan import plan


def test_each_kernel_has_its_calls():
    assert plan(1, 32, 8, 517, 1, 128)[0] == (1, 1, 1, True)            # a short context
    assert plan(4, 32, 32, 32768, 1, 128)[0][:2] == (1, 1)              # a long one
    assert plan(4, 32, 32, 32768, 1, 128)[0][2] > 1
    assert plan(16, 32, 8, 8192, 5, 128)[0][0] == 2                     # 20 rows
    assert plan(64, 32, 8, 2048, 16, 128)[0][0] == 4                    # 64 rows of many pairs
    assert plan(1, 32, 8, 10240, 2048, 128)[0][0] == 16                 # a prompt's chunk
    assert plan(1, 32, 8, 300, 300, 128)[0][0] == 1                     # a short prompt: workgroups are few
    assert plan(1, 32, 8, 10240, 2048, 128, dtype=0)[0][0] == 2         # fp32 has the two smallest only


@pytest.mark.parametrize("seed", range(8))
def test_launches_stay_within_limits(seed):
    r = random.Random(seed)
    for _ in range(400):
        Hkv, B = r.choice([1, 2, 8, 64, 65535]), r.choice([1, 2, 7, 64, 65535])
        most = max(1, 0x0fffffff // (B * Hkv))
        rows = max(1, min(most, int(2 ** r.uniform(0, 28))))
        G = r.choice([g for g in (1, 3, 4, 8) if g <= rows])
        T, d, dtype = r.choice([0, 1, 127, 129, 5000, 1 << 20]), r.choice([64, 128]), r.choice([0, 1, 2])
        (tiles, blocks, splits, alone), total = plan(B, Hkv * G, Hkv, T, rows // G, d, dtype)
        n = G * (rows // G)
        assert tiles in (1, 2, 4, 16) and splits in (1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128, 192, 256)
        assert blocks == -(-n // (16 * tiles))
        assert splits == 1 or splits <= -(-T // 128)
        along_x = blocks * splits * (B * Hkv * 512 if tiles == 16 else 512 if alone else 256)
        assert along_x < 1 << 32, (B, Hkv, n, T)
        assert not alone or (tiles, splits) == (1, 1)
        parts = B * Hkv * n * splits
        assert (total == 0) == (splits == 1) and (splits == 1 or total >= parts * (4 * d + 8))


def test_up_to_16_rows_there_is_one_kernel():
    assert all(plan(B, 4 * H, H, T, 1, 128)[0][0] == 1 for B in (1, 8, 64) for H in (1, 8, 32) for T in (1, 100, 4096, 1 << 20))
