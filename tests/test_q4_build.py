"""What the compiler made of the 4-bit cache's kernels: registers, from the metadata of the built library; needs no GPU."""
import re

from tests.test_build_resources import kernels  # noqa: F401


def test_the_attention_kernels_stay_in_registers(kernels):
    stream = {}
    for name, k in kernels.items():
        m = re.search(r"q4_stream_kernelILi(\d+)ELi(\d)ELi(\d)ELi(\d)E", name)
        if m:
            stream[tuple(map(int, m.groups()))] = k
    assert len(stream) == 2 * (3 * 3 + 2)   # heads of 64 and 128; three types of queries, fp32 without the four row tiles
    for (d, dtype, tiles, waves), k in stream.items():
        assert k["vgpr_spill_count"] <= (4 if (d, tiles) == (128, 4) else 0), (d, dtype, tiles, waves)
        # three waves to a SIMD for a row tile of fp16 or bf16 queries: what keeps enough requests in flight
        if tiles == 1 and dtype != 0:
            assert k["vgpr_count"] <= 168, (d, dtype, waves)
    prompt = {n: k for n, k in kernels.items() if "q4_prompt_kernel" in n}
    assert len(prompt) == 4 and all(k["vgpr_spill_count"] == 0 for k in prompt.values())


def test_the_row_kernels_fill_the_simds(kernels):
    rows = {n: k for n, k in kernels.items() if "q4_write_kernel" in n or "q4_read_kernel" in n}
    assert len(rows) > 60
    assert all(k["vgpr_count"] <= 64 and k["private_segment_fixed_size"] == 0 for k in rows.values())
