"""Rows and parts whose last wavefront has few values of its own take the way that ordinary rows take: not many times the time of rows that
fill their wavefronts."""
import pytest
import torch

from test_gpu_topk import rows, verify

pytestmark = pytest.mark.gpu


def part_time(B, N, k, kind):
    """The least mean of three times twenty launches: one that is held up from outside does not count."""
    from paper_2506_03206_amd import rdk
    x, o = rows(B, N, kind, N), rdk.TopkOutputs(B, N, k, "cuda")
    means = []
    for _ in range(3):
        rdk.rdk_topk(x, k, outputs=o)
        torch.cuda.synchronize()
        rdk.rdk_timing_read("topk_part_kernel")
        rdk.rdk_timing_select("topk_part_kernel")
        try:
            for _ in range(20):
                rdk.rdk_topk(x, k, outputs=o)
            torch.cuda.synchronize()
        finally:
            rdk.rdk_timing_select(None)
        launches, ms = rdk.rdk_timing_read("topk_part_kernel")
        assert launches == 20
        means.append(ms / launches)
    verify(o, x, k, kind)
    return min(means)


@pytest.mark.parametrize("kind,B,N,k,full", [
    ("bf16", 4, 1100, 128, 1024), ("bf16", 4, 1375, 128, 1024), ("bf16", 4, 1600, 128, 2048), ("bf16", 4, 1791, 128, 2048), ("bf16", 300, 1100, 128, 1024),
    ("bf16", 8, 128256, 128, 131072), ("bf16", 16, 128256, 100, 131072), ("f32", 4, 1100, 128, 1024),
])
def test_time_of_short_last_wavefronts(kind, B, N, k, full):
    """Searching by halving goes over a part 64 times, which is four to ten times the time of such a part; full wavefronts never take it on these rows."""
    assert part_time(B, N, k, kind) < 3 * part_time(B, full, k, kind)


@pytest.mark.parametrize("kind", ["f32", "bf16", "prob"])
@pytest.mark.parametrize("k", [97, 128])
@pytest.mark.parametrize("N", [511, 520, 767, 1017, 1023, 1030, 1100, 1281, 1375, 1536, 1543, 1600, 1791, 4096 + 1280, 49153 + 600])
def test_short_last_wavefronts(N, k, kind):
    from paper_2506_03206_amd import rdk
    x = rows(3, N, kind, N + k)
    verify(rdk.rdk_topk(x, k, "prob" if kind == "prob" else "logit"), x, k, kind)
