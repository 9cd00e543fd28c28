"""The longest row that a call takes: places in it reach the end of 32-bit numbers.  Slots outside the entries are all at 0, so that every sum is known."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def whole_row(row, value, slots):
    """Every slot of a row but those given holds the value."""
    at = row[slots].clone()
    row[slots] = value
    for part in row.split(1 << 28):
        assert bool((part == value).all())
    row[slots] = at
    return at


@pytest.mark.parametrize("g", [15.0, 60.0])                 # one reference for the row, two of them
def test_longest_row(g):
    from paper_2506_03206_amd import rdk
    n = (1 << 31) - 3
    slots = torch.tensor([0, 7, 16383, 16384, 1 << 30, n - 9, n - 1], device="cuda")
    K = slots.numel()
    z = torch.zeros((1, n), dtype=torch.bfloat16, device="cuda")
    z[0, slots] = g
    ids, v = slots.to(torch.int32)[None], torch.zeros((1, K), device="cuda")
    lse = torch.tensor([float(np.log(K) + 0.5)], device="cuda")
    t, r = np.exp(-0.5) / K, 1 - np.exp(-0.5)
    norm = np.logaddexp(np.log(K) + g, np.log(n - K))
    s, rho = np.exp(g - norm), np.exp(np.log(n - K) - norm)
    want = K * t * (np.log(t) - (g - norm)) + r * (np.log(r) - (np.log(n - K) - norm))
    outside = torch.tensor((rho - r) / (n - K), device="cuda").to(torch.bfloat16)
    o = rdk.rdk_distill_loss(None, z, ids, v, lse)
    assert abs(float(o.loss) - want) < 1e-4 * abs(want)
    dz = torch.full_like(z, float("nan"))
    out = rdk.DistillOutputs(1, n, z.dtype, "cuda", grad=dz)
    out.stats = o.stats
    for weight in (None, torch.zeros(1, device="cuda")):
        rdk.rdk_distill_grad(None, z, ids, v, out, weight=weight)
        value = dz[0, 1].clone()
        at = whole_row(dz[0], value, slots)
        if weight is None:
            assert abs(float(value) - float(outside)) <= 2 ** -7 * abs(float(outside))
            assert (at.double() - (s - t)).abs().max() <= 2 ** -8 * abs(s - t) + 1e-5
        else:
            assert float(value) == 0 and (at == 0).all()
    del dz, out
    over = rdk.DistillOutputs(1, n, z.dtype, "cuda", grad=z)
    over.stats = o.stats
    rdk.rdk_distill_grad(None, z, ids, v, over)
    assert abs(float(z[0, 1]) - float(outside)) <= 2 ** -7 * abs(float(outside))
    at = whole_row(z[0], z[0, 1].clone(), slots)
    assert (at.double() - (s - t)).abs().max() <= 2 ** -8 * abs(s - t) + 1e-5
