"""Rows of logits of any finite magnitude: masks and offsets between what a model gives and the type's limits, by rdk_topk and rdk_beam_select.
Bounds as in test_gpu_topk.py and test_gpu_beam.py, of the row's own values: masked ones are no part of a row's sum."""
import numpy as np
import pytest
import torch

from test_gpu_topk import rows, verify

pytestmark = pytest.mark.gpu

MAGNITUDES = [1e4, 1e6, 1e7, 3e7, 1e9, 1e10, 1e12, 1e20, 8e29, 1e31]


def masked_rows(N, kind, m, seed):
    """Finite masks where a lane, a wavefront or a part meets nothing else at first, and rows that lie at the magnitude themselves."""
    x = rows(12, N, kind, seed)
    at = torch.arange(N, device="cuda")
    x[0] = -m                                   # masked altogether: uniform
    x[1, : N // 2] = -m
    x[2, N // 2:] = -m
    x[3, at // 8 % 2 == 0] = -m                 # vectors
    x[4, at // 2048 % 2 == 0] = -m              # a round's
    x[5, 3:] = -m
    x[6, : N - 3] = -m
    x[7] = m
    x[8, N // 3] = m                            # one far above the others
    x[9] = torch.where(at % 3 == 0, -m, -2 * m).to(x.dtype)
    x[10] = torch.where(at // 8 % 64 < 32, -m, m).to(x.dtype)
    x[11, ::2] = -m
    return x


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("m", MAGNITUDES)
@pytest.mark.parametrize("N,T", [(50, 1.0), (5001, 0.25), (5001, 1.0), (5001, 2.0), (70001, 1.0)])
def test_topk(N, T, m, kind):
    from paper_2506_03206_amd import rdk
    x = masked_rows(N, kind, m, N)
    verify(rdk.rdk_topk(x, 32, temperature=T), x, 32, kind, T)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_topk_at_small_temperatures(kind):
    """The product with 1 / T is large where the logits are not.  (T a power of two: its reciprocal is exact.)"""
    from paper_2506_03206_amd import rdk
    for T in (2.0 ** -10, 2.0 ** -20, 2.0 ** -30):
        x = rows(4, 9001, kind, 3)
        x[1, :4500] = -1e4
        x[2] = -1e4
        x[3, 64:] = -100.0
        verify(rdk.rdk_topk(x, 16, temperature=T), x, 16, kind, T)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("m", MAGNITUDES)
@pytest.mark.parametrize("N", [50, 20001])
def test_beams(N, m, kind):
    """A beam masked altogether is a uniform one, and a mask in a row leaves the others' scores what they are."""
    from paper_2506_03206_amd import rdk
    G, W, K = 4, 3, 8
    x = rows(G * W, N, kind, N)
    r = x.view(G, W, N)
    r[0, 0] = -m
    r[1, :, : N // 2] = -m
    r[2, 1, 8:] = -m
    r[2, 2, : N - 8] = -m
    r[3] = -m
    scores = -torch.arange(W, device="cuda", dtype=torch.float32).repeat(G, 1) * 0.25
    o = rdk.rdk_beam_select(x, scores, K)
    want = (torch.log_softmax(r.double(), 2) + scores.double()[:, :, None]).flatten(1).cpu().numpy()
    got, parent, token = (t.cpu().numpy() for t in (o.scores, o.parent, o.token))
    # the logits that make up a beam's best are below 32, their scores too: an exponent's and a sum's rounding
    E = 2.0 ** -22 * 64 + 5e-6
    for g in range(G):
        chosen = parent[g].astype(np.int64) * N + token[g]
        assert (parent[g] >= 0).all() and np.unique(chosen).size == K
        assert (np.abs(want[g][chosen] - got[g]) <= E).all()
        assert (want[g][chosen] >= np.sort(want[g])[::-1][:K] - E).all()
    assert (o.parent[3] == 0).all() and torch.equal(o.token[3], torch.arange(K, dtype=torch.int32, device="cuda"))
