"""Teacher logits far from zero: the backward call's teacher is the forward call's, as exact.

A common offset of a row's logits changes nothing in the formulas, and the differences of fp32 logits are exact; so is a normaliser that is given.  The bounds are those of
test_gpu_distill.py with the logits' distance from the row's largest in the place of their magnitude."""
import numpy as np
import pytest
import torch

from test_gpu_distill import compare, run_all

pytestmark = pytest.mark.gpu


def reference(z, ids, v, lse, T):
    """ids are slots, all of them count; the drafter's logits lie about zero."""
    B, n = z.shape
    y = z / T
    log_s = y - y.max(1, keepdims=True)
    log_s -= np.log(np.exp(log_s).sum(1, keepdims=True))
    at = np.take_along_axis(log_s, ids, 1)
    d = (v - v.max(1, keepdims=True)) / T
    log_t = d - np.log(np.exp(d).sum(1, keepdims=True)) if lse is None else d - (lse[:, None] - v.max(1, keepdims=True) / T)
    t, s = np.exp(log_t), np.exp(log_s)
    R = 2.0 ** -22 * (np.abs(z).max(1) + np.abs(v - v.max(1, keepdims=True)).max(1)) / T + 5e-6
    loss, D = (t * (log_t - at)).sum(1), np.abs(log_t - at).max(1)
    g, tol = s.copy(), s * R[:, None]
    if lse is not None:
        r = np.maximum(0.0, 1.0 - t.sum(1))
        rest = s.copy()
        np.put_along_axis(rest, ids, 0.0, 1)
        rho = rest.sum(1)
        loss += r * (np.log(r) - np.log(rho))
        D = np.maximum(D, np.abs(np.log(r) - np.log(rho))) + 1.0 / np.maximum(r, 1e-3)
        g = s * (1 - r / rho)[:, None]
        tol = s * (R * (1 + 3 * r / rho) + R / rho)[:, None]
        np.put_along_axis(g, ids, np.exp(at), 1)
        np.put_along_axis(tol, ids, np.exp(at) * R[:, None], 1)
    np.put_along_axis(g, ids, np.take_along_axis(g, ids, 1) - t, 1)
    np.put_along_axis(tol, ids, np.take_along_axis(tol, ids, 1) + t * R[:, None], 1)
    return loss, g / T, (1 + D) * R, (tol + 1e-30) / T


@pytest.mark.parametrize("remainder", [False, True])
@pytest.mark.parametrize("offset,T", [(0.0, 1.0), (1e4, 1.0), (-1e5, 1.0), (20.0, 0.0078125), (1e4, 4.0)])
@pytest.mark.parametrize("B,n,K", [(5, 700, 12), (3, 20001, 64), (2, 140001, 100)])
def test_offsets(B, n, K, offset, T, remainder):
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    z = torch.randn((B, n), generator=g, device="cuda") * T
    ids = torch.argsort(torch.rand((B, n), generator=g, device="cuda"), 1)[:, :K].to(torch.int32).contiguous()
    v = torch.randn((B, K), generator=g, device="cuda") * T + offset
    lse = None
    if remainder:
        lse = (torch.logsumexp(v.double() / T, 1) + 0.4).float()
    ref = reference(z.double().cpu().numpy(), ids.cpu().numpy().astype(np.int64), v.double().cpu().numpy(),
                    None if lse is None else lse.double().cpu().numpy(), T)
    for loss, grad in run_all(None, z, ids, v, lse, T, None):
        compare(loss, grad, ref)
