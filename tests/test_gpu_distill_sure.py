"""Distillation with the remainder counted where the drafter's mass outside the entries is far below what fp32 holds beside its best logit: finite
logits give a finite loss, and the slots outside share the gradient -r.  Against the formula in 64 bits, by logarithms.

Tolerances.  Exponents are differences to the largest logit of the entries, of the slots outside or of the teacher: with the three groups' spreads, R =
2^-22 (sum of them and of the teacher's largest) / T + 5e-6 bounds the relative error of every s on A, every t and every o, the softmax over the slots outside alone.  A loss
is off by (1 + D) R, D the largest logarithm in it; outside A the gradient is s - r o: off by s R + r o R and by o times the error R of r = 1 - sum t
(there s is below r o by the gap, so its own rounding over the gap is no part of it)."""
import numpy as np
import pytest
import torch

from test_gpu_distill import compare, run_all

pytestmark = pytest.mark.gpu


def log_sum(a):
    m = a.max()
    return m + np.log(np.exp(a - m).sum()) if m > -np.inf else -np.inf


def reference(z, ids, v, lse, T, w):
    """ids are slots, distinct, all of them count."""
    B, n = z.shape
    loss, dz, tol_l, tol_g = np.zeros(B), np.zeros((B, n)), np.zeros(B), np.zeros((B, n))
    for b in range(B):
        A, out = ids[b], np.ones(n, bool)
        out[A] = False
        y = z[b] / T
        norm, outside = log_sum(y), log_sum(y[out])
        log_t, log_s = v[b] / T - lse[b], y - norm
        t, s = np.exp(log_t), np.exp(log_s)
        r = max(0.0, 1.0 - t.sum())
        loss[b] = (t * (log_t - log_s[A])).sum() + (r * (np.log(r) - (outside - norm)) if r > 0 else 0.0)
        o = np.where(out, np.exp(y - y[out].max()), 0.0)
        o /= o.sum()
        g = np.where(out, s - r * o, s)
        g[A] -= t
        R = 2.0 ** -22 * (np.ptp(z[b][A]) + np.ptp(z[b][out]) + np.abs(v[b]).max()) / T + 5e-6
        D = max(np.abs(log_t - log_s[A]).max(), abs(np.log(r) - (outside - norm)) + 1.0 / max(r, 1e-3) if r > 0 else 0.0)
        tol = s * R + (r + 1.0) * o * R
        tol[A] += t * R
        loss[b] *= w[b]
        dz[b], tol_l[b], tol_g[b] = g * w[b] / T, (1 + D) * R * abs(w[b]), (tol + 1e-30) * abs(w[b]) / T
    return loss, dz, tol_l, tol_g


def sure_rows(B, n, K, gap, T, dtype, seed, bottom=None):
    """Entries' logits `gap` above the others, which lie about zero or all at `bottom`."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    z = torch.randn((B, n), generator=g, device="cuda") if bottom is None else torch.full((B, n), bottom, device="cuda")
    ids = torch.argsort(torch.rand((B, n), generator=g, device="cuda"), 1)[:, :K].to(torch.int32).contiguous()
    z.scatter_(1, ids.long(), gap + torch.randn((B, K), generator=g, device="cuda"))
    v = torch.randn((B, K), generator=g, device="cuda") * T
    lse = (torch.logsumexp(v.double() / T, 1) + 0.1).float()
    return z.to(dtype), ids, v, lse


def check(z, ids, v, lse, T):
    B = z.shape[0]
    w = torch.linspace(0.5, 1.5, B, device="cuda")
    ref = reference(z.double().cpu().numpy(), ids.cpu().numpy(), v.double().cpu().numpy(), lse.double().cpu().numpy(), T, w.double().cpu().numpy())
    assert np.isfinite(ref[0]).all()
    for loss, grad in run_all(None, z, ids, v, lse, T, w):
        compare(loss, grad, ref)


# a row in the registers of a workgroup; the loss in rounds; both in parts; both in rounds (of many rows)
SIZES = [(3, 513, 5), (3, 7999, 33), (3, 40001, 64), (2, 140001, 128), (130, 130601, 7)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gap,T", [(60.0, 1.0), (86.0, 1.0), (88.5, 1.0), (100.0, 1.0), (130.0, 1.0), (1000.0, 1.0), (22.0, 0.25), (16.0, 0.125), (500.0, 4.0)])
@pytest.mark.parametrize("B,n,K", SIZES[:4])
def test_gaps(B, n, K, gap, T, dtype):
    check(*sure_rows(B, n, K, gap, T, dtype, n + K), T)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gap,T", [(100.0, 1.0), (22.0, 0.25)])
def test_gaps_of_many_long_rows(gap, T, dtype):
    B, n, K = SIZES[4]
    check(*sure_rows(B, n, K, gap, T, dtype, n + K), T)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bottom", [-1e4, -1e9, "lowest"])
@pytest.mark.parametrize("B,n,K", SIZES[:4])
def test_finite_masks_outside_the_entries(B, n, K, bottom, dtype):
    """A mask of the type's lowest value is a number: the loss is large, not infinite.  (Everything outside equal: shares of 1 / (n - K).)"""
    check(*sure_rows(B, n, K, 3.0, 1.0, dtype, n, torch.finfo(dtype).min if bottom == "lowest" else bottom), 1.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_smallest_case(dtype):
    """Four slots, one entry: loss t (log t - log s) + r (log r - log rho) = 8.003, a third of r on every slot outside."""
    from paper_2506_03206_amd import rdk
    z = torch.tensor([[88.5, 0.0, 0.0, 0.0]], device="cuda").to(dtype)
    ids, v, lse = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.zeros((1, 1), device="cuda"), torch.full((1,), 0.1, device="cuda")
    o = rdk.rdk_distill_loss_grad(None, z, ids, v, lse)
    t = np.exp(-0.1)
    r = 1 - t
    want = t * -0.1 + r * (np.log(r) + 88.5 - np.log(3.0))
    assert abs(want - 8.003) < 2e-3
    assert abs(float(o.loss) - want) < 1e-4
    np.testing.assert_allclose(o.grad.float().cpu().numpy()[0], [r, -r / 3, -r / 3, -r / 3], rtol=2 ** -8 if dtype == torch.bfloat16 else 1e-5)


@pytest.mark.parametrize("dtype,n", [(torch.bfloat16, 16384), (torch.bfloat16, 16385), (torch.bfloat16, 100003), (torch.float32, 8192), (torch.float32, 8193),
                                     (torch.float32, 50001)])
def test_gradient_over_the_logits(dtype, n):
    """The backward call over z itself, where one workgroup or several share a row, of rows on both sides of where the gap parts them: the same bits
    as apart from z, row by row."""
    from paper_2506_03206_amd import rdk
    z, ids, v, lse = sure_rows(64, n, 100, 0.0, 1.0, dtype, n)
    z.scatter_add_(1, ids.long(), torch.linspace(0.0, 120.0, 64, device="cuda")[:, None].expand(64, 100).to(dtype))
    apart = rdk.DistillOutputs(64, n, dtype, "cuda")
    rdk.rdk_distill_loss(None, z, ids, v, lse, outputs=apart)
    rdk.rdk_distill_grad(None, z, ids, v, apart)
    w = torch.ones(64, device="cuda")
    ref = reference(z.double().cpu().numpy(), ids.cpu().numpy(), v.double().cpu().numpy(), lse.double().cpu().numpy(), 1.0, w.double().cpu().numpy())
    compare(apart.loss, apart.grad, ref)
    over = rdk.DistillOutputs(64, n, dtype, "cuda", grad=z)
    over.stats = apart.stats
    rdk.rdk_distill_grad(None, z, ids, v, over)
    assert torch.equal(z.view(torch.int16), apart.grad.view(torch.int16))
