"""The distillation calls where they can go wrong, against their formulas in 64 bits (numpy), the gradient against differences too.

Tolerances.  With R = 2^-22 (max |z| + max |v|) / T + 5e-6 (roundings of exponents and of fp32 sums) every log s and log t is off by at most R, every s and t
by the relative R: a loss by (1 + D) R, D the largest |log t - log s| that counts; an entry of the gradient by (s + t) R, and outside A by
s R (1 + 3 r / rho) + s / rho R, the second for the remainder r = 1 - sum t.  A bf16 gradient is rounded once: 2^-8 of it."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def reference(z, ids, v, lse, T, w, slot_of):
    """z [B,n], ids, v [B,K], lse [B] or None, w [B]; slot_of: dict-like array id -> slot or -1.  float64 loss, dz and their tolerances."""
    B, n = z.shape
    loss, dz = np.zeros(B), np.zeros((B, n))
    tol_l, tol_g = np.zeros(B), np.zeros((B, n))
    with np.errstate(all="ignore"):
        for b in range(B):
            if w[b] == 0:
                continue
            m = z[b].max()
            e = np.exp((z[b] - (m if m > -np.inf else 0.0)) / T)
            total = e.sum()
            s = e / total if total > 0 else np.zeros(n)
            log_s = (z[b] - m) / T - np.log(total) if total > 0 else np.full(n, -np.inf)
            slot = np.array([slot_of[i] if 0 <= i < len(slot_of) else -1 for i in ids[b]])
            on = (slot >= 0) & (v[b] != -np.inf)
            A, va = slot[on], v[b][on] / T
            assert np.unique(A).size == A.size
            remainder = lse is not None and A.size < n
            if A.size:
                log_t = va - (lse[b] if remainder else va.max() + np.log(np.exp(va - va.max()).sum()))
                t = np.exp(log_t)
                loss[b] = np.where(t > 0, t * (log_t - log_s[A]), 0.0).sum()
                D = np.abs(np.where(t > 1e-30, log_t - log_s[A], 0.0)).max()
            else:
                t, D = np.zeros(0), 0.0
            finite = lambda a: np.abs(a[np.isfinite(a)]).max(initial=0.0)  # noqa: E731
            R = 2.0 ** -22 * (finite(z[b]) + finite(va * T)) / T + 5e-6
            g = s * (1.0 if A.size else 0.0)
            tol = s * R
            if remainder:
                r = max(0.0, 1.0 - t.sum())
                out = np.ones(n, bool)
                out[A] = False
                rho = s[out].sum()
                if r > 0:
                    loss[b] += r * (np.log(r) - np.log(rho))
                D = max(D, np.abs(np.log(r) - np.log(rho)) if r > 0 and rho > 0 else 0.0)
                D += 1.0 / max(r, 1e-3) if r > 0 else 0.0       # r itself is a difference: its logarithm is off by R / r
                g = np.where(out, s * (1.0 - r / rho) if rho > 0 else s, s)
                tol = np.where(out, s * R * (1 + 3 * r / rho) + s / rho * R if rho > 0 else 0.0, tol)
            g[A] -= t
            tol[A] += t * R
            dz[b], tol_g[b] = g * w[b] / T, (tol + 1e-30) * abs(w[b]) / T
            loss[b] *= w[b]
            tol_l[b] = (1 + D) * R * abs(w[b])
    return loss, dz, tol_l, tol_g


def vocabulary(N, n, seed):
    from paper_2506_03206_amd import rdk
    rng = np.random.default_rng(seed)
    kept = np.sort(rng.choice(N, size=n, replace=False)).astype(np.int32)
    slot_of = np.full(N, -1)
    slot_of[kept] = np.arange(n)
    return rdk.rdk_build_kernel(N, torch.from_numpy(kept).cuda(), rdk.IDENTITY), kept, slot_of


def inputs(B, N, n, K, dtype, seed, T, kept, sigma=3.0):
    """Drafter logits, the teacher's top entries and its normaliser."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    p = torch.randn((B, N), generator=g, device="cuda") * sigma
    v, ids = torch.topk(p, K, dim=1)
    z = (p[:, torch.from_numpy(kept).cuda().long()] + torch.randn((B, n), generator=g, device="cuda")).to(dtype)
    return z.contiguous(), ids.to(torch.int32), v.contiguous(), torch.logsumexp(p.double() / T, 1).float()


def run_all(kernel, z, ids, v, lse, T, w):
    """Loss and gradient from the single calls, from both at once, and from both at once over z itself."""
    from paper_2506_03206_amd import rdk
    B, n = z.shape
    a = rdk.DistillOutputs(B, n, z.dtype, "cuda")
    a.grad.fill_(float("nan"))
    rdk.rdk_distill_loss(kernel, z, ids, v, lse, T, w, a)
    rdk.rdk_distill_grad(kernel, z, ids, v, a, T, w)
    b = rdk.DistillOutputs(B, n, z.dtype, "cuda")
    b.grad.fill_(float("nan"))
    rdk.rdk_distill_loss_grad(kernel, z, ids, v, lse, T, w, b)
    own = torch.empty((B, z.stride(0)), dtype=z.dtype, device="cuda")[:, :n].copy_(z)
    c = rdk.DistillOutputs(B, n, z.dtype, "cuda", grad=own)
    rdk.rdk_distill_loss_grad(kernel, own, ids, v, lse, T, w, c)
    apart = torch.empty((B, z.stride(0)), dtype=z.dtype, device="cuda")[:, :n].copy_(z)
    d = rdk.DistillOutputs(B, n, z.dtype, "cuda", grad=apart)
    d.stats = a.stats
    rdk.rdk_distill_grad(kernel, apart, ids, v, d, T, w)
    assert torch.equal(d.grad.view(torch.int16), a.grad.view(torch.int16))         # over z itself, the same bits
    return [(a.loss, a.grad), (b.loss, b.grad), (c.loss, c.grad)]


def check(kernel, slot_of, z, ids, v, lse, T, w):
    B, n = z.shape
    w64 = np.ones(B) if w is None else w.double().cpu().numpy()
    ref = reference(z.double().cpu().numpy(), ids.cpu().numpy(), v.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy(), T, w64,
                    slot_of)
    for loss, grad in run_all(kernel, z, ids, v, lse, T, w):
        compare(loss, grad, ref)
    return ref


def compare(loss, grad, ref):
    want_l, want_g, tol_l, tol_g = ref
    got_l, got_g = loss.double().cpu().numpy(), grad.double().cpu().numpy()
    fine = np.isfinite(want_l)
    np.testing.assert_array_equal(got_l[~fine], want_l[~fine])
    assert (np.abs(got_l - want_l)[fine] <= tol_l[fine]).all(), np.max((np.abs(got_l - want_l) - tol_l)[fine])
    fine = np.isfinite(want_g)
    np.testing.assert_array_equal(got_g[~fine], want_g[~fine])
    tol = tol_g + (2.0 ** -8 * np.abs(want_g) if grad.dtype == torch.bfloat16 else 2.0 ** -23 * np.abs(want_g)) + 1e-38
    bad = (np.abs(got_g - want_g) > tol) & fine
    assert not bad.any(), (np.argwhere(bad)[:5], got_g[bad][:5], want_g[bad][:5])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("remainder", [False, True])
@pytest.mark.parametrize("B,N,n,K,T", [(1, 1, 1, 1, 1.0), (3, 9, 2, 4, 1.0), (5, 40, 7, 9, 0.5), (2, 100, 8, 100, 2.0), (4, 300, 299, 128, 1.0),
                                       (16, 1024, 256, 8, 1.0), (3, 5000, 1023, 64, 3.0), (7, 9001, 2047, 65, 1.0), (2, 40000, 8193, 33, 1.0),
                                       (3, 40000, 16385, 128, 2.0), (2, 70001, 32769, 100, 1.0), (2, 70001, 65537, 64, 1.0),
                                       (1, 140000, 131072, 16, 1.0), (2, 140000, 131081, 16, 1.0), (1, 300007, 262147, 128, 1.0),
                                       (600, 2000, 501, 20, 1.0), (260, 20000, 5003, 12, 1.0)])
def test_sizes(B, N, n, K, T, remainder, dtype):
    kernel, kept, slot_of = vocabulary(N, n, N + n)
    z, ids, v, lse = inputs(B, N, n, min(K, N), dtype, B + K, T, kept)
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    w = torch.rand(B, generator=g, device="cuda") + 0.1
    if B > 2:
        w[1] = 0.0
    check(kernel, slot_of, z, ids, v, lse if remainder else None, T, w)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1001, 20003, 70003])
def test_rows_at_odd_strides_and_ids_that_are_slots(n, dtype):
    B, K = 3, 31
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    wide = torch.full((B, n + 5), float("nan"), dtype=dtype, device="cuda")
    z = wide[:, :n]
    z.copy_(torch.randn((B, n), generator=g, device="cuda") * 2)
    ids = torch.stack([torch.randperm(n, generator=g, device="cuda")[:K] for _ in range(B)]).to(torch.int32)
    v = torch.randn((B, K), generator=g, device="cuda")
    check(None, np.arange(n), z, ids, v, None, 1.0, None)
    check(None, np.arange(n), z, ids, v, torch.logsumexp(v, 1) + 0.3, 1.0, None)
    assert torch.isnan(wide[:, n:]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("remainder", [False, True])
@pytest.mark.parametrize("n", [513, 30001, 140001])
def test_masks_and_rows_without_entries(n, remainder, dtype):
    """Entries out of the vocabulary or masked, none that count, drafter rows masked in part, where the teacher has mass, and altogether; rows of
    weight 0 that hold NaN; a drafter sure of its top entry, whose remainder is far below what 1 - sum can hold."""
    N, K, T = n + 100, 16, 1.0
    kernel, kept, slot_of = vocabulary(N, n, 5)
    z, ids, v, lse = inputs(10, N, n, K, dtype, 6, T, kept)
    pruned = torch.from_numpy(np.setdiff1d(np.arange(N), kept)[:K].astype(np.int32)).cuda()
    held = torch.from_numpy(kept[:K].copy()).cuda()
    w = torch.ones(10, device="cuda")
    ids[0] = pruned                                     # nothing held
    ids[1], v[1] = held, -float("inf")                  # held, but masked
    ids[2, 3:] = -1
    v[2, 3:] = -float("inf")
    ids[3, ::2] = N + 7                                 # ids beyond the vocabulary
    ids[3, 1] = -5
    ids[4] = held
    z[4, : K // 2] = -float("inf")                      # the loss is infinite there
    z[5] = -float("inf")                                # the whole drafter row
    z[6, n // 2:] = torch.finfo(dtype).min
    z[7], w[7] = float("nan"), 0.0
    ids[8] = held
    v[8] = torch.linspace(0, -3, K, device="cuda")
    lse[8] = float(torch.logsumexp(v[8], 0)) + 1e-3
    z[8] = -20.0 + 0.5 * torch.randn(n, device="cuda")
    z[8, 0] = 20.0
    ids[9] = held
    z[9, K:] = -float("inf")                            # no mass outside the entries
    check(kernel, slot_of, z, ids, v, lse if remainder else None, T, w)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_nan_and_infinity_show(dtype):
    from paper_2506_03206_amd import rdk
    n, K = 3001, 8
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    z = torch.randn((4, n), generator=g, device="cuda").to(dtype)
    ids = torch.arange(K, dtype=torch.int32, device="cuda").repeat(4, 1)
    v = torch.randn((4, K), generator=g, device="cuda")
    z[0, 2000] = float("nan")
    z[1, 3] = float("inf")
    v[2, 1] = float("nan")
    for lse in (None, torch.logsumexp(v, 1) + 0.5):
        for o in (rdk.rdk_distill_loss(None, z, ids, v, lse), rdk.rdk_distill_loss_grad(None, z, ids, v, lse)):
            assert torch.isnan(o.loss[:3]).all() and torch.isfinite(o.loss[3])


@pytest.mark.parametrize("remainder", [False, True])
@pytest.mark.parametrize("T", [1.0, 2.5])
def test_gradient_against_differences(T, remainder):
    """Central differences of the 64-bit loss over steps of 1e-4: truncation about h^2, fp32 gradient about 1e-5."""
    n, K, B = 40, 6, 3
    rng = np.random.default_rng(3)
    z, v = rng.normal(size=(B, n)) * 2, rng.normal(size=(B, K))
    z = z.astype(np.float32).astype(np.float64)
    ids = np.stack([rng.choice(n, K, replace=False) for _ in range(B)]).astype(np.int32)
    v = v.astype(np.float32).astype(np.float64)
    lse = (np.log(np.exp(v / T).sum(1)) + 0.4).astype(np.float32) if remainder else None
    slots = np.arange(n)
    f = lambda x: reference(x, ids, v, lse, T, np.ones(B), slots)[0]  # noqa: E731
    h, want = 1e-4, np.empty((B, n))
    for j in range(n):
        step = np.zeros((B, n))
        step[:, j] = h
        want[:, j] = (f(z + step) - f(z - step)) / (2 * h)
    t = lambda a, dt: torch.from_numpy(np.ascontiguousarray(a)).cuda().to(dt)  # noqa: E731
    for _, grad in run_all(None, t(z, torch.float32), t(ids, torch.int32), t(v, torch.float32), None if lse is None else t(lse, torch.float32), T, None):
        assert np.abs(grad.double().cpu().numpy() - want).max() < 2e-5


def test_differentiation_through_torch():
    """rdk_distill under autograd: a head's weights get the gradient that the formula gives through torch, and a mean over tokens reaches it."""
    from paper_2506_03206_amd import rdk
    N, n, K, B, D = 3000, 700, 12, 20, 24
    kernel, kept, slot_of = vocabulary(N, n, 1)
    _, ids, v, lse = inputs(B, N, n, K, torch.float32, 2, 1.0, kept)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    h, head = torch.randn((B, D), generator=g, device="cuda"), torch.randn((D, n), generator=g, device="cuda").mul_(0.3).requires_grad_()
    rdk.rdk_distill(kernel, h @ head, ids, v, lse).mean().backward()
    z = (h @ head).detach()
    _, dz, _, _ = reference(z.double().cpu().numpy(), ids.cpu().numpy(), v.double().cpu().numpy(), lse.double().cpu().numpy(), 1.0, np.full(B, 1.0 / B), slot_of)
    want = h.double().cpu().numpy().T @ dz
    got = head.grad.double().cpu().numpy()
    assert np.abs(got - want).max() <= 1e-4 * np.abs(want).max()


def test_rows_beyond_32_bits():
    from paper_2506_03206_amd import rdk
    n, K, ld = 5003, 16, (1 << 31) + 8
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    flat = torch.empty(ld + n, dtype=torch.bfloat16, device="cuda")
    z = flat.as_strided((2, n), (ld, 1))
    z.copy_(torch.randn((2, n), generator=g, device="cuda"))
    ids = torch.stack([torch.randperm(n, generator=g, device="cuda")[:K] for _ in range(2)]).to(torch.int32)
    v = torch.randn((2, K), generator=g, device="cuda")
    ref = reference(z.double().cpu().numpy(), ids.cpu().numpy(), v.double().cpu().numpy(), None, 1.0, np.ones(2), np.arange(n))
    o = rdk.DistillOutputs(2, n, z.dtype, "cuda", grad=z)                           # over z itself: strides alike
    rdk.rdk_distill_loss_grad(None, z, ids, v, outputs=o)
    compare(o.loss, o.grad, ref)


def test_other_streams_and_replays():
    from paper_2506_03206_amd import rdk
    N, n, K, B = 20000, 9001, 24, 12
    kernel, kept, slot_of = vocabulary(N, n, 1)
    z, ids, v, lse = inputs(B, N, n, K, torch.bfloat16, 2, 1.0, kept)
    o = rdk.DistillOutputs(B, n, z.dtype, "cuda")
    want = lambda: reference(z.double().cpu().numpy(), ids.cpu().numpy(), v.double().cpu().numpy(), lse.double().cpu().numpy(), 1.0, np.ones(B),  # noqa: E731
                             slot_of)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        rdk.rdk_distill_loss_grad(kernel, z, ids, v, lse, outputs=o)
    torch.cuda.current_stream().wait_stream(side)
    compare(o.loss, o.grad, want())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rdk.rdk_distill_loss(kernel, z, ids, v, lse, outputs=o)
        rdk.rdk_distill_grad(kernel, z, ids, v, o)
    for i in range(4):
        a, b, c, d = inputs(B, N, n, K, torch.bfloat16, 20 + i, 1.0, kept)
        z.copy_(a), ids.copy_(b), v.copy_(c), lse.copy_(d)
        graph.replay()
        torch.cuda.synchronize()
        ref = want()
        compare(o.loss, o.grad, ref)
        e = rdk.rdk_distill_loss_grad(kernel, z, ids, v, lse)
        compare(e.loss, e.grad, ref)


def test_refusals_of_the_binding():
    from paper_2506_03206_amd import rdk
    z = torch.zeros((2, 100), device="cuda")
    ids, v = torch.zeros((2, 4), dtype=torch.int32, device="cuda"), torch.zeros((2, 4), device="cuda")
    kernel, _, _ = vocabulary(500, 99, 1)
    with pytest.raises(rdk.RdkError):
        rdk.rdk_distill_loss(kernel, z, ids, v)                                     # another vocabulary
    with pytest.raises(rdk.RdkError):
        rdk.rdk_distill_loss(None, z, ids, v, temperature=-1.0)
    for bad in ({"z": z.half()}, {"ids": ids.long()}, {"v": v[:, :3]}, {"ids": ids[:1], "v": v[:1]}, {"lse": torch.zeros(3, device="cuda")},
                {"w": torch.ones(2, device="cuda", dtype=torch.float64)}):
        a = dict({"z": z, "ids": ids, "v": v, "lse": None, "w": None}, **bad)
        with pytest.raises(AssertionError):
            rdk.rdk_distill_loss(None, a["z"], a["ids"], a["v"], a["lse"], weight=a["w"])
    with pytest.raises(AssertionError):
        rdk.rdk_distill_loss_grad(None, z, ids, v, outputs=rdk.DistillOutputs(2, 100, torch.bfloat16, "cuda"))
    with pytest.raises(AssertionError):
        rdk.rdk_distill_grad(None, z, ids, v, rdk.DistillOutputs(2, 100, torch.float32, "cuda", grad=False))
