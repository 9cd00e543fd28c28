"""Every kernel and variant of the operators beside the decoding step at a size that takes it, at the ends of its range: which kernels were
launched, and the results against torch in 64 bits (tolerances as in test_gpu_distill.py, test_gpu_topk.py)."""
import numpy as np
import pytest
import torch

from test_gpu_distill import compare
from test_gpu_topk import verify

pytestmark = pytest.mark.gpu

ROW, LOOP, PART, FINISH, GRAD = "distill_row_kernel", "distill_loop_kernel", "distill_part_kernel", "distill_finish_kernel", "distill_grad_kernel"
DISTILL = [ROW, LOOP, PART, FINISH, GRAD]


def launched(names, call):
    from paper_2506_03206_amd import rdk
    for name in names:
        rdk.rdk_timing_read(name)
    rdk.rdk_timing_select("*")
    try:
        call()
        torch.cuda.synchronize()
    finally:
        rdk.rdk_timing_select(None)
    return [name for name in names if rdk.rdk_timing_read(name)[0]]


def reference(z, ids, v, lse, w):
    """Loss, gradient and their tolerances in 64 bits, on the device; ids are slots, T = 1, every entry counts."""
    z64 = z.double()
    log_s = torch.log_softmax(z64, 1)
    s, i = log_s.exp(), ids.long()
    at = log_s.gather(1, i)
    R = 2.0 ** -22 * (z64.abs().amax(1) + v.abs().amax(1).double()) + 5e-6
    if lse is None:
        log_t = torch.log_softmax(v.double(), 1)
        t = log_t.exp()
        loss, D = (t * (log_t - at)).sum(1), (log_t - at).abs().amax(1)
        g, tol = s.clone(), s * R[:, None]
    else:
        log_t = v.double() - lse.double()[:, None]
        t = log_t.exp()
        r = (1 - t.sum(1)).clamp(min=0)
        rest = s.scatter(1, i, 0.0)
        rho = rest.sum(1)
        loss = (t * (log_t - at)).sum(1) + r * (r.log() - rho.log())
        D = torch.maximum((log_t - at).abs().amax(1), (r.log() - rho.log()).abs()) + 1 / r.clamp(min=1e-3)
        g = s * (1 - r / rho)[:, None]
        tol = s * (R * (1 + 3 * r / rho))[:, None] + s * (R / rho)[:, None]
        g.scatter_(1, i, s.gather(1, i))
        tol.scatter_(1, i, s.gather(1, i) * R[:, None])
    g.scatter_add_(1, i, -t)
    tol.scatter_add_(1, i, t * R[:, None])
    w = w.double()
    return [x.cpu().numpy() for x in (loss * w, g * w[:, None], (1 + D) * R * w, (tol + 1e-30) * w[:, None])]


@pytest.mark.parametrize("remainder", [False, True])
@pytest.mark.parametrize("dtype,B,n,loss_by,both_by", [
    (torch.bfloat16, 2, 4608, [ROW], [ROW]), (torch.bfloat16, 2, 4609, [ROW], [ROW]), (torch.bfloat16, 2, 13824, [ROW], [ROW]),
    (torch.bfloat16, 2, 13825, [ROW], [ROW]), (torch.bfloat16, 3, 17921, [ROW], [ROW]), (torch.bfloat16, 3, 32256, [ROW], [ROW]),
    (torch.bfloat16, 3, 32257, [LOOP], [ROW]), (torch.bfloat16, 3, 60928, [LOOP], [ROW]), (torch.bfloat16, 2, 60929, [PART, FINISH], [ROW]),
    (torch.bfloat16, 129, 60935, [LOOP], [ROW]), (torch.bfloat16, 65, 69120, [PART, FINISH], [ROW]), (torch.bfloat16, 64, 69121, [PART, FINISH], [PART, FINISH, GRAD]),
    (torch.bfloat16, 65, 69127, [PART, FINISH], [ROW]), (torch.bfloat16, 66, 130560, [PART, FINISH], [ROW]), (torch.bfloat16, 129, 130561, [LOOP], [LOOP, GRAD]),
    (torch.bfloat16, 2, 491521, [PART, FINISH], [PART, FINISH, GRAD]), (torch.bfloat16, 130, 491519, [LOOP], [LOOP, GRAD]),
    (torch.float32, 2, 2304, [ROW], [ROW]), (torch.float32, 2, 6913, [ROW], [ROW]), (torch.float32, 3, 16128, [ROW], [ROW]),
    (torch.float32, 3, 16129, [LOOP], [ROW]), (torch.float32, 2, 30465, [PART, FINISH], [ROW]), (torch.float32, 66, 34561, [PART, FINISH], [ROW]),
    (torch.float32, 3, 34561, [PART, FINISH], [PART, FINISH, GRAD]), (torch.float32, 131, 65281, [LOOP], [LOOP, GRAD]), (torch.float32, 130, 65280, [LOOP], [ROW]),
])
def test_distill_kernels(dtype, B, n, loss_by, both_by, remainder):
    from paper_2506_03206_amd import rdk
    K = 61
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    wide = torch.full((B, n + 1), float("nan"), dtype=dtype, device="cuda")
    z = wide[:, :n]
    z.copy_(torch.randn((B, n), generator=g, device="cuda") * 2)
    ids = torch.argsort(torch.rand((B, n), generator=g, device="cuda"), 1)[:, :K].to(torch.int32).contiguous()
    ids[0, 0] = n - 1 if not (ids[0] == n - 1).any() else ids[0, 0]               # the last slot is an entry of the first row
    v = torch.randn((B, K), generator=g, device="cuda") + 3
    lse = (torch.logsumexp(v.double(), 1) + 0.4).float() if remainder else None
    w = torch.rand(B, generator=g, device="cuda") + 0.5
    a, b = rdk.DistillOutputs(B, n, dtype, "cuda"), rdk.DistillOutputs(B, n, dtype, "cuda")
    ref = reference(z, ids, v, lse, w)
    assert launched(DISTILL, lambda: rdk.rdk_distill_loss(None, z, ids, v, lse, weight=w, outputs=a)) == loss_by
    assert launched(DISTILL, lambda: rdk.rdk_distill_grad(None, z, ids, v, a, weight=w)) == [GRAD]
    compare(a.loss, a.grad, ref)
    assert launched(DISTILL, lambda: rdk.rdk_distill_loss_grad(None, z, ids, v, lse, weight=w, outputs=b)) == both_by
    compare(b.loss, b.grad, ref)
    assert torch.isnan(wide[:, n:]).all()


TOP = ["topk_part_kernel", "topk_merge_kernel", "beam_merge_kernel"]


@pytest.mark.parametrize("dtype,B,N,k,merges", [
    (torch.bfloat16, 1, 49152, 20, False), (torch.bfloat16, 1, 49153, 20, True), (torch.bfloat16, 191, 49153, 128, True), (torch.bfloat16, 192, 49153, 128, False),
    (torch.float32, 2, 24576, 128, False), (torch.float32, 2, 24577, 128, True), (torch.float32, 1, 300001, 128, True), (torch.float32, 1, 300001, 3, True),
])
def test_topk_kernels(dtype, B, N, k, merges):
    from paper_2506_03206_amd import rdk
    g = torch.Generator(device="cuda")
    g.manual_seed(N + k)
    x = torch.randn((B, N), generator=g, device="cuda").to(dtype)
    x[0, 5:] = -float("inf")
    o = rdk.TopkOutputs(B, N, k, "cuda")
    assert launched(TOP, lambda: rdk.rdk_topk(x, k, outputs=o)) == TOP[:1 + merges]
    verify(o, x, k, "f32")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("k", [1, 40, 128])
@pytest.mark.parametrize("N", [30000, 200003])
def test_rows_whose_best_crowd(N, k, dtype):
    """More noted than there is room for, more than fits behind the bound, bounds equal to their sixteenth bit, in one part and in several."""
    from paper_2506_03206_amd import rdk
    g = torch.Generator(device="cuda")
    g.manual_seed(N)
    at, noise = torch.arange(N, device="cuda"), torch.randn(N, generator=g, device="cuda")
    few = at % 2048 < 8                                                            # one thread's vectors in a wavefront's
    rows = [at.float(), at.float() / 1000 + noise * 0.01, 1 + noise * 1e-5, torch.where(few, 50 + noise, noise), torch.where(at > N - 3000, 9.0, noise.clamp(max=8)),
            torch.where(few, 7.25, 0.0), torch.full((N,), 0.1, device="cuda"), torch.where(at < N // 2, 3.5, 3.5 + 1e-6)]
    x = torch.stack(rows).to(dtype).repeat_interleave(25, 0) if N < 50000 else torch.stack(rows).to(dtype)
    verify(rdk.rdk_topk(x, k), x, k, "f32")


def test_many_beams_of_one_request():
    """Sixteen wavefronts merge; beams of which one has all the best, and entries that tie by the thousand."""
    from paper_2506_03206_amd import rdk
    G, W, N, K = 2, 64, 9001, 128
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn((G * W, N), generator=g, device="cuda")
    x[W:] = 0.0                                                                    # the second request: every score is the same
    scores = torch.full((G, W), -2.0, device="cuda")
    scores[0] = -torch.arange(W, device="cuda") * 20.0                             # the first beam has all the best
    o = rdk.rdk_beam_select(x, scores, K)
    assert (o.parent[0] == 0).all()
    ids = torch.sort(x[0], descending=True, stable=True).indices[:K]
    assert torch.equal(o.token[0].long(), ids)
    assert (o.parent[1] == 0).all() and torch.equal(o.token[1].long(), torch.arange(K, device="cuda"))
    want = torch.log_softmax(x[0].double(), 0)[ids]
    assert (o.scores[0].double() - want).abs().max() < 1e-5
