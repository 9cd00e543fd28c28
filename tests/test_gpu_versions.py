"""What a call writes counts as written for torch: a backward pass whose saved tensors were overwritten by a call raises torch's error."""
import pytest
import torch

pytestmark = pytest.mark.gpu

B, N, n, K = 6, 500, 200, 8


def rows(seed, width=n):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn((B, width), generator=g, device="cuda")


def test_saved_entries_overwritten():
    """A second micro-batch's top entries in the buffers of the first, before the first one's backward pass."""
    from paper_2506_03206_amd import rdk
    top = rdk.rdk_topk(rows(1), K)
    z = rows(2).requires_grad_()
    loss = rdk.rdk_distill(None, z, top.ids, top.values, top.lse).sum()
    rdk.rdk_topk(rows(3), K, outputs=top)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_saved_logits_overwritten_by_a_gradient():
    from paper_2506_03206_amd import rdk
    top = rdk.rdk_topk(rows(1), K)
    z = rows(2, 16) @ torch.ones((16, n), device="cuda").requires_grad_()
    loss = rdk.rdk_distill(None, z, top.ids, top.values, top.lse).sum()
    rdk.rdk_distill_loss_grad(None, z.detach(), top.ids, top.values, top.lse, outputs=rdk.DistillOutputs(B, n, z.dtype, "cuda", grad=z.detach()))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_two_batches_of_their_own():
    """Outputs of their own for each micro-batch: both backward passes run, before and after calls into other buffers."""
    from paper_2506_03206_amd import rdk
    grads = []
    for apart in (False, True):
        z, losses, tops = rows(2).requires_grad_(), [], []
        for seed in (1, 3):
            tops.append(rdk.rdk_topk(rows(seed), K))
            losses.append(rdk.rdk_distill(None, z, tops[-1].ids, tops[-1].values, tops[-1].lse).sum())
            if not apart:
                losses.pop().backward()
        for loss in losses:
            loss.backward()
        grads.append(z.grad)
    assert torch.equal(*grads)


def test_every_output_counts_as_written():
    from paper_2506_03206_amd import rdk
    x, scores = rows(1), torch.zeros((2, 3), device="cuda")
    top, beam, out = rdk.rdk_topk(x, K), rdk.rdk_beam_select(x, scores, 3), rdk.DistillOutputs(B, n, x.dtype, "cuda")
    state, other = rows(5), rows(6)

    def written(tensors, call):
        before = [t._version for t in tensors]
        call()
        return [t._version - v for t, v in zip(tensors, before)]

    assert written([x, top.ids, top.values, top.lse], lambda: rdk.rdk_topk(x, K, outputs=top)) == [0, 1, 1, 1]
    a = (None, x, top.ids, top.values)
    assert written([x, top.ids, out.loss, out.stats, out.grad], lambda: rdk.rdk_distill_loss(*a, outputs=out)) == [0, 0, 1, 1, 0]
    assert written([x, top.ids, out.loss, out.stats, out.grad], lambda: rdk.rdk_distill_grad(*a, out)) == [0, 0, 0, 0, 1]
    assert written([x, top.ids, out.loss, out.stats, out.grad], lambda: rdk.rdk_distill_loss_grad(*a, outputs=out)) == [0, 0, 1, 1, 1]
    assert written([x, scores, beam.scores, beam.parent, beam.token, beam.finished],
                   lambda: rdk.rdk_beam_select(x, scores, 3, outputs=beam)) == [0, 0, 1, 1, 1, 1]
    assert written([state, beam.parent], lambda: rdk.rdk_beam_reorder([state], beam.parent)) == [1, 0]
    assert written([state, other, beam.parent], lambda: rdk.rdk_beam_reorder([state], beam.parent, out=[other])) == [0, 1, 0]
    bad = rdk.TopkOutputs(B, n, K, "cuda")
    with pytest.raises(rdk.RdkError):
        written([bad.ids], lambda: rdk.rdk_topk(x, K, temperature=-1.0, outputs=bad))
    assert bad.ids._version == 0                                                       # nothing was written


def test_inference_mode():
    """Tensors without versions, outputs of every call among them."""
    from paper_2506_03206_amd import rdk
    with torch.inference_mode():
        x, scores = rows(1), torch.zeros((2, 3), device="cuda")
        top = rdk.rdk_topk(x, K)
        out = rdk.rdk_distill_loss_grad(None, x, top.ids, top.values, top.lse)
        beam = rdk.rdk_beam_select(x, scores, 3)
        moved = rdk.rdk_beam_reorder([x], beam.parent)[0]
        assert torch.isfinite(out.loss).all() and torch.isfinite(moved).all()
    rdk.rdk_topk(rows(2), K, outputs=rdk.TopkOutputs(B, n, K, "cuda"))
