"""Rows that the forward call passed over (weight 0) have gradient 0 in the backward call whatever weight it has, and whatever the row holds."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("remainder", [False, True])
@pytest.mark.parametrize("n", [257, 20003, 40001, 140001])     # a row in registers, in rounds, in parts
def test_weight_of_the_forward_call(n, remainder, dtype):
    from paper_2506_03206_amd import rdk
    B, K = 6, 9
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    z = torch.randn((B, n), generator=g, device="cuda").to(dtype)
    ids = torch.argsort(torch.rand((B, n), generator=g, device="cuda"), 1)[:, :K].to(torch.int32).contiguous()
    v = torch.randn((B, K), generator=g, device="cuda") + 2
    lse = torch.logsumexp(v, 1) + 0.2 if remainder else None
    z[1], z[3], z[5, ::2] = 200.0, float("nan"), float("inf")
    w = torch.ones(B, device="cuda")
    w[1::2] = 0.0
    o = rdk.DistillOutputs(B, n, dtype, "cuda")
    rdk.rdk_distill_loss(None, z, ids, v, lse, weight=w, outputs=o)
    for above in (None, torch.full((B,), 0.7, device="cuda")):
        o.grad.fill_(float("nan"))
        rdk.rdk_distill_grad(None, z, ids, v, o, weight=above)
        assert (o.grad[1::2] == 0).all()
        assert torch.isfinite(o.grad[::2]).all() and (o.grad[::2] != 0).any(1).all()
    both = rdk.rdk_distill_loss_grad(None, z, ids, v, lse, weight=w)
    o.grad.fill_(float("nan"))
    rdk.rdk_distill_grad(None, z, ids, v, rebind(o, both.stats))                  # the statistics of the other call
    assert (o.grad[1::2] == 0).all() and (o.loss[1::2] == 0).all()


def rebind(outputs, stats):
    outputs.stats = stats
    return outputs
