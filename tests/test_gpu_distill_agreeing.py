"""The loss of a drafter that agrees with its teacher: roundings of exponentials leave it to first order.

One entry at g, all slots outside at 0, the teacher's mass on the entry and its remainder those of the drafter: with every exponential outside 1 and their sum exact, what
is rounded is exp(-g / T), by d = 2^-24 g log2(e) / T ln 2 and an instruction's last place, up to 1e-6.  It stands in the row's sum and in rho: the loss is off by
(rho - r) d, and so by next to nothing, where rho and the sum take the same exponential (rho d where each takes its own).  What else is rounded: the sum 2^-24 once, t and with it r by
2^-24 t: 2.5 * 2^-24 in all."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [32001, 60001, 500001])         # in registers, in rounds, in parts
def test_loss_of_an_agreeing_drafter(n, dtype):
    from paper_2506_03206_amd import rdk
    B = 128
    rng = np.random.default_rng(n)
    g = torch.from_numpy((np.log(n) - rng.uniform(0.5, 2.5, B)).astype(np.float32)).cuda().to(dtype)
    z = torch.zeros((B, n), dtype=dtype, device="cuda")
    ids = torch.from_numpy(rng.integers(0, n, (B, 1)).astype(np.int32)).cuda()
    z.scatter_(1, ids.long(), g[:, None])
    y = g.double().cpu().numpy()
    norm = np.logaddexp(y, np.log(n - 1.0))
    v = torch.zeros((B, 1), device="cuda")
    lse = torch.from_numpy((norm - y).astype(np.float32)).cuda()
    log_t = -lse.double().cpu().numpy()
    t = np.exp(log_t)
    r, log_rho = 1 - t, np.log(n - 1.0) - norm
    want = t * (log_t - (y - norm)) + r * (np.log(r) - log_rho)
    for o in (rdk.rdk_distill_loss(None, z, ids, v, lse), rdk.rdk_distill_loss_grad(None, z, ids, v, lse)):
        assert np.abs(o.loss.double().cpu().numpy() - want).max() <= 2.5 * 2.0 ** -24
