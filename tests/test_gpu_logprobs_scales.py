"""Logits and temperatures of any size together: distances from the largest value that are ordinary numbers only over T.  Tolerances: those of test_gpu_logprobs.py."""
import pytest
import torch

from test_gpu_logprobs import check_forward, check_gradients, dtype_of, rows, some_tokens

pytestmark = pytest.mark.gpu
INF = float("inf")
SIZES = [(6, 300), (6, 3000), (6, 9001), (40, 20000), (130, 40000), (6, 140001)]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("B,N", SIZES)
def test_logits_of_the_temperatures_size(kind, B, N):
    """Logits of a few T: the gradient of the entropy alone and with others.  Powers of two, so that 1 / T is exact."""
    for e in (-20, 40, 70, 100):
        x, gen = rows("f32", B, N, N, sigma=1.5)
        x = (x * 2.0 ** e).to(dtype_of(kind))
        x[1, ::2] = -INF
        tokens = some_tokens(B, N, 2, gen)
        tokens[2:, 1] = x[2:].float().argmax(1).to(torch.int32)
        g, h = torch.randn((B, 2), generator=gen, device="cuda"), torch.randn(B, generator=gen, device="cuda")
        check_forward(x, tokens, kind, 2.0 ** e, 3)
        check_gradients(x, tokens, kind, 2.0 ** e, None, h)
        check_gradients(x, tokens, kind, 2.0 ** e, g, h)
