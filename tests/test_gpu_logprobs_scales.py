"""Logits and temperatures of any size together: distances from the largest value that are ordinary numbers only over T, differences of logits that are no number of 32
bits, the lowest finite value as a mask at temperatures that see it.  Tolerances: those of test_gpu_logprobs.py."""
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


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("B,N", SIZES)
def test_the_lowest_and_the_largest_value(kind, B, N):
    """Half of the ids at the lowest finite value beside ordinary ones, beside the largest finite value, and beside one of it: at 2^127 these are 2 or 4 apart."""
    low, high = torch.finfo(dtype_of(kind)).min, torch.finfo(dtype_of(kind)).max
    for e, size in ((0, 1.0), (1, 1.0), (60, 1.0), (120, 2.0 ** 30), (126, 2.0 ** 40), (127, 2.0 ** 40)):
        x, gen = rows(kind, B, N, N + e)
        half = torch.rand(x.shape, generator=gen, device="cuda") < 0.5
        x[0].masked_fill_(half[0], low)
        x[1] = torch.where(half[1], torch.tensor(low, device="cuda"), torch.tensor(high, device="cuda")).to(x.dtype)
        x[2] = low
        x[2, N // 3] = high
        x[3].masked_fill_(half[3], low)
        x[3, ::3] = -INF
        x[4] = low
        tokens = some_tokens(B, N, 3, gen)
        tokens[:, 1] = half.float().argmax(1).to(torch.int32)
        tokens[2, 2] = N // 3
        g, h = torch.randn((B, 3), generator=gen, device="cuda") * size, torch.randn(B, generator=gen, device="cuda") * size
        check_forward(x, tokens, kind, 2.0 ** e, 3)
        check_gradients(x, tokens, kind, 2.0 ** e, g, h)
        check_gradients(x, tokens, kind, 2.0 ** e, None, h)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("B,N", SIZES)
def test_large_logits_at_high_temperatures(kind, B, N):
    """Logits of a few T = 2^120, whose distances' sums over a row are no number of 32 bits before they are taken over T."""
    x, gen = rows("f32", B, N, N + 3, sigma=1.5)
    x = (x * 2.0 ** 120).to(dtype_of(kind))
    tokens = some_tokens(B, N, 2, gen)
    g, h = torch.randn((B, 2), generator=gen, device="cuda") * 2.0 ** 30, torch.randn(B, generator=gen, device="cuda") * 2.0 ** 30
    check_forward(x, tokens, kind, 2.0 ** 120, 3)
    check_gradients(x, tokens, kind, 2.0 ** 120, None, h)
    check_gradients(x, tokens, kind, 2.0 ** 120, g, h)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("N", [3, 300, 3000, 9001, 20000, 140001])
def test_sure_rows_at_low_temperatures(kind, N):
    """Rows that are sure of an entry, with logits of T's size: products of an exponential and a distance that are no normal number before they are taken over T."""
    gaps = torch.tensor([7.0, 25.0, 40.0, 60.0, 70.0, 78.0], device="cuda")
    for e in (-9, -11, -20, -37, -100, -120):
        x, gen = rows("f32", 6, N, N - e, sigma=0.5)
        x = x - x.amax(1, keepdim=True)
        at = torch.randint(0, N, (6, 1), generator=gen, device="cuda")
        x = (x.scatter(1, at, gaps[:, None]) * 2.0 ** e).to(dtype_of(kind))
        tokens = torch.cat([at.to(torch.int32), some_tokens(6, N, 1, gen)], 1)
        _, ref = check_forward(x, tokens, kind, 2.0 ** e, min(N, 3))
        assert (ref["tol_h"][:5] < 2e-4 * ref["entropy"][:5]).all()
        if e >= -40:
            g, h = torch.randn((6, 2), generator=gen, device="cuda"), torch.randn(6, generator=gen, device="cuda")
            check_gradients(x, tokens, kind, 2.0 ** e, g, h)
            check_gradients(x, tokens, kind, 2.0 ** e, None, h)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("B,N", SIZES)
def test_large_logits_at_low_temperatures(kind, B, N):
    """Rows whose largest value over T is no number of 32 bits: it has all of the row, or shares it with those that tie, tokens among them or not."""
    for e, size in ((-20, 110), (-40, 95), (-40, 120), (-126, 2), (-126, 100)):
        x, gen = rows("f32", B, N, N - e, sigma=1.0)
        x = (x * 2.0 ** size).to(dtype_of(kind))
        x[1] = -x[1].abs()
        x[2] = (x[2].float() / 2.0 ** (size + 1)).round().to(x.dtype) * 2.0 ** (size + 1)
        x[3, ::2] = -INF
        x[4] = -(2.0 ** size)
        x[5, 1:] = x[5, :1]
        tokens = some_tokens(B, N, 3, gen)
        tokens[::2, 1] = x[::2].float().argmax(1).to(torch.int32)
        check_forward(x, tokens, kind, 2.0 ** e, 3)
        if e >= -40:
            g, h = torch.randn((B, 3), generator=gen, device="cuda"), torch.randn(B, generator=gen, device="cuda")
            check_gradients(x, tokens, kind, 2.0 ** e, g, h)
            check_gradients(x, tokens, kind, 2.0 ** e, None, h)
