"""Gradients of log probabilities at tokens of the row's largest value: flat rows, where the largest entry is next to nothing, and sure rows whose token is given several times.

Tolerance.  With q = Z' / (1 + Z'), s = 1 / (1 + Z'), a the sum of g over the tokens there, o over the row's other tokens, u = U / (1 + Z'), the gradient is
1 / T (a q - o s + h u s).  Z' is off by the relative D of test_gpu_logprobs.py, so q by D s and s by D q; a and o are sums of up to C numbers, and every term is rounded in
a few products and sums: (C + 8) 2^-24 of the sum of its magnitudes.  u: D (3 |u| + 6 q).  2^-22 of the result, half a step more where it is bf16; n 2^-126 of Z' as there."""
import pytest
import torch

from test_gpu_logprobs import check_forward, dtype_of, near, place, reference, rows

pytestmark = pytest.mark.gpu


def at_largest(x, tokens, kind, T, g, h):
    """The gradient at every token and its tolerance, in float64, NaN at tokens that are not their row's largest value."""
    B, n = x.shape
    C = tokens.shape[1]
    x64, g64 = x.double(), torch.where((tokens >= 0) & (tokens < n), g.double(), 0.0)
    M = x64.amax(1, keepdim=True)
    d = (x64 - M) / T
    e = torch.exp(d)
    others = e.scatter(1, torch.argmax(d, 1, keepdim=True), 0.0)
    rest = others.sum(1, keepdim=True)
    s, q = 1 / (1 + rest), rest / (1 + rest)
    u = torch.where(e > 0, e * d, 0.0).sum(1, keepdim=True) * s
    d1 = torch.where(others > 0, d, -torch.inf).scatter(1, torch.argmax(d, 1, keepdim=True), -torch.inf).amax(1, keepdim=True).clamp(min=-1e4).neg().nan_to_num(nan=0.0)
    D = 2.0 ** -22 * (d1 + 20) + (28 + n // (2048 if kind == "bf16" else 1024)) * 2.0 ** -24
    h64 = h.double()[:, None] if h is not None else torch.zeros_like(M)
    same = tokens[:, :, None] == tokens[:, None, :]
    a, o = [(torch.where(w, g64[:, None, :], 0.0)).sum(2) for w in (same, ~same)]
    size_a, size_o = [(torch.where(w, g64[:, None, :].abs(), 0.0)).sum(2) for w in (same, ~same)]
    u24 = (C + 8) * 2.0 ** -24
    want = (a * q - o * s + h64 * u * s) / T
    tol = size_a * q * (D * s + u24) + size_o * s * (D * q + u24) + h64.abs() * s * (D * (3 * u.abs() + 6 * q) + u24 * u.abs())
    tol = tol + n * 2.0 ** -126 * (size_a + size_o + 105 * h64.abs())
    tol = tol / T + want.abs() * (2.0 ** -22 + (2.0 ** -8 if kind == "bf16" else 0.0)) + 1e-38
    held = (tokens >= 0) & (tokens < n)
    there = held & (torch.gather(x64, 1, torch.where(held, tokens, 0).long()) == M)
    return torch.where(there, want, torch.nan), tol


def check(x, tokens, kind, T, g, h):
    """Every call that gives a gradient: its entries at tokens of the largest value."""
    from paper_2506_03206_amd import rdk
    want, tol = at_largest(x, tokens, kind, T, g, h)
    there = ~torch.isnan(want)
    at = torch.where(there, tokens, 0).long()
    forward = rdk.rdk_logprobs(x, tokens, temperature=T)
    rdk.rdk_logprobs_grad(x, tokens, forward, g, h, temperature=T)
    step = rdk.rdk_logprobs_step(x, tokens, g, h, temperature=T)
    own = x.clone()
    rdk.rdk_logprobs_step(own, tokens, g, h, temperature=T, outputs=rdk.LogprobsOutputs(x.shape[0], tokens.shape[1], 0, "cuda", grad=own))
    ref = reference(x, place(tokens, x.shape[1]), kind, T, g=g, h=h)
    for what, grad in (("backward", forward.grad), ("step", step.grad), ("step over x", own)):
        near(torch.gather(grad, 1, at)[there], want[there], tol[there], what)
        near(grad, ref["dx"], ref["tol_dx"], what + ": all entries")


SIZES = [(8, 300), (8, 3000), (8, 9000), (40, 20000), (130, 40000), (8, 140000)]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("B,N", SIZES)
def test_flat_rows(kind, B, N):
    """The largest entry has about 1 / N of the row; its own weight is 0, as small as its share, or as large as the other tokens' weights."""
    x, gen = rows("f32", B, N, N, sigma=0.01)
    at = torch.randint(0, N, (B, 1), generator=gen, device="cuda")
    x = x.scatter(1, at, 0.125).to(dtype_of(kind))
    tokens = torch.randint(0, N, (B, 4), generator=gen, device="cuda", dtype=torch.int32)
    tokens[:, :1] = at
    tokens[1::4, 2], tokens[2::4, 3] = -1, N
    g = torch.randn((B, 4), generator=gen, device="cuda")
    g[0::4, 0], g[1::4, 0], g[2::4, 0] = 0.0, 1.1 / N, -0.3 / N
    for T, h in ((1.0, None), (0.5, torch.randn(B, generator=gen, device="cuda"))):
        check(x, tokens, kind, T, g, h)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("B,N", SIZES)
def test_the_token_of_sure_rows_given_again(kind, B, N):
    """Sixteen times the entry that the row is sure of, with unequal gradients; some of them padding or unknown ids; another token beside it."""
    gaps = torch.tensor([7.0, 12.0, 17.0, 25.0, 40.0, 55.0, 62.0, 70.0], device="cuda")
    x, gen = rows("f32", B, N, N + 1, sigma=0.5)
    x = x - x.amax(1, keepdim=True)
    at = torch.randint(0, N, (B, 1), generator=gen, device="cuda")
    x = x.scatter(1, at, gaps[torch.arange(B, device="cuda") % 8][:, None]).to(dtype_of(kind))
    tokens = at.to(torch.int32).repeat(1, 16)
    check_forward(x, tokens, kind)
    g = torch.randn((B, 16), generator=gen, device="cuda") * 10.0 ** torch.randint(-3, 3, (B, 16), generator=gen, device="cuda")
    check(x, tokens, kind, 1.0, g, None)
    tokens[1::2, 3], tokens[1::2, 9] = -1, N
    check(x, tokens, kind, 1.0, g, None)
    check(x, tokens, kind, 0.75, g, torch.full((B,), 0.5, device="cuda"))
    tokens[::3, 5] = (tokens[::3, 0] + 1) % N
    check(x, tokens, kind, 1.0, g, None)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_ties_of_the_largest(kind):
    """Several tokens at entries that tie for the largest value, one of them twice, in one vector and in others."""
    for B, N in SIZES:
        x, gen = rows(kind, B, N, N + 2, sigma=1.0)
        top = x.float().amax(1, keepdim=True).to(x.dtype)
        for j in (0, 1, 2, N // 2, N - 1):
            x[:, j:j + 1] = top
        tokens = torch.tensor([[0, 1, 1, N // 2, N - 1, 3]], device="cuda", dtype=torch.int32).repeat(B, 1)
        check(x, tokens, kind, 1.0, torch.randn((B, 6), generator=gen, device="cuda"), torch.randn(B, generator=gen, device="cuda"))
