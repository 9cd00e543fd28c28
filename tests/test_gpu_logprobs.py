"""Log probabilities of given tokens, ranks, entropy, top entries and gradients where they can go wrong, against their definitions in 64 bits.

Tolerances.  With d = (x - M) / T, Z' = sum of exp(d) over all but the largest, U = sum exp(d) d: an exponent d is rounded when the difference is taken, in
1 / T and log2(e) / T, and in their product: 2^-22 |d| in all; the exponential itself and d in U add 2^-22.  Terms that lie 20 below the largest of the others come to
nothing beside it, so Z' and U are off by the relative D = 2^-22 (D1 + 20) + A 2^-24, D1 the distance of the second largest entry (0 for ties), A the
additions that a term goes through: at most one for each of 8 entries, vectors of a lane (n / 2048 of bf16, n / 1024 of fp32) and 20 to bring lanes and parts together.
The distances in U are first taken to a reference that a lane's largest value, in units of log 2, lies at most 8.5 above, and are brought to the largest value after
the sums: |d| <= (distance) + 8.5 log 2, so that U is off by D (|U| + 6 Z') (where nearly all entries tie, U comes to much less than Z').
  log probability:  2^-22 |d| (its own distance) + D Z' / (1 + Z') + 2^-23 of it
  entropy:          D (7 Z' / (1 + Z') + 2 |U| / (1 + Z')) + 2^-23 of it
  s:                the relative S = 2^-22 (|d| + 1) + D Z' / (1 + Z')
  gradient:         1/T (s S (|G| + |h| (|d| + |u|)) + s |h| (2^-22 |d| + D (|u| + 6 Z' / (1 + Z'))) + s 2^-20 sum |g| + 2^-20 sum |g| at the tokens), u = U / (1 + Z'), 2^-22 of it,
                    and where it is rounded to bf16 half a step, 2^-8 of it.  (G is a sum of up to 16 numbers, off by 16 2^-24 sum |g|, however small it is.
                    The exponential of the hardware gives 0 where the result is below 2^-126: s there is off by that, in units of 1 / (1 + Z'), Z' by n 2^-126, and U by 104 times that: beyond a
                    distance of 104 it is less than 2^-149 of anything.)  At a token that is the largest entry, alone: |g| Z' / (1 + Z') D in the place of 2^-20 |g|."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
INF = math.inf


def dtype_of(kind):
    return torch.bfloat16 if kind == "bf16" else torch.float32


def reference(x, tokens, kind, T=1.0, slots=None, g=None, h=None):
    """Everything in float64 on x's device.  tokens [B,C] places in the row (-1: an unknown id, -2: nothing asked)."""
    x64 = x.double()
    B, n = x64.shape
    if kind == "prob":
        y = torch.log(x64)
        M = y.amax(1, keepdim=True)
        d = y - M
    else:
        M = x64.amax(1, keepdim=True)
        d = (x64 - M) / T
    masked = (M == -INF)[:, 0]
    bad = torch.isnan(x64).any(1) | (x64 == INF).any(1)
    d = torch.where(masked[:, None], torch.full_like(d, -INF), d)
    e = torch.exp(d)
    top = torch.argmax(torch.nan_to_num(d, nan=INF), 1, keepdim=True)
    others = e.scatter(1, top, 0.0)
    rest = others.sum(1)
    U = torch.where(e > 0, e * d, 0.0).sum(1)
    all_ = 1 + rest
    s = e / all_[:, None]
    u = U / all_
    entropy = torch.where(masked, torch.zeros_like(rest), torch.log1p(rest) - u)
    d1 = torch.where(others > 0, d, -INF).scatter(1, top, -INF).amax(1).clamp(min=-1e4).neg().nan_to_num(nan=0.0)
    adds = 28 + n // (2048 if kind == "bf16" else 1024)
    D = 2.0 ** -22 * (d1 + 20) + adds * 2.0 ** -24
    share = rest / all_
    at = tokens.clamp(min=0).long()
    dt = torch.gather(d, 1, at)
    lp = torch.where(masked[:, None], torch.full_like(dt, -INF), dt - torch.log1p(rest)[:, None])
    lp = torch.where(tokens == -2, torch.zeros_like(lp), torch.where(tokens == -1, torch.full_like(lp, -INF), lp))
    lp = torch.where(lp < -torch.finfo(torch.float32).max, -INF, lp)     # no number of 32 bits: 4 / T at T = 2^-126 is 3.4e38 already
    dfin = lambda a: torch.where(torch.isfinite(a), a, torch.zeros_like(a)).abs()  # noqa: E731
    tol_lp = 2.0 ** -22 * dfin(dt) + (D * share)[:, None] + 2.0 ** -23 * dfin(lp) + n * 2.0 ** -126
    tol_h = D * (7 * share + 2 * u.abs()) + 2.0 ** -23 * entropy.abs() + 105 * n * 2.0 ** -126
    v = torch.gather(x64, 1, at)
    place = torch.arange(n, device=x.device)
    ranks = torch.stack([(x64 > v[:, c:c + 1]).sum(1) + ((x64 == v[:, c:c + 1]) & (place < at[:, c:c + 1])).sum(1) for c in range(tokens.shape[1])], 1)
    ranks = torch.where((tokens >= 0) & (lp > -INF) & ~bad[:, None], ranks, -1)
    out = {"logprob": lp, "tol_lp": tol_lp, "entropy": entropy, "tol_h": tol_h, "rank": ranks, "masked": masked, "bad": bad}
    if g is None and h is None:
        return out
    C = tokens.shape[1]
    g64 = torch.where(tokens >= 0, g.double(), 0.0) if g is not None else torch.zeros(B, C, dtype=torch.float64, device=x.device)
    h64 = h.double() if h is not None else torch.zeros(B, dtype=torch.float64, device=x.device)
    live = ((g64 != 0).any(1) | (h64 != 0)) & ~masked
    G = g64.sum(1, keepdim=True)
    dd = torch.where(e > 0, d, 0.0)
    factor = G + h64[:, None] * (dd - u[:, None])
    dx = -s * factor
    S = 2.0 ** -22 * (dd.abs() + 1) + (D * share)[:, None]
    tol = s * S * (G.abs() + h64[:, None].abs() * (dd.abs() + u[:, None].abs())) + s * h64[:, None].abs() * (2.0 ** -22 * dd.abs() + (D * (u.abs() + 6 * share))[:, None])
    # at the tokens; of a sure row 1 - s = Z' / (1 + Z') is formed without a difference, here too
    add = torch.zeros_like(dx).scatter_add_(1, at, g64)
    met = torch.zeros_like(dx).scatter_add_(1, at, (tokens >= 0).double()) > 0
    largest = met & (d == 0)
    dx = torch.where(largest, (add - G) + (G * share[:, None] + h64[:, None] * u[:, None] / all_[:, None]), dx + add)
    total = g64.abs().sum(1, keepdim=True)
    tol = tol + s * 2.0 ** -20 * total
    far = torch.where(torch.isfinite(d), d, 0.0).abs().clamp(max=200.0)
    tol = tol + 2.0 ** -126 / all_[:, None] * (G.abs() + h64[:, None].abs() * (far + u[:, None].abs()))
    alone = largest & (add == G) & (g64.ne(0).sum(1, keepdim=True) == 1)
    tol = torch.where(alone, (D * share)[:, None] * total + h64[:, None].abs() * (D * (u.abs() * 3 + 6 * share))[:, None] / all_[:, None], tol + met * 2.0 ** -20 * total)
    tol = tol + n * 2.0 ** -126 * (G.abs() + 105 * h64[:, None].abs())       # of Z' and U
    dx, tol = dx / T, tol / T
    tol = tol + dx.abs() * (2.0 ** -22 + (2.0 ** -8 if x.dtype == torch.bfloat16 else 0.0)) + 1e-38
    out["dx"], out["tol_dx"] = torch.where(live[:, None], dx, torch.zeros_like(dx)), torch.where(live[:, None], tol, torch.zeros_like(tol))
    return out


def near(got, want, tol, what):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what + ": NaN elsewhere"
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    off = torch.where(same, torch.zeros_like(want), (got - want).abs() - tol)
    assert not torch.isnan(off).any() and float(off.max()) <= 0, "%s off by %.3g beyond %.3g" % (what, float(off.max()), float(tol.flatten()[off.argmax()]))


def place(tokens, N):
    """Places of tokens without a pruned vocabulary."""
    return torch.where(tokens < 0, -2, torch.where(tokens >= N, -1, tokens)).long()


def rows(kind, B, N, seed, ld=None, sigma=3.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = torch.randn((B, N), generator=gen, device="cuda") * sigma
    if kind == "prob":
        x = torch.softmax(x, 1)
    out = torch.empty((B, ld or N), dtype=dtype_of(kind), device="cuda")[:, :N]
    return out.copy_(x), gen


def some_tokens(B, N, C, gen):
    t = torch.randint(0, N, (B, C), generator=gen, device="cuda", dtype=torch.int32)
    t[0, 0] = N - 1
    if C > 1:
        t[-1, -1] = t[-1, 0]                       # the same token twice
    return t


def check_forward(x, tokens, kind, T=1.0, k=0, kernel=None, places=None):
    if k:                                                               # without top entries, too: other kernels
        check_forward(x, tokens, kind, T, 0, kernel, places)
    from paper_2506_03206_amd import rdk
    B, N = x.shape
    o = rdk.LogprobsOutputs(B, tokens.shape[1], k, "cuda")
    for t in (o.logprob, o.entropy, o.top_logprobs, o.stats):
        t.fill_(float("nan"))
    o.rank.fill_(-77), o.top_ids.fill_(-77)
    rdk.rdk_logprobs(x, tokens, "prob" if kind == "prob" else "logit", k=k, kernel=kernel, temperature=T, outputs=o)
    ref = reference(x, place(tokens, N) if places is None else places, kind, T)
    near(o.logprob, ref["logprob"], ref["tol_lp"], "logprob")
    near(o.entropy, ref["entropy"], ref["tol_h"], "entropy")
    assert torch.equal(o.rank.long(), ref["rank"]), "ranks"
    if k:
        top = rdk.rdk_topk(x, k, "prob" if kind == "prob" else "logit")
        want = reference(x, torch.where(top.ids < 0, -1, top.ids).long(), kind, T)
        near(o.top_logprobs, want["logprob"], want["tol_lp"], "top_logprobs")
        assert torch.equal(o.top_ids, top.ids if kernel is None else torch.where(top.ids < 0, -1, kernel.kept[top.ids.clamp(min=0).long()]))
    return o, ref


def check_gradients(x, tokens, kind, T, g, h, kernel=None, places=None):
    """The backward call, the step, and both over x itself."""
    from paper_2506_03206_amd import rdk
    B, N = x.shape
    ref = reference(x, place(tokens, N) if places is None else places, kind, T, g=g, h=h)
    a = rdk.rdk_logprobs(x, tokens, kernel=kernel, temperature=T)
    a.grad = torch.full_like(x, float("nan"))
    rdk.rdk_logprobs_grad(x, tokens, a, g, h, kernel=kernel, temperature=T)
    near(a.grad, ref["dx"], ref["tol_dx"], "gradient")
    b = rdk.LogprobsOutputs(B, tokens.shape[1], 0, "cuda", grad=torch.full_like(x, float("nan")))
    rdk.rdk_logprobs_step(x, tokens, g, h, kernel=kernel, temperature=T, outputs=b)
    near(b.logprob, ref["logprob"], ref["tol_lp"], "step: logprob")
    near(b.entropy, ref["entropy"], ref["tol_h"], "step: entropy")
    near(b.grad, ref["dx"], ref["tol_dx"], "step: gradient")
    for both in (False, True):
        own = torch.empty((B, x.stride(0)), dtype=x.dtype, device="cuda")[:, :N].copy_(x)
        c = rdk.LogprobsOutputs(B, tokens.shape[1], 0, "cuda", grad=own)
        if both:
            rdk.rdk_logprobs_step(own, tokens, g, h, kernel=kernel, temperature=T, outputs=c)
            near(c.logprob, ref["logprob"], ref["tol_lp"], "step over x: logprob")
        else:
            c.stats = a.stats
            rdk.rdk_logprobs_grad(own, tokens, c, g, h, kernel=kernel, temperature=T)
        near(own, ref["dx"], ref["tol_dx"], "gradient over x")
    return a, ref


SIZES = [(1, 1), (3, 2), (2, 7), (5, 63), (2, 64), (4, 257), (7, 1000), (3, 8191), (2, 8197), (40, 16385), (1, 50001), (2, 128257), (300, 9000)]


@pytest.mark.parametrize("kind", ["bf16", "f32", "prob"])
@pytest.mark.parametrize("B,N", SIZES)
def test_sizes(kind, B, N):
    for C, k, T, ld in ((1, 0, 1.0, N), (3, min(5, N), 2.0, N + 3), (16, min(128, N), 0.25, N + 1)):
        if kind == "prob":
            T = 1.0
        x, gen = rows(kind, B, N, B * N + C, ld)
        check_forward(x, some_tokens(B, N, C, gen), kind, T, k)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("B,N", SIZES + [(3, 65536), (2, 65537), (2, 131072), (2, 131073), (3, 4096), (3, 32768), (3, 32769), (3, 2048), (3, 2049)])
def test_gradients(kind, B, N):
    for C, T, entropy, ld in ((1, 1.0, False, N), (3, 2.0, True, N + 5), (16, 0.5, True, N)):
        x, gen = rows(kind, B, N, 7 * B * N + C, ld)
        tokens = some_tokens(B, N, C, gen)
        g = torch.randn((B, C), generator=gen, device="cuda")
        h = torch.randn(B, generator=gen, device="cuda") if entropy else None
        check_gradients(x, tokens, kind, T, g, h)
    check_gradients(x, tokens, kind, 1.0, None, torch.randn(B, generator=gen, device="cuda"))


@pytest.mark.parametrize("kind", ["bf16", "f32", "prob"])
@pytest.mark.parametrize("N", [5, 700, 5000, 20000, 60000, 90001])
def test_masks(kind, N):
    """Half of the ids masked, all, all but one, the type's lowest value as a mask, tokens that are masked, unknown, or padding."""
    B = 8
    x, gen = rows(kind, B, N, N)
    none = 0.0 if kind == "prob" else -INF
    x[0, torch.rand(N, generator=gen, device="cuda") < 0.5] = none
    x[1] = none
    x[2] = none
    x[2, N // 2] = 0.75
    if kind != "prob":
        x[3, torch.rand(N, generator=gen, device="cuda") < 0.5] = torch.finfo(x.dtype).min
        x[4] = torch.finfo(x.dtype).min
    x[5, : N - 1] = none
    x[6] = x[6, 0]                                                      # all equal
    tokens = torch.randint(0, N, (B, 4), generator=gen, device="cuda", dtype=torch.int32)
    tokens[:, 1] = torch.tensor([-1, N, -5, 2 ** 31 - 1, 0, N - 1, N // 2, -2 ** 31], device="cuda", dtype=torch.int32)
    tokens[2, 0] = tokens[2, 2] = N // 2
    tokens[5, 3] = N - 1
    check_forward(x, tokens, kind, 1.0, min(3, N))
    if kind != "prob":
        g = torch.randn((B, 4), generator=gen, device="cuda")
        check_gradients(x, tokens, kind, 1.0, g, None)
        check_gradients(x, tokens, kind, 3.0, g, torch.randn(B, generator=gen, device="cuda"))


@pytest.mark.parametrize("kind", ["bf16", "f32", "prob"])
@pytest.mark.parametrize("N", [9, 3001, 10000, 20000, 40000, 90001])
def test_nan_and_infinity(kind, N):
    """A NaN or an infinity shows in its row and in no other; masked tokens of such a row stay -inf."""
    B = 6
    x, gen = rows(kind, B, N, N + 1)
    x[1, N // 2] = float("nan")
    x[2, N - 1] = INF
    x[3, 0] = float("nan")
    x[3, 1:] = 0.0 if kind == "prob" else -INF
    tokens = torch.tensor([[0, 1], [0, N // 2], [0, N - 1], [0, 1], [1, 2], [2, N - 1]], device="cuda", dtype=torch.int32)
    from paper_2506_03206_amd import rdk
    o = rdk.rdk_logprobs(x, tokens, "prob" if kind == "prob" else "logit")
    assert torch.isnan(o.entropy[1:4]).all() and (o.rank[1:4] == -1).all()
    assert torch.isnan(o.logprob[1:3]).all() and torch.isnan(o.logprob[3, 0]) and o.logprob[3, 1] == -INF
    fine = [0, 4, 5]
    check_forward(x[fine].contiguous(), tokens[fine].contiguous(), kind)
    want = rdk.rdk_logprobs(x[fine].contiguous(), tokens[fine].contiguous(), "prob" if kind == "prob" else "logit")
    assert torch.isfinite(o.entropy[fine]).all() and torch.isfinite(o.logprob[fine]).all()
    near(o.entropy[fine], want.entropy.double(), 1e-5 * want.entropy.double().abs(), "rows beside it")
    if kind == "prob":
        return
    g, h = torch.ones((B, 2), device="cuda"), torch.ones(B, device="cuda")
    rdk.rdk_logprobs_grad(x, tokens, o, g, h)
    s = rdk.rdk_logprobs_step(x, tokens, g, h)
    for grad in (o.grad, s.grad):
        assert torch.isnan(grad[1:4]).all() and torch.isfinite(grad[fine].float()).all()
    # a row of which nothing is asked is not read by the backward call
    g[1:4], h[1:4] = 0.0, 0.0
    rdk.rdk_logprobs_grad(x, tokens, o, g, h)
    s = rdk.rdk_logprobs_step(x, tokens, g, h)
    for grad in (o.grad, s.grad):
        assert (grad[1:4] == 0).all() and torch.isfinite(grad[fine].float()).all() and (grad[fine].float().abs().amax(1) > 0).all()


@pytest.mark.parametrize("kind", ["bf16", "f32", "prob"])
@pytest.mark.parametrize("N", [2, 300, 6000, 15000, 30000, 60000, 130000])
def test_sure_rows(kind, N):
    """Rows that are sure of one entry: the others together come to 1e-3 down to 1e-30 of it; the entropy, that entry's log probability and its gradient keep
    their own last bits, wherever in the row the entry stands."""
    gaps = [7.0, 12.0, 17.0, 25.0, 40.0, 70.0]
    x, gen = rows("f32", len(gaps), N, N + 2, sigma=0.5)
    x = x - x.amax(1, keepdim=True)
    at = torch.randint(0, N, (len(gaps), 1), generator=gen, device="cuda")
    at[0], at[1] = 0, N - 1
    x = x.scatter(1, at, torch.tensor(gaps, device="cuda")[:, None])
    x = torch.exp(x - 60.0).float() if kind == "prob" else x.to(dtype_of(kind))
    tokens = at.to(torch.int32)
    o, ref = check_forward(x, tokens, kind)
    assert (ref["tol_lp"] < 2e-4 * ref["logprob"].abs()).all() and (ref["tol_h"] < 2e-4 * ref["entropy"]).all()
    if kind != "prob":
        g = torch.full((len(gaps), 1), -0.37, device="cuda")
        _, ref = check_gradients(x, tokens, kind, 1.0, g, None)
        assert (ref["tol_dx"].gather(1, at) < 0.01 * ref["dx"].abs().gather(1, at)).all()
        check_gradients(x, tokens, kind, 1.0, g, torch.full((len(gaps),), 0.5, device="cuda"))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1e4, 1e10, 1e30])
def test_large_logits(kind, scale):
    """Logits far from zero and far apart; a mask of -1e10 instead of -inf."""
    x, gen = rows("f32", 6, 20001, 5)
    x = torch.cat([x[:3] * scale, x[3:] + scale]).to(dtype_of(kind))
    x[5, ::2] = -1e10
    tokens = some_tokens(6, 20001, 3, gen)
    tokens[:, 2] = x.float().argmax(1).to(torch.int32)
    g, h = torch.randn((6, 3), generator=gen, device="cuda"), torch.randn(6, generator=gen, device="cuda")
    check_forward(x, tokens, kind, 1.0, 4)
    check_gradients(x, tokens, kind, 1.0, g, h)
    check_gradients(x, tokens, kind, 1e4, g, h)


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-3, 7.0, 1e30])
def test_weights_of_any_scale(scale):
    x, gen = rows("prob", 5, 10007, 6)
    x = x * scale
    x[1, 17] = 3.0 * scale                                              # sure of it
    tokens = some_tokens(5, 10007, 2, gen)
    tokens[1, 0] = 17
    tokens[:, 1] = x.argmax(1).to(torch.int32)
    if scale == 1e-38:                                                  # weights that are not normal numbers are sums of fewer bits: what they are worth
        from paper_2506_03206_amd import rdk
        o = rdk.rdk_logprobs(x, tokens, "prob")
        ref = reference(x, place(tokens, 10007), "prob")
        assert torch.equal(o.rank.long(), ref["rank"])
        near(o.logprob, ref["logprob"], ref["logprob"].abs().nan_to_num(posinf=0) * 0.05 + 0.05, "logprob of the smallest weights")
        return
    check_forward(x, tokens, "prob", k=9)


def test_ranks_of_ties():
    """Equal entries in order of their places, across vectors, rounds and parts, and zeros of both signs."""
    for kind in ("bf16", "f32"):
        for B, N in ((3, 13), (3, 2050), (3, 7001), (3, 16001), (3, 30001), (33, 31001), (3, 70001)):
            x = torch.randint(-2, 3, (B, N), device="cuda").to(dtype_of(kind))
            x[1] = torch.where(x[1] == 0, torch.tensor(-0.0, device="cuda", dtype=x.dtype), x[1])
            x[2, ::3] = -0.0
            tokens = torch.stack([torch.randperm(N, device="cuda")[:13].to(torch.int32) for _ in range(B)])
            tokens[0, 0], tokens[0, 1] = 0, N - 1
            check_forward(x, tokens, kind, k=5)


@pytest.mark.parametrize("kind", ["bf16", "f32", "prob"])
def test_pruned_vocabulary(kind):
    """Rows over kept slots, target ids as tokens: ids are brought to slots and back; pruned ids are unknown."""
    from paper_2506_03206_amd import rdk
    N, n, B = 4000, 1111, 9
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    kept = torch.sort(torch.randperm(N, generator=gen, device="cuda")[:n]).values.to(torch.int32)
    kernel = rdk.rdk_build_kernel(N, kept, rdk.IDENTITY)
    kernel.kept = kept
    slot_of = torch.full((N,), -1, dtype=torch.int64, device="cuda")
    slot_of[kept.long()] = torch.arange(n, device="cuda")
    x, _ = rows(kind, B, n, 4)
    tokens = torch.randint(0, N, (B, 6), generator=gen, device="cuda", dtype=torch.int32)
    tokens[0, 0], tokens[1, 1], tokens[2] = -1, N, kept[:6]
    slots = torch.where(tokens < 0, -2, torch.where(tokens >= N, -1, slot_of[tokens.clamp(0, N - 1).long()]))
    check_forward(x, tokens, kind, k=7, kernel=kernel, places=slots)
    if kind != "prob":
        g, h = torch.randn((B, 6), generator=gen, device="cuda"), torch.randn(B, generator=gen, device="cuda")
        check_gradients(x, tokens, kind, 1.0, g, h, kernel, slots)
        check_gradients(x, tokens, kind, 1.0, g, None, kernel, slots)
    with pytest.raises(rdk.RdkError):
        rdk.rdk_logprobs(torch.zeros((B, n + 1), device="cuda"), tokens, kernel=kernel)


def test_gradient_against_differences():
    """The objective in 64 bits from the library's own formulas at x +- e: differences of it, and the gradient that the library returns."""
    x, gen = rows("f32", 3, 50, 11)
    tokens = torch.randint(0, 50, (3, 2), generator=gen, device="cuda", dtype=torch.int32)
    g, h = torch.randn((3, 2), generator=gen, device="cuda"), torch.randn(3, generator=gen, device="cuda")
    from paper_2506_03206_amd import rdk
    leaf = x.clone().requires_grad_(True)
    lp, entropy = rdk.rdk_token_logprobs(leaf, tokens, temperature=1.5)
    ((lp * g).sum() + (entropy * h).sum()).backward()

    def objective(y):
        log_s = torch.log_softmax(y / 1.5, 1)
        return (log_s.gather(1, tokens.long()) * g.double()).sum(1) - ((log_s.exp() * log_s).sum(1) * h.double())

    e, y = 1e-5, x.double()
    for j in range(50):
        step = torch.zeros_like(y)
        step[:, j] = e
        slope = (objective(y + step) - objective(y - step)) / (2 * e)
        # a difference of 64-bit numbers of about 20: 20 2^-52 / e, its third-order term: 20 e^2; the gradient itself: 1e-5 of numbers up to 20
        assert (leaf.grad[:, j].double() - slope).abs().max() < 2e-4


def test_under_torch():
    """Automatic differentiation: one of the outputs unused, a broadcast gradient, tokens of one dimension, and outputs that were written over."""
    from paper_2506_03206_amd import rdk
    x, gen = rows("bf16", 4, 1000, 12)
    tokens = torch.randint(0, 1000, (4,), generator=gen, device="cuda", dtype=torch.int32)
    for use in ("logprob", "entropy", "none"):
        leaf = x.clone().requires_grad_(True)
        lp, entropy = rdk.rdk_token_logprobs(leaf, tokens)
        assert lp.shape == (4,) and entropy.shape == (4,)
        if use == "none":
            (leaf.sum() * 2).backward()
            continue
        (lp if use == "logprob" else entropy).mean().backward()
        quarter = torch.full((4,), 0.25, device="cuda")
        ref = reference(x, tokens[:, None].long(), "bf16", g=quarter[:, None] if use == "logprob" else None, h=None if use == "logprob" else quarter)
        near(leaf.grad, ref["dx"], ref["tol_dx"], use)
    leaf = x.clone().requires_grad_(True)
    y = leaf * 1.0
    lp, _ = rdk.rdk_token_logprobs(y, tokens)
    rdk.rdk_logprobs_step(y.detach(), tokens, torch.ones(4, device="cuda"), outputs=rdk.LogprobsOutputs(4, 1, 0, "cuda", grad=y.detach()))
    with pytest.raises(RuntimeError):
        lp.sum().backward()


def test_streams_and_graphs():
    """On a stream of its own, and captured into a graph that is replayed between eager calls on new inputs."""
    from paper_2506_03206_amd import rdk
    for B, N, k in ((4, 128256, 5), (64, 3001, 0)):
        x, gen = rows("bf16", B, N, 13)
        tokens = some_tokens(B, N, 2, gen)
        g, h = torch.randn((B, 2), generator=gen, device="cuda"), torch.randn(B, generator=gen, device="cuda")
        o = rdk.LogprobsOutputs(B, 2, k, "cuda", grad=torch.empty_like(x))
        s = rdk.LogprobsOutputs(B, 2, 0, "cuda", grad=torch.empty_like(x))

        def both(o, s):
            rdk.rdk_logprobs(x, tokens, k=k, outputs=o)
            rdk.rdk_logprobs_grad(x, tokens, o, g, h)
            rdk.rdk_logprobs_step(x, tokens, g, h, outputs=s)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            both(o, s)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            both(o, s)
        for i in range(4):
            x.copy_(rows("bf16", B, N, 20 + i)[0])
            e, es = rdk.LogprobsOutputs(B, 2, k, "cuda"), rdk.LogprobsOutputs(B, 2, 0, "cuda")
            both(e, es)
            for t in (o.logprob, o.entropy, o.grad, s.logprob, s.grad):
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            for name in ("logprob", "rank", "entropy", "top_ids", "top_logprobs", "grad"):
                assert torch.equal(getattr(o, name), getattr(e, name)), name
            for name in ("logprob", "entropy", "grad"):
                assert torch.equal(getattr(s, name), getattr(es, name)), name


def test_what_is_not_asked_for_stays():
    """Ranks that are not asked for and rows behind the batch are left as they were; without statistics and entropy the rest is the same."""
    import ctypes
    from paper_2506_03206_amd import rdk
    x, gen = rows("bf16", 5, 777, 14)
    tokens = some_tokens(5, 777, 2, gen)
    o = rdk.LogprobsOutputs(5, 2, 0, "cuda")
    o.rank.fill_(-77)
    rdk.rdk_logprobs(x, tokens, ranks=False, outputs=o)
    assert (o.rank == -77).all()
    room = torch.full((9, 777), 5.0, dtype=torch.bfloat16, device="cuda")
    o.grad = room[:5]
    rdk.rdk_logprobs_grad(x, tokens, o, torch.ones((5, 2), device="cuda"))
    assert (room[5:] == 5.0).all()
    lp = torch.empty((5, 2), device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    p = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    d = rdk.LogprobsDesc(B=5, N=777, C=2, k=0, temperature=1.0)
    st = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert rdk.lib().rdk_logprobs(ctypes.byref(d), None, p(x), 2, 777, p(tokens), p(lp), None, None, None, None, None, p(ws), ws.numel(), st) == 0
    assert torch.equal(lp, o.logprob)
    dx = torch.empty_like(x)
    g = torch.ones((5, 2), device="cuda")
    assert rdk.lib().rdk_logprobs_step(ctypes.byref(d), None, p(x), 2, 777, p(tokens), p(g), None, p(lp), None, None, p(dx), 777, p(ws), ws.numel(),
                                       st) == 0
    ref = reference(x, tokens.long(), "bf16", g=g)
    near(dx, ref["dx"], ref["tol_dx"], "step without statistics")
    long = torch.randn((2, 140000), device="cuda").bfloat16()
    both = torch.empty_like(long)
    d = rdk.LogprobsDesc(B=2, N=140000, C=1, k=0, temperature=1.0)
    t = torch.tensor([5, 139999], dtype=torch.int32, device="cuda")
    assert rdk.lib().rdk_logprobs_step(ctypes.byref(d), None, p(long), 2, 140000, p(t), p(g), None, p(lp), None, None, p(both), 140000, p(ws), ws.numel(),
                                       st) == 0
    ref = reference(long, t[:, None].long(), "bf16", g=g.view(-1)[:2, None])
    near(both, ref["dx"], ref["tol_dx"], "step of long rows without statistics")


def test_far_rows():
    """Rows that begin beyond 2^32 bytes and 2^31 elements."""
    from paper_2506_03206_amd import rdk
    B, N = 17000, 128256
    x = torch.zeros((B, N), dtype=torch.bfloat16, device="cuda")
    last, gen = rows("bf16", 3, N, 15)
    x[-3:] = last
    tokens = torch.zeros((B, 1), dtype=torch.int32, device="cuda")
    tokens[-3:] = some_tokens(3, N, 1, gen)
    g = torch.ones((B, 1), device="cuda")
    o = rdk.rdk_logprobs(x, tokens)
    rdk.rdk_logprobs_step(x, tokens, g, outputs=rdk.LogprobsOutputs(B, 1, 0, "cuda", grad=x))
    ref = reference(last, tokens[-3:].long(), "bf16", g=g[-3:])
    near(o.logprob[-3:], ref["logprob"], ref["tol_lp"], "logprob")
    near(x[-3:], ref["dx"], ref["tol_dx"], "gradient")
    assert (o.logprob[:-3] + math.log(N)).abs().max() < 1e-5


@pytest.mark.parametrize("sigma", [40.0, 80.0])
def test_weights_far_apart(sigma):
    """Weights that are next to nothing beside the largest, whose ratios to it are no normal numbers."""
    for B, N in ((3, 1000), (2, 50001)):
        x, gen = rows("prob", B, N, N, None, sigma)
        tokens = torch.randint(0, N, (B, 16), generator=gen, device="cuda", dtype=torch.int32)
        tokens[:, 0] = torch.where(x >= 2.0 ** -126, x, 2.0).argmin(1).to(torch.int32)
        check_forward(x, tokens, "prob", 1.0, min(N, 128))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_rows_of_ties(kind):
    """Few values, far from 0, that many entries have: of entropy gradients alone and with others."""
    for B, N, step in ((33, 33703, 16.0), (5, 513, 0.25)):
        x, gen = rows(kind, B, N, N, None, 10.0)
        x.copy_((x / step).round() * step + 3008.0)
        tokens = some_tokens(B, N, 1, gen)
        tokens[::2, 0] = x[::2].float().argmax(1).to(torch.int32)
        g, h = torch.randn((B, 1), generator=gen, device="cuda"), torch.randn(B, generator=gen, device="cuda")
        g[::4] = 0
        check_forward(x, tokens, kind, 0.3)
        check_gradients(x, tokens, kind, 0.3, g, h)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_ranks_of_the_lowest_value(kind):
    """Tokens of the type's lowest finite value among others like it and masked ones, of rows that take every kernel."""
    for B, N in ((3, 301), (3, 5003), (40, 20000), (8, 20000), (8, 45001), (8, 90001)):
        x, gen = rows(kind, B, N, N)
        u = torch.rand(x.shape, generator=gen, device="cuda")
        x.masked_fill_(u < 0.4, torch.finfo(x.dtype).min)
        x.masked_fill_(u > 0.8, -INF)
        tokens = u.argsort(1)[:, :8].to(torch.int32)
        tokens[:, 5:] = some_tokens(B, N, 3, gen)
        check_forward(x, tokens, kind, 1.0, 7)


@pytest.mark.parametrize("kind", ["bf16", "f32", "prob"])
def test_many_tokens_of_many_rows(kind):
    """Sixteen tokens of rows that one large workgroup reads each, the same token among them, tokens that lie side by side and at both ends."""
    for B, N in ((200, 20003), (130, 8193)):
        x, gen = rows(kind, B, N, N)
        tokens = some_tokens(B, N, 16, gen)
        tokens[:, 1] = 0
        tokens[:, 2] = N - 1
        tokens[:, 3] = (tokens[:, 0] + 1).clamp(max=N - 1)
        tokens[::3, 5] = -1
        tokens[1::3, 6] = N
        check_forward(x, tokens, kind)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_temperatures(kind):
    """Temperatures at both ends of their range, powers of two (1 / T is exact): every kernel's forward call, and gradients from 2^-40 on."""
    for B, N in ((6, 300), (6, 9001), (40, 20000), (6, 90001)):
        x, gen = rows(kind, B, N, N)
        x[1] = 1.0                                                          # all of them tie
        x[2, ::2] = -INF
        tokens = some_tokens(B, N, 2, gen)
        tokens[:, 1] = x.float().argmax(1).to(torch.int32)
        g, h = torch.randn((B, 2), generator=gen, device="cuda"), torch.randn(B, generator=gen, device="cuda")
        for e in (-126, -70, -40, -20, 20, 100, 127):
            check_forward(x, tokens, kind, 2.0 ** e, 3)
            if e >= -40:
                check_gradients(x, tokens, kind, 2.0 ** e, g, h)
