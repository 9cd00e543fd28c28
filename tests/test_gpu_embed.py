"""Embedding rows and the table's gradient where they can go wrong, against their definitions: the lookup bit for bit, the gradient in 64 bits.

Tolerance of the gradient.  A sum of m terms x in fp32, in any order and any grouping, is off by at most m 2^-24 sum |x|; its product with the scale and the
addition to what the table holds are rounded once each, 2^-24 of the result and of the product; a bf16 result half a step more, 2^-8 of it."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def strided(t, ld, dtype):
    """t in rows of a larger stride."""
    return torch.empty((t.shape[0], max(ld, t.shape[1])), dtype=dtype, device="cuda")[:, : t.shape[1]].copy_(t)


def tokens(how, B, V, gen):
    if how == "uniform":
        t = torch.randint(0, V, (B,), generator=gen, device="cuda")
    elif how == "zipf":
        cdf = torch.cumsum(1.0 / torch.arange(1, V + 1, device="cuda", dtype=torch.float64), 0)
        t = torch.searchsorted(cdf, torch.rand(B, generator=gen, device="cuda", dtype=torch.float64) * cdf[-1]).clamp(max=V - 1)
        t = torch.randperm(V, generator=gen, device="cuda")[t]
    elif how == "one":
        t = torch.full((B,), V // 2, device="cuda")
    elif how == "none":
        t = torch.where(torch.arange(B, device="cuda") % 2 == 0, -1, V)
    else:                                                               # ends, unknown ids among them
        t = torch.randint(-2, V + 2, (B,), generator=gen, device="cuda")
        t[0], t[-1] = V - 1, 0
    return t.to(torch.int32)


def check_lookup(ids, table, scale, out, kernel=None, slots=None):
    from paper_2506_03206_amd import rdk
    out.fill_(float("nan"))
    rdk.rdk_embed(ids, table, scale, kernel, out)
    at = ids.long() if slots is None else slots
    held = (at >= 0) & (at < table.shape[0])
    want = torch.where(held[:, None], table[torch.where(held, at, 0)].float() * scale, 0.0).to(out.dtype)
    assert torch.equal(out, want)


@pytest.mark.parametrize("table,rows", [(BF16, BF16), (BF16, F32), (F32, BF16), (F32, F32)])
@pytest.mark.parametrize("d", [1, 7, 8, 64, 515, 2048, 2056, 5001])
def test_lookup(table, rows, d):
    for B, V, how, ld in ((1, 1, "uniform", 0), (37, 200, "ends", d + 3), (300, 8000, "zipf", d + 1), (5000, 33, "ends", d)):
        gen = generator(B + d)
        t = strided(torch.randn((V, d), generator=gen, device="cuda"), ld, table)
        out = strided(torch.zeros((B, d), device="cuda"), ld + 5 if ld else 0, rows)
        for scale in (1.0, 0.3, -64.0, 0.0):
            check_lookup(tokens(how, B, V, gen), t, scale, out)


def added(at, rows, V):
    """Sums of the rows of equal places in 64 bits, small ones on the CPU (atomics on one address take half a minute)."""
    where = "cpu" if rows.numel() <= 1 << 23 else rows.device
    return torch.zeros((V, rows.shape[1]), dtype=torch.float64, device=where).index_add_(0, at.to(where), rows.to(where)).to(rows.device)


def check_gradient(ids, d_out, V, dtype, scale, accumulate, ld=0, kernel=None, slots=None):
    from paper_2506_03206_amd import rdk
    d = d_out.shape[1]
    at = ids.long() if slots is None else slots
    held = (at >= 0) & (at < V)
    gen = generator(99)
    old = torch.randn((V, d), generator=gen, device="cuda").to(dtype)
    grad = strided(old if accumulate else torch.full((V, d), float("nan"), device="cuda"), ld, dtype)
    o = rdk.EmbedGradOutputs(V, d, dtype, "cuda", grad=grad)
    rdk.rdk_embed_grad(ids, d_out, o, scale, kernel, accumulate)
    rows = torch.where(held[:, None], d_out.double(), 0.0)
    at = torch.where(held, at, 0)
    total, absolute, m = added(at, rows, V), added(at, rows.abs(), V), added(at, held.double()[:, None], V)
    base = old.double() if accumulate else torch.zeros_like(total)
    scale = float(torch.tensor(scale, dtype=F32))
    want = base + total * scale
    u = 2.0 ** -24
    tol = m * u * absolute * abs(scale) + u * (total * scale).abs() + u * want.abs() + (2.0 ** -8 * want.abs() if dtype == BF16 else 0.0) + 1e-37
    tol = torch.where(m > 0, tol * (1 + 2.0 ** -7), torch.zeros_like(tol))    # (a bound of the rounded result, of the exact one's size)
    off = (grad.double() - want).abs() - tol
    assert not torch.isnan(off).any() and float(off.max()) <= 0, float(off.max())
    again = rdk.EmbedGradOutputs(V, d, dtype, "cuda", grad=strided(old if accumulate else torch.zeros_like(old), ld, dtype))
    rdk.rdk_embed_grad(ids, d_out, again, scale, kernel, accumulate)
    assert torch.equal(again.grad, grad)                                # the same bits
    return grad


@pytest.mark.parametrize("how", ["uniform", "zipf", "one", "none", "ends"])
@pytest.mark.parametrize("B", [1, 2, 63, 300, 1023, 1024, 1025, 2049, 5000, 16384, 20480, 20481, 40000])
def test_gradient(how, B):
    i = 0
    for V, d in ((1, 5), (513, 64), (8000, 24), (300000, 8)):
        for table, rows, accumulate in ((F32, BF16, False), (BF16, F32, True), (BF16, BF16, False), (F32, F32, True))[i % 2::2]:
            gen = generator(B + V)
            ids = tokens(how, B, V, gen)
            d_out = strided(torch.randn((B, d), generator=gen, device="cuda"), d + (3 if i % 3 == 0 else 0), rows)
            check_gradient(ids, d_out, V, table, 0.7 if accumulate else 1.0, accumulate, d + (5 if i % 2 else 0))
        i += 1


@pytest.mark.parametrize("d", [1, 8, 9, 63, 512, 515, 1024, 2048, 2050, 4100])
@pytest.mark.parametrize("B", [40, 1500, 17000])
def test_gradient_widths(B, d):
    gen = generator(d)
    for table, rows in ((BF16, BF16), (F32, F32), (F32, BF16), (BF16, F32)):
        ids = tokens("zipf", B, 700, gen)
        check_gradient(ids, torch.randn((B, d), generator=gen, device="cuda").to(rows), 700, table, 2.0, False)


def test_gradient_of_long_runs():
    """A run over many pieces beside others that begin and end at their borders, in every position of a piece."""
    gen = generator(5)
    for first in (0, 1, 3, 4, 7, 8, 31, 32, 33):
        for length in (1, 4, 31, 32, 33, 64, 65, 2500):
            ids = torch.cat([torch.zeros(first), torch.ones(length), torch.full((2700,), 2.0), torch.arange(3, 60)]).to(torch.int32).cuda()
            ids = ids[torch.randperm(ids.numel(), generator=gen, device="cuda")]
            check_gradient(ids, torch.randn((ids.numel(), 16), generator=gen, device="cuda"), 64, F32, 1.0, False)
    ids = torch.full((70000,), 7, dtype=torch.int32, device="cuda")      # more than 64 pieces of 64
    check_gradient(ids, torch.randn((70000, 8), generator=gen, device="cuda"), 9, F32, 1.0, False)
    ids[:100] = 3
    check_gradient(ids, torch.randn((70000, 8), generator=gen, device="cuda").bfloat16(), 9, F32, 1.0, True)


def test_rows_without_tokens_are_left():
    """With accumulate nothing but the named rows is touched, NaN there included; rows behind the table stay as they are either way."""
    from paper_2506_03206_amd import rdk
    for B in (10, 3000):
        room = torch.full((600, 32), float("nan"), device="cuda")
        room[::2] = 1.0
        ids = (torch.randint(0, 250, (B,), device="cuda") * 2).to(torch.int32)
        before = room.clone()
        rdk.rdk_embed_grad(ids, torch.ones((B, 32), device="cuda"), rdk.EmbedGradOutputs(500, 32, F32, "cuda", grad=room[:500]), accumulate=True)
        named = torch.zeros(600, dtype=torch.bool, device="cuda")
        named[ids.long()] = True
        assert torch.equal(torch.nan_to_num(room[~named], nan=-5.0), torch.nan_to_num(before[~named], nan=-5.0))
        assert torch.equal(room[named][:, 0], 1.0 + torch.bincount(ids.long(), minlength=600)[named].float())
        rdk.rdk_embed_grad(ids, torch.ones((B, 32), device="cuda"), rdk.EmbedGradOutputs(500, 32, F32, "cuda", grad=room[:500]))
        assert (room[:500][~named[:500]] == 0).all() and torch.equal(torch.nan_to_num(room[500:], nan=-5.0), torch.nan_to_num(before[500:], nan=-5.0))


@pytest.mark.parametrize("B", [50, 3000, 20000])
def test_pruned_table(B):
    from paper_2506_03206_amd import rdk
    N, n, d = 5000, 1234, 40
    gen = generator(B)
    kept = torch.sort(torch.randperm(N, generator=gen, device="cuda")[:n]).values.to(torch.int32)
    kernel = rdk.rdk_build_kernel(N, kept, rdk.IDENTITY)
    slot_of = torch.full((N,), -1, dtype=torch.int64, device="cuda")
    slot_of[kept.long()] = torch.arange(n, device="cuda")
    ids = torch.randint(-1, N + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
    slots = torch.where((ids >= 0) & (ids < N), slot_of[ids.clamp(0, N - 1).long()], -1)
    table = torch.randn((n, d), generator=gen, device="cuda")
    check_lookup(ids, table, 2.0, torch.empty((B, d), device="cuda"), kernel, slots)
    for accumulate in (False, True):
        check_gradient(ids, torch.randn((B, d), generator=gen, device="cuda"), n, F32, 0.5, accumulate, 0, kernel, slots)
    with pytest.raises(rdk.RdkError):
        rdk.rdk_embed(ids, torch.zeros((n + 1, d), device="cuda"), 1.0, kernel)


def test_under_torch():
    """Automatic differentiation against torch's own in 64 bits, with ids of several dimensions and a gradient that is broadcast."""
    from paper_2506_03206_amd import rdk
    gen = generator(8)
    table = torch.randn((300, 24), generator=gen, device="cuda").requires_grad_(True)
    ids = torch.randint(0, 300, (6, 50), generator=gen, device="cuda", dtype=torch.int32)
    weight = torch.randn((6, 50, 24), generator=gen, device="cuda")
    rows = rdk.rdk_embedding(ids, table, 3.0)
    assert rows.shape == (6, 50, 24)
    (rows * weight).sum().backward()
    exact = table.detach().double().requires_grad_(True)
    (exact[ids.long()] * 3.0 * weight.double()).sum().backward()
    assert (table.grad.double() - exact.grad).abs().max() <= 50 * 2.0 ** -24 * 3 * 20
    table.grad = None
    rdk.rdk_embedding(ids, table, 3.0).sum().backward()
    assert torch.equal(table.grad[:, 0], 3.0 * torch.bincount(ids.long().flatten(), minlength=300).float())
    e = 1e-3                                                            # linear in the table: a difference of any size
    other = table.detach().clone()
    other[5, 7] += e
    base = (rdk.rdk_embed(ids, table.detach(), 3.0).double() * weight.double()).sum()
    slope = ((rdk.rdk_embed(ids, other, 3.0).double() * weight.double()).sum() - base) / (other[5, 7].double() - table[5, 7].detach().double())
    assert abs(float(slope - exact.grad[5, 7])) < 1e-2                   # roundings 2^-23 of numbers up to 12 over a step of 1e-3


def test_streams_and_graphs():
    """On a stream of its own, and captured into graphs that are replayed between eager calls on new inputs."""
    from paper_2506_03206_amd import rdk
    for B, V, d in ((40, 500, 64), (3000, 5000, 64), (20000, 70000, 32)):
        gen = generator(B)
        ids, d_out = tokens("zipf", B, V, gen), torch.randn((B, d), generator=gen, device="cuda").bfloat16()
        table, out = torch.randn((V, d), generator=gen, device="cuda").bfloat16(), torch.empty((B, d), device="cuda")
        o = rdk.EmbedGradOutputs(V, d, F32, "cuda")

        def both(out, o):
            rdk.rdk_embed(ids, table, 2.0, out=out)
            rdk.rdk_embed_grad(ids, d_out, o, 2.0)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            both(out, o)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            both(out, o)
        for i in range(4):
            ids.copy_(tokens("zipf", B, V, gen))
            d_out.copy_(torch.randn((B, d), generator=gen, device="cuda"))
            e, eo = torch.empty_like(out), rdk.EmbedGradOutputs(V, d, F32, "cuda")
            both(e, eo)
            out.zero_(), o.grad.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, e) and torch.equal(o.grad, eo.grad)


def test_far_rows():
    """Rows of a table and of a batch that begin beyond 2^32 bytes and 2^31 elements."""
    V, d = 600000, 4096
    gen = generator(4)
    table = torch.zeros((V, d), dtype=BF16, device="cuda")
    table[-4:] = torch.randn((4, d), generator=gen, device="cuda")
    ids = torch.randint(V - 4, V, (50,), generator=gen, device="cuda", dtype=torch.int32)
    check_lookup(ids, table, 1.0, torch.empty((50, d), dtype=BF16, device="cuda"))
    from paper_2506_03206_amd import rdk
    rows = torch.randn((50, d), generator=gen, device="cuda")
    o = rdk.EmbedGradOutputs(V, d, BF16, "cuda", grad=table)
    rdk.rdk_embed_grad(ids, rows, o)
    want = torch.zeros((4, d), dtype=torch.float64, device="cuda").index_add_(0, ids.long() - (V - 4), rows.double())
    assert ((table[-4:].double() - want).abs() <= 2.0 ** -8 * want.abs() + 50 * 2.0 ** -24 * 200).all()
    assert not table[:-4].any()
    del table, o
    B = 2200000
    big = torch.ones((B, 1024), dtype=BF16, device="cuda")
    ids = (torch.arange(B, device="cuda") % 3).to(torch.int32)
    ids[-1] = 5
    big[-1] = 7.0
    o = rdk.rdk_embed_grad(ids, big, rdk.EmbedGradOutputs(6, 1024, F32, "cuda"))
    assert (o.grad[5] == 7.0).all() and (o.grad[3:5] == 0).all()
    count = torch.bincount(ids.long(), minlength=6)[:3].float()
    assert torch.equal(o.grad[:3], count[:, None].expand(3, 1024))       # whole numbers below 2^24 are exact


@pytest.mark.parametrize("types", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32)])
def test_few_tokens_of_wide_rows(types):
    """More columns to a workgroup, from more than 8192 workgroups of 64 threads across on."""
    for B, d in ((513, 8195), (900, 5000)):
        gen = generator(B)
        ids = tokens("zipf", B, 700, gen)
        x = strided(torch.randn((B, d), generator=gen, device="cuda"), d, types[1])
        check_gradient(ids, x, 700, types[0], 0.5, False, d)
        check_gradient(ids, x, 700, types[0], 0.5, True, d + 3)
