"""rdk_topk where it can go wrong, against numpy in 64 bits: ids and values exactly (descending, equal entries by id), the logarithm of the
normaliser within what fp32 sums allow (about 2^-22 of the largest exponent and a few units of the last place of the result)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

KINDS = ["f32", "bf16", "prob"]


def reference(x, k, prob, T=1.0):
    """x [B,N] float64.  Sorted by value, NaN first, then id; masked entries left out."""
    B, N = x.shape
    ids, values = np.full((B, k), -1, np.int64), np.full((B, k), 0.0 if prob else -np.inf)
    lse = np.empty(B)
    for b in range(B):
        row = x[b]
        unmasked = np.nonzero(np.isnan(row) | (row > (0.0 if prob else -np.inf)))[0]
        value = np.where(np.isnan(row[unmasked]), np.inf, row[unmasked])
        order = unmasked[np.lexsort((unmasked, -value, ~np.isnan(row[unmasked])))][:k]
        ids[b, :order.size], values[b, :order.size] = order, row[order]
        with np.errstate(all="ignore"):
            if prob:
                lse[b] = np.log(row.sum())
            else:
                m = row.max()
                if np.isnan(m) or m == np.inf:
                    lse[b] = np.nan
                else:
                    lse[b] = m / T + np.log(np.exp((row - m) / T).sum()) if m > -np.inf else -np.inf
    return ids, values, lse


def check(x, k, kind, T=1.0, outputs=None):
    from paper_2506_03206_amd import rdk
    o = rdk.rdk_topk(x, k, "prob" if kind == "prob" else "logit", temperature=T, outputs=outputs)
    verify(o, x, k, kind, T)
    return o


def verify(o, x, k, kind, T=1.0):
    x64 = x.double().cpu().numpy()
    ids, values, lse = reference(x64, k, kind == "prob", T)
    np.testing.assert_array_equal(o.ids.cpu().numpy(), ids)
    np.testing.assert_array_equal(o.values.cpu().numpy().astype(np.float64), values)
    got = o.lse.cpu().numpy().astype(np.float64)
    finite = np.isfinite(lse)
    np.testing.assert_array_equal(got[~finite], lse[~finite])
    assert (np.abs(got - lse)[finite] <= 4e-6 + 4e-7 * np.abs(lse[finite])).all()


def rows(B, N, kind, seed, sigma=3.0, pad=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((B, N), generator=g, device="cuda") * sigma
    if kind == "prob":
        x = torch.softmax(x, 1)
    x = x.to(torch.bfloat16 if kind == "bf16" else torch.float32)
    if pad:
        x = torch.nn.functional.pad(x, (0, pad), value=float("nan"))[:, :N]
    return x


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("B,N,k", [(1, 1, 1), (3, 2, 2), (5, 7, 3), (2, 8, 8), (4, 9, 1), (3, 63, 63), (2, 127, 127), (7, 129, 128), (2, 1023, 128),
                                   (5, 1024, 16), (3, 1025, 100), (2, 2049, 128), (300, 4099, 5), (1, 16385, 64), (2, 32003, 33), (1, 65537, 128),
                                   (9, 128256, 16), (1, 256000, 1), (1, 1000003, 77), (1030, 5001, 20)])
def test_sizes(B, N, k, kind):
    check(rows(B, N, kind, B + N, pad=3 if N % 2 else 0), k, kind)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("T", [0.25, 2.0, 10.0])
def test_temperature(T, kind):
    check(rows(4, 20001, kind, 5), 10, kind, T)


def special(N, kind, k):
    """Rows whose largest entries lie where a selection by parts, lanes or thresholds could lose them."""
    g = torch.Generator(device="cuda")
    g.manual_seed(N + k)
    dt = torch.bfloat16 if kind == "bf16" else torch.float32
    one = lambda f: f.to(dt)  # noqa: E731
    base = torch.randn(N, generator=g, device="cuda")
    at = torch.arange(N, device="cuda")
    out = [torch.zeros(N, device="cuda"),                                          # all equal
           at.float(), -at.float(),                                               # rising, falling
           torch.where(at < k, 5.0, base), torch.where(at >= N - k, 5.0, base),       # a block of equal ones at either end
           torch.where(at % 256 == 3, base + 20, base), torch.where(at % 8 == 7, base + 20, base), torch.where(at // 8 % 256 == 9, base + 20, base),
           torch.where(at // 4 % 256 == 17, base + 20, base), torch.where(at // 8 % 64 == 1, base + 20, base),
           torch.round(base), torch.round(base * 0.3),                               # many ties
           torch.where(at % 2 == 0, -0.0, 0.0)]                                   # zeros of both signs are equal
    return torch.stack([one(r) for r in out])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("N,k", [(300, 100), (5000, 7), (40001, 64), (130000, 128)])
def test_ties_and_unlucky_orders(N, k, kind):
    x = special(N, kind, k)
    from paper_2506_03206_amd import rdk
    o = rdk.rdk_topk(x, k)
    x64 = x.double().cpu().numpy() + 0.0                                           # -0 and 0 alike
    ids, values, lse = reference(x64, k, False)
    np.testing.assert_array_equal(o.ids.cpu().numpy(), ids)
    np.testing.assert_array_equal(o.values.cpu().numpy().astype(np.float64), values)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("N", [50, 5001, 70001])
def test_masks_infinities_and_nan(N, kind):
    x = rows(12, N, kind, N)
    k = 32
    low = torch.finfo(x.dtype).min
    x[0] = -float("inf")                        # nothing left
    x[1, 5:] = -float("inf")                    # five entries left
    x[2, : N // 2] = -float("inf")
    x[3] = low                                  # all at the lowest finite value: ties, a uniform row
    x[4, 3:] = low
    x[5, N // 2] = float("nan")
    x[6, [1, N - 1]] = float("nan")
    x[7, N - 2] = float("inf")
    x[8, N // 3] = torch.finfo(x.dtype).max     # differences leave the range of a float
    x[9] = float("nan")
    x[10, 0] = -float("nan")
    x[11, ::2] = -float("inf")
    check(x, k, kind)


def test_weights_of_zero_are_masked():
    x = rows(6, 9001, "prob", 3)
    x[0] = 0
    x[1, 7:] = 0
    x[2, :4500] = 0
    x[3] = 1.0 / 9001
    x[4, 8999] = 1e-42                          # a subnormal weight is one
    x[4, :8990] = 0
    check(x, 20, "prob")


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_rows_beyond_32_bits(kind):
    dt = torch.bfloat16 if kind == "bf16" else torch.float32
    N, ld = 5003, (1 << 31) + 8
    flat = torch.empty(2 * ld + N, dtype=dt, device="cuda")
    x = flat.as_strided((3, N), (ld, 1))
    x.copy_(rows(3, N, kind, 1))
    check(x, 12, kind)


def test_other_streams_and_replays():
    """Launched on a stream of its own, and recorded into a graph that is replayed over changing rows with eager work between."""
    from paper_2506_03206_amd import rdk
    x, B, N, k = rows(6, 100003, "bf16", 1), 6, 100003, 24
    o = rdk.TopkOutputs(B, N, k, "cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        rdk.rdk_topk(x, k, outputs=o)
    torch.cuda.current_stream().wait_stream(side)
    verify(o, x, k, "bf16")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rdk.rdk_topk(x, k, outputs=o)
    for i in range(4):
        x.copy_(rows(B, N, "bf16", 10 + i))
        graph.replay()
        torch.cuda.synchronize()
        verify(o, x, k, "bf16")
        verify(rdk.rdk_topk(x, k), x, k, "bf16")


def test_every_call_gives_the_same_bits():
    from paper_2506_03206_amd import rdk
    x = rows(16, 128256, "bf16", 4)
    first = rdk.rdk_topk(x, 64)
    for _ in range(5):
        again = rdk.rdk_topk(x, 64)
        assert torch.equal(first.ids, again.ids) and torch.equal(first.values, again.values) and torch.equal(first.lse, again.lse)


def test_refusals_of_the_binding():
    from paper_2506_03206_amd import rdk
    x = rows(2, 100, "f32", 1)
    with pytest.raises(rdk.RdkError):
        rdk.rdk_topk(x, 101)
    with pytest.raises(rdk.RdkError):
        rdk.rdk_topk(x, 4, temperature=0.0)
    with pytest.raises(AssertionError):
        rdk.rdk_topk(x, 4, outputs=rdk.TopkOutputs(3, 100, 4, "cuda"))
    with pytest.raises(AssertionError):
        rdk.rdk_topk(x.double(), 4)
    with pytest.raises(AssertionError):
        rdk.rdk_topk(x.t(), 2)
