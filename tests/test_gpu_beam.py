"""Beam search's selection and the reordering of states, against numpy.

Scores are formed in fp32: with Z = max |x| and S = max |score| one is off by at most E = 2^-22 (Z + S) + 5e-6.  The chosen candidates are compared by their
64-bit scores: in order, distinct, none better left out, each within E; where the 64-bit scores are further apart than that, ids are equal."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def candidates(x, scores, finished, eos, prob):
    """Per request {(beam, id): score} as arrays: flat 64-bit scores [G, W, N], -inf where there is none."""
    G, W = scores.shape
    x = x.reshape(G, W, -1)
    with np.errstate(all="ignore"):
        if prob:
            lp = np.log(x) - np.log(x.sum(2, keepdims=True))
        else:
            m = x.max(2, keepdims=True)
            m = np.where(m > -np.inf, m, 0.0)
            lp = (x - m) - np.log(np.exp(x - m).sum(2, keepdims=True))
        out = scores[:, :, None] + lp
    out[np.isnan(out)] = -np.inf
    for g in range(G):
        for w in range(W):
            if scores[g, w] == -np.inf:
                out[g, w] = -np.inf
            elif finished is not None and finished[g, w]:
                out[g, w] = -np.inf
                out[g, w, eos] = scores[g, w]
    return out


def verify(o, x, scores, K, kind, finished=None, eos=-1):
    G, W = scores.shape
    N = x.shape[1]
    s64, x64 = scores.double().cpu().numpy(), x.double().cpu().numpy()
    fin = None if finished is None else finished.cpu().numpy()
    cand = candidates(x64, s64, fin, eos, kind == "prob")
    got, parent, token, done = (t.cpu().numpy() for t in (o.scores, o.parent, o.token, o.finished))
    for g in range(G):
        flat = cand[g].reshape(-1)
        n = min(K, int((flat > -np.inf).sum()))
        order = np.argsort(-flat, kind="stable")[:n + 1]
        best = flat[order]
        assert (parent[g, n:] == -1).all() and (token[g, n:] == -1).all() and (got[g, n:] == -np.inf).all() and (done[g, n:] == 0).all()
        if not n:
            continue
        E = 2.0 ** -22 * (np.abs(x64[np.isfinite(x64)]).max() + np.abs(best[:n]).max()) + 5e-6
        chosen = parent[g, :n].astype(np.int64) * N + token[g, :n]
        assert (parent[g, :n] >= 0).all() and (parent[g, :n] < W).all() and (token[g, :n] >= 0).all() and (token[g, :n] < N).all()
        assert np.unique(chosen).size == n
        assert (np.abs(flat[chosen] - got[g, :n]) <= E).all()
        assert (np.diff(got[g, :n]) <= 0).all()
        assert (flat[chosen] >= best[:n] - E).all()
        clear = np.ones(n, bool)                                                # ranks whose neighbours are further away than roundings
        gap = best[:-1] - best[1:] if best.size > n else np.append(best[:-1] - best[1:], np.inf)
        gap = gap[:n]
        clear &= gap > 2 * E
        clear[1:] &= gap[:-1] > 2 * E
        np.testing.assert_array_equal(chosen[clear], order[:n][clear])
        want = np.zeros(n, bool) if fin is None else fin[g][parent[g, :n]] != 0
        want |= token[g, :n] == eos
        np.testing.assert_array_equal(done[g, :n] != 0, want)


def make(G, W, N, kind, seed, sigma=3.0, pad=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((G * W, N), generator=g, device="cuda") * sigma
    if kind == "prob":
        x = torch.softmax(x, 1)
    x = x.to(torch.bfloat16 if kind == "bf16" else torch.float32)
    if pad:
        x = torch.nn.functional.pad(x, (0, pad), value=float("nan"))[:, :N]
    return x, -torch.cumsum(torch.rand((G, W), generator=g, device="cuda"), 1)


@pytest.mark.parametrize("kind", ["f32", "bf16", "prob"])
@pytest.mark.parametrize("G,W,N,K", [(1, 1, 1, 1), (2, 1, 5, 3), (1, 2, 3, 6), (3, 4, 17, 4), (2, 64, 33, 128), (1, 3, 1000, 128), (5, 5, 4099, 10),
                                     (1, 4, 128256, 4), (2, 8, 32003, 16), (1, 64, 9001, 64), (70, 4, 1025, 4), (3, 7, 70001, 100), (1, 2, 1000003, 5),
                                     (40, 16, 2049, 16)])
def test_sizes(G, W, N, K, kind):
    from paper_2506_03206_amd import rdk
    x, scores = make(G, W, N, kind, G + W + N, pad=3 if N % 2 else 0)
    o = rdk.rdk_beam_select(x, scores, K, "prob" if kind == "prob" else "logit")
    verify(o, x, scores, K, kind)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("N", [50, 20001])
def test_finished_dead_and_masked_beams(N, kind):
    """Beams that are finished (their rows hold NaN), dead, masked in part or altogether; requests without any candidate, with fewer than K."""
    from paper_2506_03206_amd import rdk
    G, W, K, eos = 6, 5, 10, 3
    x, scores = make(G, W, N, kind, N)
    finished = torch.zeros((G, W), dtype=torch.uint8, device="cuda")
    rows = x.view(G, W, N)
    finished[0, 1] = finished[0, 3] = 1
    rows[0, 1] = rows[0, 3] = float("nan")
    scores[1, 1:] = -float("inf")                       # the first step: one beam
    rows[1, 1:] = float("nan")
    scores[2] = -float("inf")                           # nothing
    finished[3] = 1                                     # all finished: W candidates
    rows[3] = float("nan")
    rows[4, 0] = -float("inf")
    rows[4, 1, 4:] = -float("inf")
    rows[4, 2:] = -float("inf")                         # four candidates in the request
    rows[5, :, 7:] = torch.finfo(x.dtype).min
    finished[5, 2], scores[5, 2] = 1, -float("inf")     # finished and dead
    o = rdk.rdk_beam_select(x, scores, K, finished=finished, eos=eos)
    verify(o, x, scores, K, kind, finished, eos)


def test_ties_go_to_the_lower_beam_then_id():
    from paper_2506_03206_amd import rdk
    G, W, N, K = 2, 4, 9000, 12
    x = torch.zeros((G * W, N), device="cuda")
    x[:, [5, 17, 8999]] = 4.0                           # the same three in every beam
    scores = torch.full((G, W), -1.5, device="cuda")
    scores[1, 0] = -float("inf")
    o = rdk.rdk_beam_select(x, scores, K)
    want = [(w, j) for w in range(4) for j in (5, 17, 8999)]
    assert list(zip(o.parent[0].tolist(), o.token[0].tolist())) == want
    want = [(w, j) for w in (1, 2, 3) for j in (5, 17, 8999)] + [(1, 0), (1, 1), (1, 2)]
    assert list(zip(o.parent[1].tolist(), o.token[1].tolist())) == want


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_nan_and_infinity_show(bad):
    from paper_2506_03206_amd import rdk
    x, scores = make(2, 3, 5001, "f32", 1)
    x[1, 77] = bad
    o = rdk.rdk_beam_select(x, scores, 4)
    assert torch.isnan(o.scores[0]).all() and (o.parent[0] == 1).all() and int(o.token[0, 0]) == 77
    assert torch.isfinite(o.scores[1]).all()


def test_selection_on_other_streams_and_replays():
    from paper_2506_03206_amd import rdk
    G, W, N, K = 3, 4, 50001, 4
    x, scores = make(G, W, N, "bf16", 1)
    finished = torch.zeros((G, W), dtype=torch.uint8, device="cuda")
    o = rdk.BeamOutputs(G, W, N, K, "cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        rdk.rdk_beam_select(x, scores, K, finished=finished, eos=9, outputs=o)
    torch.cuda.current_stream().wait_stream(side)
    verify(o, x, scores, K, "bf16", finished, 9)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rdk.rdk_beam_select(x, scores, K, finished=finished, eos=9, outputs=o)
    for i in range(4):
        y, s = make(G, W, N, "bf16", 30 + i)
        x.copy_(y), scores.copy_(s)
        finished[i % G, i] = 1
        graph.replay()
        torch.cuda.synchronize()
        verify(o, x, scores, K, "bf16", finished, 9)
        verify(rdk.rdk_beam_select(x, scores, K, finished=finished, eos=9), x, scores, K, "bf16", finished, 9)


# ------------------------------------------------------------------------------------------------------------- states
def moved(src, parent, W):
    G, K = parent.shape
    rows = (parent.long() + torch.arange(G, device="cuda")[:, None] * W).reshape(-1)
    return src[rows]


@pytest.mark.parametrize("dtype", [torch.uint8, torch.bfloat16, torch.float32, torch.float64])
@pytest.mark.parametrize("G,W,shape", [(1, 2, (1,)), (3, 4, (7,)), (2, 1, (9, 5)), (5, 3, (2, 33)), (1, 64, (130,)), (2, 33, (3, 5, 7)), (2, 17, (1025,)),
                                       (4, 8, (40001,)), (70, 5, (64,))])
def test_rows_in_place_and_apart(G, W, shape, dtype):
    from paper_2506_03206_amd import rdk
    g = torch.Generator(device="cuda")
    g.manual_seed(G + W)
    for K in sorted({W, max(1, W - 1), min(64, 2 * W)}):
        x = torch.randint(0, 250, (G * W,) + shape, generator=g, device="cuda").to(dtype)
        parent = torch.randint(0, W, (G, K), generator=g, device="cuda", dtype=torch.int32)
        out = torch.zeros((G * K,) + shape, dtype=dtype, device="cuda")
        rdk.rdk_beam_reorder([x], parent, W, [out])
        assert torch.equal(out, moved(x, parent, W))
        if K == W:
            want = moved(x, parent, W)
            rdk.rdk_beam_reorder([x], parent)
            assert torch.equal(x, want)


@pytest.mark.parametrize("shift", range(0, 17, 1))
def test_any_alignment(shift):
    from paper_2506_03206_amd import rdk
    G, W, n = 2, 5, 333
    flat = torch.arange(0, 7000, device="cuda").to(torch.uint8)
    x = flat.as_strided((G * W, n), (n + shift, 1), shift)
    before = flat.clone()
    parent = torch.tensor([[4, 3, 2, 1, 0], [1, 1, 1, 1, 1]], dtype=torch.int32, device="cuda")
    want = moved(x.clone(), parent, W)
    rdk.rdk_beam_reorder([x], parent)
    assert torch.equal(x, want)
    touched = torch.zeros_like(flat)
    touched.as_strided((G * W, n), (n + shift, 1), shift).fill_(1)
    assert torch.equal(flat[touched == 0], before[touched == 0])                    # nothing beside the rows


def test_caches_of_which_a_part_is_filled():
    """Many states at once (more than one launch holds), pieces with gaps, an empty one, a cache stored head by head; what lies behind the filled part
    stays; a compact source into a roomy destination."""
    from paper_2506_03206_amd import rdk
    G, W, H, room, D = 3, 4, 5, 40, 24
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    parent = torch.randint(0, W, (G, W), generator=g, device="cuda", dtype=torch.int32)
    parent[1, 2] = -1                                                               # left as it is
    rows = parent.clone()
    rows[1, 2] = 2
    full = [torch.randn((G * W, H, room, D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(30)]
    lengths = [i + 1 for i in range(29)] + [0]
    views = [f[:, :, :n] for f, n in zip(full, lengths)]
    by_head = torch.randn((H, G * W, room, D), generator=g, device="cuda")
    views.append(by_head.transpose(0, 1)[:, :, :7])
    full.append(by_head.transpose(0, 1))
    before = [f.clone() for f in full]
    rdk.rdk_beam_reorder(views, parent)
    for f, b, v in zip(full, before, views):
        n = v.shape[2]
        assert torch.equal(f[:, :, :n], moved(b[:, :, :n], rows, W)) and torch.equal(f[:, :, n:], b[:, :, n:])
    small = torch.randn((G, H, 9, D), generator=g, device="cuda")                    # after the prompt: one row a request, W beams of it
    wide = torch.zeros((G * W, H, room, D), device="cuda")
    rdk.rdk_beam_reorder([small], torch.zeros((G, W), dtype=torch.int32, device="cuda"), 1, [wide[:, :, :9]])
    assert torch.equal(wide[:, :, :9], small.repeat_interleave(W, 0)) and (wide[:, :, 9:] == 0).all()


def test_rows_whose_memory_has_another_order():
    """Caches stored position by position and looked at head by head, and a source and a destination of one such order."""
    from paper_2506_03206_amd import rdk
    G, W, H, room, D = 2, 3, 5, 11, 6
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    parent = torch.randint(0, W, (G, W), generator=g, device="cuda", dtype=torch.int32)
    for n in (room, 7):
        memory = torch.randn((G * W, room, H, D), generator=g, device="cuda")
        x = memory[:, :n].transpose(1, 2)                                            # [rows, heads, positions, D]
        before = memory.clone()
        out = torch.zeros((G * W, n, H, D), device="cuda")
        rdk.rdk_beam_reorder([x], parent, W, [out.transpose(1, 2)])
        assert torch.equal(out, moved(before[:, :n], parent, W))
        rdk.rdk_beam_reorder([x], parent)
        assert torch.equal(memory[:, :n], moved(before[:, :n], parent, W)) and torch.equal(memory[:, n:], before[:, n:])
    with pytest.raises(AssertionError):                                              # rows of one shape, but not of one order
        rdk.rdk_beam_reorder([x], parent, W, [torch.zeros((G * W, H, n, D), device="cuda")])


def test_more_requests_than_a_launch_has_workgroups():
    from paper_2506_03206_amd import rdk
    G = (1 << 24) + 5                                                                # a workgroup each, and 2^24 - 1 at once
    x = torch.arange(2 * G, device="cuda").to(torch.uint8).view(2 * G, 1)
    parent = torch.ones((G, 1), dtype=torch.int32, device="cuda")
    out = torch.zeros((G, 1), dtype=torch.uint8, device="cuda")
    other = torch.full((G, 1), 7, dtype=torch.uint8, device="cuda")
    twin = torch.stack([other, x.view(G, 2, 1)[:, 0]], 1).reshape(2 * G, 1)
    rdk.rdk_beam_reorder([x, twin], parent, 2, [out, other])
    assert torch.equal(out[:, 0], x[1::2, 0]) and torch.equal(other[:, 0], x[0::2, 0])


def test_offsets_beyond_32_bits():
    from paper_2506_03206_amd import rdk
    W, n, stride = 3, 1 << 20, (1 << 32) + 4096
    flat = torch.empty(2 * stride + n, dtype=torch.uint8, device="cuda")
    x = flat.as_strided((W, n), (stride, 1))
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x.copy_(torch.randint(0, 256, (W, n), generator=g, device="cuda"))
    parent = torch.tensor([[2, 0, 1]], dtype=torch.int32, device="cuda")
    want = x[parent[0].long()].clone()
    rdk.rdk_beam_reorder([x], parent)
    assert torch.equal(x, want)
    long = torch.empty((2, (1 << 32) + 48), dtype=torch.uint8, device="cuda")       # a row of more than 2^32 bytes
    long[0].fill_(1), long[1].fill_(2)
    long[0, -7:], long[1, -7:] = 3, 4
    rdk.rdk_beam_reorder([long], torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"))
    assert int(long[0, 0]) == 2 and int(long[1, 0]) == 1 and (long[0, -7:] == 4).all() and (long[1, -7:] == 3).all()
    assert bool((long[0, :-7] == 2).all()) and bool((long[1, :-7] == 1).all())


def test_reordering_on_other_streams_and_replays():
    from paper_2506_03206_amd import rdk
    G, W = 2, 4
    x = torch.arange(G * W * 1000, dtype=torch.float32, device="cuda").view(G * W, 1000)
    parent = torch.tensor([[1, 0, 3, 2], [0, 0, 3, 1]], dtype=torch.int32, device="cuda")
    want = moved(x, parent, W)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        rdk.rdk_beam_reorder([x], parent)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(x, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rdk.rdk_beam_reorder([x], parent)
    for i in range(4):
        x.copy_(torch.randn((G * W, 1000), device="cuda"))
        parent.copy_(torch.randint(0, W, (G, W), device="cuda", dtype=torch.int32))
        want = moved(x, parent, W)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x, want)


def test_refusals_of_the_binding():
    from paper_2506_03206_amd import rdk
    x, scores = make(2, 3, 100, "f32", 1)
    with pytest.raises(rdk.RdkError):
        rdk.rdk_beam_select(x, scores, 129)
    with pytest.raises(rdk.RdkError):
        rdk.rdk_beam_select(x, scores, 3, finished=torch.zeros((2, 3), dtype=torch.uint8, device="cuda"))   # no eos
    with pytest.raises(AssertionError):
        rdk.rdk_beam_select(x[:5], scores, 3)
    with pytest.raises(AssertionError):
        rdk.rdk_beam_select(x, scores.double(), 3)
    parent = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    with pytest.raises(AssertionError):
        rdk.rdk_beam_reorder([x[:5]], parent)
    with pytest.raises(AssertionError):
        rdk.rdk_beam_reorder([x], parent.long())
    with pytest.raises(AssertionError):
        rdk.rdk_beam_reorder([torch.zeros((6, 4, 4, 4), device="cuda")[:, ::2, :, ::2]], parent)            # two gaps
    with pytest.raises(rdk.RdkError):
        rdk.rdk_beam_reorder([x], parent[:, :2].contiguous(), 3, [x[:4]])                                   # overlaps
