"""Operators beside the decoding step: what a vocabulary-pruned drafter is trained on, and beam search over the same rows.

  topk     the target's k largest logits of every row and the logarithm of its normaliser: what is kept of a teacher
  distill  a drafter over ``n`` of the target's ``N`` ids against the teacher's top logits: the loss alone (evaluation), the loss and
           then its gradient (two calls: what comes from above arrives in between), or both at once (row weights known beforehand)
  beam     beam search's selection over ``W`` beams and the vocabulary in each of ``G`` requests
  reorder  the states of the beams (key-value caches of which a part is filled, token histories) after the selection

Rows have the values of section 5.1 of the paper: Gaussian logits of a standard deviation of 2-3 on a Zipf rank bias, a drafter that
sees a noisy target, kept ids = the most frequent ones and 10 % random ones.
"""
import math

import torch

own = False


# ---------------------------------------------------------------------------------------------------------------- cases
def _topk(name, B, N, k, dtype="bf16", temperature=1.0, masked=0.0, sigma=3.0):
    c = {"op": "topk", "B": B, "N": N, "k": k, "dtype": dtype, "temperature": temperature, "masked": masked, "sigma": sigma, "zipf": 1.0}
    return dict(c, name=name) if name else c


def _distill(name, path, B, N, n, K, dtype="bf16", temperature=1.0, remainder=False, live=1.0, sigma=3.0):
    c = {"op": "distill", "path": path, "B": B, "N": N, "n": n, "K": K, "dtype": dtype, "temperature": temperature, "remainder": remainder,
         "live": live, "sigma": sigma, "zipf": 1.0}
    return dict(c, name=name) if name else c


def _beam(name, G, W, K, N, dtype="bf16", finished=0.0, masked=0.0, sigma=3.0):
    c = {"op": "beam", "G": G, "W": W, "K": K, "N": N, "dtype": dtype, "finished": finished, "masked": masked, "sigma": sigma, "zipf": 1.0}
    return dict(c, name=name) if name else c


def _reorder(name, G, W, K, buffers, heads, length, room, width, history, dtype="bf16"):
    c = {"op": "reorder", "G": G, "W": W, "K": K, "buffers": buffers, "heads": heads, "length": length, "room": room, "width": width,
         "history": history, "dtype": dtype}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the rows of one sequence's verification step, kept for training while serving
        _topk("topk_one_seq", 8, 128256, 16),
        # an odd vocabulary in 32 bits, softened, a third of the ids masked (a grammar's mask)
        _topk("topk_odd", 37, 32003, 33, dtype="f32", temperature=2.0, masked=0.33, sigma=2.0),
        # a teacher's batch: 1024 tokens of the largest serving vocabulary
        _topk("topk_teacher", 1024, 151936, 64),
        # the smallest training step: 4 sequences of 4 tokens over a toy vocabulary
        _distill("distill_step_tiny", "step", 16, 1024, 256, 8, dtype="f32", sigma=2.0),
        # evaluation of a drafter of an odd vocabulary, softened, the remainder counted, an eighth of the tokens not
        _distill("distill_loss_odd", "loss", 300, 32003, 7999, 33, dtype="f32", temperature=2.0, remainder=True, live=0.875, sigma=2.0),
        # forward and backward apart, as a framework's automatic differentiation calls them
        _distill("distill_both_qwen", "both", 1024, 151936, 16384, 64, remainder=True, live=0.875),
        # a training batch of the headline vocabulary: 2048 tokens, loss and gradient at once
        _distill("distill_step_llama3", "step", 2048, 128256, 32064, 64, live=0.875),
        # one request with four beams: latency
        _beam("beam_one", 1, 4, 4, 128256),
        # a few requests of an odd vocabulary in 32 bits, twice as many candidates as beams, finished beams and masked ids among them
        _beam("beam_odd", 3, 5, 10, 32003, dtype="f32", finished=0.2, masked=0.33, sigma=2.0),
        # a serving batch: 16 requests with 8 beams
        _beam("beam_batch", 16, 8, 8, 128256, finished=0.1),
        # two requests, five beams: a token history and a little state of odd widths; launches are all of it
        _reorder("reorder_small", 2, 5, 5, 1, 3, 1, 1, 33, 77, dtype="f32"),
        # 16 requests with 4 beams: keys and values of two layers, 1000 of 1024 places filled
        _reorder("reorder_cache", 16, 4, 4, 4, 8, 1000, 1024, 128, 1000),
    ]


def _log_int(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v + 1 if v == 3072 else v


def draw(rng):
    op = rng.choice(["topk", "distill", "distill", "beam", "reorder"])
    dtype = rng.choice(["bf16", "f32"])
    e = 2 if dtype == "bf16" else 4
    sigma = round(rng.uniform(2.0, 3.0), 2)
    while True:
        N = _log_int(rng, 1000, 260000)
        if op == "topk":
            B = _log_int(rng, 1, 2048)
            if B * N * e <= 1024 * 151936 * 2:
                return _topk(None, B, N, _log_int(rng, 1, 128), dtype, rng.choice([1.0, 1.0, 2.0]), rng.choice([0.0, 0.33]), sigma)
        elif op == "distill":
            B, n = _log_int(rng, 1, 4096), max(100, int(N * rng.choice([0.1, 0.25, 0.4, 1.0])))
            n = n + 1 if n == 3072 else n
            if B * n * e <= 2048 * 32064 * 2 and B * N <= 2048 * 128256:
                return _distill(None, rng.choice(["loss", "both", "step", "step"]), B, N, n, _log_int(rng, 4, 128), dtype,
                                rng.choice([1.0, 2.0]), rng.choice([False, True]), rng.choice([1.0, 0.875]), sigma)
        elif op == "beam":
            G, W = _log_int(rng, 1, 64), rng.randint(1, 16)
            K = rng.choice([W, W, 2 * W])
            if G * W * N * e <= 256 * 128256 * 2 and G * K * K <= 2048:
                return _beam(None, G, W, K, N, dtype, rng.choice([0.0, 0.2]), rng.choice([0.0, 0.33]), sigma)
        else:
            G, W, length, heads, width = _log_int(rng, 1, 32), rng.randint(1, 12), _log_int(rng, 1, 4000), rng.randint(1, 8), rng.choice([33, 64, 128])
            K, buffers = rng.choice([W, W, W, rng.randint(1, 12)]), rng.randint(1, 8)
            if K == W == 1:
                continue
            if buffers * G * (W + K) * heads * length * width * e <= 4 * 2 * 64 * 8 * 1000 * 128 * 2:
                return _reorder(None, G, W, K, buffers, heads, length, length + rng.randint(0, 64), width, _log_int(rng, 1, 4000), dtype)


# ---------------------------------------------------------------------------------------------------------------- inputs
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return gen


def _rank_bias(case, gen):
    perm = torch.randperm(case["N"], generator=gen, device="cuda")     # rank of id j is 1 + perm[j]
    return perm, -case["zipf"] * torch.log1p(perm.to(torch.float32))


def _logits(case, B, bias, gen):
    return torch.randn((B, case["N"]), generator=gen, device="cuda").mul_(case["sigma"]).add_(bias)


def _mask(x, share, gen):
    if share:
        x.masked_fill_(torch.rand(x.shape, generator=gen, device="cuda") < share, -math.inf)
    return x


def _inputs(case, seed):
    """What the case's tensors hold, made from the seed alone."""
    gen, st = _generator(seed), {"case": case}
    if case["op"] == "topk":
        _, bias = _rank_bias(case, gen)
        st["x"] = _mask(_logits(case, case["B"], bias, gen), case["masked"], gen).to(_dtype(case))
    elif case["op"] == "distill":
        N, n, B, K = case["N"], case["n"], case["B"], case["K"]
        perm, bias = _rank_bias(case, gen)
        by_rank, n_top = torch.argsort(perm), (9 * n) // 10
        rest = by_rank[n_top:]
        kept = torch.cat([by_rank[:n_top], rest[torch.randperm(N - n_top, generator=gen, device="cuda")[:n - n_top]]])
        kept = torch.sort(kept).values
        st["kept"] = kept.to(torch.int32)
        st["z"] = torch.empty((B, n), dtype=_dtype(case), device="cuda")
        st["ids"] = torch.empty((B, K), dtype=torch.int32, device="cuda")
        st["top"] = torch.empty((B, K), device="cuda")
        st["lse"] = torch.empty(B, device="cuda")
        for r in range(0, B, 256):
            p = _logits(case, min(B, r + 256) - r, bias, gen)
            v, i = torch.topk(p, K, dim=1)
            st["top"][r:r + 256], st["ids"][r:r + 256] = v, i.to(torch.int32)
            st["lse"][r:r + 256] = torch.logsumexp(p / case["temperature"], 1)
            q = p[:, kept]
            st["z"][r:r + 256] = q.add_(torch.randn(q.shape, generator=gen, device="cuda")).to(_dtype(case))
        live = (torch.rand(B, generator=gen, device="cuda") < case["live"]).float()
        st["weight"] = live / live.sum().clamp(min=1.0)               # the mean over the tokens that count
    elif case["op"] == "beam":
        G, W = case["G"], case["W"]
        _, bias = _rank_bias(case, gen)
        st["x"] = _mask(_logits(case, G * W, bias, gen), case["masked"], gen).to(_dtype(case))
        st["scores"] = -torch.cumsum(torch.rand((G, W), generator=gen, device="cuda"), 1)
        st["finished"] = (torch.rand((G, W), generator=gen, device="cuda") < case["finished"]).to(torch.uint8)
    else:
        G, W, K = case["G"], case["W"], case["K"]
        shape = (G * W, case["heads"], case["room"], case["width"])
        st["states"] = [torch.randn(shape, generator=gen, device="cuda").to(_dtype(case)) for _ in range(case["buffers"])]
        st["history"] = torch.randint(0, 128256, (G * W, case["history"]), generator=gen, device="cuda", dtype=torch.int32)
        st["parent"] = torch.randint(0, W, (G, K), generator=gen, device="cuda", dtype=torch.int32)
    return st


EOS = 7


def prepare(case, seed):
    st = _inputs(case, seed)
    if case["op"] == "reorder":
        views = [s[:, :, :case["length"]] for s in st["states"]] + [st["history"]]
        st["views"] = views
        # beams that stay as many are reordered where they lie, others into buffers that the program keeps
        st["out"] = None if case["K"] == case["W"] else [torch.empty((case["G"] * case["K"],) + v.shape[1:], dtype=v.dtype, device="cuda") for v in views]
    if own:
        from paper_2506_03206_amd import rdk
        st["rdk"] = rdk
        if case["op"] == "topk":
            st["o"] = rdk.TopkOutputs(case["B"], case["N"], case["k"], "cuda")
        elif case["op"] == "distill":
            st["kernel"] = rdk.rdk_build_kernel(case["N"], st["kept"], rdk.IDENTITY)   # the drafter's vocabulary
            st["o"] = rdk.DistillOutputs(case["B"], case["n"], _dtype(case), "cuda")
        elif case["op"] == "beam":
            st["o"] = rdk.BeamOutputs(case["G"], case["W"], case["N"], case["K"], "cuda")
    elif case["op"] == "distill":
        st["slot_of"] = torch.full((case["N"],), -1, dtype=torch.int64, device="cuda")
        st["slot_of"][st["kept"].long()] = torch.arange(case["n"], device="cuda")
    return st


# ---------------------------------------------------------------------------------------------------------------- one pass
def run(st):
    case = st["case"]
    return (_run_own if own else _run_plain)[case["op"]](st, case)


def _own_topk(st, case):
    o = st["rdk"].rdk_topk(st["x"], case["k"], "logit", temperature=case["temperature"], outputs=st["o"])
    return {"ids": o.ids, "values": o.values, "lse": o.lse}


def _own_distill(st, case):
    rdk, lse = st["rdk"], st["lse"] if case["remainder"] else None
    args, T = (st["kernel"], st["z"], st["ids"], st["top"]), case["temperature"]
    if case["path"] == "step":
        o = rdk.rdk_distill_loss_grad(*args, teacher_lse=lse, temperature=T, weight=st["weight"], outputs=st["o"])
        return {"loss": o.loss, "grad": o.grad}
    o = rdk.rdk_distill_loss(*args, teacher_lse=lse, temperature=T, weight=st["weight"], outputs=st["o"])
    if case["path"] == "loss":
        return {"loss": o.loss}
    rdk.rdk_distill_grad(*args, o, temperature=T, weight=st["weight"])
    return {"loss": o.loss, "grad": o.grad}


def _own_beam(st, case):
    o = st["rdk"].rdk_beam_select(st["x"], st["scores"], case["K"], "logit", finished=st["finished"], eos=EOS, outputs=st["o"])
    return {"scores": o.scores, "parent": o.parent, "token": o.token, "finished": o.finished}


def _own_reorder(st, case):
    return st["rdk"].rdk_beam_reorder(st["views"], st["parent"], case["W"], out=st["out"])


def _plain_topk(st, case):
    x = st["x"].float()
    values, ids = torch.sort(x, dim=1, descending=True, stable=True)
    values, ids = values[:, :case["k"]], ids[:, :case["k"]].to(torch.int32)
    y = x / case["temperature"]
    m = y.amax(1, keepdim=True)
    lse = (m + torch.log(torch.exp(y - m).sum(1, keepdim=True)))[:, 0]
    return {"ids": torch.where(values > -math.inf, ids, -1).contiguous(), "values": values.contiguous(), "lse": lse}


def _plain_distill(st, case):
    T, w = case["temperature"], st["weight"]
    y = st["z"].float() / T
    m = y.amax(1, keepdim=True)
    e = torch.exp(y - m)
    total = e.sum(1, keepdim=True)
    slot = torch.where(st["ids"] >= 0, st["slot_of"][st["ids"].clamp(min=0).long()], -1)
    held = (slot >= 0) & (st["top"] > -math.inf)
    at = torch.where(held, slot, 0)
    v = torch.where(held, st["top"] / T, -math.inf)
    log_s = torch.gather(y, 1, at) - m - torch.log(total)
    if case["remainder"]:
        log_t = v - st["lse"][:, None]
    else:
        c = v.amax(1, keepdim=True)
        c = torch.where(c > -math.inf, c, 0.0)
        norm = torch.where(held, torch.exp(v - c), 0.0).sum(1, keepdim=True)
        log_t = v - (c + torch.log(norm))
    t = torch.where(held, torch.exp(log_t), 0.0)
    loss = torch.where(t > 0, t * (log_t - log_s), 0.0).sum(1)
    some = held.any(1)
    if case["remainder"]:
        others = torch.ones_like(e).scatter_reduce_(1, at, torch.where(held, 0.0, 1.0), "amin")
        rho = (e * others).sum(1) / total[:, 0]
        r = (1.0 - t.sum(1)).clamp(min=0.0)
        loss = loss + torch.where(r > 0, r * (torch.log(r) - torch.log(rho)), 0.0)
        factor = torch.where(others > 0, 1.0 - (r / rho)[:, None], 1.0)
    else:
        factor = some.float()[:, None]
    loss = torch.where(w == 0, 0.0, w * loss)
    if case["path"] == "loss":
        return {"loss": loss}
    grad = (factor * e / total).scatter_add_(1, at, -t) * (w / T)[:, None]
    return {"loss": loss, "grad": torch.where(w[:, None] == 0, 0.0, grad).to(st["z"].dtype)}


def _plain_beam(st, case):
    G, W, K, N = case["G"], case["W"], case["K"], case["N"]
    x = st["x"].float()
    y = x - x.amax(1, keepdim=True)
    y = y - torch.log(torch.exp(y).sum(1, keepdim=True))
    y = st["scores"].reshape(G * W, 1) + y
    done = st["finished"].bool()
    ended = torch.full_like(y, -math.inf)
    ended[:, EOS] = st["scores"].reshape(-1)
    y = torch.where(done.reshape(-1, 1), ended, y).reshape(G, W * N)
    scores, at = torch.sort(y, dim=1, descending=True, stable=True)
    scores, at = scores[:, :K].contiguous(), at[:, :K]
    some = scores > -math.inf
    parent, token = torch.where(some, at // N, -1), torch.where(some, at % N, -1)
    finished = some & (torch.gather(done, 1, parent.clamp(min=0)) | (token == EOS))
    return {"scores": scores, "parent": parent.to(torch.int32), "token": token.to(torch.int32), "finished": finished.to(torch.uint8)}


def _plain_reorder(st, case):
    rows = (st["parent"].long() + torch.arange(case["G"], device="cuda")[:, None] * case["W"]).reshape(-1)
    out = st["out"] or st["views"]
    return [o.copy_(v[rows]) for o, v in zip(out, st["views"])]


_run_own = {"topk": _own_topk, "distill": _own_distill, "beam": _own_beam, "reorder": _own_reorder}
_run_plain = {"topk": _plain_topk, "distill": _plain_distill, "beam": _plain_beam, "reorder": _plain_reorder}


# ---------------------------------------------------------------------------------------------------------------- what it costs
def work(case):
    """Every input read once and every output written once; rows without a weight, finished beams and beams that stay are not touched."""
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "topk":
        B, N = case["B"], case["N"]
        return {"bytes": B * (N * e + 8 * case["k"] + 4), "flops": 4.0 * B * N}
    if case["op"] == "distill":
        B, n, live = case["B"], case["n"], case["live"]
        reads, grads = (2 if case["path"] == "both" else 1), (0 if case["path"] == "loss" else 1)
        return {"bytes": B * n * e * (reads * live + grads) + B * (12 * case["K"] + 12), "flops": (4.0 + 4.0 * grads) * B * n * live}
    if case["op"] == "beam":
        rows = case["G"] * case["W"] * (1.0 - case["finished"])
        return {"bytes": rows * case["N"] * e + case["G"] * (5 * case["W"] + 13 * case["K"]), "flops": 5.0 * rows * case["N"]}
    G, W, K = case["G"], case["W"], case["K"]
    row = case["buffers"] * case["heads"] * case["length"] * case["width"] * e + 4 * case["history"]
    if K == W:   # of W beams with parents at random: those that change, and those that another one needs
        written, read = W - 1.0, W * (1.0 - (1.0 - 1.0 / W) ** (W - 1))
    else:
        written, read = float(K), W * (1.0 - (1.0 - 1.0 / W) ** K)
    return {"bytes": G * (written + read) * row + 4 * G * K, "flops": 0.0}


# ---------------------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    st = _inputs(case, seed)
    if case["op"] == "topk":
        x = st["x"].double()
        return {"ids": None, "values": torch.topk(x, case["k"], dim=1).values, "lse": torch.logsumexp(x / case["temperature"], 1)}
    if case["op"] == "beam":
        G, W, K = case["G"], case["W"], case["K"]
        y = torch.log_softmax(st["x"].double(), 1).reshape(G, W, -1) + st["scores"].double()[:, :, None]
        best = torch.topk(y, min(K, y.shape[2]), dim=2).values                  # no beam has more than K of the best
        alone = torch.full_like(best, -math.inf)
        alone[:, :, 0] = st["scores"].double()
        best = torch.where(st["finished"].bool()[:, :, None], alone, best)
        return {"scores": torch.topk(best.reshape(G, -1), K, dim=1).values, "parent": None, "token": None, "finished": None}
    if case["op"] == "reorder":
        G, W, parent = case["G"], case["W"], st["parent"].long()
        groups = torch.arange(G, device="cuda")[:, None]
        pick = lambda s: s.reshape((G, W) + s.shape[1:])[groups, parent].flatten(0, 1)  # noqa: E731
        return [pick(s[:, :, :case["length"]]).double() for s in st["states"]] + [pick(st["history"])]
    # the loss as a function of the logits, and its gradient by differentiation
    T, n = case["temperature"], case["n"]
    z = st["z"].double().requires_grad_(case["path"] != "loss")
    log_s = torch.log_softmax(z / T, 1)
    place = torch.searchsorted(st["kept"], st["ids"].contiguous()).clamp(max=n - 1)
    held = st["kept"][place] == st["ids"]
    row, col = torch.nonzero(held, as_tuple=True)
    teacher = torch.full((case["B"], n), -math.inf, dtype=torch.float64, device="cuda")
    teacher[row, place[row, col]] = st["top"][row, col].double() / T
    member = teacher > -math.inf
    if case["remainder"]:
        t = torch.exp(teacher - st["lse"].double()[:, None])
        r = (1.0 - t.sum(1)).clamp(min=0.0)
        log_rho = torch.logsumexp(log_s.masked_fill(member, -math.inf), 1)
        loss = torch.xlogy(t, t).sum(1) - (t * log_s).sum(1) + torch.xlogy(r, r) - r * log_rho
    else:
        t = torch.where(member, torch.softmax(teacher, 1), 0.0)
        loss = (torch.xlogy(t, t) - t * log_s).sum(1)
    loss = loss * st["weight"].double()
    if case["path"] == "loss":
        return {"loss": loss}
    return {"loss": loss.detach(), "grad": torch.autograd.grad(loss.sum(), z)[0]}
