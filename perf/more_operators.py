"""Operators around a model's ends: what a model says of given tokens, and the embedding rows its tokens come in by, both with their gradients.

  score   log probabilities of given tokens of every row, their ranks, the row's entropy and its top alternatives: scoring a text, the
          log probabilities that a server returns, candidates held against redistributed rows
  train   a drafter or a target trained on tokens, with a gradient of the entropy where a policy is kept from collapsing: forward and then
          backward (two calls: what comes from above arrives in between), or both at once (weights known beforehand)
  embed   rows of an embedding table for a batch of tokens
  embed_grad  the table's gradient: rows of equal tokens summed

Rows have the values of section 5.1 of the paper: Gaussian logits of a standard deviation of 2-3 on a Zipf rank bias; tokens follow the Zipf law of the
same ranks.  Where a vocabulary is pruned (n < N) the kept ids are the most frequent ones and 10 % random ones, and tokens are target ids.
"""
import math

import numpy as np
import torch

own = False


# ---------------------------------------------------------------------------------------------------------------- cases
def _score(name, B, N, C, k=0, kind="bf16", temperature=1.0, masked=0.0, sigma=3.0):
    c = {"op": "score", "B": B, "N": N, "n": N, "C": C, "k": k, "kind": kind, "temperature": temperature, "masked": masked, "sigma": sigma}
    return dict(c, name=name) if name else c


def _train(name, path, B, N, n, C, kind="bf16", temperature=1.0, entropy=False, live=1.0, sigma=3.0):
    c = {"op": "train", "path": path, "B": B, "N": N, "n": n, "C": C, "k": 0, "kind": kind, "temperature": temperature, "masked": 0.0, "sigma": sigma,
         "entropy": entropy, "live": live}
    return dict(c, name=name) if name else c


def _embed(name, B, N, n, d, table="bf16", rows="bf16", scale=1.0):
    c = {"op": "embed", "B": B, "N": N, "n": n, "d": d, "table": table, "rows": rows, "scale": scale}
    return dict(c, name=name) if name else c


def _embed_grad(name, B, N, n, d, table="bf16", rows="bf16", scale=1.0):
    return dict(_embed(name, B, N, n, d, table, rows, scale), op="embed_grad")


def listed():
    return [
        # the positions of one sequence's verification step, with five alternatives each, as a server returns them
        _score("score_one_seq", 8, 128256, 1, 5),
        # an odd vocabulary in 32 bits, softened, a third of the ids masked (a grammar's mask), three tokens a row
        _score("score_odd", 37, 32003, 3, kind="f32", temperature=2.0, masked=0.33, sigma=2.0),
        # a text of 1024 tokens scored over the largest serving vocabulary
        _score("score_text", 1024, 151936, 1),
        # a prompt's log probabilities with twenty alternatives
        _score("score_top", 256, 128256, 1, 20),
        # eight candidates a position held against redistributed rows (weights)
        _score("score_weights", 256, 32000, 8, kind="prob"),
        # the smallest training step: 4 sequences of 4 tokens over a toy vocabulary
        _train("train_step_tiny", "step", 16, 1024, 256, 1, kind="f32", sigma=2.0),
        # forward and backward apart, as a framework's automatic differentiation calls them, with the entropy's gradient
        _train("train_both_qwen", "both", 1024, 151936, 16384, 1, entropy=True, live=0.875),
        # a training batch of the pruned headline vocabulary: 2048 tokens, an eighth of them padding, loss and gradient at once
        _train("train_step_llama3", "step", 2048, 128256, 32064, 1, live=0.875),
        # one decoding step of eight beams: latency
        _embed("embed_decode", 8, 128256, 128256, 4096),
        # a prompt
        _embed("embed_prompt", 8192, 128256, 128256, 4096, scale=64.0),
        # a few sequences and a pruned table of an odd width in 32 bits
        _embed_grad("embed_grad_odd", 301, 32003, 7999, 515, "f32", "f32", scale=0.5),
        # a training batch of 16384 tokens
        _embed_grad("embed_grad_batch", 16384, 128256, 128256, 2048),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["score", "score", "train", "embed", "embed_grad"])
    sigma = round(rng.uniform(2.0, 3.0), 2)
    while True:
        N, B = _log_int(rng, 1000, 260000), _log_int(rng, 1, 20000 if op.startswith("embed") else 2048)
        n = max(100, int(N * rng.choice([0.1, 0.25, 0.4, 1.0])))
        if op == "score":
            kind = rng.choice(["bf16", "f32", "prob"])
            if B * N * (2 if kind == "bf16" else 4) <= 1024 * 151936 * 2:
                return _score(None, B, N, rng.choice([1, 1, rng.randint(2, 16)]), rng.choice([0, 0, _log_int(rng, 1, 64)]), kind,
                              1.0 if kind == "prob" else rng.choice([1.0, 1.0, 2.0]), rng.choice([0.0, 0.33]), sigma)
        elif op == "train":
            kind = rng.choice(["bf16", "f32"])
            if B * n * (2 if kind == "bf16" else 4) <= 2048 * 32064 * 2:
                return _train(None, rng.choice(["both", "step"]), B, N, n, rng.choice([1, 1, rng.randint(2, 16)]), kind, rng.choice([1.0, 1.0, 2.0]), rng.choice([False, True]),
                              rng.choice([1.0, 0.875]), sigma)
        else:
            d, table, rows = _log_int(rng, 16, 8192), rng.choice(["bf16", "f32"]), rng.choice(["bf16", "f32"])
            if (B + n) * d * 4 <= (16384 + 128256) * 2048 * 2:
                return (_embed if op == "embed" else _embed_grad)(None, B, N, n, d, table, rows, rng.choice([1.0, 0.5, round(math.sqrt(d), 3)]))


# ---------------------------------------------------------------------------------------------------------------- inputs
def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return gen


def _tokens(case, by_rank, count, gen):
    """`count` target ids: the id of rank r with a probability proportional to 1 / (1 + r)."""
    cdf = torch.cumsum(1.0 / torch.arange(1, case["N"] + 1, device="cuda", dtype=torch.float64), 0)
    at = torch.searchsorted(cdf, torch.rand(count, generator=gen, device="cuda", dtype=torch.float64) * cdf[-1]).clamp(max=case["N"] - 1)
    return by_rank[at].to(torch.int32)


def _inputs(case, seed):
    """What the case's tensors hold, made from the seed alone."""
    gen, st = _generator(seed), {"case": case}
    N, n, B = case["N"], case["n"], case["B"]
    perm = torch.randperm(N, generator=gen, device="cuda")              # rank of id j
    by_rank, st["kept"] = torch.argsort(perm), None
    if n < N:
        n_top = (9 * n) // 10
        rest = by_rank[n_top:]
        kept = torch.cat([by_rank[:n_top], rest[torch.randperm(N - n_top, generator=gen, device="cuda")[:n - n_top]]])
        st["kept"] = torch.sort(kept).values.to(torch.int32)
    if case["op"] in ("score", "train"):
        bias = -torch.log1p(perm.float())
        if n < N:
            bias = bias[st["kept"].long()]
        x = torch.randn((B, n), generator=gen, device="cuda").mul_(case["sigma"]).add_(bias)
        if case["masked"]:
            x.masked_fill_(torch.rand(x.shape, generator=gen, device="cuda") < case["masked"], -math.inf)
        st["x"] = torch.softmax(x, 1) if case["kind"] == "prob" else x.to(_dtype(case["kind"]))
        st["tokens"] = _tokens(case, by_rank, B * case["C"], gen).reshape(B, case["C"])
        if case["op"] == "train":
            live = (torch.rand((B, case["C"]), generator=gen, device="cuda") < case["live"]).float()
            st["above"] = -live / live.sum().clamp(min=1.0)             # the mean of the tokens that count
            st["tokens"].masked_fill_(live == 0, -1)                    # padding
            st["above_entropy"] = live.amax(1) * (-0.01 / B) if case["entropy"] else None
    else:
        st["ids"] = _tokens(case, by_rank, B, gen)
        shape, kind = ((n, case["d"]), case["table"]) if case["op"] == "embed" else ((B, case["d"]), case["rows"])
        st["x"] = torch.randn(shape, generator=gen, device="cuda").to(_dtype(kind))
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:
        from paper_2506_03206_amd import rdk
        st["rdk"], B, n = rdk, case["B"], case["n"]
        st["kernel"] = None if st["kept"] is None else rdk.rdk_build_kernel(case["N"], st["kept"], rdk.IDENTITY)   # the pruned vocabulary
        if case["op"] in ("score", "train"):
            st["o"] = rdk.LogprobsOutputs(B, case["C"], case["k"], "cuda", grad=torch.empty_like(st["x"]) if case["op"] == "train" else None)
        elif case["op"] == "embed":
            st["out"] = torch.empty((B, case["d"]), dtype=_dtype(case["rows"]), device="cuda")
        else:
            st["o"] = rdk.EmbedGradOutputs(n, case["d"], _dtype(case["table"]), "cuda")
    elif st["kept"] is not None:
        st["slot_of"] = torch.full((case["N"],), -1, dtype=torch.int64, device="cuda")
        st["slot_of"][st["kept"].long()] = torch.arange(case["n"], device="cuda")
    return st


# ---------------------------------------------------------------------------------------------------------------- one pass
def run(st):
    case = st["case"]
    return (_run_own if own else _run_plain)[case["op"]](st, case)


def _own_score(st, case):
    o = st["rdk"].rdk_logprobs(st["x"], st["tokens"], "prob" if case["kind"] == "prob" else "logit", k=case["k"], temperature=case["temperature"],
                               outputs=st["o"])
    out = {"logprob": o.logprob, "rank": o.rank, "entropy": o.entropy}
    return dict(out, top_ids=o.top_ids, top_logprobs=o.top_logprobs) if case["k"] else out


def _own_train(st, case):
    rdk, x, tokens = st["rdk"], st["x"], st["tokens"]
    args, above = {"kernel": st["kernel"], "temperature": case["temperature"]}, (st["above"], st["above_entropy"])
    if case["path"] == "step":
        o = rdk.rdk_logprobs_step(x, tokens, *above, outputs=st["o"], **args)
    else:
        o = rdk.rdk_logprobs(x, tokens, ranks=False, outputs=st["o"], **args)
        rdk.rdk_logprobs_grad(x, tokens, o, *above, **args)
    return {"logprob": o.logprob, "entropy": o.entropy, "grad": o.grad}


def _own_embed(st, case):
    return st["rdk"].rdk_embed(st["ids"], st["x"], scale=case["scale"], kernel=st["kernel"], out=st["out"])


def _own_embed_grad(st, case):
    return st["rdk"].rdk_embed_grad(st["ids"], st["x"], st["o"], scale=case["scale"], kernel=st["kernel"]).grad


def _slots(st, ids):
    """Places of target ids in the vocabulary, -1 where it does not hold them."""
    ids = ids.long()
    return ids if st["kept"] is None else torch.where(ids >= 0, st["slot_of"][ids.clamp(min=0)], -1)


def _plain_rows(st, case):
    """Shares s, their logarithms (0 s for s = 0), log probabilities of the tokens and the entropy."""
    x, tokens = st["x"].float(), st["tokens"]
    if case["kind"] == "prob":
        y = torch.log(x)
    else:
        y = x / case["temperature"]
    y = y - y.amax(1, keepdim=True)
    e = torch.exp(y)
    total = e.sum(1, keepdim=True)
    s, log_s = e / total, y - torch.log(total)
    entropy = -torch.where(s > 0, s * log_s, 0.0).sum(1)
    slot = _slots(st, tokens)
    at = slot.clamp(min=0)
    logprob = torch.where(slot >= 0, torch.gather(log_s, 1, at), -math.inf)
    logprob = torch.where(tokens < 0, 0.0, logprob)
    return x, s, log_s, slot, logprob, entropy


def _plain_score(st, case):
    x, s, log_s, slot, logprob, entropy = _plain_rows(st, case)
    place, ranks = torch.arange(case["n"], device="cuda"), []
    for c in range(case["C"]):
        at = slot[:, c:c + 1]
        v = torch.gather(x, 1, at)
        before = (x > v).sum(1) + ((x == v) & (place < at)).sum(1)
        ranks.append(torch.where(logprob[:, c] > -math.inf, before, -1))
    out = {"logprob": logprob, "rank": torch.stack(ranks, 1).to(torch.int32), "entropy": entropy}
    if case["k"]:
        values, ids = torch.sort(x, dim=1, descending=True, stable=True)
        ids = ids[:, :case["k"]]
        top = torch.gather(log_s, 1, ids)
        out.update(top_ids=torch.where(top > -math.inf, ids, -1).to(torch.int32), top_logprobs=top)
    return out


def _plain_train(st, case):
    x, s, log_s, slot, logprob, entropy = _plain_rows(st, case)
    above = torch.where(slot >= 0, st["above"], 0.0)
    pull = above.sum(1, keepdim=True)
    if case["entropy"]:
        pull = pull + st["above_entropy"][:, None] * (log_s + entropy[:, None])
    grad = (-s * pull).scatter_add_(1, slot.clamp(min=0), above) / case["temperature"]
    return {"logprob": logprob, "entropy": entropy, "grad": grad.to(st["x"].dtype)}


def _plain_embed(st, case):
    slot = _slots(st, st["ids"])
    rows = st["x"][slot.clamp(min=0)].float() * case["scale"]
    return torch.where(slot[:, None] >= 0, rows, 0.0).to(_dtype(case["rows"]))


def _plain_embed_grad(st, case):
    slot = _slots(st, st["ids"])
    rows = torch.where(slot[:, None] >= 0, st["x"].float(), 0.0)
    grad = torch.zeros((case["n"], case["d"]), device="cuda").index_add_(0, slot.clamp(min=0), rows)
    return (grad * case["scale"]).to(_dtype(case["table"]))


_run_own = {"score": _own_score, "train": _own_train, "embed": _own_embed, "embed_grad": _own_embed_grad}
_run_plain = {"score": _plain_score, "train": _plain_train, "embed": _plain_embed, "embed_grad": _plain_embed_grad}


# ---------------------------------------------------------------------------------------------------------------- what it costs
def _size(name):
    return 2 if name == "bf16" else 4


def work(case):
    """Every input read once and every output written once; of a table the rows that the tokens are expected to name."""
    B, n = case["B"], case["n"]
    if case["op"] == "score":
        return {"bytes": B * (n * _size(case["kind"]) + 12 * case["C"] + 4 + 8 * case["k"]), "flops": (5.0 + case["C"]) * B * n}
    if case["op"] == "train":
        read_again = 1.0 - (1.0 - case["live"]) ** case["C"]            # rows of padding alone have no gradient that depends on them
        reads = read_again + 1.0 if case["path"] == "both" else 1.0
        return {"bytes": B * ((reads + 1.0) * n * _size(case["kind"]) + 12 * case["C"] + 8), "flops": (12.0 if case["entropy"] else 9.0) * B * n}
    d = case["d"]
    if case["op"] == "embed":
        p = 1.0 / np.arange(1, n + 1)
        named = float((1.0 - (1.0 - p / (p.sum() + math.log(case["N"] / n))) ** B).sum())
        return {"bytes": B * (4 + d * _size(case["rows"])) + named * d * _size(case["table"]), "flops": float(B * d)}
    return {"bytes": B * (4 + d * _size(case["rows"])) + n * d * _size(case["table"]), "flops": float(B * d)}


# ---------------------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    st = _inputs(case, seed)
    n = case["n"]

    def places(ids):
        if st["kept"] is None:
            return ids.long(), ids >= 0
        place = torch.searchsorted(st["kept"], ids.contiguous()).clamp(max=n - 1)
        return place, st["kept"][place] == ids

    if case["op"] == "embed":
        place, held = places(st["ids"])
        return st["x"].double()[place.clamp(min=0)] * (case["scale"] * held.double())[:, None]
    if case["op"] == "embed_grad":
        place, held = places(st["ids"])
        order = torch.argsort(torch.where(held, place, n), stable=True)
        sums = torch.cumsum(torch.bincount(torch.where(held, place, n), minlength=n + 1)[:n], 0)
        grad = torch.zeros((n, case["d"]), dtype=torch.float64, device="cuda")
        for first in range(0, case["d"], 256):                          # sums of runs as differences would cancel: segment by segment
            part = st["x"][order, first:first + 256].double()
            lengths = torch.diff(sums, prepend=sums.new_zeros(1))
            grad[:, first:first + 256] = torch.segment_reduce(part[:int(sums[-1])], "sum", lengths=lengths, initial=0.0) if int(sums[-1]) else 0.0
        return grad * case["scale"]
    x = st["x"].double()
    if case["op"] == "score":
        logits = torch.log(x) if case["kind"] == "prob" else x / case["temperature"]
        log_s = torch.log_softmax(logits, 1)
        out = {"logprob": torch.gather(log_s, 1, st["tokens"].long()), "rank": None, "entropy": torch.special.entr(log_s.exp()).sum(1)}
        return dict(out, top_ids=None, top_logprobs=torch.topk(log_s, case["k"], dim=1).values) if case["k"] else out
    # the objective as a function of the logits, and its gradient by differentiation
    x.requires_grad_(True)
    log_s = torch.log_softmax(x / case["temperature"], 1)
    place, held = places(st["tokens"])
    held &= st["tokens"] >= 0
    picked = torch.gather(log_s, 1, place.clamp(min=0))
    entropy = -(log_s.exp() * log_s).sum(1)
    objective = (torch.where(held, picked, 0.0) * st["above"].double()).sum()
    if case["entropy"]:
        objective = objective + (entropy * st["above_entropy"].double()).sum()
    logprob = torch.where(held, picked.detach(), torch.where(st["tokens"] < 0, 0.0, -math.inf))
    return {"logprob": logprob, "entropy": entropy.detach(), "grad": torch.autograd.grad(objective, x)[0]}
