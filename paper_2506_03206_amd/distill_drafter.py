#!/usr/bin/env python3
"""A pruned drafter distilled from its target's top logits, another trained on its target's tokens, and beam search with the target and with the trained drafter.

The target is a small recurrent model with random weights: a state s, s' = tanh(s A + E[token]), and logits s U on a Zipf rank bias over N ids.
The drafter sees the same state and has a trainable head V over the n most frequent ids.

  training   the target's rows of a batch of states -> rdk_topk keeps K logits and the normaliser of each (all that is stored of a teacher)
             -> rdk_distill_loss_grad gives the loss and its gradient with respect to the drafter's logits -> the head's weights by one product
  tokens     a drafter that reads one state less and the token that followed, by an embedding over its own vocabulary (rdk_embed), trained on the
             tokens that the target drew: rdk_logprobs_step gives their log probabilities and the gradient with respect to the logits, rdk_embed_grad that of the
             embedding
  scoring    the target's own text under its rows: log probabilities, ranks, entropy and the top alternatives (rdk_logprobs)
  check      the acceptance rate alpha of the drafter under redistribution (Eq. 3), before and after, by rdk_redistribute_verify
  decoding   beam search over the target's rows and over the drafter's redistributed rows: rdk_beam_select picks the beams, rdk_beam_reorder moves
             their recurrent states and token histories

  python -m paper_2506_03206_amd.distill_drafter [--N 32000] [--n 8000] [--steps 200]
"""
import argparse
import json

import torch

from . import rdk


class Target:
    """Random recurrent model: rows over N ids from states [B, d]."""

    def __init__(self, N, d, seed, device):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        rand = lambda *shape: torch.randn(shape, generator=g, device=device)  # noqa: E731
        self.A, self.E, self.U = rand(d, d) * (0.6 / d ** 0.5), rand(N, d) * 0.8, rand(d, N) * (3.0 / d ** 0.5)
        rank = torch.randperm(N, generator=g, device=device)
        self.bias = -torch.log1p(rank.float())
        self.by_frequency = torch.argsort(rank)
        self.N, self.d, self.gen = N, d, g

    def step(self, state, token):
        return torch.tanh(state @ self.A + rdk.rdk_embed(token.to(torch.int32).contiguous(), self.E))

    def rows(self, state, dtype=torch.bfloat16):
        return (state @ self.U + self.bias).to(dtype)

    def states(self, B, steps=4):
        """States after a few tokens drawn from the model itself."""
        s = torch.zeros((B, self.d), device=self.E.device)
        for _ in range(steps):
            p = torch.softmax(self.rows(s).float(), 1)
            s = self.step(s, torch.multinomial(p, 1, generator=self.gen)[:, 0])
        return s

    def draw(self, state):
        """A token of every row."""
        return torch.multinomial(torch.softmax(self.rows(state).float(), 1), 1, generator=self.gen)[:, 0].to(torch.int32)


class Drafter:
    """A head over the kept ids on the target's state."""

    def __init__(self, target, n):
        self.kept = torch.sort(target.by_frequency[:n]).values.to(torch.int32)
        self.kernel = rdk.rdk_build_kernel(target.N, self.kept, rdk.IDENTITY)
        self.V = torch.zeros((target.d + 1, n), device=self.kept.device)      # the last row is a bias

    def rows(self, state):
        return torch.addmm(self.V[-1], state, self.V[:-1]).to(torch.bfloat16)


class TokenDrafter(Drafter):
    """A head on the state before the last token and an embedding of that token over the kept ids (zero for others)."""

    def __init__(self, target, n):
        super().__init__(target, n)
        self.E = torch.zeros((n, target.d), device=self.kept.device)

    def step(self, state, token, following, weight, entropy_weight=None):
        """Log probabilities of the following tokens [B], entropies, and the gradients of sum(weight * logprob) + sum(entropy_weight * entropy) with respect to
        the head and the embedding.  Tokens that the vocabulary does not hold have a log probability of -inf and no gradient."""
        h = state + rdk.rdk_embed(token, self.E, kernel=self.kernel)
        o = rdk.rdk_logprobs_step(self.rows(h), following, weight, entropy_weight, kernel=self.kernel)
        dz = o.grad.float()
        head = torch.cat([h.t() @ dz, dz.sum(0, keepdim=True)])
        table = rdk.EmbedGradOutputs(self.E.shape[0], self.E.shape[1], torch.float32, self.E.device)
        rdk.rdk_embed_grad(token, dz @ self.V[:-1].t(), table, kernel=self.kernel)
        return o.logprob[:, 0], o.entropy, head, table.grad


def train(target, drafter, steps, B, K, temperature, rate, remainder=True):
    """Mean losses, one a step.  Adam on the head's weights."""
    first, second, losses = torch.zeros_like(drafter.V), torch.zeros_like(drafter.V), []
    weight = torch.full((B,), 1.0 / B, device=drafter.V.device)
    top = rdk.TopkOutputs(B, target.N, K, drafter.V.device)
    out = rdk.DistillOutputs(B, drafter.kept.numel(), torch.bfloat16, drafter.V.device)
    for t in range(1, steps + 1):
        s = target.states(B)
        rdk.rdk_topk(target.rows(s), K, temperature=temperature, outputs=top)
        rdk.rdk_distill_loss_grad(drafter.kernel, drafter.rows(s), top.ids, top.values, teacher_lse=top.lse if remainder else None,
                                  temperature=temperature, weight=weight, outputs=out)
        losses.append(out.loss.sum())
        dz = out.grad.float()
        grad = torch.cat([s.t() @ dz, dz.sum(0, keepdim=True)])
        first.mul_(0.9).add_(grad, alpha=0.1)
        second.mul_(0.99).addcmul_(grad, grad, value=0.01)
        drafter.V -= rate * (first / (1 - 0.9 ** t)) / ((second / (1 - 0.99 ** t)).sqrt() + 1e-8)
    return torch.stack(losses).tolist()


def train_on_tokens(target, drafter, steps, B, rate, entropy=0.0):
    """Mean losses of the tokens that the drafter's vocabulary holds, one a step.  Adam on its head and its embedding; entropy: weight of the mean entropy, which is
    held up by it."""
    params = [drafter.V, drafter.E]
    first, second, losses = [torch.zeros_like(p) for p in params], [torch.zeros_like(p) for p in params], []
    weight = torch.full((B,), -1.0 / B, device=drafter.V.device)
    for t in range(1, steps + 1):
        s = target.states(B)
        token = target.draw(s)
        following = target.draw(target.step(s, token))
        logprob, _, *grads = drafter.step(s, token, following, weight, weight * entropy if entropy else None)
        held = logprob > -float("inf")
        losses.append(-torch.where(held, logprob, 0.0).sum() / held.sum().clamp(min=1))
        for p, m, v, g in zip(params, first, second, grads):
            m.mul_(0.9).add_(g, alpha=0.1)
            v.mul_(0.99).addcmul_(g, g, value=0.01)
            p -= rate * (m / (1 - 0.9 ** t)) / ((v / (1 - 0.99 ** t)).sqrt() + 1e-8)
    return torch.stack(losses).tolist()


def score(target, B, top):
    """The target's own next tokens under its rows: mean log probability, mean entropy, the share of them that is among the top entries."""
    s = target.states(B)
    o = rdk.rdk_logprobs(target.rows(s), target.draw(s), k=top)
    return float(o.logprob.mean()), float(o.entropy.mean()), float((o.rank < top).float().mean())


def acceptance(target, drafter, B=512):
    """Mean acceptance rate of the drafter's rows under Eq. 3."""
    s = target.states(B)
    o = rdk.rdk_redistribute_verify(drafter.kernel, rdk.LINEAR_TAYLOR, target.rows(s), drafter.rows(s), seed=1, p_kind="logit", q_kind="logit")
    return float(o.alpha.mean())


def beam_search(target, G, W, length, eos, drafter=None):
    """Best sequences of G requests: token histories [G, W, length], scores [G, W].  With a drafter the rows are its redistributed ones."""
    dev = target.E.device
    state = target.states(G).repeat_interleave(W, 0)
    history = torch.full((G * W, length), -1, dtype=torch.int32, device=dev)
    scores = torch.full((G, W), -float("inf"), device=dev)
    scores[:, 0] = 0.0                                                   # the beams of a request are one at first
    finished = torch.zeros((G, W), dtype=torch.uint8, device=dev)
    start = state.clone()
    for t in range(length):
        if drafter is None:
            x, kind = target.rows(state), "logit"
        else:
            x, kind = rdk.rdk_redistribute_linear(drafter.kernel, rdk.LINEAR_SPARSE, drafter.rows(state), "logit"), "prob"
        o = rdk.rdk_beam_select(x, scores, W, kind, finished=finished, eos=eos)
        rdk.rdk_beam_reorder([state, history], o.parent)
        token = o.token.reshape(-1)
        history[:, t] = token
        state = target.step(state, token.clamp(min=0).long())
        scores, finished = o.scores, o.finished
    return history.view(G, W, length), scores, start


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--N", type=int, default=32000)
    ap.add_argument("--n", type=int, default=8000)
    ap.add_argument("--d", type=int, default=64)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--batch", type=int, default=512)
    ap.add_argument("--top", type=int, default=64)
    ap.add_argument("--temperature", type=float, default=1.0)
    ap.add_argument("--rate", type=float, default=0.02)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    target = Target(a.N, a.d, a.seed, "cuda")
    drafter = Drafter(target, a.n)
    before = acceptance(target, drafter)
    losses = train(target, drafter, a.steps, a.batch, a.top, a.temperature, a.rate)
    after = acceptance(target, drafter)
    eos = int(target.by_frequency[0])
    history, scores, _ = beam_search(target, 4, 4, 12, eos)
    draft_history, draft_scores, _ = beam_search(target, 4, 4, 12, eos, drafter)
    by_tokens = TokenDrafter(target, a.n)
    token_losses = train_on_tokens(target, by_tokens, a.steps, a.batch, a.rate)
    logprob, entropy, among_top = score(target, a.batch, 5)
    print(json.dumps({"N": a.N, "n": a.n, "loss_first": losses[0], "loss_last": losses[-1], "alpha_before": before, "alpha_after": after,
                      "best_scores": scores[:, 0].tolist(), "best_tokens": history[:, 0].tolist(),
                      "drafter_best_scores": draft_scores[:, 0].tolist(), "drafter_best_tokens": draft_history[:, 0].tolist(),
                      "token_loss_first": token_losses[0], "token_loss_last": token_losses[-1], "text_logprob": logprob, "text_entropy": entropy,
                      "text_among_top": among_top}))


if __name__ == "__main__":
    main()
