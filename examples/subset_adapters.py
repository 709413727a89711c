"""Trying a choice of training data out: the brittleness test of data valuation, with adapters.

A frozen model (one residual block and a vocabulary of logits) is valued and then tuned on synthetic data:

  1. the projected gradients of every training example are logged, the queries' gradients preconditioned, and each
     training example is scored by its summed influence on the queries;
  2. four subsets are formed: all data, all without the most valuable examples, all without as many random ones, and
     the most valuable ones alone;
  3. an adapter is trained on each subset, all four in the same batches: a row of a batch names its adapter;
  4. the queries' loss under each adapter tells whether the examples named valuable were.

The logits' gradient of step 1, which the logging reads, and the steps of 3 come from the same operators
(logra_token_loss, logra_dropout, logra_adapter_forward and _backward).  Run on an MI355X:

    python examples/subset_adapters.py
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2405_13954_amd as P  # noqa: E402

DEV = "cuda"


class Frozen:
    """h = x + drop(relu(x W1)), logits = h W2: the frozen model, with dropout in its residual block."""

    def __init__(self, n, vocab, gen):
        self.w1 = (torch.randn(n, n, generator=gen, device=DEV) * n ** -0.5).to(torch.bfloat16)
        self.w2 = (torch.randn(n, vocab, generator=gen, device=DEV) * n ** -0.5).to(torch.bfloat16)

    def hidden(self, x, p=0.0, seed=0, offset=0):
        h = torch.empty_like(x)
        P.logra_dropout(torch.relu(x @ self.w1), h, p, seed, offset, residual=x)
        return h


def make_data(model, n, vocab, examples, tokens, gen, shift):
    """Inputs [examples, tokens, n] and targets drawn from the model with a shift of its last layer."""
    x = torch.randn(examples, tokens, n, generator=gen, device=DEV).to(torch.bfloat16)
    z = (model.hidden(x.view(-1, n)).float() @ (model.w2.float() + shift)) * 2
    target = torch.multinomial(torch.softmax(z, 1), 1, generator=gen).view(examples, tokens)
    return x, target


def losses_and_gradients(model, x, target):
    """Per-token losses and logit gradients of the bare model."""
    h = model.hidden(x.view(-1, x.shape[-1]))
    z = h @ model.w2
    loss, dz = torch.empty(z.shape[0], device=DEV), torch.empty_like(z)
    P.logra_token_loss(z, target.reshape(-1), loss, dlogits=dz)
    return h, loss, dz


def value(model, train, query, k, gen):
    """Influence of every training example on the queries' loss, summed over the queries (the projected gradients of
    the logits' layer, Sec. 3.1; damped inverse, Sec. 2; scores, Eq. (2))."""
    n, vocab = model.w2.shape
    p_in = (torch.randn(k, n, generator=gen, device=DEV) * k ** -0.5).to(torch.bfloat16)
    p_out = (torch.randn(k, vocab, generator=gen, device=DEV) * k ** -0.5).to(torch.bfloat16)
    rows = []
    for x, target in (train, query):
        B, T, _ = x.shape
        h, _, dz = losses_and_gradients(model, x, target)
        g = torch.empty(B, k * k, device=DEV)
        P.logra_project_layer(h.view(B, T, n), dz.view(B, T, vocab), p_in, p_out, g)
        rows.append(g)
    S = torch.zeros(k * k, k * k, device=DEV)
    P.logra_cov_accumulate(rows[0], S)
    pre = torch.empty_like(rows[1])
    P.logra_precondition(S, rows[0].shape[0], 0.1, rows[1], pre)
    scores = torch.empty(rows[1].shape[0], rows[0].shape[0], device=DEV)
    P.logra_influence_scores(pre, rows[0], scores=scores)
    return scores.sum(0)


def train_adapters(model, train, subsets, rank, steps, batch, gen, lr=0.01, p=0.1, seed=11):
    """One adapter of the logits' layer per subset (lists of example numbers), trained together; returns (a, b)."""
    x, target = train
    n, vocab = model.w2.shape
    m, tokens = len(subsets), x.shape[1]
    a = torch.randn(m, rank, n, generator=gen, device=DEV) * n ** -0.5
    b = torch.zeros(m, rank, vocab, device=DEV)
    rows = m * batch * tokens
    # the rows' adapters are the same in every step: one plan, one workspace
    ids = torch.arange(m, dtype=torch.int32, device=DEV).repeat_interleave(batch * tokens)
    plan = P.logra_adapter_plan(ids, m)
    ws = torch.empty(P.logra_adapter_ws_size(rows, n, vocab, rank, m), dtype=torch.uint8, device=DEV)
    scale = torch.full((m,), 2.0, device=DEV)
    weight = torch.full((rows,), 1.0 / (batch * tokens), device=DEV)
    u, loss = torch.empty(rows, rank, device=DEV), torch.empty(rows, device=DEV)
    y = torch.empty(rows, vocab, dtype=torch.bfloat16, device=DEV)
    da, db = torch.empty_like(a), torch.empty_like(b)
    moments = [torch.zeros_like(t) for t in (a, a, b, b)]
    for step in range(steps):
        picks = torch.cat([s[torch.randint(len(s), (batch,), generator=gen, device=DEV)] for s in subsets])
        h = model.hidden(x[picks].view(-1, n), p, seed, 2 * step)
        a16, b16 = a.to(torch.bfloat16), b.to(torch.bfloat16)
        drop = dict(p=p, seed=seed, offset=2 * step + 1)
        base = h @ model.w2
        P.logra_adapter_forward(h, a16, b16, plan, y, base=base, scale=scale, u=u, ws=ws, **drop)
        P.logra_token_loss(y, target[picks].reshape(-1), loss, dlogits=y, weight=weight)
        P.logra_adapter_backward(h, y, a16, b16, plan, u, da, db, scale=scale, ws=ws, **drop)
        for t, g, m1, m2 in ((a, da, *moments[:2]), (b, db, *moments[2:])):      # Adam
            m1.lerp_(g, 0.1)
            m2.lerp_(g * g, 0.05)
            fix1, fix2 = 1 - 0.9 ** (step + 1), 1 - 0.95 ** (step + 1)
            t -= lr * (m1 / fix1) / ((m2 / fix2).sqrt() + 1e-8)
    return a.to(torch.bfloat16), b.to(torch.bfloat16), scale


def query_loss(model, query, adapters):
    """Mean loss of the queries under each adapter, and under the bare model (last): every query once per adapter, one
    batch, the bare model's rows without an adapter."""
    x, target = query
    a, b, scale = adapters
    m, n = a.shape[0], x.shape[-1]
    h = model.hidden(x.view(-1, n)).repeat(m + 1, 1)
    per = x.shape[0] * x.shape[1]
    ids = torch.arange(m + 1, dtype=torch.int32, device=DEV).repeat_interleave(per)
    ids[m * per:] = -1
    y = h @ model.w2
    P.logra_adapter_forward(h, a, b, P.logra_adapter_plan(ids, m), y, base=y, scale=scale)
    loss = torch.empty(y.shape[0], device=DEV)
    P.logra_token_loss(y, target.reshape(-1).repeat(m + 1), loss)
    return loss.view(m + 1, per).mean(1).tolist()


def run(n=256, vocab=1000, examples=256, tokens=32, queries=32, k=16, rank=8, steps=150, batch=16, seed=0):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    model = Frozen(n, vocab, gen)
    shift = torch.randn(n, 4, generator=gen, device=DEV) @ torch.randn(4, vocab, generator=gen, device=DEV) * (0.7 / n ** 0.5)
    train = make_data(model, n, vocab, examples, tokens, gen, shift)
    noise = torch.randperm(examples, generator=gen, device=DEV)[:examples // 2]    # half of the examples teach nothing
    train[1][noise] = torch.randint(vocab, (len(noise), tokens), generator=gen, device=DEV)
    query = make_data(model, n, vocab, queries, tokens, gen, shift)
    scores = value(model, train, query, k, gen)
    order = scores.argsort(descending=True)
    drop = examples // 4
    shuffled = torch.randperm(examples, generator=gen, device=DEV)
    subsets = {"all data": order, "without the most valuable quarter": order[drop:],
               "without a random quarter": shuffled[drop:], "the most valuable quarter alone": order[:drop]}
    adapters = train_adapters(model, train, list(subsets.values()), rank, steps, batch, gen)
    losses = query_loss(model, query, adapters)
    informative = 1.0 - torch.isin(order[:drop], noise).float().mean().item()
    return dict(zip([*subsets, "no adapter"], losses)), informative


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=150)
    ap.add_argument("--seed", type=int, default=0)
    args = ap.parse_args()
    losses, informative = run(steps=args.steps, seed=args.seed)
    print(f"of the quarter valued most, {100 * informative:.0f}% is not noise (half of all data is noise)")
    for name, loss in losses.items():
        print(f"  query loss {loss:.4f}  {name}")


if __name__ == "__main__":
    main()
