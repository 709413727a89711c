"""Valuing preference data, and trying the choice out: which pairs of answers teach a model what its users prefer.

The data are pairs of answers to the same inputs, one chosen and one rejected.  A frozen model (one residual block, a layer
norm and a vocabulary of logits) is valued and then tuned on synthetic pairs:

  1. the projected gradient of every training pair's preference loss is logged, the held-out pairs' gradients are
     preconditioned, and each training pair is scored by its summed influence on the held-out loss;
  2. three subsets are formed: all pairs, all without the most valuable quarter, all without a random quarter;
  3. a model is tuned on each subset, all of them in the same batches: an adapter of the logits' layer and a gain of the
     norm for each, their states kept in 8 bits;
  4. the held-out pairs' loss under each tells whether the pairs named valuable were.

Some of the training pairs are mislabelled (the rejected answer is called the chosen one); the valuation does not know.
Run on an MI355X:

    python examples/preference_subsets.py
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2405_13954_amd as P  # noqa: E402

DEV = "cuda"
BF16 = torch.bfloat16


class Frozen:
    """h = x + relu(x W1), logits = norm(h) W2: the frozen model."""

    def __init__(self, n, vocab, gen):
        self.w1 = (torch.randn(n, n, generator=gen, device=DEV) * n ** -0.5).to(BF16)
        self.w2 = (torch.randn(n, vocab, generator=gen, device=DEV) * n ** -0.5).to(BF16)
        self.w2t = self.w2.t().contiguous()
        self.gain, self.bias = torch.ones(n, dtype=BF16, device=DEV), torch.zeros(n, dtype=BF16, device=DEV)

    def hidden(self, x):
        """(norm(h), h, mean, rstd): what the logits' layer reads, and what the norm's backward pass needs."""
        h, y = torch.empty_like(x), torch.empty_like(x)
        mean, rstd = torch.empty(2, x.shape[0], device=DEV)
        P.logra_layer_norm_forward(x, y, gain=self.gain, bias=self.bias, residual=torch.relu(x @ self.w1), h=h, mean=mean,
                                   rstd=rstd)
        return y, h, mean, rstd


def offsets_of(pairs, tokens):
    """Rows of pairs: the chosen answer's tokens, then the rejected one's."""
    return torch.arange(2 * pairs + 1, device=DEV) * tokens


def make_pairs(model, n, vocab, pairs, tokens, gen, shift):
    """Inputs [pairs * 2 * tokens, n] and targets: the chosen answer is drawn from the model with a shift of its last layer,
    the rejected one from the model as it is."""
    x = torch.randn(pairs, 1, tokens, n, generator=gen, device=DEV).to(BF16).expand(-1, 2, -1, -1).reshape(-1, n)
    y = model.hidden(x)[0].float()
    prefer = torch.softmax(2 * (y @ (model.w2.float() + shift)), 1).view(pairs, 2, tokens, vocab)[:, 0]
    plain = torch.softmax(2 * (y @ model.w2.float()), 1).view(pairs, 2, tokens, vocab)[:, 1]
    draw = lambda p: torch.multinomial(p.reshape(-1, vocab), 1, generator=gen).view(pairs, tokens)  # noqa: E731
    return x, torch.stack([draw(prefer), draw(plain)], 1)


def swapped(target, which):
    """The targets with the two answers of the pairs `which` exchanged."""
    out = target.clone()
    out[which] = target[which].flip(1)
    return out


def pair_losses(z, target, ref=None, dz=None, beta=0.1, weight=None):
    """(losses, log probabilities) of the pairs, and in dz the gradient of the logits."""
    pairs, _, tokens = target.shape
    loss, logp = torch.empty(pairs, device=DEV), torch.empty(2 * pairs, device=DEV)
    P.logra_preference_loss(z, target.reshape(-1), offsets_of(pairs, tokens), logp, loss=loss, dlogits=dz, ref=ref,
                            weight=weight, beta=beta)
    return loss, logp


def value(model, train, query, k, gen):
    """Influence of every training pair on the held-out pairs' loss, summed over these (the projected gradients of the
    logits' layer, Sec. 3.1; damped inverse, Sec. 2; scores, Eq. (2)).  The frozen model is its own reference, so every
    pair starts at a log ratio of zero."""
    n, vocab = model.w2.shape
    p_in = (torch.randn(k, n, generator=gen, device=DEV) * k ** -0.5).to(BF16)
    p_out = (torch.randn(k, vocab, generator=gen, device=DEV) * k ** -0.5).to(BF16)
    rows = []
    for x, target in (train, query):
        pairs, _, tokens = target.shape
        y = model.hidden(x)[0]
        z = y @ model.w2
        ref = pair_losses(z, target)[1]
        dz = torch.empty_like(z)
        pair_losses(z, target, ref, dz)
        g = torch.empty(pairs, k * k, device=DEV)
        P.logra_project_layer(y.view(pairs, 2 * tokens, n), dz.view(pairs, 2 * tokens, vocab), p_in, p_out, g)
        rows.append(g)
    S = torch.zeros(k * k, k * k, device=DEV)
    P.logra_cov_accumulate(rows[0], S)
    pre = torch.empty_like(rows[1])
    P.logra_precondition(S, rows[0].shape[0], 0.1, rows[1], pre)
    scores = torch.empty(rows[1].shape[0], rows[0].shape[0], device=DEV)
    P.logra_influence_scores(pre, rows[0], scores=scores)
    return scores.sum(0)


class Models:
    """One tuned model for each of m subsets: an adapter (a, b) of the logits' layer and a gain of the norm, with the
    optimizer's states in 8 bits.  fp32 parameters, bf16 copies for the products."""

    def __init__(self, model, m, rank, gen, lr=0.002, max_norm=1.0):
        n, vocab = model.w2.shape
        self.model, self.m, self.rank, self.lr, self.max_norm = model, m, rank, lr, max_norm
        self.param = [torch.randn(m, rank, n, generator=gen, device=DEV) * n ** -0.5, torch.zeros(m, rank, vocab, device=DEV),
                      torch.ones(m, n, device=DEV)]
        self.work = [p.to(BF16) for p in self.param]
        self.grad = [torch.empty_like(p) for p in self.param]
        tensors = []
        for i, (p, w, g) in enumerate(zip(self.param, self.work, self.grad)):
            blocks = m * -(-(p.numel() // m) // P.ADAMW_BLOCK)
            tensors.append(P.AdamwTensor(p, g, torch.zeros(p.shape, device=DEV).to(torch.float8_e4m3fn),
                                         torch.zeros(p.shape, device=DEV).to(torch.float8_e5m2), torch.zeros(blocks, device=DEV),
                                         torch.zeros(blocks, device=DEV), work=w, slices=m, decay=i < 2))
        self.optimizer = P.logra_adamw_plan(tensors, m)
        self.step = torch.zeros(1, dtype=torch.int64, device=DEV)
        self.norms = torch.empty(m, device=DEV)
        self.scale = torch.full((m,), 2.0, device=DEV)

    def logits(self, x, keep=None):
        """Logits of the rows of m equal parts, each under its own model; keep: a dict for what the backward pass needs."""
        m, per = self.m, x.shape[0] // self.m
        ids = torch.arange(m, dtype=torch.int32, device=DEV).repeat_interleave(per)
        plan = P.logra_adapter_plan(ids, m)
        h, y = torch.empty_like(x), torch.empty_like(x)
        mean, rstd = torch.empty(2, x.shape[0], device=DEV)
        inner = torch.relu(x @ self.model.w1)
        for s in range(m):
            part = slice(s * per, (s + 1) * per)
            P.logra_layer_norm_forward(x[part], y[part], gain=self.work[2][s], bias=self.model.bias, residual=inner[part],
                                       h=h[part], mean=mean[part], rstd=rstd[part])
        z, u = y @ self.model.w2, torch.empty(x.shape[0], self.rank, device=DEV)
        P.logra_adapter_forward(y, self.work[0], self.work[1], plan, z, base=z, scale=self.scale, u=u)
        if keep is not None:
            keep.update(plan=plan, h=h, y=y, mean=mean, rstd=rstd, u=u)
        return z

    def gradients(self, dz, kept):
        """Fills grad from the logits' gradient."""
        m, per = self.m, dz.shape[0] // self.m
        dy = dz @ self.model.w2t
        P.logra_adapter_backward(kept["y"], dz, self.work[0], self.work[1], kept["plan"], kept["u"], self.grad[0], self.grad[1],
                                 dx=dy, base=dy, scale=self.scale)
        for s in range(m):
            part = slice(s * per, (s + 1) * per)
            P.logra_layer_norm_backward(kept["h"][part], dy[part], kept["rstd"][part], mean=kept["mean"][part],
                                        gain=self.work[2][s], dgain=self.grad[2][s])

    def train_step(self, x, target, ref, beta=0.1):
        """One step of every model on its part of the batch; returns the pairs' losses."""
        kept = {}
        z = self.logits(x, kept)
        pairs = target.shape[0] // self.m
        weight = torch.full((target.shape[0],), 1.0 / pairs, device=DEV)
        loss, _ = pair_losses(z, target, ref, z, beta, weight)
        self.gradients(z, kept)
        P.logra_adamw_step(self.optimizer, self.step, self.lr, beta2=0.95, weight_decay=0.01, max_norm=self.max_norm,
                           norms=self.norms, seed=5)
        return loss * pairs


def run(n=64, vocab=200, pairs=512, tokens=32, queries=128, k=16, rank=4, steps=80, batch=16, seed=0):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    model = Frozen(n, vocab, gen)
    shift = torch.randn(n, 4, generator=gen, device=DEV) @ torch.randn(4, vocab, generator=gen, device=DEV) * (1.5 / n ** 0.5)
    x, target = make_pairs(model, n, vocab, pairs, tokens, gen, shift)
    wrong = torch.randperm(pairs, generator=gen, device=DEV)[:pairs // 3]
    target = swapped(target, wrong)
    query = make_pairs(model, n, vocab, queries, tokens, gen, shift)
    scores = value(model, (x, target), query, k, gen)
    order, quarter = scores.argsort(descending=True), pairs // 4
    shuffled = torch.randperm(pairs, generator=gen, device=DEV)
    subsets = {"all pairs": order, "without the most valuable quarter": order[quarter:],
               "without a random quarter": shuffled[quarter:]}
    ref = pair_losses(model.hidden(x)[0] @ model.w2, target)[1].view(pairs, 2)
    models = Models(model, len(subsets), rank, gen)
    x = x.view(pairs, 2 * tokens, n)
    for _ in range(steps):
        picks = torch.cat([s[torch.randint(len(s), (batch,), generator=gen, device=DEV)] for s in subsets.values()])
        models.train_step(x[picks].view(-1, n), target[picks], ref[picks].view(-1))
    qx, qt = query
    m = len(subsets)
    q_ref = pair_losses(model.hidden(qx)[0] @ model.w2, qt)[1]
    loss, _ = pair_losses(models.logits(qx.repeat(m, 1)), qt.repeat(m, 1, 1), q_ref.repeat(m))
    right = 1.0 - torch.isin(order[:quarter], wrong).float().mean().item()
    return dict(zip(subsets, loss.view(m, -1).mean(1).tolist())), right


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=80)
    ap.add_argument("--seed", type=int, default=0)
    args = ap.parse_args()
    losses, right = run(steps=args.steps, seed=args.seed)
    print(f"of the quarter valued most, {100 * right:.0f}% is labelled right (two thirds of all pairs are)")
    print(f"  held-out loss {0.6931:.4f}  the frozen model")
    for name, loss in losses.items():
        print(f"  held-out loss {loss:.4f}  {name}")


if __name__ == "__main__":
    main()
