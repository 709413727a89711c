"""Norm, adapters, preference loss and optimizer together, as a tuning step uses them: the gradients against float64, a
captured step against eager ones, and the example."""
import importlib.util
import os

import numpy as np
import pytest

from oracle import adapters as OA
from oracle import tuning as O
from tuning_util import U, host, within

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("preference_subsets", os.path.join(ROOT, "examples", "preference_subsets.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _small(seed=1, m=3, pairs=2, tokens=5, n=64, vocab=104, rank=4):
    import torch
    ex = _example()
    gen = torch.Generator(device="cuda").manual_seed(seed)
    model = ex.Frozen(n, vocab, gen)
    models = ex.Models(model, m, rank, gen)
    models.param[1].normal_(generator=gen).mul_(0.1)
    models.param[2].normal_(1.0, 0.1, generator=gen)
    for p, w in zip(models.param, models.work):
        w.copy_(p)
    x = torch.randn(m * pairs * 2 * tokens, n, generator=gen, device="cuda").to(torch.bfloat16)
    target = torch.randint(vocab, (m * pairs, 2, tokens), generator=gen, device="cuda")
    ref = torch.randn(2 * m * pairs, generator=gen, device="cuda") * 3
    return ex, models, x, target, ref


def test_gradients_of_a_step_against_float64():
    """Every operator's gradient by the oracle's, fed with the values that the step computed in front of it; the bf16 roundings
    of these are their own.  Bounds: the tests of each operator hold them at their own tolerances, here 2^-8 for the one
    bf16 rounding of dz and dy (which the next operator reads), and 2^-12 of a sum's terms for everything in fp32."""
    import torch
    ex, models, x, target, ref = _small()
    kept = {}
    z = models.logits(x, kept)
    dz = torch.empty_like(z)
    loss, logp = ex.pair_losses(z, target, ref, dz)
    offsets = host(ex.offsets_of(target.shape[0], target.shape[2])).astype(int)
    t = target.reshape(-1).cpu().numpy()
    want_loss, want_logp, want_dz = O.preference_loss(host(z), t, offsets, host(ref), None, 0.1)
    within(host(loss), want_loss, 2.0 ** -16 * (1 + np.abs(want_loss)), "loss")
    within(host(logp), want_logp, 2.0 ** -16 * (1 + np.abs(want_logp)), "logp")
    within(host(dz), want_dz, 2.0 ** -8 * np.abs(want_dz) + 2.0 ** -14, "dz")
    models.gradients(dz, kept)
    a, b = host(models.work[0]), host(models.work[1])
    m, per = models.m, x.shape[0] // models.m
    ids = np.repeat(np.arange(m), per)
    u = OA.adapter_forward(host(kept["y"]), a, b, ids, scale=np.full(m, 2.0))[1]
    within(host(kept["u"]), u, 2.0 ** -12 * (1 + np.abs(u)), "u")
    base = (dz @ models.model.w2t)                                       # as the step computed it
    dzn = host(dz)
    for s in range(m):
        rows = slice(s * per, (s + 1) * per)
        du = 2.0 * dzn[rows] @ b[s].T
        dn = np.abs(dzn[rows])
        within(host(models.grad[0][s]), du.T @ host(kept["y"])[rows], 2.0 ** -12 * np.abs(du).T @ np.abs(host(kept["y"])[rows]) + 1e-6, "da")
        within(host(models.grad[1][s]), 2.0 * u[rows].T @ dzn[rows], 2.0 ** -12 * 2 * np.abs(u[rows]).T @ dn + 1e-6, "db")
        dy = host(base)[rows] + du @ a[s]
        xh = (host(kept["h"])[rows] - host(kept["mean"])[rows, None]) * host(kept["rstd"])[rows, None]
        bound = np.sum(np.abs(xh) * (2.0 ** -8 * np.abs(dy) + 2.0 ** -12 * (np.abs(host(base)[rows]) + np.abs(du) @ np.abs(a[s]))), 0)
        within(host(models.grad[2][s]), np.sum(dy * xh, 0), bound + 1e-6, "dgain")


def test_gradients_of_a_step_against_differences():
    """(loss(w + h) - loss(w - h)) against grad . (w+ - w-), w+ and w- being the bf16 copies as they are after rounding.  The
    losses' own errors: a logit is off by 2^-8 of itself (one rounding) and by what y's rounding does to it, 2^-8 of |y| |w2|
    at most, which moves the loss by |dz| as much; random signs make the sum over N terms a root of N smaller, of which this
    takes six, for both losses.  What curvature leaves of a central difference is a third of h^2, h = 2^-4 of the weights."""
    import torch
    ex, models, x, target, ref = _small(seed=2, pairs=4)
    kept = {}
    z = models.logits(x, kept)
    dz = torch.empty_like(z)
    ex.pair_losses(z, target, ref, dz)
    y = kept["y"]
    models.gradients(dz.clone(), kept)
    loose = dz.double().abs() * (z.double().abs() + (y.double().abs() @ models.model.w2.double().abs())) * 2.0 ** -8
    noise = 2 * 6 * float(loose.square().sum().sqrt())
    start = [p.clone() for p in models.param]
    h = 2.0 ** -4 * float(sum(w.double().square().sum() for w in models.work).sqrt())
    length = float(sum(g.double().square().sum() for g in models.grad).sqrt())
    ends, losses = [], []
    for sign in (1, -1):
        for p, s, g, w in zip(models.param, start, models.grad, models.work):
            p.copy_(s + sign * h / length * g)
            w.copy_(p)
        ends.append([w.double() for w in models.work])
        losses.append(float(ex.pair_losses(models.logits(x), target, ref)[0].double().sum()))
    want = float(sum((g.double() * (a - b)).sum() for g, a, b in zip(models.grad, *ends)))
    assert want > 10 * noise, (want, noise)
    assert abs(losses[0] - losses[1] - want) <= noise + want / 16, (losses[0] - losses[1], want, noise)


def test_a_captured_step_is_the_eager_one():
    import torch
    outs = []
    for captured in (False, True):
        ex, models, x, target, ref = _small(seed=3)
        losses = torch.empty(5, target.shape[0], device="cuda")
        here = torch.empty(target.shape[0], device="cuda")

        def step():
            here.copy_(models.train_step(x, target, ref))

        if captured:
            state = [t.clone() for t in (*models.param, *models.work, models.step)]
            moments = [(t.m.clone(), t.v.clone(), t.m_scale.clone(), t.v_scale.clone()) for t in models.optimizer.tensors]
            step()                                            # library handles and memory before the capture
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
            for t, s in zip((*models.param, *models.work, models.step), state):
                t.copy_(s)
            for t, old in zip(models.optimizer.tensors, moments):
                for dst, src in zip((t.m, t.v, t.m_scale, t.v_scale), old):
                    dst.view(torch.uint8).copy_(src.view(torch.uint8)) if dst.element_size() == 1 else dst.copy_(src)
        for k in range(5):
            graph.replay() if captured else step()
            torch.cuda.synchronize()
            losses[k] = here
            x.mul_(0.97)
        assert int(models.step) == 5
        outs.append([losses, *models.param, *models.work, *models.grad, models.norms]
                    + [t for d in models.optimizer.tensors for t in (d.m.view(torch.uint8), d.v.view(torch.uint8), d.m_scale, d.v_scale)])
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_eight_bit_states_train_like_fp32_ones():
    """The same adapters for 60 steps with states of either kind: the 8-bit ones' losses are finite and the parameters moved
    about as far (between half and twice the distance)."""
    import torch
    import paper_2405_13954_amd as P
    moved = []
    for eight in (True, False):
        ex, models, x, target, ref = _small(seed=4)
        if not eight:
            tensors = [P.AdamwTensor(t.param, t.grad, torch.zeros_like(t.param), torch.zeros_like(t.param), work=t.work,
                                     slices=t.slices, decay=t.decay) for t in models.optimizer.tensors]
            models.optimizer = P.logra_adamw_plan(tensors, models.m)
        start = [p.clone() for p in models.param]
        for _ in range(60):
            loss = models.train_step(x, target, ref)
        assert bool(torch.isfinite(loss).all())
        moved.append([float((p - s).norm()) for p, s in zip(models.param, start)])
    for a, b in zip(*moved):
        assert 0.5 < a / b < 2.0, moved


def test_the_example_runs():
    import torch
    ex = _example()
    losses, right = ex.run(n=64, vocab=200, pairs=24, tokens=6, queries=8, k=8, rank=4, steps=6, batch=4)
    assert len(losses) == 3 and all(np.isfinite(v) and v > 0 for v in losses.values()) and 0.0 <= right <= 1.0
    torch.cuda.synchronize()
