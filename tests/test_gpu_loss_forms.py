"""Every form of the token loss (threads, kept vectors, the vectors that go by twice) against the float64 oracle, with
bounds that follow the kernel's sum, so that one lost logit of an ordinary row shows, and rows whose probability sits in
single places, so that a lost vector shows.

Bounds, in units of 2^-24 and with d = max - z >= 0, derived before any run.  A term exp(z - max) carries 2 units of
the hardware exponential, and 2.23 d of its argument: the difference, the constant log2(e) (0.23) and the product each
round relative to d.  The running maximum changes the argument's parts and not their sum, and costs 5 units (exponential,
product) a change.  With v vectors a thread: 8 additions in a vector, v of vectors, 6 of lanes, 16 of waves, and at most
v / 4 + 2 changes of the maximum.  So the relative error of the sum is
    E = 24 + 8 + v + 5 (v / 4 + 3) + 2.23 sum_j p_j d_j
and a loss is within |w| (E + 4 |log(sum)| + |max - z_target|) + 3 |loss|; a gradient element within
|w| p (E + 2.23 d + 5) + |g| and one rounding to bf16 (2^-8 of it).  One per cent covers products of the errors.
"""
import numpy as np
import pytest

from oracle import adapters as O

UNIT = 2.0 ** -24


def _bounds(z, target, weight, want, grad, dtype):
    rows, vocab = z.shape
    per = 8 if dtype == "bf16" else 4
    vec = -(-vocab // per)
    v = max(4, -(-vec // 1024) + 1)
    w = np.ones(rows) if weight is None else np.abs(weight.astype(np.float64))
    top = z.max(1)
    d = top[:, None] - z
    e = np.exp(-d)
    total = e.sum(1)
    p = e / total[:, None]
    E = 24 + 8 + v + 5 * (v / 4 + 3) + 2.23 * (p * d).sum(1)
    zt = z[np.arange(rows), np.clip(target, 0, vocab - 1)]
    loss = 1.01 * UNIT * (w * (E + 4 * np.abs(np.log(total)) + np.abs(top - zt)) + 3 * np.abs(want)) + 1e-37
    bound = 1.01 * UNIT * (w[:, None] * p * (E[:, None] + 2.23 * d + 5) + np.abs(grad)) + 1e-37
    return loss, bound + (2.0 ** -8 * np.abs(grad) if dtype == "bf16" else 0.0)


def _places(vocab, per):
    """Logits at the edges of what a thread keeps, what goes by twice and the last, partial vector, for every width that
    a launch may have."""
    out = {0, per - 1, per, vocab // 2, vocab - 1, vocab // per * per - 1, vocab // per * per}
    for threads in (256, 512, 1024):
        for kept in (4, 12):
            edge = threads * kept * per
            out |= {edge - 1, edge, edge + per, edge - threads * per, edge + threads * per, edge + 4 * threads * per}
    return sorted(k for k in out if 0 <= k < vocab)


def _case(rows, vocab, dtype):
    """Ordinary rows, and for each place a row with nearly all probability there and the target elsewhere."""
    import torch
    per = 8 if dtype == "bf16" else 4
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    places = _places(vocab, per)
    rows = max(rows, len(places) + 6)
    g = np.random.default_rng([rows, vocab])
    z = (g.standard_normal((rows, vocab)) * 2.5).astype(np.float32)
    target = g.integers(0, vocab, rows)
    weight = g.uniform(0.5, 2.0, rows).astype(np.float32)
    for k, at in enumerate(places):
        z[k, at] = 25.0
        target[k] = (at + vocab // 2 + 1) % vocab
    tail = vocab // per * per          # all of the last, partial vector
    z[len(places), tail:] = 22.0
    target[-1] = -100
    weight[len(places) + 1] = 0.0
    z = torch.from_numpy(z).to(dt)
    return z, z.double().numpy(), target, weight


def _run(z, target, weight, inplace, pad):
    import torch
    import paper_2405_13954_amd as P
    rows, vocab = z.shape
    width = -(-vocab // 8) * 8
    buf = torch.full((rows, width + pad), 7.0, dtype=z.dtype, device="cuda")
    zz = buf[:, :vocab]
    zz.copy_(z)
    out = buf if inplace else torch.full((rows, width), 7.0, dtype=z.dtype, device="cuda")
    loss = torch.empty(rows, device="cuda")
    P.logra_token_loss(zz, target, loss, dlogits=out[:, :vocab], weight=weight)
    assert bool((out[:, vocab:] == 7.0).all()), "a store outside the rows"
    if not inplace:
        assert torch.equal(zz, z.cuda()), "the logits changed"
    return loss, out[:, :vocab]


SIZES = [("bf16", 6, v) for v in (9, 1021, 8191, 8193, 16391, 32763, 32775, 98301, 98311, 131079)] + \
        [("f32", 6, v) for v in (5, 1001, 4099, 8195, 16385, 49157, 65537)] + \
        [("bf16", 300, 33001), ("bf16", 300, 40963), ("bf16", 270, 100003), ("f32", 300, 16389), ("f32", 270, 50001)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,rows,vocab", SIZES)
def test_loss_of_every_form(dtype, rows, vocab):
    import torch
    z, z64, target, weight = _case(rows, vocab, dtype)
    rows = len(target)
    print("[loss]", dtype, rows, vocab, flush=True)
    t, w = torch.from_numpy(target).cuda(), torch.from_numpy(weight).cuda()
    want, grad = O.token_loss(z64, target, weight.astype(np.float64))
    lb, gb = _bounds(z64, target, weight, want, grad, dtype)

    def check(loss, d, part, what):
        err = np.abs(loss.double().cpu().numpy() - want[part]) - lb[part]
        assert (err <= 0).all(), f"{what}: loss {err.max():.3e} beyond the bound in row {err.argmax()}"
        err = np.abs(d.double().cpu().numpy() - grad[part]) - gb[part]
        assert (err <= 0).all(), f"{what}: gradient {err.max():.3e} beyond the bound at {np.unravel_index(err.argmax(), err.shape)}"

    first = _run(z, t, w, False, 0)
    check(*first, slice(None), "apart")
    again = _run(z, t, w, True, 16)
    assert all(torch.equal(p, q) for p, q in zip(first, again)), "in place differs"
    # the same tokens a few at a time (up to 256 of them may take another form)
    for at in range(0, rows, 200):
        part = slice(at, min(at + 200, rows))
        check(*_run(z[part], t[part].contiguous(), w[part].contiguous(), at == 0, 8), part, f"rows from {at}")


def test_bounds_notice_lost_vectors():
    # the oracle without one vector of logits, at the edges of every form, is beyond the bound in some row; in an ordinary
    # row it is at 8,193 logits, where the last vector has a single one
    for dtype, vocab in (("bf16", 8193), ("bf16", 131079), ("f32", 65537)):
        z, z64, target, weight = _case(6, vocab, dtype)
        want, grad = O.token_loss(z64, target, weight.astype(np.float64))
        bound, _ = _bounds(z64, target, weight, want, grad, dtype)
        per = 8 if dtype == "bf16" else 4
        places = _places(vocab, per)
        for at in places:
            rows = np.r_[0:len(places), len(target) - 2]
            cut, t = z64[rows].copy(), target[rows]
            lost = slice(at // per * per, at // per * per + per)
            cut[:, lost] = np.where(np.arange(vocab)[None, lost] == t[:, None], cut[:, lost], -np.inf)
            other, _ = O.token_loss(cut, t, weight[rows].astype(np.float64))
            assert (np.abs(other - want[rows]) > bound[rows]).any(), (dtype, vocab, at)
            if vocab == 8193:
                assert np.abs(other - want[rows])[-1] > bound[rows][-1]


@pytest.mark.gpu
def test_far_rows():
    # 40 rows at a stride of 2^27 elements: byte offsets to 2^33 and beyond, of logits and gradient
    import torch
    import paper_2405_13954_amd as P
    for dt, elements in ((torch.bfloat16, 40 << 27), (torch.float32, 20 << 27)):
        wide = torch.empty(elements, dtype=dt, device="cuda").view(40, -1)
        g = torch.Generator().manual_seed(1)
        z = torch.randn(40, 1001, generator=g).to(dt)
        near = torch.empty(40, 1008, dtype=dt, device="cuda")
        near[:, :1001] = z.cuda()
        t = torch.randint(0, 1001, (40,), generator=g).cuda()
        want, got = torch.empty(40, device="cuda"), torch.empty(40, device="cuda")
        d = torch.empty_like(near)
        P.logra_token_loss(near[:, :1001], t, want, dlogits=d[:, :1001])
        far = wide[:, 8:1009]
        far.copy_(near[:, :1001])
        P.logra_token_loss(far, t, got, dlogits=wide[:, 2048:3049])
        assert torch.equal(got, want) and torch.equal(wide[:, 2048:3049], d[:, :1001])
        P.logra_token_loss(far, t, got, dlogits=far)
        assert torch.equal(got, want) and torch.equal(far, d[:, :1001])
        del wide, far
