"""Every logit's part in the preference loss: rows whose sums of exponentials are known whole numbers, rows whose probability
sits in single places, and the gradient against differences of the loss.

Equal logits.  Row 2b has z = 0 where bit b of the token's number is set and -inf elsewhere, row 2b + 1 the opposite, each a
sequence of one token.  exp(0) is 1 and a whole number below 2^24 is exact in fp32 in whatever order it is counted, so lp is
-log(count) but for the logarithm's last bits (4 U |lp|, U = 2^-24) and its rounding (U |lp|).  A logit that is lost or counted
twice is off by 1 / count at least, and no two logits are in the same rows, so that one cannot stand in for another.

Ordinary logits.  In units of U, with d = max - z: a term exp(z - max) carries 2 of the hardware exponential and 2.23 d of its
argument (the difference, the constant log2(e), the product).  With v <= 17 vectors a thread: 8 additions in a vector, v of
vectors, 6 of lanes, 4 of waves, 16 of a row's ranges; a change of the maximum costs 5 (exponential, product), of which there are v / 4 + 2
in a thread, one in the workgroup and one between ranges.  So the relative error of the sum is
    E = 36 + v + 5 (v / 4 + 4) + 2.23 sum_j p_j d_j
and lp of a token is within E + 4 |log(sum)| + |max - z_target|, and its rounding.
"""
import numpy as np
import pytest

from oracle import tuning as O
from tuning_util import HALF, U, dt, f32, guarded, host, room, within

V = 17


def members(vocab):
    """[2 bits, vocab]: the tokens whose number has bit b, then those that have it not, for each bit in turn."""
    bits = (np.arange(vocab) >> np.arange((vocab - 1).bit_length())[:, None]) & 1
    return np.stack([bits == 1, bits == 0], 1).reshape(-1, vocab)


def flat_bound(count):
    return 5 * U * np.log(count)


FLAT = [("bf16", v) for v in (2, 9, 1000, 8192, 8193, 16385, 32769, 65544, 131079)] + \
       [("f32", v) for v in (3, 1001, 4096, 4097, 16385, 32769, 40001, 65537)]


# many: rows enough that a row is one range, or few
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,vocab,many", [(d, v, 1) for d, v in FLAT] +
                         [("bf16", 8193, 80), ("bf16", 32769, 66), ("bf16", 131079, 20), ("f32", 16385, 75), ("f32", 40001, 20)])
def test_equal_logits_are_counted(dtype, vocab, many):
    import torch
    import paper_2405_13954_amd as P
    print("[equal logits]", dtype, vocab, many, flush=True)
    of = members(vocab)
    few = len(of)
    rows, n = few * many, few * many // 2
    one = torch.from_numpy(np.where(of, 0.0, -np.inf)).to(dt(dtype)).cuda()
    z, _ = room(rows, vocab, dtype)
    d, full = room(rows, vocab, dtype, 8)
    for part in z.split(few):
        part.copy_(one)
    count = of.sum(1)
    target = np.where(np.arange(few) % 2 == 0, 1 << (np.arange(few) // 2), 0)           # the first of each row's tokens
    t, o = torch.from_numpy(np.tile(target, many)).cuda(), torch.arange(rows + 1).cuda()
    loss, logp = f32(n), f32(2 * n)
    P.logra_preference_loss(z, t, o, logp, loss=loss, dlogits=d, beta=0.5, smoothing=0.1)
    lp, bound = -np.log(count), flat_bound(count)
    within(host(logp).reshape(many, few), lp[None], bound[None], "logp")
    dif = 0.5 * (lp[0::2] - lp[1::2])
    want = 0.9 * O.softplus(-dif) + 0.1 * O.softplus(dif)
    ed = 0.5 * (bound[0::2] + bound[1::2])
    within(host(loss).reshape(many, -1), want[None], (ed + 2 * U * want)[None], "loss")
    slope = np.repeat(0.5 * (0.1 - 1 / (1 + np.exp(dif))), 2) * np.where(np.arange(few) % 2 == 0, 1, -1)
    hot = torch.zeros(few, vocab, dtype=torch.float64, device="cuda")
    hot[torch.arange(few), torch.from_numpy(target).cuda()] = 1.0
    p = torch.from_numpy(of / count[:, None]).cuda()
    col = lambda a: torch.from_numpy(a).cuda()[:, None]  # noqa: E731
    exact = col(slope) * (hot - p)
    # the slope's own error, its rounding, the quotient's and the product's, and one of the type
    most = col(0.5 / 4 * np.repeat(ed, 2) + 4 * U * np.abs(slope)) * (hot + p) + (HALF[dtype] + U) * exact.abs()
    for part in d.split(few):
        assert bool(((part.double() - exact).abs() <= most).all()), (part.double() - exact).abs().sub(most).max()
    guarded(full, rows, vocab)


def test_the_counts_notice_one_logit():
    # one logit lost, one counted twice, or one in the place of another: beyond the bound in some row
    for _, vocab in FLAT:
        of = members(vocab)
        count = of.sum(1)
        spots = sorted({0, 1, vocab // 2, vocab - 1, vocab - 2} | {k for k in range(0, vocab, 1021)})
        for at in spots:
            for change in (-1, 1):
                other = count + change * of[:, at]
                some = other > 0
                assert (np.abs(np.log(other[some]) - np.log(count[some])) > flat_bound(count[some])).any() or not some.all(), (vocab, at)
        for a, b in zip(spots, spots[1:]):
            other = count - of[:, a] + of[:, b]
            some = other > 0
            assert (np.abs(np.log(other[some]) - np.log(count[some])) > flat_bound(count[some])).any() or not some.all(), (vocab, a, b)


def _places(vocab, per):
    """Tokens at the edges of vectors, of a thread's rounds, of the ranges that a row may be cut into and of the partial vector."""
    whole = vocab // per
    out = {0, per - 1, per, vocab // 2, vocab - 1, whole * per - 1, whole * per}
    for k in (256, 768, 1024, 4096):
        out |= {k * per - 1, k * per, (k + 1) * per}
    for ranges in (2, 3, 5, 16):
        each = -(-whole // ranges) * per
        out |= {each - 1, each, (ranges - 1) * each}
    return sorted(k for k in out if 0 <= k < vocab)


def _bounds(z, target):
    """(log probability, its bound in fp32, probabilities) of every row."""
    top = z.max(1)
    d = top[:, None] - z
    e = np.exp(-d)
    total = e.sum(1)
    p = e / total[:, None]
    E = 36 + V + 5 * (V / 4 + 4) + 2.23 * (p * d).sum(1)
    zt = z[np.arange(len(z)), target]
    lp = zt - top - np.log(total)
    return lp, 1.01 * U * (E + 4 * np.log(total) + top - zt), p, d


def _case(vocab, dtype):
    import torch
    per = 8 if dtype == "bf16" else 4
    places = _places(vocab, per)
    rows = len(places) + 4 + len(places) % 2
    g = np.random.default_rng(vocab)
    z = (g.standard_normal((rows, vocab)) * 2.5).astype(np.float32)
    target = g.integers(0, vocab, rows)
    for k, at in enumerate(places):                # nearly all probability in one place, below and above what comes before it
        z[k, at] = 25.0
        target[k] = (at + vocab // 2 + 1) % vocab
    z[len(places), vocab // per * per:] = 22.0     # all of the last, partial vector
    z[len(places) + 1] = np.linspace(-20, 20, vocab)   # a maximum that grows all the way, and one that shrinks
    z[len(places) + 2] = np.linspace(20, -20, vocab)
    z = torch.from_numpy(z).to(dt(dtype))
    return z, z.double().numpy(), target


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,vocab,many", [(d, v, 1) for d, v in FLAT if v > 8] +
                         [("bf16", 32769, 60), ("bf16", 131079, 12), ("f32", 16385, 60), ("f32", 65537, 12)])
def test_probability_in_single_places(dtype, vocab, many):
    import torch
    import paper_2405_13954_amd as P
    print("[single places]", dtype, vocab, many, flush=True)
    one, z64, target = _case(vocab, dtype)
    few = len(target)
    rows, n = few * many, few * many // 2
    z, _ = room(rows, vocab, dtype)
    for part in z.split(few):
        part.copy_(one)
    t, o = torch.from_numpy(np.tile(target, many)).cuda(), torch.arange(rows + 1).cuda()
    lp, bound, p, far = _bounds(z64, target)
    ref = (lp + np.random.default_rng(1).standard_normal(few)).astype(np.float32)     # ratios near one, where the slope is not 0
    d, full = room(rows, vocab, dtype, 8)
    loss, logp = f32(n), f32(2 * n)
    P.logra_preference_loss(z, t, o, logp, loss=loss, dlogits=d, ref=torch.from_numpy(np.tile(ref, many)).cuda(), beta=0.5)
    within(host(logp).reshape(many, few), lp[None], (bound + U * np.abs(lp))[None], "logp")
    ratio = lp - ref.astype(np.float64)
    dif, ed = 0.5 * (ratio[0::2] - ratio[1::2]), 0.5 * (bound[0::2] + bound[1::2])
    want = O.softplus(-dif)
    within(host(loss).reshape(many, -1), want[None], (ed + 2 * U * want)[None], "loss")
    slope = np.repeat(-0.5 / (1 + np.exp(dif)), 2) * np.where(np.arange(few) % 2 == 0, 1, -1)
    hot = np.zeros_like(p)
    hot[np.arange(few), target] = 1.0
    exact = slope[:, None] * (hot - p)
    E = 36 + V + 5 * (V / 4 + 4) + 2.23 * (p * far).sum(1)
    most = (0.5 / 4 * np.repeat(ed, 2) + U * np.abs(slope))[:, None] * (hot + p)
    most += 1.01 * U * np.abs(slope)[:, None] * p * (E[:, None] + 2.23 * far + 5) + (HALF[dtype] + U) * np.abs(exact) + 1e-37
    exact, most = torch.from_numpy(exact).cuda(), torch.from_numpy(most).cuda()
    for part in d.split(few):
        assert bool(((part.double() - exact).abs() <= most).all()), (part.double() - exact).abs().sub(most).max()
    guarded(full, rows, vocab)


def test_single_places_notice_a_lost_vector():
    for dtype, vocab in (("bf16", 8193), ("bf16", 131079), ("f32", 40001)):
        per = 8 if dtype == "bf16" else 4
        _, z64, target = _case(vocab, dtype)
        lp, bound, _, _ = _bounds(z64, target)
        for at in _places(vocab, per):
            cut = z64.copy()
            lost = np.arange(at // per * per, min(vocab, at // per * per + per))
            cut[:, lost] = np.where(lost[None] == target[:, None], cut[:, lost], -1e4)
            other = _bounds(cut, target)[0]
            assert (np.abs(other - lp) > bound + U * np.abs(lp)).any(), (dtype, vocab, at)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,smoothing", [(24, 0.1), (24, 0.0), (600, 0.1)])   # (600 rows of two pairs: three launches)
def test_gradient_against_differences_along_it(rows, smoothing):
    """(loss(z + h e) - loss(z - h e)) / 2h against |dz|, e = dz / |dz| for each pair, fp32, beta 1.

    What is left of a central difference is h^2 / 6 times the third derivative along e.  For d = lp_c - lp_r of n tokens the
    first is at most sqrt(2 n) (onehot - p has a norm of sqrt(2) at most), the second 1 and the third 2 (cumulants of numbers
    whose squares add up to 1); the loss' third is sigma'' d'^3 + 3 sigma' d' d'' + sigma d''', with factors below 0.1, 1/4 and 1.
    lp of each token is within the bound above, and the rounding of z + h e moves it by U |z + h e| of the target and as much
    of the others' mean; the loss has a rounding of its own."""
    import torch
    import paper_2405_13954_amd as P
    g = torch.Generator().manual_seed(5)
    vocab = 256
    z, t = torch.randn(rows, vocab, generator=g).cuda(), torch.randint(0, vocab, (rows,), generator=g).cuda()
    cuts = [0, 5, 12, 20, 24] if rows == 24 else [0, 10, 24, rows - 12, rows]
    t[24:cuts[3]] = -1                                      # (long, but most of it does not count)
    o = torch.tensor(cuts).cuda()
    loss, logp, d, h = f32(2), f32(4), torch.empty_like(z), 2.0 ** -5
    kw = dict(beta=1.0, smoothing=smoothing)
    P.logra_preference_loss(z, t, o, logp, **kw)
    kw["ref"] = (logp + torch.tensor([0.25, -0.5, 0.5, 0.25]).cuda()).contiguous()     # ratios near one, where the slope is not 0
    P.logra_preference_loss(z, t, o, logp, loss=loss, dlogits=d, **kw)
    parts = (slice(0, cuts[2]), slice(cuts[2], cuts[4]))
    norm = torch.stack([d[p].double().norm() for p in parts])
    assert cuts[4] == rows and not d[t < 0].any()
    e = torch.cat([(d[p].double() / n).float() for p, n in zip(parts, norm)])
    ends = []
    for s in (h, -h):
        out = f32(2)
        P.logra_preference_loss(z + s * e, t, o, logp, loss=out, **kw)
        ends.append(out.double())
    diff, want = (ends[0] - ends[1]) / (2 * h), torch.stack([(d[p].double() * e[p].double()).sum() for p in parts])
    z64, live = host(z), host(t) >= 0
    _, bound, prob, _ = _bounds(z64[live], host(t)[live].astype(int))
    zt = np.abs(z64[live][np.arange(live.sum()), host(t)[live].astype(int)])
    each = bound + 2 * U * ((prob * (np.abs(z64[live]) + h)).sum(1) + zt + h)
    for i, p in enumerate(parts):
        mine = np.zeros(rows, dtype=bool)
        mine[p] = True
        noise = each[mine[live]].sum() + 2 * U * float(loss[i])
        n = mine[live].sum()
        bound_i = noise / h + h * h / 6 * (0.1 * (2 * n) ** 1.5 + 0.75 * (2 * n) ** 0.5 + 2)
        assert float(want[i]) > 10 * bound_i, (float(want[i]), bound_i)
        assert abs(float(diff[i] - want[i])) <= bound_i, (float(diff[i]), float(want[i]), bound_i)
