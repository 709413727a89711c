"""The preference loss against the float64 oracle.

Tolerances: a token's log probability is within T = 2^-20 + vocab 2^-24 of 1 + |lp| (the exponential's and logarithm's few
2^-23, at most vocab additions); a sequence's sum within the sum of those, and one rounding to fp32.  So d is within beta
times both sequences' bounds; the loss, whose slope in d is w at most, within w times that and a few roundings; a gradient
element within T of its terms, w beta / 4 times d's bound of onehot + p (the sigmoid's slope is 1/4 at most), and its rounding.
"""
import numpy as np
import pytest

from oracle import tuning as O
from tuning_util import HALF, U, dt, f32, guarded, host, mk, room, within

pytestmark = pytest.mark.gpu


def check(z, z64, target, offsets, dtype, ref=None, weight=None, beta=0.1, smoothing=0.0, inplace=False, note=""):
    import torch
    import paper_2405_13954_amd as P
    rows, vocab = z64.shape
    n = len(offsets) // 2
    print("[pairs]", rows, vocab, n, dtype, note, flush=True)
    as64 = lambda a: None if a is None else a.astype(np.float64)  # noqa: E731
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    with np.errstate(over="ignore", invalid="ignore"):
        want, want_lp, want_g = O.preference_loss(z64, target, offsets, as64(ref), as64(weight), beta, smoothing)
    t, o, r, w = dev(target), dev(np.asarray(offsets, dtype=np.int64)), dev(ref), dev(weight)
    kw = dict(ref=r, weight=w, beta=beta, smoothing=smoothing)
    loss, logp, only = f32(n), f32(2 * n), f32(2 * n)
    P.logra_preference_loss(z, t, o, only, **kw)
    d, full = (z, None) if inplace else room(rows, vocab, dtype, 8)
    P.logra_preference_loss(z, t, o, logp, loss=loss, dlogits=d, **kw)
    assert torch.equal(only, logp) or bool(torch.isnan(logp).any())
    tol = 2.0 ** -20 + vocab * 2.0 ** -24
    lp_bound, p = np.zeros(2 * n), np.zeros((rows, vocab))
    pair_of, live = np.full(rows, -1), np.zeros(rows, dtype=bool)
    for s in range(2 * n):
        for i in range(offsets[s], offsets[s + 1]):
            if 0 <= target[i] < vocab:
                with np.errstate(over="ignore", invalid="ignore"):
                    lp, prob = O.token_logp(z64[i], target[i])
                if np.isfinite(lp):
                    lp_bound[s] += tol * (1 + abs(lp))
                pair_of[i], live[i] = s // 2, True
                if prob is not None:
                    p[i] = prob
    lp_bound += U * np.abs(np.where(np.isfinite(want_lp), want_lp, 0))
    same = lambda a, b: np.array_equal(np.isnan(a), np.isnan(b)) and np.array_equal(a[np.isinf(b)], b[np.isinf(b)])  # noqa: E731
    got_lp, got = host(logp), host(loss)
    assert same(got_lp, want_lp) and same(got, want)
    fin = np.isfinite(want_lp)
    within(got_lp[fin], want_lp[fin], lp_bound[fin], "logp")
    size = np.ones(n) if weight is None else np.abs(weight.astype(np.float64))
    ed = abs(beta) * (lp_bound[0::2] + lp_bound[1::2])
    fin = np.isfinite(want)
    within(got[fin], want[fin], (size * ed + 4 * U * np.abs(want))[fin] + 1e-38, "loss")
    got_g = host(d)
    assert np.array_equal(np.isnan(got_g), np.isnan(want_g))
    pair = np.maximum(pair_of, 0)
    hot = np.zeros_like(p)
    hot[np.nonzero(live)[0], target[live]] = 1.0
    slope = np.zeros(rows)
    slope[live] = (size * abs(beta))[pair[live]]
    bound = (slope * ed[pair] / 4)[:, None] * (hot + p) + 2 * tol * slope[:, None] * (hot + p) + (HALF[dtype] + U) * np.abs(want_g) + 1e-37
    ok = ~np.isnan(want_g)
    within(np.where(ok, got_g, 0), np.where(ok, want_g, 0), np.where(ok, bound, 0), "gradient")
    assert np.all(got_g[~live] == 0)
    if full is not None:
        guarded(full, rows, vocab)
    return d


def ragged(g, rows, n, gap=0):
    """Offsets of 2 n sequences within the rows, some of them empty, `gap` rows before the first and behind the last."""
    return np.concatenate([[gap], np.sort(g.integers(gap, rows - gap + 1, 2 * n - 1)), [rows - gap]]).astype(np.int64)


# on either side of the vectors', the pieces' and the ranges' limits
@pytest.mark.parametrize("dtype,vocab", [("bf16", v) for v in (1, 5, 8, 1000, 8192, 8193, 32768, 32769, 65544, 131079)] +
                         [("f32", v) for v in (1, 3, 4, 1001, 4096, 4097, 16384, 16385, 40001)])
def test_vocabularies(dtype, vocab):
    g = np.random.default_rng(vocab)
    rows = 12
    z, z64, _ = mk(g, rows, vocab, 3.0, dtype)
    target = g.integers(0, vocab, rows)
    target[1], target[4], target[2] = -100, vocab, vocab - 1
    offsets = np.array([1, 4, 4, 7, 11], dtype=np.int64)
    ref = g.standard_normal(4).astype(np.float32) * 5
    check(z, z64, target, offsets, dtype, ref=ref)
    weight = np.array([-1.5, 0.25], dtype=np.float32)
    check(z, z64, target, offsets, dtype, ref=ref, weight=weight, beta=0.7, smoothing=0.15, inplace=True)


@pytest.mark.parametrize("rows,n,vocab", [(2, 1, 300), (3, 1, 77), (300, 1, 500), (700, 40, 260), (1030, 3, 129)])
def test_rows_and_pairs(rows, n, vocab):
    g = np.random.default_rng(rows)
    for dtype in ("bf16", "f32"):
        z, z64, _ = mk(g, rows, vocab, 2.0, dtype, 8)
        target = np.where(g.random(rows) < 0.2, -1, g.integers(0, vocab, rows))
        offsets = ragged(g, rows, n, min(2, rows // 2 - 1))
        ref = np.array([-np.log(vocab) * (b - a) for a, b in zip(offsets, offsets[1:])], dtype=np.float32)
        check(z, z64, target, offsets, dtype, ref=ref, weight=g.uniform(0.5, 2, n).astype(np.float32), beta=0.05, smoothing=0.3)


# on either side of the limits of the form for few rows: pairs, rows a pair, the gradient's workgroups (1,536 rows in one
# piece each, 40 rows in 39)
@pytest.mark.parametrize("rows,n,vocab", [(1, 1, 9), (40, 127, 300), (40, 128, 300), (256, 2, 130), (257, 2, 130),
                                          (1536, 20, 520), (1537, 20, 520), (39, 3, 159700), (40, 3, 159700)])
def test_few_rows_and_more(rows, n, vocab):
    g = np.random.default_rng([rows, n])
    z, z64, _ = mk(g, rows, vocab, 2.0, "bf16", 8)
    target = np.where(g.random(rows) < 0.3, vocab, g.integers(0, vocab, rows))
    ref = (g.standard_normal(2 * n) * 3).astype(np.float32)
    weight = np.where(g.random(n) < 0.2, 0.0, g.uniform(0.5, 2, n)).astype(np.float32)
    check(z, z64, target, ragged(g, rows, n, min(1, rows // 3)), "bf16", ref=ref, weight=weight, smoothing=0.1)
    if vocab < 1000:   # all rows in one sequence, the others empty; then in place of the logits
        for s in (0, 2 * n - 1):
            check(z, z64, target, [0] * (s + 1) + [rows] * (2 * n - s), "bf16", ref=ref, inplace=s > 0)


@pytest.mark.parametrize("smoothing", [0.0, 1.0])
def test_far_ratios(smoothing):
    # d of thousands: the loss is linear on one side and zero on the other, with no overflow
    g = np.random.default_rng(8)
    z, z64, _ = mk(g, 8, 100, 1.0, "f32")
    target = g.integers(0, 100, 8)
    for far in (3e4, -3e4, 1e30):
        check(z, z64, target, [0, 3, 5, 6, 8], "f32", ref=np.array([far, 0, 0, far], dtype=np.float32), smoothing=smoothing)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [100, 40000])
def test_forbidden_and_extreme_logits(vocab, dtype):
    import torch
    g = np.random.default_rng(vocab)
    z, z64, _ = mk(g, 10, vocab, 2.0, dtype)
    target = g.integers(0, vocab, 10)
    low = float(torch.finfo(dt(dtype)).min)
    z64[0, g.random(vocab) < 0.9] = -np.inf       # forbidden tokens, but not the target
    z64[0, target[0]] = 1.0
    z64[2, :] = low                               # masked by the lowest value: uniform
    z64[3, :] = low
    z64[3, target[3]] = 0.0                       # and all but the target
    z64[4, :] = -np.inf
    z64[4, target[4]] = 3.0
    z64[5] += 60.0 if dtype == "bf16" else 1000.0
    z64[6, :] = -np.inf                           # nothing is possible: the rejected sequence has probability zero
    z64[8, target[8]] = -np.inf                   # the chosen target is forbidden
    zt = torch.from_numpy(z64).to(dt(dtype))
    z.copy_(zt)
    #                                  pair 0    pair 1 (rejected: -inf)   pair 2 (chosen: -inf)
    check(z, zt.double().numpy(), target, [0, 3, 5, 6, 8, 9, 10], dtype)
    check(z, zt.double().numpy(), target, [0, 3, 5, 6, 8, 9, 10], dtype, smoothing=0.25, beta=-0.5)


@pytest.mark.parametrize("rows", [9, 300])   # (three launches from 257 rows of two pairs on)
def test_what_is_not_read_may_hold_anything(rows):
    import torch
    import paper_2405_13954_amd as P
    full = torch.randn(rows, 780, generator=torch.Generator().manual_seed(0)).cuda()
    z = full[:, :777]
    z[0], z[8:], z[3] = float("nan"), float("nan"), float("nan")     # before, behind, masked
    z[6, 5] = float("nan")                                          # in pair 1
    target = torch.tensor([3, 4, 5, -1, 776, 0, 9, 2] + [1] * (rows - 8)).cuda()
    offsets = torch.tensor([1, 3, 5, 6, 8]).cuda()
    loss, logp, d = f32(2), f32(4), torch.empty(rows, 780, device="cuda")[:, :777]
    P.logra_preference_loss(z, target, offsets, logp, loss=loss, dlogits=d)
    assert torch.isnan(loss).tolist() == [False, True] and torch.isnan(logp).tolist() == [False, False, False, True]
    assert not d[[0, 3]].any() and not d[8:].any() and bool(torch.isfinite(d[[1, 2, 4]]).all())
    # a pair that does not count, whatever it holds
    P.logra_preference_loss(z, target, offsets, logp, loss=loss, dlogits=d, weight=torch.tensor([1.0, 0.0]).cuda())
    assert loss[1] == 0 and not d[5:8].any() and bool(torch.isfinite(d).all())


@pytest.mark.parametrize("rows", [6, 300])
def test_offsets_of_any_kind_are_safe(rows):
    # values out of range or decreasing: results are unspecified, memory is not touched outside the outputs
    import torch
    import paper_2405_13954_amd as P
    for cuts in ([-5, 3, 100, 2, 1 << 40], [-(1 << 62), 1 << 62, 0, 6, 3], [6, 6, 6, 6, 6], [9, 9, 9, 9, 9], [5, 4, 3, 2, 1]):
        z, _, _ = mk(np.random.default_rng(0), rows, 50, 1.0, "f32")
        d, full = room(rows, 50, "f32")
        loss, logp = f32(3), f32(5)
        P.logra_preference_loss(z, (torch.arange(rows) % 50).cuda(), torch.tensor(cuts).cuda(), logp[:4], loss=loss[:2], dlogits=d)
        guarded(full, rows, 50)
        assert loss[2] == 12345.0 and logp[4] == 12345.0
    assert logp[:4].tolist() == [0.0] * 4


def test_no_rows_and_no_pairs():
    import torch
    import paper_2405_13954_amd as P
    z, loss, logp = torch.empty(0, 48, device="cuda"), f32(1), f32(2)
    none = torch.zeros(3, dtype=torch.int64, device="cuda")
    P.logra_preference_loss(z, none[:0], none, logp, loss=loss, dlogits=z, ref=torch.tensor([2.0, 0.0]).cuda(), beta=0.5)
    assert logp.tolist() == [0, 0] and abs(float(loss[0]) - np.log1p(np.exp(1.0))) < 1e-6
    P.logra_preference_loss(z, none[:0], none[:1], logp[:0])


def test_more_rows_and_pairs_than_one_line_of_the_grid():
    import torch
    import paper_2405_13954_amd as P
    rows = (1 << 21) + 7
    z = torch.randn(rows, 8, device="cuda").to(torch.bfloat16)
    t = torch.randint(0, 8, (rows,), device="cuda")
    o = torch.tensor([0, rows - 9, rows - 4, rows - 4, rows - 1]).cuda()
    d, loss, logp = torch.empty_like(z), f32(2), f32(4)
    P.logra_preference_loss(z, t, o, logp, loss=loss, dlogits=d)
    few, l2, p2 = torch.empty(9, 8, dtype=torch.bfloat16, device="cuda"), f32(1), f32(2)
    P.logra_preference_loss(z[-9:], t[-9:], torch.tensor([5, 5, 8]).cuda(), p2, loss=l2, dlogits=few)
    assert torch.equal(few[5:], d[-4:]) and torch.equal(l2, loss[1:]) and torch.equal(p2, logp[2:]) and not d[-1].any()
    lse = torch.logsumexp(z.double(), 1)
    want = (z.double().gather(1, t[:, None])[:, 0] - lse)[:rows - 9].sum()
    assert abs(float(logp[0]) - float(want)) <= rows * (2.0 ** -20 + 8 * 2.0 ** -24) * 4 + U * abs(float(want))
    pairs = (1 << 21) + 3
    loss, logp = f32(pairs), f32(2 * pairs)
    P.logra_preference_loss(z[:0], t[:0], torch.zeros(2 * pairs + 1, dtype=torch.int64, device="cuda"), logp, loss=loss)
    assert not logp.any() and bool((loss == loss[0]).all()) and abs(float(loss[0]) - np.log(2)) < 1e-7


def test_far_rows():
    # rows at a stride of 2^27 elements: offsets beyond 32 bits
    import torch
    import paper_2405_13954_amd as P
    wide = torch.empty(36 << 27, dtype=torch.bfloat16, device="cuda").view(36, -1)
    z = wide[:, :120]
    z.copy_(torch.randn(36, 120).to(torch.bfloat16))
    t, o = torch.randint(0, 120, (36,)).cuda(), torch.tensor([0, 9, 20, 30, 36]).cuda()
    near, out = torch.empty(36, 120, dtype=torch.bfloat16, device="cuda"), wide[:, 128:248]
    lp1, lp2 = f32(4), f32(4)
    P.logra_preference_loss(z.contiguous(), t, o, lp1, dlogits=near)
    P.logra_preference_loss(z, t, o, lp2, dlogits=out)
    assert torch.equal(out, near) and torch.equal(lp1, lp2)


def test_gradient_against_differences():
    # fp32, beta 0.5, along e with a step of 2^-6 in every logit of a pair's 12 tokens: the loss' third derivative along e is
    # below (12 |e|)^3 (d's derivatives times the sigmoid's, each below 1), and each loss is within beta 12 (2^-20 + 2^-15)(1 + 8)
    import torch
    import paper_2405_13954_amd as P
    g = torch.Generator().manual_seed(5)
    z, e = torch.randn(24, 512, generator=g).cuda(), torch.randn(24, 512, generator=g).cuda() / 12
    t, o = torch.randint(0, 512, (24,), generator=g).cuda(), torch.tensor([0, 5, 12, 20, 24]).cuda()
    h, losses, logp = 2.0 ** -6, [], f32(4)
    for s in (h, -h):
        losses.append(f32(2))
        P.logra_preference_loss(z + s * e, t, o, logp, loss=losses[-1], beta=0.5, smoothing=0.1)
    loss, d = f32(2), torch.empty_like(z)
    P.logra_preference_loss(z, t, o, logp, loss=loss, dlogits=d, beta=0.5, smoothing=0.1)
    diff = (losses[0] - losses[1]).double() / (2 * h)
    along = (d.double() * e.double()).sum(1)
    want = torch.stack([along[:12].sum(), along[12:].sum()])
    big = float(e.abs().max()) * 12
    bound = h * h * big ** 3 / 6 + 0.5 * 12 * (2.0 ** -20 + 2.0 ** -15) * 9 / h
    assert bool(((diff - want).abs() <= bound).all()), (diff, want, bound)


def test_one_pair_against_the_token_loss():
    # with d far on the losing side the slope is w beta: the gradient is the token loss' of weight +-w beta
    import torch
    import paper_2405_13954_amd as P
    z = torch.randn(6, 1000, generator=torch.Generator().manual_seed(1)).cuda()
    t, o = torch.randint(0, 1000, (6,)).cuda(), torch.tensor([0, 4, 6]).cuda()
    a, b, loss, logp = torch.empty_like(z), torch.empty_like(z), f32(6), f32(2)
    P.logra_preference_loss(z, t, o, logp, dlogits=a, ref=torch.tensor([1e4, 0.0]).cuda(), beta=0.25)
    P.logra_token_loss(z, t, loss, dlogits=b, weight=torch.tensor([0.25] * 4 + [-0.25] * 2).cuda())
    within(host(a), host(b), 0.5 * 2 * (2.0 ** -19 + 1000 * 2.0 ** -23), "gradient")
    within(host(logp), -np.array([host(loss)[:4].sum() * 4, -host(loss)[4:].sum() * 4]), 6 * 4 * 20 * (2.0 ** -20 + 1000 * 2.0 ** -24), "logp")


@pytest.mark.parametrize("rows", [300, 150])
def test_reruns_streams_and_graphs(rows):
    import torch
    import paper_2405_13954_amd as P
    z = torch.randn(rows, 9000, device="cuda").to(torch.bfloat16)
    t, o = torch.randint(0, 9000, (rows,), device="cuda"), torch.tensor([0, 40, 100, 120, rows]).cuda()
    d, loss, logp = torch.empty_like(z), f32(2), f32(4)
    ws = torch.empty(P.logra_preference_loss_ws_size(rows, 2), dtype=torch.uint8, device="cuda")

    def step(ws=ws):
        P.logra_preference_loss(z, t, o, logp, loss=loss, dlogits=d, ws=ws)

    step()
    first = [x.clone() for x in (d, loss, logp)]
    ws.fill_(255)
    step()
    assert all(torch.equal(x, y) for x, y in zip(first, (d, loss, logp)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for x in (d, loss, logp):
            x.fill_(1.0)
        step(ws=None)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(first, (d, loss, logp)))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        z.mul_(0.9)
        step()
        want = [x.clone() for x in (d, loss, logp)]
        for x in (d, loss, logp):
            x.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip((d, loss, logp), want))
