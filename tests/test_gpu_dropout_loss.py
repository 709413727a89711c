"""Dropout and the token loss against the float64 oracle.

Tolerances are bounds: a dropout output carries one product, one addition and one rounding (2^-8 of the value for
bf16, 2^-23 of the terms for fp32).  A loss sums vocab exponentials of relative error below 2^-21 in fp32 (the
hardware exponential and the product of z - max, below 2^7 where it matters, with log2 e), so it is within
(2^-20 + vocab 2^-24) of 1 + |loss|; a gradient element within (2^-19 + vocab 2^-24) of its terms w p and w [target]
and one rounding.
"""
import numpy as np
import pytest

from oracle import adapters as O

pytestmark = pytest.mark.gpu
SENTINEL = 12345.0


def _dt(name):
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _mk(g, rows, cols, std, dtype, extra=0):
    """(device view [rows, cols], float64 copy, the whole buffer): row strides are multiples of 16 bytes, and one row
    of sentinels follows."""
    import torch
    t = torch.from_numpy((g.standard_normal((rows, cols)) * std).astype(np.float32)).to(_dt(dtype))
    full = torch.full((rows + 1, -(-cols // 8) * 8 + extra), SENTINEL, dtype=_dt(dtype))
    full[:rows, :cols] = t
    full = full.cuda()
    return full[:rows, :cols], t.double().numpy(), full


def _guarded(full, rows, cols):
    keep = full.clone()
    keep[:rows, :cols] = SENTINEL
    assert bool((keep == SENTINEL).all()), "a store outside the rows"


def _within(err, bound, what):
    bad = ~(err <= bound)
    at = np.argwhere(bad)[:4].tolist()
    assert not bad.any(), f"{what}: {int(bad.sum())} beyond the bound, first at {at}: {err[bad][:4]} > {bound[bad][:4]}"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (3, 8), (5, 9), (64, 33), (37, 130), (2, 1031), (9, 2056)])
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_dropout(rows, cols, p, dtype):
    import torch
    import paper_2405_13954_amd as P
    print("[dropout]", rows, cols, p, dtype, flush=True)
    g = np.random.default_rng([rows, cols])
    x, x64, _ = _mk(g, rows, cols, 1.0, dtype)
    r, r64, _ = _mk(g, rows, cols, 1.0, dtype, 16)
    seed, offset = 0xFEDCBA9876543210, 0x1234567890ABCDEF
    f = O.drop_factor(rows, cols, p, seed, offset)
    u = 2.0 ** -8 if dtype == "bf16" else 0.0
    for res, res64 in ((None, None), (r, r64)):
        out, _, full = _mk(g, rows, cols, 1.0, dtype, 8)
        P.logra_dropout(x, out, p, seed, offset, residual=res)
        want = O.dropout(x64, res64, p, seed, offset)
        bound = u * np.abs(want) + 2.0 ** -22 * (np.abs(x64 * f) + (0 if res64 is None else np.abs(res64)))
        _within(np.abs(out.double().cpu().numpy() - want), bound, "out")
        if res is None:
            assert np.array_equal(out.double().cpu().numpy() == 0, (want == 0))
        _guarded(full, rows, cols)
    # in place, of either input
    want = torch.empty_like(x)
    P.logra_dropout(x, out, p, seed, offset, residual=r)
    x2, r2 = x.clone(memory_format=torch.preserve_format), r
    buf, _, full = _mk(g, rows, cols, 1.0, dtype)
    buf.copy_(x2)
    P.logra_dropout(buf, buf, p, seed, offset, residual=r)
    assert torch.equal(buf, out)
    _guarded(full, rows, cols)
    keep = out.clone()
    P.logra_dropout(x, r2, p, seed, offset, residual=r2)
    assert torch.equal(r2, keep)


def test_dropout_is_the_adapters_dropout_and_its_own_backward():
    import torch
    import paper_2405_13954_amd as P
    g = torch.Generator().manual_seed(3)
    x = torch.randn(90, 264, generator=g).cuda()
    d = torch.empty_like(x)
    P.logra_dropout(x, d, 0.5, 77, 88)                       # scale 2: exact
    a, b = torch.randn(2, 5, 264, generator=g).cuda(), torch.randn(2, 5, 32, generator=g).cuda()
    plan = P.logra_adapter_plan(torch.randint(0, 2, (90,), generator=g, dtype=torch.int32).cuda(), 2)
    y, z = torch.empty(90, 32, device="cuda"), torch.empty(90, 32, device="cuda")
    P.logra_adapter_forward(x, a, b, plan, y, p=0.5, seed=77, offset=88)
    P.logra_adapter_forward(d, a, b, plan, z)
    assert torch.equal(y, z)
    # linear, with a diagonal matrix: the gradient of sum(out * dy) is drop(dy)
    dy, back = torch.randn(90, 264, generator=g).cuda(), torch.empty_like(x)
    P.logra_dropout(dy, back, 0.5, 77, 88)
    assert torch.equal((back * x), (dy * d))


def test_dropout_selects():
    import torch
    import paper_2405_13954_amd as P
    f = O.drop_factor(8, 40, 0.5, 1, 2)
    for dtype in ("bf16", "f32"):
        x = torch.ones(8, 40, dtype=_dt(dtype), device="cuda")
        x[torch.from_numpy(f == 0).cuda()] = float("nan")
        out = torch.empty_like(x)
        P.logra_dropout(x, out, 0.5, 1, 2)
        assert np.array_equal(out.float().cpu().numpy(), f.astype(np.float32))


def test_dropout_of_far_rows():
    # rows at a stride of 2^26 elements: offsets beyond 32 bits, and the rows' masks are those of near rows
    import torch
    import paper_2405_13954_amd as P
    wide = torch.empty(70 << 26, dtype=torch.bfloat16, device="cuda").view(70, -1)
    x = wide[:, :24]
    x.copy_(torch.randn(70, 24).to(torch.bfloat16))
    near, out = torch.empty(70, 24, dtype=torch.bfloat16, device="cuda"), wide[:, 64:88]
    P.logra_dropout(x.contiguous(), near, 0.25, 9, 1)
    P.logra_dropout(x, out, 0.25, 9, 1, residual=None)
    assert torch.equal(out, near)


# ------------------------------------------------------------------- loss --
def _check_loss(z, z64, target, weight, dtype, inplace=False, vocab_note=""):
    import torch
    import paper_2405_13954_amd as P
    rows, vocab = z64.shape
    print("[loss]", rows, vocab, dtype, vocab_note, flush=True)
    want, wantg = O.token_loss(z64, target, None if weight is None else weight.astype(np.float64))
    w = np.ones(rows) if weight is None else np.abs(weight.astype(np.float64))
    loss = torch.full((rows,), SENTINEL, device="cuda")
    t = torch.from_numpy(target).cuda()
    wt = None if weight is None else torch.from_numpy(weight).cuda()
    only = torch.empty_like(loss)
    P.logra_token_loss(z, t, only, weight=wt)
    full = None
    if inplace:
        d = z
    else:
        d, _, full = _mk(np.random.default_rng(0), rows, vocab, 1.0, dtype, 8)
    P.logra_token_loss(z, t, loss, dlogits=d, weight=wt)
    assert torch.equal(loss, only)
    got, gotg = loss.double().cpu().numpy(), d.double().cpu().numpy()
    fin = np.isfinite(want)
    assert np.array_equal(np.isinf(got) & (got > 0), ~fin)
    tol = 2.0 ** -20 + vocab * 2.0 ** -24
    _within(np.abs(got[fin] - want[fin]), (tol * (w + np.abs(want)))[fin], "loss")
    hot = np.zeros_like(wantg)
    live = (target >= 0) & (target < vocab) & (w != 0)
    hot[np.nonzero(live)[0], target[live]] = 1.0
    bound = 2 * tol * (np.abs(wantg) + 2 * w[:, None] * hot) + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23) * np.abs(wantg) + 1e-37
    _within(np.abs(gotg - wantg), bound, "gradient")
    assert np.all(gotg[~live] == 0)
    if full is not None:
        _guarded(full, rows, vocab)


# one size for each width of the kernel, on either side of its limits, and odd ones
@pytest.mark.parametrize("dtype,vocab", [("bf16", v) for v in (1, 5, 8, 1000, 8192, 8193, 16391, 32768, 32775, 65537, 131072, 131079)] +
                         [("f32", v) for v in (1, 3, 4, 1001, 4096, 4097, 8195, 16385, 32769, 65536, 65537)])
def test_loss(dtype, vocab):
    g = np.random.default_rng(vocab)
    rows = 6
    z, z64, _ = _mk(g, rows, vocab, 3.0, dtype)
    target = g.integers(0, vocab, rows)
    target[1], target[4] = -100, vocab
    target[2] = vocab - 1
    _check_loss(z, z64, target, None, dtype)
    weight = g.uniform(0.5, 2.0, rows).astype(np.float32)
    weight[3], weight[5] = 0.0, -1.5
    _check_loss(z, z64, target, weight, dtype, inplace=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [100, 5000, 140000])
def test_loss_of_forbidden_and_extreme_logits(vocab, dtype):
    import torch
    g = np.random.default_rng(vocab)
    z, z64, _ = _mk(g, 6, vocab, 2.0, dtype)
    target = g.integers(0, vocab, 6)
    low = float(torch.finfo(_dt(dtype)).min)
    z64[0, g.random(vocab) < 0.9] = -np.inf       # forbidden tokens, the target maybe among them
    z64[1, :] = -np.inf                           # nothing is possible
    z64[2, :] = low                               # masked by the lowest value: uniform
    z64[3, :] = low
    z64[3, target[3]] = 0.0                       # and all but the target
    z64[4, :] = -np.inf
    z64[4, target[4]] = 3.0
    z64[5] += 60.0 if dtype == "bf16" else 1000.0
    zt = torch.from_numpy(z64).to(_dt(dtype))
    z.copy_(zt)
    _check_loss(z, zt.double().numpy(), target, None, dtype)


def test_loss_never_reads_masked_tokens_and_keeps_nan_in_its_row():
    import torch
    import paper_2405_13954_amd as P
    z = torch.randn(4, 777, generator=torch.Generator().manual_seed(0)).cuda()
    full = torch.zeros(4, 780, device="cuda")
    full[:, :777] = z
    z = full[:, :777]
    z[1] = float("nan")
    z[2, 5] = float("nan")
    loss, d = torch.empty(4, device="cuda"), torch.empty(4, 780, device="cuda")[:, :777]
    P.logra_token_loss(z, torch.tensor([3, -1, 4, 776]).cuda(), loss, dlogits=d)
    assert torch.isnan(loss).tolist() == [False, False, True, False]
    assert loss[1] == 0 and bool((d[1] == 0).all()) and bool(torch.isfinite(d[[0, 1, 3]]).all())


def test_loss_gradient_against_differences():
    # fp32: (loss(z + h e) - loss(z - h e)) / 2h with h = 2^-6; the third derivative along e bounds the difference by
    # h^2 |e|^3 max / 6 < 1e-3 here, and the losses' rounding by 2^-20 (1 + |loss|) / h
    import torch
    import paper_2405_13954_amd as P
    g = torch.Generator().manual_seed(5)
    z, e = torch.randn(8, 512, generator=g).cuda(), torch.randn(8, 512, generator=g).cuda()
    t = torch.randint(0, 512, (8,), generator=g).cuda()
    h, losses = 2.0 ** -6, []
    for s in (h, -h):
        losses.append(torch.empty(8, device="cuda"))
        P.logra_token_loss(z + s * e, t, losses[-1])
    loss, d = torch.empty(8, device="cuda"), torch.empty(8, 512, device="cuda")
    P.logra_token_loss(z, t, loss, dlogits=d)
    diff = (losses[0] - losses[1]).double() / (2 * h)
    bound = h * h * e.abs().max(1)[0].double() ** 3 / 6 + 2.0 ** -19 * (1 + loss.double()) / h
    assert bool(((diff - (d.double() * e.double()).sum(1)).abs() <= bound).all())


def test_dropout_and_loss_in_a_graph():
    import torch
    import paper_2405_13954_amd as P
    z = torch.randn(20, 1000, device="cuda").to(torch.bfloat16)
    t = torch.randint(0, 1000, (20,), device="cuda")
    h, d, loss = torch.empty_like(z), torch.empty_like(z), torch.empty(20, device="cuda")

    def step():
        P.logra_dropout(z, h, 0.1, 4, 5, residual=z)
        P.logra_token_loss(h, t, loss, dlogits=d)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        z.mul_(0.9)
        step()
        want = [x.clone() for x in (h, d, loss)]
        for x in (h, d, loss):
            x.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip((h, d, loss), want))


def test_refusals():
    import torch
    import paper_2405_13954_amd as P
    x = torch.zeros(4, 16, device="cuda")
    for kw in (dict(p=1.0), dict(p=float("nan")), dict(p=-1e-9), dict(p=1 - 2.0 ** -20)):
        with pytest.raises(P.LograError):
            P.logra_dropout(x, torch.empty_like(x), kw["p"], 1)
    with pytest.raises(ValueError):
        P.logra_dropout(x, torch.empty(4, 12, device="cuda"), 0.1, 1)
    with pytest.raises(P.LograError):
        P.logra_dropout(torch.zeros(4, 15, device="cuda"), torch.empty(4, 15, device="cuda"), 0.1, 1)   # stride of 60 bytes
    with pytest.raises(P.LograError):
        P.logra_dropout(torch.zeros(4, 16), torch.empty(4, 16), 0.1, 1)                                # host memory
    with pytest.raises(ValueError):
        P.logra_token_loss(x, torch.zeros(4, dtype=torch.int32, device="cuda"), torch.empty(4, device="cuda"))
    with pytest.raises(ValueError):
        P.logra_token_loss(x, torch.zeros(4, dtype=torch.int64, device="cuda"), torch.empty(3, device="cuda"))
