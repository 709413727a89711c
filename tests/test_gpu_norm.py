"""Layer norm, forward and backward, against the float64 oracle.

Tolerances count roundings of u = 2^-24.  A sum over a row is at most 64 additions in a thread, 6 between lanes and 16
between waves, and its terms have a few roundings each: 95 u of the terms' magnitudes (`ROW`).  So, forward: mean within
ROW avg|h| (em); the variance within its own ROW and 3 em^2 (the difference of means enters squared); rstd by half of that,
relative, and 4 u; y by its terms.  Backward, from exact statistics: xh and c carry 2 u and u, their averages ROW, and dgain and dbias are
sums of at most rows / 512 + 1 additions in a thread, 16 between teams, 512 / 16 + 16 between workgroups (`ROWS`); of up to 1,024 rows
8 in a thread, 16 and 8 between threads.  Then one rounding to the output's type.
"""
import numpy as np
import pytest

from oracle import tuning as O
from tuning_util import HALF, U, dt, f32, guarded, host, mk, room, vector, within

pytestmark = pytest.mark.gpu
ROW = 95 * U


def forward_bounds(h, y, mean, rstd, gain, bias, eps, rms):
    avg = np.mean(np.abs(h), 1)
    em = np.zeros(len(h)) if rms else ROW * avg
    d = h - mean[:, None]
    var = np.mean(d * d, 1)
    er = rstd * (0.5 * (ROW * var + 3 * em ** 2) / (var + eps) + 4 * U)
    g = np.abs(gain) if gain is not None else 1.0
    ey = g * (rstd[:, None] * (em[:, None] + 2 * U * np.abs(d)) + np.abs(d) * er[:, None]) + 3 * U * np.abs(y)
    if bias is not None:
        ey = ey + 2 * U * np.abs(bias)
    return em + 2 * U * np.abs(mean), er + 2 * U * rstd, ey


def check_forward(rows, cols, dtype, rms, residual, mask_share=0.0, extra=0, shift=0.3, affine=True, eps=1e-5, seed=0):
    import torch
    import paper_2405_13954_amd as P
    print("[norm forward]", rows, cols, dtype, "rms" if rms else "", "residual" if residual else "", mask_share, extra, flush=True)
    g = np.random.default_rng([rows, cols, seed])
    x, x64, _ = mk(g, rows, cols, 1.0, dtype, extra, shift)
    r, r64, _ = mk(g, rows, cols, 2.0, dtype) if residual else (None, 0.0, None)
    gain, gain64 = vector(g, cols, 0.3, dtype, 1.0) if affine else (None, None)
    bias, bias64 = vector(g, cols, 0.3, dtype) if affine and not rms else (None, None)
    live = g.random(rows) >= mask_share
    mask = torch.from_numpy(live.astype(np.uint8) * 3).cuda() if mask_share else None   # (anything but 0 counts)
    if mask_share:
        x[~torch.from_numpy(live).cuda()] = float("nan")     # rows that are not read
    y, full_y = room(rows, cols, dtype, 8)
    h, full_h = room(rows, cols, dtype, 16)
    mean, rstd = (None if rms else f32(rows)), f32(rows)
    P.logra_layer_norm_forward(x, y, gain=gain, bias=bias, eps=eps, rms=rms, mask=mask, residual=r, h=h, mean=mean, rstd=rstd)
    h64 = host(h)
    want_h = np.where(live[:, None], x64 + r64, 0.0)
    within(h64, want_h, HALF[dtype] * np.abs(want_h) + U * np.abs(want_h) if residual else 0.0, "h")
    want_y, want_mean, want_rstd = O.norm_forward(h64, gain64, bias64, eps, rms, live)
    em, er, ey = forward_bounds(h64, want_y, want_mean, want_rstd, gain64, bias64, eps, rms)
    ey = ey + HALF[dtype] * (np.abs(want_y) + ey)
    within(host(rstd), want_rstd, np.where(live, er, 0), "rstd")
    if not rms:
        within(host(mean), want_mean, np.where(live, em, 0), "mean")
    within(host(y), want_y, np.where(live[:, None], ey, 0), "y")
    guarded(full_y, rows, cols)
    guarded(full_h, rows, cols)
    # without h and the statistics, and in place of x and of the residual: the same bits
    y2, _ = room(rows, cols, dtype)
    P.logra_layer_norm_forward(x, y2, gain=gain, bias=bias, eps=eps, rms=rms, mask=mask, residual=r)
    assert torch.equal(y2, y)
    if residual:
        x2, r2 = x.clone(), r.clone()
        x2, full_x = room(rows, cols, dtype)
        x2.copy_(x)
        r2, full_r = room(rows, cols, dtype)
        r2.copy_(r)
        P.logra_layer_norm_forward(x2, x2, gain=gain, bias=bias, eps=eps, rms=rms, mask=mask, residual=r2, h=r2)
        assert torch.equal(x2, y) and torch.equal(r2, h)
        guarded(full_x, rows, cols)
        guarded(full_r, rows, cols)
    return x, h, y, mean, rstd


# widths on either side of every team's limits, odd ones, and the smallest
@pytest.mark.parametrize("dtype,cols", [("bf16", c) for c in (1, 7, 8, 33, 256, 257, 511, 520, 768, 1001, 1024, 1031, 2049,
                                                              4096, 4104, 8200, 12289, 16377, 16384)] +
                         [("f32", c) for c in (1, 3, 4, 130, 129, 260, 513, 1001, 2048, 4100, 6145, 8193, 12289, 16381, 16384)])
def test_forward_widths(cols, dtype):
    check_forward(5, cols, dtype, False, True, mask_share=0.3)
    check_forward(3, cols, dtype, True, False, extra=24)


@pytest.mark.parametrize("rows", [1, 2, 63, 1024, 1025, 2050])
@pytest.mark.parametrize("cols", [24, 257, 768, 2056])
def test_forward_rows(rows, cols):
    check_forward(rows, cols, "bf16", False, rows % 2 == 0, mask_share=0.2 if rows > 2 else 0.0)
    check_forward(rows, cols, "f32", True, rows % 2 == 1)


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_forward_plain_and_far_from_zero(dtype, rms):
    check_forward(9, 640, dtype, rms, False, affine=False)
    # a mean 1000 times the spread: the variance is that of the differences
    check_forward(9, 640, dtype, rms, False, shift=1000.0)
    check_forward(4, 5000, dtype, rms, False, shift=-300.0, eps=1e-12)


def test_forward_constant_and_extreme_rows():
    import torch
    import paper_2405_13954_amd as P
    x = torch.zeros(6, 64, device="cuda")
    x[1], x[2] = 7.25, 1e15
    x[3, 5] = float("nan")
    x[4, 5] = float("inf")
    x[5] = 1e-20
    y, mean, rstd = torch.empty_like(x), f32(6), f32(6)
    P.logra_layer_norm_forward(x, y, eps=1e-6, mean=mean, rstd=rstd)
    assert bool((y[:3] == 0).all()) and bool((y[5] == 0).all()) and mean[1] == 7.25
    within(host(rstd[:3]), np.full(3, 1000.0), 1000.0 * 4 * U + 1e-4, "rstd")        # (1e-6 itself is rounded to fp32)
    assert bool(torch.isnan(y[3]).all()) and bool(torch.isnan(y[4]).all())


def test_forward_far_rows():
    # rows at a stride of 2^27 elements: offsets beyond 32 bits
    import torch
    import paper_2405_13954_amd as P
    wide = torch.empty(36 << 27, dtype=torch.bfloat16, device="cuda").view(36, -1)
    x = wide[:, :40]
    x.copy_(torch.randn(36, 40).to(torch.bfloat16))
    near = torch.empty(36, 40, dtype=torch.bfloat16, device="cuda")
    P.logra_layer_norm_forward(x.contiguous(), near)
    out = wide[:, 64:104]
    P.logra_layer_norm_forward(x, out)
    assert torch.equal(out, near)


def test_more_rows_than_one_line_of_the_grid():
    import torch
    import paper_2405_13954_amd as P
    rows = (1 << 24) + 9                                       # 2^21 workgroups of eight rows, and two more
    x = torch.empty(rows, 8, dtype=torch.bfloat16, device="cuda")
    for part in x.split(1 << 21):
        part.copy_(torch.randn(part.shape, device="cuda"))
    y, dx, mean, rstd, dgain = torch.empty_like(x), torch.empty_like(x), f32(rows), f32(rows), f32(8)
    P.logra_layer_norm_forward(x, y, mean=mean, rstd=rstd)
    P.logra_layer_norm_backward(x, y, rstd, mean=mean, dx=dx, dgain=dgain)
    for at in (0, (1 << 24) - 8, rows - 8):                    # the same rows by themselves
        part, few = x[at:at + 8].contiguous(), torch.empty(8, 8, dtype=torch.bfloat16, device="cuda")
        m, r, d = f32(8), f32(8), torch.empty_like(few)
        P.logra_layer_norm_forward(part, few, mean=m, rstd=r)
        P.logra_layer_norm_backward(part, few, r, mean=m, dx=d)
        assert torch.equal(few, y[at:at + 8]) and torch.equal(m, mean[at:at + 8]) and torch.equal(d, dx[at:at + 8])
    want = torch.zeros(8, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(want)
    for a, b, m, r in zip(x.split(1 << 21), y.split(1 << 21), mean.split(1 << 21), rstd.split(1 << 21)):
        t = b.double() * (a.double() - m.double()[:, None]) * r.double()[:, None]
        want, size = want + t.sum(0), size + t.abs().sum(0)
    # a workgroup's team adds 2^24 / (256 * 16) = 4,096 rows in a line, the rest as ROWS has it
    within(host(dgain), host(want), (4097 + 70) * U * host(size), "dgain")


def check_backward(rows, cols, dtype, rms, base, mask_share=0.0, extra=0, affine=True, seed=0):
    import torch
    import paper_2405_13954_amd as P
    print("[norm backward]", rows, cols, dtype, "rms" if rms else "", "base" if base else "", mask_share, extra, flush=True)
    g = np.random.default_rng([rows, cols, seed, 7])
    h, h64, _ = mk(g, rows, cols, 1.0, dtype, extra, 0.3)
    dy, dy64, _ = mk(g, rows, cols, 1e-2, dtype, 8)
    b, b64, _ = mk(g, rows, cols, 1e-2, dtype, 16) if base else (None, None, None)
    gain, gain64 = vector(g, cols, 0.3, dtype, 1.0) if affine else (None, None)
    live = g.random(rows) >= mask_share
    _, mean64, rstd64 = O.norm_forward(h64, rms=rms)
    mean, rstd = (None if rms else torch.from_numpy(mean64).float().cuda()), torch.from_numpy(rstd64).float().cuda()
    mean64, rstd64 = (np.zeros(rows) if rms else host(mean)), host(rstd)     # as the kernel has them
    mask = None
    if mask_share:
        off = torch.from_numpy(~live).cuda()
        mask = (~off).to(torch.uint8)
        h[off], dy[off], rstd[off] = float("nan"), float("nan"), float("nan")
    want_dx, want_g, want_b = O.norm_backward(h64, dy64, mean64, rstd64, gain64, rms, live, b64)
    xh = (h64 - mean64[:, None]) * rstd64[:, None]
    c = dy64 * (1.0 if gain64 is None else gain64)
    term = np.abs(c) + (0 if rms else np.mean(np.abs(c), 1)[:, None]) + np.abs(xh) * np.mean(np.abs(c * xh), 1)[:, None]
    near = np.abs(h64) + np.abs(mean64)[:, None]     # the rounding of h - mean
    ex = U * near * rstd64[:, None]
    ed = np.abs(rstd64)[:, None] * ((ROW + 6 * U) * term + 2 * np.abs(c) * ex + np.mean(np.abs(c) * ex, 1)[:, None] * np.abs(xh)
                                    + ex * np.mean(np.abs(c * xh), 1)[:, None])
    ed = np.where(live[:, None], ed, 0.0) + HALF[dtype] * np.abs(want_dx) + 2 * U * (np.abs(want_dx) + (0 if b64 is None else np.abs(b64)))
    rows_u = (rows / 512 + 70) * U
    lm = live[:, None]
    eg = rows_u * np.sum(np.where(lm, np.abs(dy64 * xh), 0), 0) + np.sum(np.where(lm, np.abs(dy64) * (ex + 3 * U * np.abs(xh)), 0), 0)
    eb = rows_u * np.sum(np.where(lm, np.abs(dy64), 0), 0)
    dx, full = room(rows, cols, dtype, 8)
    dgain, dbias = f32(cols), (None if rms else f32(cols))
    args = dict(mean=mean, gain=gain, rms=rms, mask=mask, base=b)
    P.logra_layer_norm_backward(h, dy, rstd, dx=dx, dgain=dgain, dbias=dbias, **args)
    within(host(dx), want_dx, ed, "dx")
    within(host(dgain), want_g, eg + 1e-38, "dgain")
    if not rms:
        within(host(dbias), want_b, eb + 1e-38, "dbias")
    guarded(full, rows, cols)
    # one gradient at a time and added to what is there
    twice, only = dgain.clone(), torch.empty_like(dx)
    only, _ = room(rows, cols, dtype)
    P.logra_layer_norm_backward(h, dy, rstd, dgain=twice, accumulate=True, **{**args, "base": None})
    assert torch.equal(twice, dgain + dgain)
    P.logra_layer_norm_backward(h, dy, rstd, dx=only, **args)
    assert torch.equal(only, dx)
    if not rms:
        again = torch.ones_like(dbias)
        P.logra_layer_norm_backward(h, dy, rstd, dbias=again, **{**args, "base": None})
        assert torch.equal(again, dbias)
    # in place of each input
    for name in ("h", "dy", "base") if base else ("h", "dy"):
        src = {"h": h, "dy": dy, "base": b}[name]
        buf, whole = room(rows, cols, dtype)
        buf.copy_(src)
        use = {"h": h, "dy": dy, "base": b, name: buf}
        P.logra_layer_norm_backward(use["h"], use["dy"], rstd, dx=buf, dgain=twice, **{**args, "base": use["base"]})
        assert torch.equal(buf, dx) and torch.equal(twice, dgain), name
        guarded(whole, rows, cols)


@pytest.mark.parametrize("dtype,cols", [("bf16", c) for c in (1, 7, 8, 33, 256, 512, 520, 768, 1001, 1024, 1031, 2049, 4096, 4104,
                                                              8200, 12289, 16377, 16384)] +
                         [("f32", c) for c in (1, 3, 4, 130, 256, 260, 513, 1001, 2048, 4100, 6145, 8193, 12289, 16381, 16384)])
def test_backward_widths(cols, dtype):
    check_backward(5, cols, dtype, False, True, mask_share=0.3)
    check_backward(3, cols, dtype, True, False, extra=24)


# (more rows than one launch takes)
@pytest.mark.parametrize("dtype,cols", [("bf16", c) for c in (1, 33, 257, 520, 1001, 2049, 4104, 8200, 12289, 16384)] +
                         [("f32", c) for c in (3, 129, 513, 1001, 2049, 4100, 6145, 8193, 12289, 16381)])
def test_backward_widths_of_many_rows(cols, dtype):
    check_backward(1030, cols, dtype, cols % 2 == 0, True, mask_share=0.3, extra=8)


@pytest.mark.parametrize("rows", [1, 2, 17, 511, 513, 1025, 9000])
@pytest.mark.parametrize("cols", [24, 257, 768])
def test_backward_rows(rows, cols):
    check_backward(rows, cols, "bf16", False, rows % 2 == 0, mask_share=0.4 if rows > 2 else 0.0)
    check_backward(rows, cols, "f32", True, rows % 2 == 1, affine=rows != 17)


def test_backward_of_wide_rows_of_many_workgroups():
    check_backward(1500, 4096, "bf16", True, True, mask_share=0.2)
    check_backward(700, 8200, "f32", False, False)


def test_backward_of_masked_batches_and_no_rows():
    import torch
    import paper_2405_13954_amd as P
    nan = torch.full((5, 72), float("nan"), device="cuda")
    base, dx = torch.randn(5, 72, device="cuda"), f32(5 * 72).view(5, 72)
    dgain, dbias = f32(72), f32(72)
    stat = torch.full((5,), float("nan"), device="cuda")
    none = torch.zeros(5, dtype=torch.uint8, device="cuda")
    P.logra_layer_norm_backward(nan, nan, stat, mean=stat, mask=none, dx=dx, base=base, dgain=dgain, dbias=dbias)
    assert torch.equal(dx, base) and not dgain.any() and not dbias.any()
    P.logra_layer_norm_backward(nan, nan, stat, mean=stat, mask=none, dx=dx, dgain=dgain)
    assert not dx.any()
    dgain.fill_(3.0)
    dbias.fill_(3.0)
    empty = nan[:0]
    P.logra_layer_norm_backward(empty, empty, stat[:0], mean=stat[:0], dx=dx[:0], dgain=dgain, dbias=dbias, accumulate=True)
    assert bool((dgain == 3).all()) and bool((dbias == 3).all())
    P.logra_layer_norm_backward(empty, empty, stat[:0], mean=stat[:0], dx=dx[:0], dgain=dgain, dbias=dbias)
    assert not dgain.any() and not dbias.any()
    y, rstd = f32(5 * 72).view(5, 72), f32(5)
    P.logra_layer_norm_forward(nan, y, mask=none, rstd=rstd)
    assert not y.any() and not rstd.any()
    P.logra_layer_norm_forward(empty, y[:0])


@pytest.mark.parametrize("rows", [4, 1040])
def test_backward_of_rows_without_variance(rows):
    # rstd = 1 / sqrt(eps) up to 10^15, whose cube no fp32 holds: dx = rstd (c - avg(c))
    import torch
    import paper_2405_13954_amd as P
    g = torch.Generator().manual_seed(3)
    dy = torch.randn(rows, 96, generator=g).cuda()
    h = torch.tensor([0.0, 3.0, -1e-3, 1e4]).cuda().repeat(rows // 4)[:, None].expand(rows, 96).contiguous()
    for eps in (1e-5, 1e-20, 1e-30):
        y, mean, rstd, dx, dgain = torch.empty_like(h), f32(rows), f32(rows), torch.empty_like(h), f32(96)
        P.logra_layer_norm_forward(h, y, eps=eps, mean=mean, rstd=rstd)
        P.logra_layer_norm_backward(h, dy, rstd, mean=mean, dx=dx, dgain=dgain)
        c = host(dy)
        # (a mean that is not its row's value exactly leaves differences of one last bit of h, and then a variance)
        exact = host(mean) == host(h)[:, 0]
        assert exact[0] and exact[1]
        want = host(rstd)[:, None] * (c - c.mean(1, keepdims=True))
        within(host(dx)[exact], want[exact], (host(rstd)[:, None] * ROW * 2 * (np.abs(c) + np.abs(c).mean(1, keepdims=True)))[exact], "dx")
        assert bool(torch.isfinite(dx).all()) and bool(torch.isfinite(dgain).all())


def test_nan_stays_in_its_row():
    import torch
    import paper_2405_13954_amd as P
    g = torch.Generator().manual_seed(0)
    h, dy = torch.randn(6, 200, generator=g).cuda(), torch.randn(6, 200, generator=g).cuda()
    dy[2, 7] = float("nan")
    y, dx, mean, rstd, dgain, dbias = torch.empty_like(h), torch.empty_like(h), f32(6), f32(6), f32(200), f32(200)
    P.logra_layer_norm_forward(h, y, mean=mean, rstd=rstd)
    P.logra_layer_norm_backward(h, dy, rstd, mean=mean, dx=dx, dgain=dgain, dbias=dbias)
    rows = torch.isnan(dx).any(1)
    assert rows.tolist() == [False, False, True, False, False, False]
    assert torch.isnan(dgain).nonzero().flatten().tolist() == [7] and torch.isnan(dbias).nonzero().flatten().tolist() == [7]


@pytest.mark.parametrize("rows,cols", [(6, 72), (6, 2048), (6, 8200), (6, 12296), (1100, 72), (1100, 2048), (1100, 12296)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masked_rows_under_a_gain_that_is_not_finite(dtype, rows, cols):
    import torch
    import paper_2405_13954_amd as P
    g = torch.Generator().manual_seed(cols)
    h, dy, base = (torch.randn(rows, cols, generator=g).to(dt(dtype)).cuda() for _ in range(3))
    gain = torch.ones(cols, dtype=dt(dtype), device="cuda")
    gain[3], gain[cols - 2] = float("nan"), float("inf")
    mask = torch.tensor([1, 0, 1, 0, 0, 1], dtype=torch.uint8, device="cuda").repeat(rows // 6 + 1)[:rows]
    off = mask == 0
    y, dx, mean, rstd, dgain, dbias = torch.empty_like(h), torch.empty_like(h), f32(rows), f32(rows), f32(cols), f32(cols)
    P.logra_layer_norm_forward(h, y, gain=gain, mask=mask, mean=mean, rstd=rstd)
    assert not y[off].any() and bool(torch.isnan(y[~off][:, 3]).all())
    for rms in (False, True):
        args = dict(mean=None if rms else mean, gain=gain, rms=rms, mask=mask, dgain=dgain, dbias=None if rms else dbias)
        P.logra_layer_norm_backward(h, dy, rstd, dx=dx, base=base, **args)
        assert torch.equal(dx[off], base[off]) and bool(torch.isnan(dx[~off]).all())
        assert bool(torch.isfinite(dgain).all()) and bool(torch.isfinite(dbias).all())   # (no gain in them)
        P.logra_layer_norm_backward(h, dy, rstd, dx=dx, **args)
        assert not dx[off].any() and bool(torch.isnan(dx[~off]).all())


@pytest.mark.parametrize("rms", [False, True])
def test_gradients_against_differences(rms):
    # sum(y dy) along a direction e of h, with a step of 2^-8 in fp32: y's third derivatives along e are below 40 |e|^3
    # here (rstd below 2, 300 columns), so the difference is off by h^2 40 |e|_inf^3 sum|dy| at most, and the two sums of y
    # are each within 200 u of their terms
    import torch
    import paper_2405_13954_amd as P
    g = torch.Generator().manual_seed(4)
    h, dy, e = (torch.randn(7, 304, generator=g).cuda() for _ in range(3))
    gain = torch.randn(304, generator=g).cuda()
    step, sums = 2.0 ** -8, []
    y, mean, rstd = torch.empty_like(h), None if rms else f32(7), f32(7)
    for s in (step, -step):
        P.logra_layer_norm_forward(h + s * e, y, gain=gain, rms=rms)
        sums.append((y.double() * dy.double()).sum(1))
    mag = (y.double() * dy.double()).abs().sum(1)
    P.logra_layer_norm_forward(h, y, gain=gain, rms=rms, mean=mean, rstd=rstd)
    assert float(rstd.max()) < 2
    dx, dgain = torch.empty_like(h), f32(304)
    P.logra_layer_norm_backward(h, dy, rstd, mean=mean, gain=gain, rms=rms, dx=dx, dgain=dgain)
    diff = (sums[0] - sums[1]) / (2 * step)
    want = (dx.double() * e.double()).sum(1)
    bound = step ** 2 * 40 * float(e.abs().max()) ** 3 * (dy * gain).abs().sum(1).double() / 6 + 200 * U * mag / step
    assert bool(((diff - want).abs() <= bound).all()), ((diff - want).abs() / bound).tolist()
    # the gain's gradient is exact in the gain: y is linear in it
    P.logra_layer_norm_forward(h, y, gain=gain + 0.5, rms=rms)
    up = (y.double() * dy.double()).sum()
    P.logra_layer_norm_forward(h, y, gain=gain - 0.5, rms=rms)
    assert abs(float(up - (y.double() * dy.double()).sum() - dgain.double().sum())) <= 400 * U * float((y * dy).abs().sum() + mag.sum())


@pytest.mark.parametrize("rows", [700, 1300])
def test_reruns_streams_and_graphs(rows):
    import torch
    import paper_2405_13954_amd as P
    g = torch.Generator().manual_seed(9)
    h, dy, r = (torch.randn(rows, 1032, generator=g).to(torch.bfloat16).cuda() for _ in range(3))
    gain, bias = torch.randn(1032, generator=g).to(torch.bfloat16).cuda(), torch.randn(1032, generator=g).to(torch.bfloat16).cuda()
    ws = torch.empty(P.logra_layer_norm_ws_size(rows, 1032), dtype=torch.uint8, device="cuda")
    out = dict(y=torch.empty_like(h), hs=torch.empty_like(h), dx=torch.empty_like(h), mean=f32(rows), rstd=f32(rows),
               dgain=f32(1032), dbias=f32(1032))

    def both(ws=ws):
        P.logra_layer_norm_forward(h, out["y"], gain=gain, bias=bias, residual=r, h=out["hs"], mean=out["mean"], rstd=out["rstd"])
        P.logra_layer_norm_backward(out["hs"], dy, out["rstd"], mean=out["mean"], gain=gain, dx=out["dx"], base=dy,
                                    dgain=out["dgain"], dbias=out["dbias"], ws=ws)

    both()
    first = {k: v.clone() for k, v in out.items()}
    both(ws=None)
    assert all(torch.equal(out[k], v) for k, v in first.items())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for v in out.values():
            v.fill_(1.0)
        both(ws=None)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(out[k], v) for k, v in first.items())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for k in range(3):
        h.mul_(0.75)
        both()
        want = {k: v.clone() for k, v in out.items()}
        for v in out.values():
            v.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], v) for k, v in want.items())
