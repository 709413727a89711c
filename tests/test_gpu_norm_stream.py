"""Layer norm of more than the 256 MB cache holds, whose loads are non-temporal, in kernels of their own: every row has the bits
that the same row has in a call of half the rows (ordinary loads, which test_gpu_norm.py compares with the oracle), y and dx of
sampled rows and the sums for the gain and the bias are within that file's bounds of float64.
"""
import numpy as np
import pytest

from oracle import tuning as O
from test_gpu_norm import check_backward, forward_bounds
from tuning_util import HALF, U, dt, f32, host, within

pytestmark = pytest.mark.gpu
CACHE = 256 << 20


def buffer(g, rows, cols, std, dtype, shift=0.0):
    """[rows, cols] at a stride of whole vectors and 8 more; NaN in what lies between the rows."""
    import torch
    full = torch.full((rows, -(-cols // 8) * 8 + 8), float("nan"), dtype=dt(dtype), device="cuda")
    for part in full.split(2048):
        part[:, :cols] = torch.randn(len(part), cols, generator=g, device="cuda") * std + shift
    return full[:, :cols]


def space(like):
    """Room for an output of the same rows and stride."""
    import torch
    return torch.full((len(like), like.stride(0)), 7.0, dtype=like.dtype, device="cuda")[:, :like.shape[1]]


def halves(rows):
    """Two calls' rows, each of more than the forms for few rows take."""
    half = rows // 2
    assert half > 1024
    return slice(0, half), slice(half, rows)


def sampled(rows, live):
    """Some rows that count, from the first to the last."""
    import torch
    at = np.unique(np.concatenate([[0, 1, rows - 2, rows - 1], np.random.default_rng(rows).integers(0, rows, 60)]))
    return torch.from_numpy(at[live[at]]).cuda()


# every team from 32 threads on, two to four vectors a thread, partial vectors, with and without the mean; enough rows for the
# four matrices of a call to be more than the cache
SHAPES = [("bf16", 250, True), ("bf16", 768, False), ("bf16", 1001, True), ("bf16", 2049, False), ("bf16", 4096, True), ("bf16", 4104, False),
          ("bf16", 8200, True), ("bf16", 12289, False), ("bf16", 16384, True), ("f32", 130, False), ("f32", 513, True), ("f32", 1001, False),
          ("f32", 2052, True), ("f32", 6145, False), ("f32", 8193, False), ("f32", 12293, True)]


def rows_for(cols, dtype, matrices=4):
    return max(2051, int(1.05 * CACHE / matrices / (cols * (2 if dtype == "bf16" else 4))) | 1)


@pytest.mark.parametrize("dtype,cols,rms", SHAPES)
def test_forward(dtype, cols, rms):
    import torch
    import paper_2405_13954_amd as P
    rows = rows_for(cols, dtype)
    print("[norm beyond the cache, forward]", rows, cols, dtype, rms, flush=True)
    g = torch.Generator(device="cuda").manual_seed(cols)
    x, r = buffer(g, rows, cols, 1.0, dtype, 0.3), buffer(g, rows, cols, 2.0, dtype)
    gain = (1 + 0.3 * torch.randn(cols, generator=g, device="cuda")).to(dt(dtype))
    bias = None if rms else (0.3 * torch.randn(cols, generator=g, device="cuda")).to(dt(dtype))
    mask = (torch.rand(rows, generator=g, device="cuda") > 0.2).to(torch.uint8)
    y, h = space(x), space(x)
    mean, rstd = (None if rms else f32(rows)), f32(rows)
    P.logra_layer_norm_forward(x, y, gain=gain, bias=bias, rms=rms, mask=mask, residual=r, h=h, mean=mean, rstd=rstd)
    for part in halves(rows):
        y2, h2, m2, r2 = space(x[part]), space(x[part]), (None if rms else f32(len(x[part]))), f32(len(x[part]))
        P.logra_layer_norm_forward(x[part], y2, gain=gain, bias=bias, rms=rms, mask=mask[part], residual=r[part], h=h2, mean=m2, rstd=r2)
        assert torch.equal(y2, y[part]) and torch.equal(h2, h[part]) and torch.equal(r2, rstd[part])
        assert rms or torch.equal(m2, mean[part])
    off = mask == 0
    assert not y[off].any() and not h[off].any() and not rstd[off].any()
    at = sampled(rows, host(mask) != 0)
    h64 = host(h[at])
    assert np.array_equal(h64, host((x[at].float() + r[at].float()).to(dt(dtype))))
    g64, b64 = host(gain), None if rms else host(bias)
    want, want_mean, want_rstd = O.norm_forward(h64, g64, b64, 1e-5, rms)
    em, er, ey = forward_bounds(h64, want, want_mean, want_rstd, g64, b64, 1e-5, rms)
    within(host(y[at]), want, ey + HALF[dtype] * (np.abs(want) + ey), "y")
    within(host(rstd[at]), want_rstd, er, "rstd")
    assert rms or np.all(np.abs(host(mean[at]) - want_mean) <= em)


@pytest.mark.parametrize("dtype,cols,rms", SHAPES)
def test_backward(dtype, cols, rms):
    import torch
    import paper_2405_13954_amd as P
    rows = rows_for(cols, dtype)
    print("[norm beyond the cache, backward]", rows, cols, dtype, rms, flush=True)
    g = torch.Generator(device="cuda").manual_seed(cols)
    h, dy, base = buffer(g, rows, cols, 1.0, dtype, 0.3), buffer(g, rows, cols, 1e-2, dtype), buffer(g, rows, cols, 1e-2, dtype)
    gain = (1 + 0.3 * torch.randn(cols, generator=g, device="cuda")).to(dt(dtype))
    mask = (torch.rand(rows, generator=g, device="cuda") > 0.2).to(torch.uint8)
    y, mean, rstd = space(h), (None if rms else f32(rows)), f32(rows)
    P.logra_layer_norm_forward(h, y, rms=rms, mean=mean, rstd=rstd)
    args = dict(gain=gain, rms=rms)
    dx, dgain, dbias = space(h), f32(cols), (None if rms else f32(cols))
    P.logra_layer_norm_backward(h, dy, rstd, mean=mean, mask=mask, base=base, dx=dx, dgain=dgain, dbias=dbias, **args)
    for part in halves(rows):
        d2 = space(h[part])
        P.logra_layer_norm_backward(h[part], dy[part], rstd[part], mean=None if rms else mean[part], mask=mask[part], base=base[part],
                                    dx=d2, **args)
        assert torch.equal(d2, dx[part])
    off = mask == 0
    assert torch.equal(dx[off], base[off])
    # in place of the gradient that comes in, whose row ahead is loaded before the row is written
    again, g2 = space(dy), f32(cols)
    again.copy_(dy)
    P.logra_layer_norm_backward(h, again, rstd, mean=mean, mask=mask, base=base, dx=again, dgain=g2, **args)
    assert torch.equal(again, dx) and torch.equal(g2, dgain)
    # sampled rows
    at = sampled(rows, host(mask) != 0)
    h64, dy64, b64, r64 = host(h[at]), host(dy[at]), host(base[at]), host(rstd[at])
    m64 = np.zeros(len(at)) if rms else host(mean[at])
    want = O.norm_backward(h64, dy64, m64, r64, host(gain), rms, base=b64)[0]
    xh, c = (h64 - m64[:, None]) * r64[:, None], np.abs(dy64 * host(gain))
    ex, along = U * (np.abs(h64) + np.abs(m64)[:, None]) * r64[:, None], np.mean(c * np.abs(xh), 1)[:, None]
    term = c + (0 if rms else np.mean(c, 1)[:, None]) + np.abs(xh) * along
    ed = r64[:, None] * ((95 + 6) * U * term + 2 * c * ex + np.mean(c * ex, 1)[:, None] * np.abs(xh) + ex * along)
    within(host(dx[at]), want, ed + (HALF[dtype] + 2 * U) * np.abs(want) + 2 * U * np.abs(b64), "dx")
    # the sums over all rows
    sums = [torch.zeros(cols, dtype=torch.float64, device="cuda") for _ in range(5)]
    for i in range(0, rows, 2048):
        live = (mask[i:i + 2048] != 0)[:, None]
        d = torch.where(live, dy[i:i + 2048].double(), 0.0)
        mm = torch.zeros(1, 1, device="cuda") if rms else mean[i:i + 2048].double()[:, None]
        rr, hh = rstd[i:i + 2048].double()[:, None], h[i:i + 2048].double()
        t = d * (hh - mm) * rr
        for s, v in zip(sums, (t, t.abs(), d.abs() * rr * (hh.abs() + mm.abs()), d, d.abs())):
            s += v.sum(0)
    # the rows that a team adds in a line: 256 workgroups, in each of them as many teams as 512 threads make
    vectors, team = -(-cols // (8 if dtype == "bf16" else 4)), 32
    while vectors > 3 * team and team < 512:
        team *= 2
    rows_u = (rows / (256 * (512 // team)) + 1 + 70) * U
    want_g, terms, near, want_b, dys = (host(s) for s in sums)
    within(host(dgain), want_g, rows_u * terms + U * (3 * terms + near), "dgain")
    if not rms:
        within(host(dbias), want_b, rows_u * dys, "dbias")


@pytest.mark.parametrize("dtype,cols", [("bf16", 520), ("bf16", 4104), ("f32", 1001), ("f32", 8193)])
@pytest.mark.parametrize("rows", [1024, 1025])
def test_backward_on_either_side_of_the_form_for_few_rows(rows, cols, dtype):
    check_backward(rows, cols, dtype, cols % 2 == 0, True, mask_share=0.3, extra=8)
