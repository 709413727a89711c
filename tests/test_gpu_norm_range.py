"""Layer norm over the whole range of fp32 magnitudes, against the float64 oracle: squares whose sum no fp32 number holds but
whose average does, statistics whose cube is subnormal or beyond fp32, and what lies beyond the range.

The bounds are those of test_gpu_norm.py: nothing in them depends on the size of the numbers.
"""
import numpy as np
import pytest

from oracle import tuning as O
from test_gpu_norm import ROW, forward_bounds
from tuning_util import HALF, U, dt, f32, host, room, vector, within

pytestmark = pytest.mark.gpu


def rows_of(g, rows, cols, size, dtype, shift=0.0):
    """([rows, cols] of N(shift, 1) size on the device, at a stride of whole vectors, and its float64 values)."""
    import torch
    t = torch.from_numpy(((g.standard_normal((rows, cols)) + shift) * size).astype(np.float32)).to(dt(dtype))
    view, _ = room(rows, cols, dtype)
    view.copy_(t)
    return view, t.double().numpy()


# 64 columns: the sum of the squares is in range where a row's average is; 16,377 and 16,384: four vectors a thread
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("rows,cols", [(5, 64), (5, 4096), (5, 9001), (5, 16384), (1030, 768), (1030, 4104), (1030, 16377)])
def test_forward_where_the_average_of_the_squares_is_in_range(rows, cols, rms, dtype):
    import torch
    import paper_2405_13954_amd as P
    g = np.random.default_rng([rows, cols, rms])
    for size, eps in ((1e17, 1e-5), (1e18, 1e-5), (1e19, 1e-5), (1e19, 1e30), (1e-12, 1e-30)):
        print("[norm range, forward]", rows, cols, dtype, rms, size, eps, flush=True)
        x, x64 = rows_of(g, rows, cols, size, dtype, 0.5)
        gain, gain64 = vector(g, cols, 0.3, dtype, 1.0)
        y, mean, rstd = room(rows, cols, dtype)[0], (None if rms else f32(rows)), f32(rows)
        P.logra_layer_norm_forward(x, y, gain=gain, eps=eps, rms=rms, mean=mean, rstd=rstd)
        eps32 = float(np.float32(eps))
        want, want_mean, want_rstd = O.norm_forward(x64, gain64, None, eps32, rms)
        em, er, ey = forward_bounds(x64, want, want_mean, want_rstd, gain64, None, eps32, rms)
        within(host(rstd), want_rstd, er, "rstd")
        if not rms:
            within(host(mean), want_mean, em, "mean")
        within(host(y), want, ey + HALF[dtype] * (np.abs(want) + ey), "y")
    assert torch.isfinite(y).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(5, 64), (5, 4096), (1030, 4104)])
def test_forward_beyond_the_range(rows, cols, dtype):
    # the average of the squares is beyond fp32: rstd is 0 and y the bias; the mean is in range up to the largest numbers
    import paper_2405_13954_amd as P
    g = np.random.default_rng([rows, cols])
    for size in (1e20, 1e37):
        x, x64 = rows_of(g, rows, cols, size, dtype, 6.0)
        bias, bias64 = vector(g, cols, 0.3, dtype)
        y, mean, rstd = room(rows, cols, dtype)[0], f32(rows), f32(rows)
        P.logra_layer_norm_forward(x, y, bias=bias, mean=mean, rstd=rstd)
        assert not rstd.any() and np.array_equal(host(y), np.broadcast_to(bias64, y.shape))
        within(host(mean), x64.mean(1), ROW * np.abs(x64).mean(1), "mean")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("rows,cols", [(5, 64), (5, 4096), (5, 16377), (1030, 768), (1030, 4104), (1030, 12296)])
def test_backward_of_rows_of_any_size(rows, cols, rms, dtype):
    # dy of 1e-6, which is what gradients are scaled to: rstd dy is a normal number of fp32 at either end, rstd^3 is not
    import torch
    import paper_2405_13954_amd as P
    g = np.random.default_rng([rows, cols, rms, 1])
    for size, eps in ((1.0, 1e-5), (1e15, 1e-5), (1e18, 1e-5), (1e19, 1e-5), (1e-14, 1e-30)):
        print("[norm range, backward]", rows, cols, dtype, rms, size, eps, flush=True)
        h, h64 = rows_of(g, rows, cols, size, dtype, 0.5)
        dy, dy64 = rows_of(g, rows, cols, 1e-6, dtype)
        gain, gain64 = vector(g, cols, 0.3, dtype, 1.0)
        _, mean64, rstd64 = O.norm_forward(h64, eps=eps, rms=rms)
        mean, rstd = (None if rms else torch.from_numpy(mean64).float().cuda()), torch.from_numpy(rstd64).float().cuda()
        mean64, rstd64 = (np.zeros(rows) if rms else host(mean)), host(rstd)
        dx, dgain, dbias = room(rows, cols, dtype)[0], f32(cols), (None if rms else f32(cols))
        P.logra_layer_norm_backward(h, dy, rstd, mean=mean, gain=gain, rms=rms, dx=dx, dgain=dgain, dbias=dbias)
        want, want_g, want_b = O.norm_backward(h64, dy64, mean64, rstd64, gain64, rms)
        xh, c = (h64 - mean64[:, None]) * rstd64[:, None], np.abs(dy64 * gain64)
        ex = U * (np.abs(h64) + np.abs(mean64)[:, None]) * rstd64[:, None]       # the rounding of h - mean
        along = np.mean(c * np.abs(xh), 1)[:, None]
        term = c + (0 if rms else np.mean(c, 1)[:, None]) + np.abs(xh) * along
        ed = rstd64[:, None] * ((ROW + 6 * U) * term + 2 * c * ex + np.mean(c * ex, 1)[:, None] * np.abs(xh) + ex * along)
        within(host(dx), want, ed + (HALF[dtype] + 2 * U) * np.abs(want), "dx")
        rows_u = (rows / 512 + 70) * U
        within(host(dgain), want_g, rows_u * np.sum(np.abs(dy64 * xh), 0) + np.sum(np.abs(dy64) * (ex + 3 * U * np.abs(xh)), 0), "dgain")
        if not rms:
            within(host(dbias), want_b, rows_u * np.sum(np.abs(dy64), 0), "dbias")


@pytest.mark.parametrize("rows,cols", [(5, 72), (1030, 4104)])
def test_backward_beyond_the_range(rows, cols):
    # rstd 0, as the forward pass leaves it: dx = base, and nothing for the gain
    import torch
    import paper_2405_13954_amd as P
    g = torch.Generator().manual_seed(cols)
    h = (torch.randn(rows, cols, generator=g) * 1e37).cuda()
    dy, base = torch.randn(rows, cols, generator=g).cuda(), torch.randn(rows, cols, generator=g).cuda()
    y, dx, mean, rstd, dgain = torch.empty_like(h), torch.empty_like(h), f32(rows), f32(rows), f32(cols)
    P.logra_layer_norm_forward(h, y, mean=mean, rstd=rstd)
    P.logra_layer_norm_backward(h, dy, rstd, mean=mean, dx=dx, base=base, dgain=dgain)
    assert not rstd.any() and torch.equal(dx, base) and not dgain.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(5, 75), (5, 1001), (5, 12289), (1030, 75), (1030, 1001), (1030, 4109), (1030, 12289)])
def test_backward_of_rows_far_from_zero_at_odd_widths(rows, cols, dtype):
    # rows of 2^123 and no variance: (h - mean) rstd is 0, while what lies behind a row's end, 0 - mean, times rstd is beyond fp32
    import torch
    import paper_2405_13954_amd as P
    g = np.random.default_rng(cols)
    h, _ = rows_of(g, rows, cols, 0.0, dtype)
    h[::2] = 2.0 ** 123
    dy, dy64 = rows_of(g, rows, cols, 1.0, dtype)
    mean, rstd = h[:, 0].float().contiguous(), torch.full((rows,), 300.0, device="cuda")
    dx, dgain, dbias = room(rows, cols, dtype)[0], f32(cols), f32(cols)
    P.logra_layer_norm_backward(h, dy, rstd, mean=mean, dx=dx, dgain=dgain, dbias=dbias)
    want = 300.0 * (dy64 - dy64.mean(1, keepdims=True))
    within(host(dx), want, 300.0 * ROW * (np.abs(dy64) + np.abs(dy64).mean(1, keepdims=True)) + (HALF[dtype] + 2 * U) * np.abs(want), "dx")
    assert not dgain.any() and bool(torch.isfinite(dbias).all())
