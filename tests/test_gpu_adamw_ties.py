"""8-bit states whose value lies on the very boundary that its random bits set: the codes are those of the formula in float64,
each product and sum rounded by itself, as the oracle computes them.

With beta = 0.9 the sum 0.9 m + 0.1 g of a code and a gradient of few digits is in decimal arithmetic exactly r / 65536 of the way
to the next value for gradients g = 10 x - 9 m, which fp32 holds.  In float64, where neither 0.9 nor 0.1 is exact, the last bit decides.
"""
import numpy as np
import pytest

from oracle import tuning as O
from tuning_util import host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("clip", [False, True])
def test_sums_on_the_boundary_of_their_random_bits(clip):
    import torch
    import paper_2405_13954_amd as P
    n, seed, at, b1, b2 = 256 * 40, 77, 5, 0.9, 0.95
    g = np.random.default_rng(2)
    for_m, _ = O.adamw_draws(n, 0, 0, at + 1, seed)
    # old codes -30 .. 30, scale 1; new values 8 .. 15 of steps of 1 (16 .. 30 of steps of 2), a largest one of 448 in each block
    old = g.choice([-30.0, -22, -15, -9, 9, 15, 22, 30], n)
    step = g.choice([1.0, 2.0], n)
    x = np.copysign((g.integers(8, 15, n) + for_m / 65536.0) * step, old)
    grad = 10 * x - 9 * old
    grad[::256] = 10 * 448 - 9 * old[::256]
    grad = grad.astype(np.float32).astype(np.float64)
    on = np.abs(0.9 * old + 0.1 * grad - x) < 1e-12
    assert on.sum() > 0.9 * n                                       # (what fp32 does not hold is off the boundary)
    m, v = torch.from_numpy(old).to(torch.float8_e4m3fn).cuda(), torch.zeros(n).to(torch.float8_e5m2).cuda()
    ms, vs = torch.ones(40, device="cuda"), torch.ones(40, device="cuda")
    param, dev = torch.zeros(n, device="cuda"), torch.from_numpy(grad).float().cuda()
    count = torch.full((1,), at, dtype=torch.int64, device="cuda")
    plan = P.logra_adamw_plan([P.AdamwTensor(param, dev, m, v, ms, vs)], 1)
    # a limit that the norm is below, so that nothing is scaled, in the way through the norms
    P.logra_adamw_step(plan, count, 1e-3, beta1=b1, beta2=b2, max_norm=1e9 if clip else 0.0, seed=seed)
    one = dict(param=np.zeros((1, n)), grad=grad[None], m=old[None], v=np.zeros((1, n)), m_scale=np.ones((1, 40)), v_scale=np.ones((1, 40)),
               first_group=0, decay=False, bits=8)
    (want,), _ = O.adamw_step([one], 1, at, 1e-3, b1, b2, seed=seed)
    assert np.array_equal(host(ms), want["m_scale"][0]) and np.array_equal(host(vs), want["v_scale"][0])
    got = host(m) * np.repeat(host(ms), 256)
    bad = got != want["m"][0]
    assert not bad.any(), (int(bad.sum()), int((bad & on).sum()))
    assert np.array_equal(host(v) * np.repeat(host(vs), 256), want["v"][0])
    up = np.abs(got[on]) > np.abs(x[on])
    assert 0.05 < up.mean() < 0.95                                  # the boundary falls on both sides
