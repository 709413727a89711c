"""Pins of the float64 oracle of the layer norm, the preference loss and the AdamW step: worked cases, gradients against
differences, the 8-bit types against torch's, the rounding's mean.  CPU only."""
import numpy as np
import pytest

from oracle import tuning as O


def test_norm_worked_example():
    # rows (1, 3) and (0, 0): mean 2 and 0, variance 1 and 0
    h = np.array([[1.0, 3.0], [0.0, 0.0], [5.0, 5.0]])
    y, mean, rstd = O.norm_forward(h, np.array([2.0, 4.0]), np.array([10.0, 20.0]), eps=3.0)
    assert mean.tolist() == [2.0, 0.0, 5.0] and rstd[0] == 0.5 and abs(rstd[1] - 3 ** -0.5) < 1e-15
    assert y[0].tolist() == [9.0, 22.0] and y[1].tolist() == [10.0, 20.0] and y[2].tolist() == [10.0, 20.0]
    y, mean, rstd = O.norm_forward(np.array([[3.0, 4.0]]), eps=12.5 * 3, rms=True)      # mean square 12.5
    assert mean[0] == 0 and abs(rstd[0] - 50 ** -0.5) < 1e-16 and np.allclose(y, [[3 / 50 ** 0.5, 4 / 50 ** 0.5]])
    y, _, rstd = O.norm_forward(np.array([[np.nan, 1.0], [1.0, 2.0]]), mask=[0, 1])
    assert y[0].tolist() == [0, 0] and rstd[0] == 0 and np.isfinite(y[1]).all()


@pytest.mark.parametrize("rms", [False, True])
def test_norm_gradients_against_differences(rms):
    g = np.random.default_rng(1)
    h, dy, gain = g.standard_normal((4, 9)), g.standard_normal((4, 9)), g.standard_normal(9)
    bias, base, mask = (None if rms else g.standard_normal(9)), g.standard_normal((4, 9)), np.array([1, 0, 1, 1])
    _, mean, rstd = O.norm_forward(h, gain, bias, 1e-3, rms, mask)
    dx, dgain, dbias = O.norm_backward(h, dy, mean, rstd, gain, rms, mask, base)

    def total(h, gain, bias):
        return np.sum(O.norm_forward(h, gain, bias, 1e-3, rms, mask)[0] * dy)

    e = 1e-6
    for at in np.ndindex(h.shape):
        step = np.zeros_like(h)
        step[at] = e
        want = (total(h + step, gain, bias) - total(h - step, gain, bias)) / (2 * e) + base[at]
        assert abs(dx[at] - want) < 1e-7
    for j in range(9):
        step = np.zeros(9)
        step[j] = e
        assert abs(dgain[j] - (total(h, gain + step, bias) - total(h, gain - step, bias)) / (2 * e)) < 1e-7
        if not rms:
            assert abs(dbias[j] - (total(h, gain, bias + step) - total(h, gain, bias - step)) / (2 * e)) < 1e-7


def test_preference_loss_worked_example_and_special_cases():
    # two tokens of two logits: lp = log(3/4) and log(1/2), each alone in its sequence
    z = np.log(np.array([[3.0, 1.0], [1.0, 1.0]]))
    loss, logp, dz = O.preference_loss(z, [0, 1], [0, 1, 2], beta=2.0)
    assert np.allclose(logp, np.log([0.75, 0.5]))
    # d = 2 log(3/2): exp(-d) = 4/9, loss = log(13/9), sigma(-d) = 4/13, slope = -8/13
    assert np.isclose(loss[0], np.log(13 / 9))
    assert np.allclose(dz, (-8 / 13) * np.array([[0.25, -0.25], [0.5, -0.5]]))
    # the frozen model's own ratios: d = 0, loss log 2
    assert np.isclose(O.preference_loss(z, [0, 1], [0, 1, 2], ref=logp)[0][0], np.log(2))
    # swapped pairs with the label smoothed by 1 are the same loss
    a = O.preference_loss(z, [0, 1], [0, 1, 2], ref=[0.3, -0.2], beta=0.7, smoothing=0.2)
    b = O.preference_loss(z[::-1], [1, 0], [0, 1, 2], ref=[-0.2, 0.3], beta=0.7, smoothing=0.8)
    assert np.isclose(a[0][0], b[0][0]) and np.allclose(a[2], b[2][::-1])
    # empty sequences, masked tokens, weight zero
    loss, logp, dz = O.preference_loss(np.full((3, 2), np.nan), [-1, 2, 0], [1, 1, 2], beta=1.0)
    assert np.isclose(loss[0], np.log(2)) and logp.tolist() == [0, 0] and not dz.any()
    assert not O.preference_loss(z, [0, 1], [0, 1, 2], weight=[0.0])[2].any()


def test_preference_gradient_against_differences():
    g = np.random.default_rng(2)
    z, target, offsets = g.standard_normal((9, 5)), g.integers(-1, 5, 9), [0, 2, 2, 5, 8]
    ref, weight = g.standard_normal(4), np.array([0.5, 2.0])
    kw = dict(ref=ref, weight=weight, beta=0.6, smoothing=0.1)
    dz = O.preference_loss(z, target, offsets, **kw)[2]
    for at in np.ndindex(z.shape):
        step = np.zeros_like(z)
        step[at] = 1e-6
        up, down = (np.sum(O.preference_loss(z + s * step, target, offsets, **kw)[0]) for s in (1, -1))
        assert abs(dz[at] - (up - down) / 2e-6) < 1e-8


def test_eight_bit_types_are_torchs():
    import torch
    for kind, dtype in ((O.E4M3, torch.float8_e4m3fn), (O.E5M2, torch.float8_e5m2)):
        every = torch.arange(128, dtype=torch.uint8).view(dtype).double()
        every = every[torch.isfinite(every)].numpy()
        assert np.array_equal(every, O.values_of(kind)) and every[-1] == torch.finfo(dtype).max


def test_block_scales():
    for kind, top in ((O.E4M3, 448.0), (O.E5M2, 57344.0)):
        assert O.block_scale(np.array([0.0, -0.0]), kind) == 1.0
        for k in (-20, -1, 0, 3):
            assert O.block_scale(np.array([1e-30, -top * 2.0 ** k]), kind) == 2.0 ** k
            assert O.block_scale(np.array([np.nextafter(top * 2.0 ** k, np.inf)]), kind) == 2.0 ** (k + 1)
        assert O.block_scale(np.array([1e-44]), kind) == 2.0 ** -126
        assert O.block_scale(np.array([np.inf, 1.0, np.nan]), kind) == O.block_scale(np.array([1.0]), kind)


def test_rounding_at_random_is_unbiased():
    # over all draws: the mean is the value, up to the draw's own steps of 2^-16 of the distance between neighbours
    draws = np.arange(65536)
    for kind in (O.E4M3, O.E5M2):
        grid = O.values_of(kind)
        for v in (0.3, 1.0, 1.0625, 17.3, 2.0 ** -7 * 1.1, 3e-4):
            got = np.abs(O.round_at_random(np.full(65536, -v), 1.0, kind, draws, False))
            gap = np.diff(grid[np.searchsorted(grid, v, side="right") - 1:][:2])[0]
            assert abs(got.mean() - v) <= gap / 65536 and len(np.unique(got)) <= 2
    assert O.round_at_random(np.array([1e-12]), 1.0, O.E5M2, [65535], True)[0] == 2.0 ** -16
    assert O.round_at_random(np.array([0.0]), 1.0, O.E5M2, [0], True)[0] == 0.0


def test_adamw_first_step_and_decay():
    # from zero states the first step moves by lr against the gradient's sign, whatever its size
    x = dict(param=np.array([[1.0, 2.0, 3.0]]), grad=np.array([[5.0, -0.1, 0.0]]), m=np.zeros((1, 3)), v=np.zeros((1, 3)),
             first_group=0, decay=True, bits=32)
    (y,), norms = O.adamw_step([x], 1, 0, 0.1, eps=1e-30, weight_decay=0.5)
    assert np.allclose(y["param"], [[0.95 - 0.1, 1.9 + 0.1, 2.85]]) and np.isclose(norms[0], np.sqrt(25.01))
    (y,), _ = O.adamw_step([dict(x, decay=False)], 1, 0, 0.1, eps=1e-30, weight_decay=0.5)
    assert np.allclose(y["param"], [[0.9, 2.1, 3.0]])


def test_adamw_against_torch():
    import torch
    g = np.random.default_rng(3)
    p = g.standard_normal((2, 40))
    t = torch.tensor(p.copy(), requires_grad=True)
    opt = torch.optim.AdamW([t], lr=0.01, betas=(0.8, 0.95), eps=1e-3, weight_decay=0.1)
    x = dict(param=p, m=np.zeros_like(p), v=np.zeros_like(p), first_group=0, decay=True, bits=32)
    for k in range(5):
        grad = g.standard_normal((2, 40))
        t.grad = torch.tensor(grad)
        opt.step()
        (y,), _ = O.adamw_step([dict(x, grad=grad)], 2, k, 0.01, 0.8, 0.95, 1e-3, 0.1)
        x.update(y)
        assert np.allclose(x["param"], t.detach().numpy(), rtol=0, atol=1e-14)


def test_adamw_groups_are_models_of_their_own():
    g = np.random.default_rng(4)
    mk = lambda s, n: dict(param=g.standard_normal((s, n)), grad=g.standard_normal((s, n)), m=np.zeros((s, n)),  # noqa: E731
                           v=np.zeros((s, n)), decay=True, bits=32)
    a, b = dict(mk(3, 7), first_group=0), dict(mk(2, 5), first_group=1)
    scale = np.array([1.0, 0.5, 2.0])
    both, norms = O.adamw_step([a, b], 3, 4, 0.1, max_norm=2.0, lr_scale=scale)
    for group in range(3):
        alone = [dict({k: v[s:s + 1] for k, v in x.items() if isinstance(v, np.ndarray)}, first_group=0, decay=True, bits=32)
                 for x, s in ((a, group), (b, group - 1)) if 0 <= s < x["param"].shape[0]]
        one, norm = O.adamw_step(alone, 1, 4, 0.1 * scale[group], max_norm=2.0)
        assert np.isclose(norm[0], norms[group])
        assert np.allclose(one[0]["param"][0], both[0]["param"][group])
        if group:
            assert np.allclose(one[1]["param"][0], both[1]["param"][group - 1])
    # a group whose gradient is not finite stays, when norms are taken
    a["grad"][1, 3] = np.nan
    some, _ = O.adamw_step([a, b], 3, 4, 0.1, max_norm=2.0)
    assert np.array_equal(some[0]["param"][1], a["param"][1]) and np.array_equal(some[1]["param"][0], b["param"][0])
    assert not np.array_equal(some[0]["param"][0], a["param"][0])
