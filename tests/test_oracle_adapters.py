"""Pins of the float64 oracle of the adapters, the dropout and the token loss: published generator outputs, special
cases that reduce to a plain product, and gradients against differences.  CPU only."""
import numpy as np
import pytest

from oracle import adapters as O


def test_philox_known_answers():
    # the generator's published test vectors (all-zero and all-one inputs, 10 and 7 rounds)
    ones = 0xFFFFFFFF
    assert O.philox4x32((0,) * 4, (0, 0), 10) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert O.philox4x32((ones,) * 4, (ones, ones), 10) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert O.philox4x32((0,) * 4, (0, 0), 7) == [0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48]


def test_drop_factor_rate_and_independence():
    f = O.drop_factor(64, 257, 0.25, 5, 9)
    assert set(np.unique(f)) == {0.0, 65536.0 / (65536 - 16384)}
    # 16,448 draws: the kept share is within five standard deviations of 3/4
    assert abs((f > 0).mean() - 0.75) < 5 * np.sqrt(0.75 * 0.25 / f.size)
    for other in (O.drop_factor(64, 257, 0.25, 6, 9), O.drop_factor(64, 257, 0.25, 5, 10),
                  O.drop_factor(64, 257, 0.25, 5 | 1 << 40, 9), O.drop_factor(64, 257, 0.25, 5, 9 | 1 << 40)):
        same = ((f > 0) == (other > 0)).mean()
        assert abs(same - (0.75 ** 2 + 0.25 ** 2)) < 5 * np.sqrt(0.25 / f.size)
    # a prefix of the columns and of the rows has the prefix's mask
    assert np.array_equal(O.drop_factor(7, 100, 0.25, 5, 9), f[:7, :100])
    assert np.all(O.drop_factor(3, 5, 0.0, 5, 9) == 1.0)


def _case(seed=0):
    g = np.random.default_rng(seed)
    rows, n_in, n_out, rank, n = 11, 8, 12, 3, 3
    ids = np.array([0, 2, 2, -1, 0, 0, 7, 2, 0, 2, 0])     # adapter 1 has no row; -1 and 7 are none
    mk = lambda *s: g.standard_normal(s)  # noqa: E731
    return dict(x=mk(rows, n_in), a=mk(n, rank, n_in), b=mk(n, rank, n_out), ids=ids, base=mk(rows, n_out),
                scale=g.uniform(0.5, 2.0, n), f=O.drop_factor(rows, n_in, 0.3, 1, 2)), mk(rows, n_out), mk(rows, n_in)


def test_one_adapter_is_a_matrix_product():
    c, _, _ = _case()
    y, u, _, _ = O.adapter_forward(c["x"], c["a"][:1], c["b"][:1], np.zeros(11, int))
    assert np.allclose(u, c["x"] @ c["a"][0].T, atol=1e-14)
    assert np.allclose(y, c["x"] @ c["a"][0].T @ c["b"][0], atol=1e-13)


def test_rows_without_an_adapter_pass_through():
    c, dy, back = _case()
    c["x"][3] = np.nan
    y, u, _, _ = O.adapter_forward(**c)
    assert np.array_equal(y[[3, 6]], c["base"][[3, 6]]) and np.all(u[[3, 6]] == 0)
    dy[3] = np.nan
    (da, db, dx), _ = O.adapter_backward(c["x"], dy, c["a"], c["b"], c["ids"], u, back, c["scale"], c["f"])
    assert np.array_equal(dx[[3, 6]], back[[3, 6]]) and np.all(da[1] == 0) and np.all(db[1] == 0)
    assert np.all(np.isfinite(da)) and np.all(np.isfinite(db))


@pytest.mark.parametrize("what", ["a", "b", "x"])
def test_adapter_gradients_against_differences(what):
    # y is linear in each of a, b, x: a central difference is exact to rounding
    c, dy, _ = _case(3)
    _, u, _, _ = O.adapter_forward(**c)
    grads, _ = O.adapter_backward(c["x"], dy, c["a"], c["b"], c["ids"], u, None, c["scale"], c["f"])
    got = dict(zip(("a", "b", "x"), grads))[what]
    for _ in range(4):
        e = np.random.default_rng(_).standard_normal(c[what].shape)
        hi, lo = (O.adapter_forward(**{**c, what: c[what] + k * e})[0] for k in (0.5, -0.5))
        assert abs(((hi - lo) * dy).sum() - (got * e).sum()) < 1e-11


def test_token_loss_against_differences_and_hand():
    loss, grad = O.token_loss(np.log(np.array([[1.0, 2.0, 5.0]])), [1], [2.0])
    assert np.allclose(loss, 2 * np.log(4.0)) and np.allclose(grad, [[0.25, 0.5 - 2, 1.25]])
    g = np.random.default_rng(0)
    z, t, w = g.standard_normal((5, 9)), np.array([0, 8, -1, 9, 4]), np.array([1.0, 0.5, 1.0, 1.0, 0.0])
    loss, grad = O.token_loss(z, t, w)
    assert np.all(loss[2:] == 0) and np.all(grad[2:] == 0)
    e, h = g.standard_normal(z.shape), 1e-5
    hi, lo = O.token_loss(z + h * e, t, w)[0], O.token_loss(z - h * e, t, w)[0]
    assert np.allclose((hi - lo) / (2 * h), (grad * e).sum(1), atol=1e-9)
    loss, grad = O.token_loss(np.full((1, 4), -np.inf), [2])
    assert loss[0] == np.inf and np.all(grad == 0)
