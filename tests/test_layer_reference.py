"""The 64-bit statements that the GPU tests compare with, against differences of the functions themselves and worked examples."""
import numpy as np
import pytest

import layer_reference as ref


def differences(f, x, step=1e-5):
    d = np.zeros(x.shape)
    for i in np.ndindex(*x.shape):
        up, down = x.copy(), x.copy()
        up[i] += step
        down[i] -= step
        d[i] = (f(up) - f(down)) / (2 * step)
    return d


def test_integers_of_a_worked_row():
    q, s = ref.quantise(np.array([[127.0, 0.5, 1.5, -2.5, -126.6], [0, 0, 0, 0, 0], [1, np.inf, 0, 0, 0]]))
    assert q[0].tolist() == [127, 0, 2, -2, -127] and s[0] == 1.0
    assert q[1].tolist() == [0] * 5 and s[1] == 1.0 and np.isnan(s[2]) and q[2].tolist() == [0] * 5


@pytest.mark.parametrize("affine", [True, False])
def test_the_norms_gradient_is_that_of_the_norm(affine):
    rng = np.random.default_rng(3)
    x, g, w, b = rng.normal(size=(4, 9)), rng.normal(size=(4, 9)), rng.normal(size=9), rng.normal(size=9)
    if not affine:
        w = b = None

    def loss(x_, w_, b_):
        return (ref.norm(x_, w_, b_, 1e-3, 0)[0] * g).sum()

    _, mean, r, _, _, _ = ref.norm(x, w, b, 1e-3, 0)
    dx, dw, db, _, _, _ = ref.norm_gradient(g, x, mean, r, w, 0, 0)
    assert np.abs(dx - differences(lambda v: loss(v, w, b), x)).max() < 1e-7
    if affine:
        assert np.abs(dw - differences(lambda v: loss(x, v, b), w)).max() < 1e-7
        assert np.abs(db - differences(lambda v: loss(x, w, v), b)).max() < 1e-7


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_the_balances_gradient_is_that_of_the_loss(kind):
    rng = np.random.default_rng(4)
    logits = rng.normal(size=(6, 5))
    ids = rng.integers(-1, 5, size=(6, 2))
    logits[2, 1] = -np.inf
    logits[3] = -np.inf
    loss, counts, push, p, s, seen, _ = ref.balance(logits, ids, kind, 0.5)
    d = ref.balance_gradient(p, s, seen, push, kind)
    want = np.zeros_like(d)
    for i in np.ndindex(*d.shape):
        if np.isfinite(logits[i]):
            moved = [logits.copy(), logits.copy()]
            moved[0][i] += 1e-5
            moved[1][i] -= 1e-5
            want[i] = (ref.balance(moved[0], ids, kind, 0.5)[0] - ref.balance(moved[1], ids, kind, 0.5)[0]) / 2e-5
    assert np.abs(d - want).max() < 1e-8
    assert counts.sum() == (ids >= 0).sum()


def test_an_even_balance_costs_its_factor():
    logits = np.zeros((8, 4))
    ids = np.arange(8)[:, None] % 4
    assert abs(ref.balance(logits, ids, "softmax", 0.25)[0] - 0.25) < 1e-12
