"""Pins of the 64-bit cross-attention branch: closed forms, and its gradients against central differences."""
import numpy as np
import pytest

from oracle import branch


def rng(seed=0):
    return np.random.default_rng(seed)


def slope(f, x, direction, h=1e-5):
    """Central difference of the scalar f along a direction; its error is h^2 / 6 times the third derivative plus 1e-16 / h."""
    return (f(x + h * direction) - f(x - h * direction)) / (2 * h)


def agrees(f, x, grad, seed):
    g = rng(seed)
    for _ in range(3):
        d = g.standard_normal(x.shape)
        got, want = float((grad * d).sum()), slope(f, x, d)
        # sums of some hundred terms of order one, third derivatives of order ten
        assert abs(got - want) <= 1e-7 * (1 + abs(want)), (got, want)


@pytest.mark.parametrize("modulated", [False, True])
@pytest.mark.parametrize("per", [1, 3, 7])
def test_layer_norm_gradient(modulated, per):
    g = rng(1)
    x, w, b = g.standard_normal((7, 10)), g.standard_normal((-(-7 // per), 10)), g.standard_normal((-(-7 // per), 10))
    dy, res = g.standard_normal((7, 10)), g.standard_normal((7, 10))
    _, mean, rstd = branch.layer_norm(x, w, b, per, modulated, 1e-6)
    dx, dw, db = branch.layer_norm_grad(x, w, per, modulated, mean, rstd, dy, res)
    loss = lambda x, w, b: float((branch.layer_norm(x, w, b, per, modulated, 1e-6)[0] * dy).sum() + (x * res).sum())  # noqa: E731
    agrees(lambda t: loss(t, w, b), x, dx, 2)
    agrees(lambda t: loss(x, t, b), w, dw, 3)
    agrees(lambda t: loss(x, w, t), b, db, 4)


def test_layer_norm_closed_form():
    y, mean, rstd = branch.layer_norm([[1.0, 3.0]], [[2.0, 4.0]], [[1.0, 1.0]], 1, False, 1e-30)
    assert np.allclose(mean, 2) and np.allclose(rstd, 1) and np.allclose(y, [[-1, 5]])
    y, _, _ = branch.layer_norm([[1.0, 3.0]], [[2.0, 4.0]], None, 1, True, 1e-30)
    assert np.allclose(y, [[-3, 5]])


def test_cross_attention_closed_form():
    # equal keys: the mean of the values that count; an empty prompt: zeros and -inf
    q, k = rng(5).standard_normal((2, 3, 2, 4)), np.ones((2, 5, 1, 4))
    v = np.arange(40.0).reshape(2, 5, 1, 4)
    out, lse = branch.cross_attention(q, k, v, [1, 0], [0, 3])
    assert np.allclose(out[0], v[1, :3, 0].mean(0)) and np.allclose(lse[0], (q[0].sum(2) / 2 + np.log(3)).T)
    assert not out[1].any() and np.isneginf(lse[1]).all()
    # clamped lengths and indexes
    same = branch.cross_attention(q, k, v, [7, -1], [-4, 3])
    assert np.array_equal(same[0], out)


def test_cross_attention_gradient():
    g = rng(6)
    q, k, v = g.standard_normal((3, 4, 4, 8)), g.standard_normal((3, 5, 2, 8)), g.standard_normal((3, 5, 2, 8))
    index, lengths, dout = [2, 0, 2], [3, 5, 4], g.standard_normal((3, 4, 4, 8))
    out, lse = branch.cross_attention(q, k, v, index, lengths)
    dq, dk, dv = branch.cross_attention_grad(q, k, v, out, lse, dout, index, lengths)
    loss = lambda q, k, v: float((branch.cross_attention(q, k, v, index, lengths)[0] * dout).sum())  # noqa: E731
    agrees(lambda t: loss(t, k, v), q, dq, 7)
    agrees(lambda t: loss(q, t, v), k, dk, 8)
    agrees(lambda t: loss(q, k, t), v, dv, 9)
    assert not dk[1].any() and not dk[0, 3:].any() and not dv[2, 4:].any()


@pytest.mark.parametrize("per", [1, 2, 9])
def test_adapters_gradient(per):
    g = rng(10)
    x, down, up = g.standard_normal((9, 6)), g.standard_normal((3, 2, 6)), g.standard_normal((3, 5, 2))
    s, dy, res = g.standard_normal(3), g.standard_normal((9, 5)), g.standard_normal((9, 6))
    index = (np.arange(-(-9 // per)) * 2) % 4 - 1
    _, u = branch.adapters(x, down, up, s, index, per)
    dx, dd, du = branch.adapters_grad(x, down, up, u, dy, s, index, per, res)
    loss = lambda x, d, u: float((branch.adapters(x, d, u, s, index, per)[0] * dy).sum() + (x * res).sum())  # noqa: E731
    agrees(lambda t: loss(t, down, up), x, dx, 11)
    agrees(lambda t: loss(x, t, up), down, dd, 12)
    agrees(lambda t: loss(x, down, t), up, du, 13)


def test_adapters_closed_form():
    out, u = branch.adapters([[1.0, 2.0], [3.0, 4.0]], [[[1.0, 1.0]]], [[[2.0], [3.0]]], [0.5], [0, -1], 1,
                             [[1.0, 1.0], [1.0, 1.0]], [1.0, 2.0])
    assert np.allclose(u, [[3], [0]]) and np.allclose(out, [[4, 10], [1, 1]])
