"""The oracle of the layers beside the normalization, against hand values, closed forms, differences and plain loops."""

import math

import numpy as np
import pytest

from oracle import layers_oracle as Y

ACTS = ["none", "relu", "gelu", "silu"]


def _differences(f, a, step=1e-6):
    """Gradient of the number f(a) by central differences."""
    g = np.zeros_like(a)
    for i in np.ndindex(*a.shape):
        old = a[i]
        a[i] = old + step
        up = f(a)
        a[i] = old - step
        down = f(a)
        a[i] = old
        g[i] = (up - down) / (2 * step)
    return g


def test_activations_at_known_points():
    z = np.array([-1.0, 0.0, 2.0])
    assert np.allclose(Y.act(z, "relu"), [0, 0, 2])
    assert np.allclose(Y.act(z, "silu"), [-1 / (1 + math.e), 0, 2 / (1 + math.exp(-2))], rtol=1e-15)
    assert np.allclose(Y.act(z, "gelu"), [-0.15865525393145707, 0, 1.9544997361036416], rtol=1e-12)
    assert np.array_equal(Y.act(np.array([-800.0, 800.0]), "silu"), [-0.0, 800.0])


@pytest.mark.parametrize("name", ACTS)
def test_slopes_are_the_derivatives(name):
    z = np.array([-3.0, -1.2, -0.3, 0.2, 0.9, 4.0])
    d = (Y.act(z + 1e-6, name) - Y.act(z - 1e-6, name)) / 2e-6
    assert np.allclose(Y.act_slope(z, name), d, atol=1e-9)


@pytest.mark.parametrize("name", ACTS)
def test_linear_gradients(name):
    rng = np.random.default_rng(1)
    x, w, b, r, dy = (rng.standard_normal(s) for s in ((3, 4), (5, 4), (5,), (3, 5), (3, 5)))
    y, z = Y.linear_forward(x, w, b, r, name)
    for i in range(3):
        for j in range(5):
            assert z[i, j] == pytest.approx(math.fsum(x[i] * w[j]) + b[j] + r[i, j], rel=1e-13)
    back = Y.linear_backward(dy, x, w, y if name == "relu" else z, name)
    loss = lambda: float((Y.linear_forward(x, w, b, r, name)[0] * dy).sum())
    for grad, a in (("dx", x), ("dw", w), ("dbias", b), ("dresidual", r)):
        assert np.allclose(back[grad], _differences(lambda _: loss(), a), atol=2e-8), grad


@pytest.mark.parametrize("name", ACTS)
def test_gated_gradients(name):
    rng = np.random.default_rng(2)
    x, wg, wu, dh = (rng.standard_normal(s) for s in ((3, 4), (5, 4), (5, 4), (3, 5)))
    _, g, u = Y.gated_forward(x, wg, wu, name)
    back = Y.gated_backward(dh, x, wg, wu, g, u, name)
    loss = lambda: float((Y.gated_forward(x, wg, wu, name)[0] * dh).sum())
    for grad, a in (("dx", x), ("dwg", wg), ("dwu", wu)):
        assert np.allclose(back[grad], _differences(lambda _: loss(), a), atol=2e-8), grad


@pytest.mark.parametrize("style", ["halves", "interleaved"])
@pytest.mark.parametrize("D,R", [(6, 6), (7, 4), (5, 0)])
def test_head_norm_gradients(D, R, style):
    rng = np.random.default_rng(3)
    x, dy, w = rng.standard_normal((4, 2, D)), rng.standard_normal((4, 2, D)), rng.standard_normal(D)
    pos = np.array([3, 0, 8, 3])
    angle = np.arange(9)[:, None] * 10.0 ** (-np.arange(R // 2) / max(1, R // 2))
    args = (1e-3, pos, np.cos(angle), np.sin(angle), R, style)
    dx, dw = Y.head_norm_backward(dy, x, w, *args)
    loss = lambda: float((Y.head_norm_forward(x, w, *args) * dy).sum())
    assert np.allclose(dx, _differences(lambda _: loss(), x), atol=2e-8)
    assert np.allclose(dw, _differences(lambda _: loss(), w), atol=2e-8)


def test_rotation_keeps_lengths_and_adds_angles():
    rng = np.random.default_rng(4)
    x = rng.standard_normal((1, 1, 8))
    angle = np.arange(12)[:, None] * np.array([0.3, 0.1, 0.05])
    for style in ("halves", "interleaved"):
        turn = lambda v, p: Y.rotate(v, np.array([p]), np.cos(angle), np.sin(angle), 6, style)
        assert np.sum(turn(x, 5) ** 2) == pytest.approx(np.sum(x ** 2), rel=1e-14)
        assert np.allclose(turn(turn(x, 5), 6), turn(x, 11), atol=1e-14)
        assert np.array_equal(turn(x, 0), x) and np.array_equal(turn(x, 7)[..., 6:], x[..., 6:])
        # a product of a turned query and a turned key depends on the positions' difference alone
        k = rng.standard_normal((1, 1, 8))
        dot = lambda a, b: float((turn(x, a) * turn(k, b)).sum())
        assert dot(7, 4) == pytest.approx(dot(5, 2), rel=1e-13)


def test_head_norm_of_a_hand_example():
    # mean(x^2) = (9 + 16) / 4: the root is 2.5
    x = np.array([[[3.0, 4.0, 0.0, 0.0]]])
    y = Y.head_norm_forward(x, np.ones(4), 0.0, np.array([1]), np.array([[1.0], [0.0]]), np.array([[0.0], [1.0]]), 2, "halves")
    # a quarter turn of (1.2, 1.6)
    assert np.allclose(y, [[[-1.6, 1.2, 0, 0]]], atol=1e-15)
