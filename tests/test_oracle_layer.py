"""The float64 oracle of projections, gated blocks and the norm and rotation of Q and K: gradients against central
differences, closed forms of the activations."""
import numpy as np
import pytest

from oracle import layer, token

ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu", "sigmoid"]


def diff(f, x, v, h=1e-6):
    return (f(x + h * v) - f(x - h * v)) / (2 * h)


@pytest.mark.parametrize("kind", ACTS)
def test_activations(kind):
    z = np.array([-30.0, -3.0, -0.7, 0.2, 1.0, 4.0, 30.0])
    a, d = layer.act(z, kind)
    np.testing.assert_allclose(d, (layer.act(z + 1e-6, kind)[0] - layer.act(z - 1e-6, kind)[0]) / 2e-6, atol=1e-8)
    far = {"sigmoid": (0.0, 1.0), "none": (-30.0, 30.0)}.get(kind, (0.0, 30.0))
    np.testing.assert_allclose(a[[0, -1]], far, atol=1e-10)
    if kind in ("gelu", "gelu_tanh"):
        np.testing.assert_allclose(a[4], 0.8413, atol=3e-4)


@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("adaptive", [False, True])
def test_linear_gradients(kind, adaptive):
    rng = np.random.default_rng(3)
    new = lambda *n: rng.normal(size=n)  # noqa: E731
    x, w, b, dy = new(2, 3, 4, 2), new(10, 6), new(10), new(2, 2, 4, 5)
    gate = new(2, 10) if adaptive else new(10)
    _, z = layer.linear(x, w, b, kind, gate)
    g = layer.linear_bwd(dy, x, w, z, kind, gate)
    loss = lambda x, w, b, gate: (layer.linear(x, w, b, kind, gate, dy)[0] * layer.flat(dy)).sum()  # noqa: E731
    for got, at, f in ((layer.unflat(g["dx"], 2, 3, 4, 2), x, lambda t: loss(t, w, b, gate)), (g["dw"], w, lambda t: loss(x, t, b, gate)),
                       (g["dbias"], b, lambda t: loss(x, w, t, gate)), (g["dgate"], gate, lambda t: loss(x, w, b, t))):
        v = new(*at.shape)
        assert abs((got * v).sum() - diff(f, at, v)) <= 1e-6 * (1 + abs((got * v).sum()))


@pytest.mark.parametrize("kind", ACTS)
def test_glu_gradients(kind):
    rng = np.random.default_rng(4)
    new = lambda *n: rng.normal(size=n)  # noqa: E731
    x, w, b, dy = new(2, 1, 3, 5), new(8, 5), new(8), new(2, 1, 3, 4)
    y, z = layer.glu(x, w, b, kind)
    want = layer.act(layer.flat(x) @ w[:4].T + b[:4], kind)[0] * (layer.flat(x) @ w[4:].T + b[4:])
    np.testing.assert_allclose(y, want, rtol=1e-12)
    g = layer.glu_bwd(dy, x, w, z, kind)
    loss = lambda x, w, b: (layer.glu(x, w, b, kind)[0] * layer.flat(dy)).sum()  # noqa: E731
    for got, at, f in ((layer.unflat(g["dx"], 2, 1, 3, 5), x, lambda t: loss(t, w, b)), (g["dw"], w, lambda t: loss(x, t, b)),
                       (g["dbias"], b, lambda t: loss(x, w, t))):
        v = new(*at.shape)
        assert abs((got * v).sum() - diff(f, at, v)) <= 1e-6 * (1 + abs((got * v).sum()))


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_qk_gradients(kind):
    rng = np.random.default_rng(5)
    x, dy, w = rng.normal(size=(2, 3, 4, 12)), rng.normal(size=(2, 3, 4, 12)), rng.normal(size=12)
    pos = rng.integers(0, 100, (2, 4, 2))
    turns, scale = token.rope_turns((4, 6))
    how = dict(kind=kind, eps=1e-3, plus_one=True, scale=1.5, layout="half")
    f = lambda x, w: (layer.qk_norm_rope(x, pos, turns, (4, 6), w, **how) * dy).sum()  # noqa: E731
    dx, dw = layer.qk_norm_rope_bwd(dy, x, pos, turns, (4, 6), w, **how)
    for got, at, g in ((dx, x, lambda t: f(t, w)), (dw, w, lambda t: f(x, t))):
        v = rng.normal(size=at.shape)
        assert abs((got * v).sum() - diff(g, at, v)) <= 1e-6 * (1 + abs((got * v).sum()))


def test_flat_and_back():
    x = np.arange(24.0).reshape(1, 2, 3, 4)
    np.testing.assert_array_equal(layer.flat(x)[1], [4, 5, 6, 7, 16, 17, 18, 19])
    np.testing.assert_array_equal(layer.unflat(layer.flat(x), 1, 2, 3, 4), x)
