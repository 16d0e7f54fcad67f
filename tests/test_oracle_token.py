"""The float64 token operators of the oracle against differences, identities and closed forms."""
import math

import numpy as np
import pytest

from oracle import token


def _directional(f, x, v, h=1e-5):
    return (f(x + h * v) - f(x - h * v)) / (2 * h)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("adaptive", [False, True])
def test_norm_gradients_against_differences(kind, adaptive):
    rng = np.random.default_rng(0)
    B, H, N, C = 2, 2, 3, 7
    x, dy = rng.normal(size=(2, B, H, N, C)) + 0.3
    w, b = rng.normal(size=(2,) + ((B, C) if adaptive else (C,)))
    y, mean, rstd = token.norm(x, w, b, kind, 1e-3, True)
    dx, dw, db = token.norm_bwd(dy, x, mean, rstd, w, kind, True, adaptive)
    for grad, at, f in ((dx, x, lambda t: (dy * token.norm(t, w, b, kind, 1e-3, True)[0]).sum()),
                        (dw, w, lambda t: (dy * token.norm(x, t, b, kind, 1e-3, True)[0]).sum()),
                        (db, b, lambda t: (dy * token.norm(x, w, t, kind, 1e-3, True)[0]).sum())):
        v = rng.normal(size=at.shape)
        assert abs(_directional(f, at, v) - (grad * v).sum()) < 1e-7


def test_norm_of_known_rows():
    y, mean, rstd = token.norm(np.array([[[[1.0, 3.0]]]]), eps=0.0)
    assert y.tolist() == [[[[-1.0, 1.0]]]] and mean == 2.0 and rstd == 1.0
    y, mean, rstd = token.norm(np.array([[[[3.0, 4.0]]]]), kind="rms", eps=0.0)
    np.testing.assert_allclose(y[0, 0, 0], np.array([3, 4]) / math.sqrt(12.5), rtol=1e-15)


@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_rope_turns_pairs_and_depends_on_distance(layout):
    rng = np.random.default_rng(1)
    turns, scale = token.rope_turns((4, 2, 2))
    assert scale == 1.0 and turns.shape == (4,)
    np.testing.assert_allclose(turns * 2 * math.pi, [1.0, 0.01, 1.0, 1.0])
    q, k = rng.normal(size=(2, 1, 1, 1, 12))
    dots = []
    for shift in (0, 5, 1000):
        p = np.array([[[7, 2, 3]]]) + shift
        r = np.array([[[1, 9, 4]]]) + shift
        a = token.rope(q, p, turns, (4, 2, 2), 1.0, layout, 12)
        b = token.rope(k, r, turns, (4, 2, 2), 1.0, layout, 12)
        dots.append((a * b).sum())
        np.testing.assert_array_equal(a[..., 8:], q[..., 8:])
        back = token.rope(a, p, turns, (4, 2, 2), 1.0, layout, 12, inverse=True)
        np.testing.assert_allclose(back, q, atol=1e-14)
    np.testing.assert_allclose(dots, dots[0], atol=1e-10)


def test_rope_scalings():
    plain, _ = token.rope_turns((64,))
    lin, s = token.rope_turns((64,), scaling="linear", factor=4.0)
    np.testing.assert_allclose(lin, plain / 4)
    ntk, _ = token.rope_turns((64,), scaling="ntk", factor=4.0)
    # the first pair keeps its frequency, the last is stretched by the factor
    assert ntk[0] == plain[0]
    np.testing.assert_allclose(ntk[-1], plain[-1] / 4, rtol=1e-12)
    yarn, s = token.rope_turns((64,), scaling="yarn", factor=4.0)
    assert s == 0.1 * math.log(4.0) + 1.0
    np.testing.assert_allclose(yarn[0], plain[0])
    np.testing.assert_allclose(yarn[-1], plain[-1] / 4)
    assert ((yarn <= plain * (1 + 1e-15)) & (yarn >= plain / 4 * (1 - 1e-15))).all()


@pytest.mark.parametrize("causal", [False, True])
def test_diff_gradients_against_differences(causal):
    rng = np.random.default_rng(2)
    B, H, Hk, N, M, d = 2, 4, 2, 3, 5, 4
    Q, dO = rng.normal(size=(2, B, H, N, d))
    K, V = rng.normal(size=(2, B, Hk, M, d))
    lam = rng.uniform(0.2, 0.8, H)
    args = ([5, 2], [2, -1], causal)
    out = token.diff_attn(Q, K, V, lam, *args, dO=dO)
    for grad, at, f in (("dQ", Q, lambda t: token.diff_attn(t, K, V, lam, *args)["O"]),
                        ("dK", K, lambda t: token.diff_attn(Q, t, V, lam, *args)["O"]),
                        ("dV", V, lambda t: token.diff_attn(Q, K, t, lam, *args)["O"]),
                        ("dlam", lam, lambda t: token.diff_attn(Q, K, V, t, *args)["O"])):
        v = rng.normal(size=at.shape)
        assert abs(_directional(lambda t: (dO * f(t)).sum(), at, v) - (out[grad] * v).sum()) < 1e-7, grad


def test_diff_rows_that_see_nothing_and_uniform_maps():
    V = np.arange(8.0).reshape(1, 1, 2, 4)
    zero = np.zeros((1, 1, 3, 4))
    out = token.diff_attn(zero, np.zeros((1, 1, 2, 4)), V, [0.25], [2], [-2], True)
    np.testing.assert_array_equal(out["O"][0, 0, :2], 0)
    assert np.isneginf(out["lse"][0, 0, :, :2]).all()
    np.testing.assert_allclose(out["O"][0, 0, 2], V[0, 0, 0] * 0.75)
    out = token.diff_attn(zero, np.zeros((1, 1, 2, 4)), V, [0.25], [2], [0], False)
    np.testing.assert_allclose(out["O"][0, 0], np.broadcast_to(V[0, 0].mean(0) * 0.75, (3, 4)))
    np.testing.assert_allclose(out["lse"], math.log(2))
