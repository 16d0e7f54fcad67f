"""Gradients of projections and gated blocks in fp16 where the gradients of the sums dZ leave that type's range: below its
subnormal numbers and above its largest, while the results are inside.

Tolerances as in test_gpu_product, but for the rounding of dZ: half a step of itself wherever it lies, or 2^-39 of the largest
dZ (which is brought to [2^14, 2^15), where 2^-25 is half a step of the smallest numbers; of a projection that is the largest
1.2 dY gate); up to 16 tokens in two numbers."""
import numpy as np
import pytest
import torch

from oracle import layer
from paper_2609_32628_amd import api
from test_gpu_product import Case, f64, half, tiny

pytestmark = pytest.mark.gpu
MOST = torch.finfo(torch.float16).max


def close(got, want, bound, what):
    """Values that fp16 holds within the bound and their rounding; those whose exact value is past its largest may be infinite."""
    t, got = got.dtype, f64(got)
    tol = bound + half(t) * (np.abs(want) + bound) + tiny(t)
    near = (np.abs(got - want) <= tol) | ((np.abs(want) + tol >= MOST) & (got * np.sign(want) >= np.minimum(np.abs(want), MOST) - tol))
    assert near.all(), (what, got[~near][:9], want[~near][:9])


def check(c):
    t, M = torch.float16, c.B * c.N
    c.outputs()
    dbias, c.dbias = c.dbias, None
    c.run()
    x, w = f64(c.X), f64(c.W)
    Z = f64(c.Z).reshape(M, 2 if c.glu else 1, -1)[:, :, :c.F].reshape(M, -1)
    dy = np.abs(layer.flat(f64(c.dY)))
    if c.glu:
        g = layer.glu_bwd(f64(c.dY), x, w, Z, c.act)
        ed = np.concatenate([2.0 ** -15 * dy * np.abs(Z[:, c.F:]), 2.0 ** -16 * dy * np.abs(layer.act(Z[:, :c.F], c.act)[0])], 1)
    else:
        g = layer.linear_bwd(f64(c.dY), x, w, Z, c.act, f64(c.gate))
        ed = 2.0 ** -15 * dy * np.abs(layer.rows_gate(f64(c.gate), c.B, c.N))
    dz = np.abs(g["dz"])
    largest = dz.max() if c.glu else 1.2 * 2.0 ** 15 * ed.max()
    er = ed + half(t) ** (2 if M <= 16 else 1) * (dz + ed) + 2.0 ** -39 * largest
    mag = dz + er
    X = np.abs(layer.flat(x))
    close(c.dX, layer.unflat(g["dx"], *c.dX.shape), layer.unflat(er @ np.abs(w) + (w.shape[0] / 16 + 24) * 2.0 ** -23 * (mag @ np.abs(w)), *c.dX.shape), "dX")
    close(c.dW, g["dw"], er.T @ X + (M / 16 + c.B + 40) * 2.0 ** -23 * (mag.T @ X), "dW")
    if c.gate is not None:
        t1 = dy * np.abs(layer.act(Z, c.act)[0])
        per = lambda v: v.reshape(c.B, c.N, c.F).sum(1) if c.gate.dim() == 2 else v.sum(0)  # noqa: E731
        close(c.dgate, g["dgate"], (2.0 ** -16 + (M + 16) * 2.0 ** -24) * per(t1), "dgate")
    return dz, g


ROWS = [(1, 1), (5, 1), (1, 16), (2, 20), (3, 301), (1, 4000)]


@pytest.mark.parametrize("B,N", ROWS)
@pytest.mark.parametrize("K,F", [(64, 2000), (200, 136)])
def test_below_the_smallest(B, N, K, F):
    """dZ of about 2^-26, which sum up to results of 2^-20 and more."""
    c = Case(B, N, K, F, "fp16", "gelu", gate="adaptive", residual=True, scale=8.0, dscale=2.0 ** -13)
    c.gate *= 2.0 ** -13
    dz, g = check(c)
    assert dz.max() < 2.0 ** -18 and np.median(dz) < 2.0 ** -25
    c = Case(B, N, K, F, "fp16", "silu", glu=True, scale=2.0 ** -11, dscale=2.0 ** -14)
    dz, g = check(c)
    assert dz.max() < 2.0 ** -18 and np.median(dz) < 2.0 ** -25


@pytest.mark.parametrize("B,N", ROWS)
@pytest.mark.parametrize("K,F", [(64, 2000), (200, 136)])
def test_above_the_largest(B, N, K, F):
    """dZ of up to 2^19, whose products with small rows of W and X are finite, but for some of dW over 4,000 tokens: a sum of 4,000
    products of about 2^16 and 2^-9 has a deviation of 2^13, and of 10^5 such sums the largest pass fp16's 65,504 themselves."""
    c = Case(B, N, K, F, "fp16", "gelu", gate="shared", scale=2.0 ** -8, dscale=2.0 ** 13)
    c.gate *= 16
    c.X *= 2.0 ** -9
    dz, g = check(c)
    assert 2.0 ** 16 < dz.max() and np.abs(g["dx"]).max() < 60000 and (np.abs(g["dw"]) < 60000).mean() > 0.99
    c = Case(B, N, K, F, "fp16", "silu", glu=True, bias=True, scale=2.0 ** -8, dscale=2.0 ** 13)
    c.bias[:F] = 2.0
    c.bias[F:] = 16.0
    c.X *= 2.0 ** -9
    dz, g = check(c)
    assert 2.0 ** 16 < dz.max() and np.abs(g["dx"]).max() < 60000 and (np.abs(g["dw"]) < 60000).mean() > 0.99


def test_not_a_number_and_infinities_do_not_move_the_others():
    """What is not finite stays in its rows of dX and columns of dW, and the others are what they are without it, to the rounding
    of dZ."""
    c = Case(1, 60, 64, 136, "fp16", "silu", gate="shared", dscale=2.0 ** -14)
    c.gate *= 2.0 ** -12
    check(c)
    dX, dW = c.dX.clone(), c.dW.clone()
    c.dY[0, 0, 7, 3] = float("nan")
    c.dY[0, 0, 9, 5] = float("inf")
    c.run()
    rows = [n for n in range(60) if n not in (7, 9)]
    cols = [f for f in range(136) if f not in (3, 5)]
    assert torch.equal(c.dX[0, 0, rows], dX[0, 0, rows]) and torch.equal(c.dW[cols], dW[cols])
    assert not c.dX[0, 0, [7, 9]].isfinite().any() and not c.dW[[3, 5]].isfinite().any()


def test_saturated_everywhere():
    """Derivatives of 2^-20 and less in every place, of which the scale knows nothing: dZ of 2^-27 keeps its digits."""
    c = Case(1, 200, 64, 136, "fp16", "sigmoid", bias=True, gate="shared", scale=0.25, dscale=2.0 ** -6)
    c.bias.copy_(-14.5)
    dz, g = check(c)
    assert dz.max() < 2.0 ** -22
    # dW lies below 2^-14, where fp16's half step is 2^-25 whatever the value
    assert (np.abs(f64(c.dW) - g["dw"]) <= 2.0 ** -6 * np.abs(g["dw"]).max() / 16 + 2.0 ** -25).all()


@pytest.mark.parametrize("N", [3, 200])
@pytest.mark.parametrize("glu", [False, True])
def test_captured_with_gradients_of_other_sizes(N, glu):
    """The scale of a replay is that of its own gradients: a step captured once and replayed with gradients of any size gives the
    eager results bit for bit."""
    c = Case(2, N, 136, 264, "fp16", act="gelu", bias=True, gate="none" if glu else "adaptive", residual=not glu, glu=glu)
    c.outputs()
    ws = torch.empty((api.da2_glu_ws_bytes if glu else api.da2_linear_ws_bytes)(c.X, c.W, c.Y, True), dtype=torch.uint8, device="cuda")
    names = [n for n in ("Y", "Z", "dX", "dW", "dbias", "dgate") if getattr(c, n) is not None]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run(ws=ws)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            c.run(ws=ws)
        for seed, size in enumerate((1.0, 2.0 ** -16, 2.0 ** 12, 2.0 ** -8, 2.0 ** 4)):
            g = torch.Generator(device="cuda")
            g.manual_seed(seed)
            c.dY.copy_(torch.randn(c.dY.shape, generator=g, device="cuda") * size)
            for n in names:
                getattr(c, n).fill_(float("nan"))
            ws.fill_(0xFF)
            graph.replay()
            got = {n: getattr(c, n).clone() for n in names}
            ws.fill_(0xFF)
            c.run(ws=ws)
            side.synchronize()
            for n in names:
                assert torch.equal(got[n].nan_to_num(7.0), getattr(c, n).nan_to_num(7.0)), (n, size)
