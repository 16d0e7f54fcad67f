"""Row norms on the GPU against the float64 oracle: widths on both sides of every
chunk and row-shape rule, each type, weights shared and per sample, strided and
misaligned rows, and the gradients by formula and by differences.

Tolerances. A sum of n float32 terms in the kernels' order has a chain of at most
8 * 4 additions in a thread and 6 + 8 across threads (rows up to 16,384 elements),
so it is off by at most 46 * 2^-24 of the sum of magnitudes; with the few roundings
of the products, 2^-18 bounds it (64 * 2^-24). Wider rows, whose threads add
C / 512 terms, have C / 512 more. A result rounded to the type t adds
finfo(t).eps / 2 of itself, and half the smallest subnormal."""
import numpy as np
import pytest
import torch

from oracle import token
from paper_2609_32628_amd import api

pytestmark = pytest.mark.gpu
T = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def f64(x):
    return None if x is None else x.double().cpu().numpy()


def half_step(t):
    return torch.finfo(t).eps / 2


def tiny(t):
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2


def close(got, want, bound, t, what):
    """|got - want| within the bound of the float32 arithmetic plus the rounding to t."""
    want = np.asarray(want, np.float64)
    tol = bound + half_step(t) * (np.abs(want) + bound) + tiny(t)
    err = np.abs(f64(got) - want)
    assert (err <= tol).all(), (what, float((err - tol).max()), float(err.max()))


def chain(C):
    return 2.0 ** -18 + max(0, C / 512 - 32) * 2.0 ** -24


def check(X, w, b, dY, kind, eps, plus, Y=None, in_place=False):
    """Both passes on the GPU against the oracle."""
    B, H, N, C = X.shape
    x = f64(X)
    y, mean, rstd = token.norm(x, f64(w), f64(b), kind, eps, plus)
    adaptive = w is not None and w.dim() == 2
    Y = torch.empty_like(X) if Y is None else Y
    stats = torch.full((B, H, N, 2), float("nan"), device="cuda")
    src = X.clone() if in_place else X
    api.da2_norm(src, src if in_place else Y, w, b, kind=kind, eps=eps, plus_one=plus, stats=stats)
    Y = src if in_place else Y
    c = chain(C)
    top = np.abs(x).max(-1, keepdims=True)
    f = np.abs(token.norm_factor(x, f64(w), plus))
    # the mean is off by c max|x|; the variance by twice c of itself, so rstd by c of itself
    e = c * (2 * rstd * top + 2 * np.abs((x - mean) * rstd)) * f + 2.0 ** -23 * np.abs(y)
    close(Y, y, e, X.dtype, "Y")
    s = f64(stats)
    assert (np.abs(s[..., :1] - mean) <= c * top).all()
    # an error of the mean enters the variance with its square
    assert (np.abs(s[..., 1:] - rstd) <= 2 * c * rstd + rstd ** 3 * (c * top) ** 2).all()
    if dY is None:
        return
    mean, rstd = s[..., :1], s[..., 1:]   # the backward pass reads these
    dx, dw, db = token.norm_bwd(f64(dY), x, mean, rstd, f64(w), kind, plus, adaptive)
    dX = torch.empty_like(X)
    gw = None if w is None else torch.full_like(w, float("nan"))
    gb = None if w is None else torch.full_like(w, float("nan"))
    ws = torch.empty(api.da2_norm_ws_bytes(X, w), dtype=torch.uint8, device="cuda")
    grad = dY.clone() if in_place else dY
    api.da2_norm_bwd(grad, X, stats, grad if in_place else dX, w, gw, gb, kind=kind, plus_one=plus, ws=ws)
    dX = grad if in_place else dX
    xh = np.abs((x - mean) * rstd)
    g = np.abs(f64(dY)) * f
    gm = g.max(-1, keepdims=True)
    # x - mean is rounded once relative to itself; each mean over the row is off by c of its terms' largest
    e = rstd * (4 * 2.0 ** -24 * (g + gm + xh * gm * xh.max(-1, keepdims=True)) + 2 * c * gm * (1 + xh * xh.max(-1, keepdims=True)))
    close(dX, dx, e, X.dtype, "dX")
    if w is not None:
        n = B * H * N if not adaptive else H * N
        over = (1, 2) if adaptive else (0, 1, 2)
        # one addition per row and partial, and two roundings of each term
        k = (n + 16) * 2.0 ** -24
        close(gw, dw, k * (np.abs(f64(dY)) * xh).sum(over), w.dtype, "dw")
        close(gb, db, k * np.abs(f64(dY)).sum(over), w.dtype, "db")


def make(B, H, N, C, dtype, seed, major=False, offset=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    shape = (B, N, H, C + 2 * offset) if major else (B, H, N, C + 2 * offset)
    x = torch.randn(shape, generator=g, device="cuda") * 1.5 + 0.5 * torch.randn(shape[-1], generator=g, device="cuda")
    x = x.to(T[dtype])
    x = x.transpose(1, 2) if major else x
    return x[..., offset:offset + C] if offset else x


def weights(B, C, affine, dtype, seed):
    if affine == "none":
        return None, None
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    shape = (B, C) if affine == "adaptive" else (C,)
    return tuple(torch.randn(shape, generator=g, device="cuda").to(T[dtype]) for _ in range(2))


WIDTHS = [1, 2, 3, 7, 8, 9, 31, 64, 65, 128, 257, 511, 513, 1023, 1283, 2047, 2049, 4095, 4104, 8193, 16384, 16393, 20001]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("C", WIDTHS)
def test_widths(C, dtype):
    for kind, affine, wd, plus in (("layer", "shared", "fp32", False), ("rms", "adaptive", dtype, True)):
        X, dY = make(2, 3, 7, C, dtype, C), make(2, 3, 7, C, dtype, C + 1)
        check(X, *weights(2, C, affine, wd, 5), dY, kind, 1e-6, plus)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("affine", ["none", "shared", "adaptive"])
@pytest.mark.parametrize("major,offset", [(True, 0), (False, 1), (True, 3)])
def test_strides_and_alignment(kind, affine, major, offset):
    for dtype, wd, C in (("bf16", "fp16", 128), ("fp32", "bf16", 321), ("fp16", "fp32", 2100)):
        X, dY = make(3, 2, 9, C, dtype, 1, major, offset), make(3, 2, 9, C, dtype, 2, not major, offset)
        w, b = weights(3, C, affine, wd, 3)
        check(X, w, b, dY, kind, 1e-5, affine == "adaptive", Y=make(3, 2, 9, C, dtype, 1, not major, offset))


@pytest.mark.parametrize("C,B,H,N", [(64, 1, 40, 1000), (1536, 2, 1, 700), (24, 1, 1, 70001), (17000, 1, 1, 90), (5120, 300, 1, 1)])
@pytest.mark.parametrize("affine", ["shared", "adaptive"])
def test_many_rows(C, B, H, N, affine):
    X, dY = make(B, H, N, C, "bf16", 1), make(B, H, N, C, "bf16", 2)
    check(X, *weights(B, C, affine, "fp32", 3), dY, "layer", 1e-6, True)


@pytest.mark.parametrize("C", [128, 1283, 16390])
def test_in_place(C):
    X, dY = make(2, 2, 5, C, "bf16", 1), make(2, 2, 5, C, "bf16", 2)
    check(X, *weights(2, C, "shared", "fp32", 3), dY, "layer", 1e-6, False, in_place=True)


def test_constant_zero_and_large_rows():
    """Constant rows normalise to the bias, whatever their size; a large mean costs no digits of the variance but its own."""
    X = torch.zeros(1, 1, 4, 256, device="cuda")
    X[0, 0, 1] = 1e4
    X[0, 0, 2] = torch.arange(256, device="cuda") % 2 + 2.0 ** 14   # variance 1/4 around 2^14 + 1/2, exact in float32
    X[0, 0, 3] = 1e18 * (1 - 2 * (torch.arange(256, device="cuda") % 2))
    Y = api.da2_norm(X, torch.empty_like(X), eps=1e-6)
    y = f64(Y)[0, 0]
    np.testing.assert_array_equal(y[:2], 0)
    want = (np.arange(256) % 2 - 0.5) / np.sqrt(0.25 + 1e-6)
    np.testing.assert_allclose(y[2], want, rtol=2.0 ** -21)
    np.testing.assert_allclose(y[3], 1 - 2 * (np.arange(256) % 2), rtol=2.0 ** -21)


def test_a_bad_row_stays_alone_and_gaps_stay():
    big = make(2, 3, 6, 64, "bf16", 1, offset=5)
    base = torch.full((2, 3, 6, 74), 7.0, dtype=torch.bfloat16, device="cuda")
    X, Y = big.clone(), base[..., 5:69]
    X[1, 2, 3, 10] = float("nan")
    X[0, 1, 5, 63] = float("inf")
    good = api.da2_norm(big, torch.empty_like(big))
    api.da2_norm(X, Y)
    same = torch.ones(2, 3, 6, dtype=torch.bool, device="cuda")
    same[1, 2, 3] = same[0, 1, 5] = False
    assert torch.equal(Y[same], good[same]) and Y[1, 2, 3].isnan().all()
    assert (base[..., :5] == 7).all() and (base[..., 69:] == 7).all()


def test_repeated_rows_and_partial_outputs():
    """Rows given by a stride of zero, dX alone, and one weight gradient alone."""
    X = make(2, 1, 6, 200, "fp32", 1).expand(2, 4, 6, 200)
    dY = make(2, 4, 1, 200, "fp32", 2).expand(2, 4, 6, 200)
    w, b = weights(2, 200, "shared", "fp32", 3)
    check(X, w, b, dY, "layer", 1e-6, False, Y=torch.empty(2, 4, 6, 200, device="cuda"))
    stats = torch.empty(2, 4, 6, 2, device="cuda")
    api.da2_norm(X, torch.empty(2, 4, 6, 200, device="cuda"), w, b, stats=stats)
    ws = torch.empty(api.da2_norm_ws_bytes(X, w), dtype=torch.uint8, device="cuda")
    full = [torch.empty(2, 4, 6, 200, device="cuda"), torch.empty_like(w), torch.empty_like(w)]
    api.da2_norm_bwd(dY, X, stats, full[0], w, full[1], full[2], ws=ws)
    only = [torch.empty_like(t) for t in full]
    api.da2_norm_bwd(dY, X, stats, only[0], w)
    api.da2_norm_bwd(dY, X, stats, None, w, only[1], ws=ws)
    api.da2_norm_bwd(dY, X, stats, None, w, None, only[2], ws=ws)
    for a, o in zip(full, only):
        assert torch.equal(a, o)


def test_gradient_against_differences():
    """The kernel's float32 gradients along random directions against central differences of the oracle's forward pass."""
    X, dY = make(2, 2, 5, 96, "fp32", 1), make(2, 2, 5, 96, "fp32", 2)
    w, b = weights(2, 96, "adaptive", "fp32", 3)
    stats, dX = torch.empty(2, 2, 5, 2, device="cuda"), torch.empty_like(X)
    dw, db = torch.empty_like(w), torch.empty_like(b)
    api.da2_norm(X, torch.empty_like(X), w, b, plus_one=True, stats=stats)
    api.da2_norm_bwd(dY, X, stats, dX, w, dw, db, plus_one=True,
                     ws=torch.empty(api.da2_norm_ws_bytes(X, w), dtype=torch.uint8, device="cuda"))
    x, dy, w0, b0 = f64(X), f64(dY), f64(w), f64(b)
    rng = np.random.default_rng(0)
    h = 1e-5
    for grad, at, f in ((dX, x, lambda t: token.norm(t, w0, b0, plus_one=True)[0]), (dw, w0, lambda t: token.norm(x, t, b0, plus_one=True)[0]),
                        (db, b0, lambda t: token.norm(x, w0, t, plus_one=True)[0])):
        v = rng.normal(size=at.shape)
        want = (dy * (f(at + h * v) - f(at - h * v))).sum() / (2 * h)
        # float32 gradients (2^-18 of each value's scale) and differences off by h^2 and 2^-52 / h
        assert abs((f64(grad) * v).sum() - want) <= 2.0 ** -18 * (np.abs(f64(grad)) * np.abs(v)).sum() + 1e-5


def test_offsets_beyond_32_bits():
    """Two samples 2^32 bytes apart."""
    far = (1 << 31) + 64
    room = torch.empty(far + 4096, dtype=torch.bfloat16, device="cuda")
    X = room.as_strided((2, 1, 4, 128), (far, 512, 128, 1))
    X.copy_(make(2, 1, 4, 128, "bf16", 1))
    w, b = weights(2, 128, "shared", "fp32", 3)
    check(X, w, b, make(2, 1, 4, 128, "bf16", 2), "layer", 1e-6, False, Y=torch.empty(2, 1, 4, 128, dtype=torch.bfloat16, device="cuda"))
    out = room.as_strided((2, 1, 4, 128), (far, 512, 128, 1), 2048)
    want = api.da2_norm(X, torch.empty(2, 1, 4, 128, dtype=torch.bfloat16, device="cuda"), w, b)
    api.da2_norm(X, out, w, b)
    assert torch.equal(out, want)


def test_streams_and_graph_replays():
    """On a stream of its own, and captured: three replays with new inputs and eager work in between."""
    X, dY = make(2, 1, 300, 1536, "bf16", 1), make(2, 1, 300, 1536, "bf16", 2)
    w, b = weights(2, 1536, "adaptive", "fp32", 3)
    ws = torch.empty(api.da2_norm_ws_bytes(X, w), dtype=torch.uint8, device="cuda")
    out = [torch.empty_like(X), torch.empty(2, 1, 300, 2, device="cuda"), torch.empty_like(X), torch.empty_like(w), torch.empty_like(b)]

    def both(o, scratch, stream=None):
        api.da2_norm(X, o[0], w, b, plus_one=True, stats=o[1], stream=stream)
        api.da2_norm_bwd(dY, X, o[1], o[2], w, o[3], o[4], plus_one=True, ws=scratch, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    both(out, ws, side)
    torch.cuda.current_stream().wait_stream(side)
    eager = [torch.empty_like(t) for t in out]
    both(eager, torch.empty_like(ws))
    assert all(torch.equal(a, e) for a, e in zip(out, eager))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(out, ws)
    for seed in (11, 12, 13):
        X.copy_(make(2, 1, 300, 1536, "bf16", seed))
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        both(eager, torch.empty_like(ws))
        torch.cuda.synchronize()
        assert all(torch.equal(a, e) for a, e in zip(out, eager))
