"""Projections and gated blocks on the GPU against the float64 oracle: sizes on both sides of every tile, ends of K and F inside
16-byte chunks, each type and activation, gates, residuals, heads, strides, and the gradients.

Tolerances. Sums over n products are taken 32 at a time by the matrix instructions and added up in float32: at most
n / 16 + 16 roundings (and those of a split's parts), of at most 2^-23 of the sum of magnitudes each. The activations are
off by at most 2^-16 of themselves (exponentials of arguments up to 2^6 rounded to float32, and a fitted tail of 2.3e-6), their
derivatives by 2^-15, and change by at most 1.2 times a change of their argument (1.13 for the GELU). A gradient of the sums is
rounded to the type for the products: half a step of itself, or of its smallest subnormal (up to 16 tokens in two numbers). A result rounded to the type t
adds finfo(t).eps / 2 of itself, and half the smallest subnormal."""
import numpy as np
import pytest
import torch

from oracle import layer
from paper_2609_32628_amd import api

pytestmark = pytest.mark.gpu
T = {"bf16": torch.bfloat16, "fp16": torch.float16}
NAN = float("nan")


def f64(x):
    return None if x is None else x.double().cpu().numpy()


def half(t):
    return torch.finfo(t).eps / 2


def tiny(t):
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2


def close(got, want, bound, what):
    want = np.asarray(want)
    t = got.dtype
    tol = bound + half(t) * (np.abs(want) + bound) + tiny(t)
    err = np.abs(f64(got) - want)
    assert np.isfinite(f64(got)).all() and (err <= tol).all(), (what, float((err - tol).max()), float(err.max()))


def rows(B, H, N, C, dtype, major=False, pad=0):
    """Rows in memory that holds NaN around them: each padded to 16 bytes and `pad` chunks more."""
    wide = -(-C // 8) * 8 + 8 * pad
    shape = (B, N, H, wide) if major else (B, H, N, wide)
    x = torch.full(shape, NAN, dtype=T[dtype], device="cuda")
    return (x.transpose(1, 2) if major else x)[..., :C]


def fill(x, g, scale=1.0):
    x.copy_(torch.randn(x.shape, generator=g, device="cuda") * scale)
    return x


def matrix(R, C, dtype, pad=0):
    return torch.full((R, -(-C // 8) * 8 + 8 * pad), NAN, dtype=T[dtype], device="cuda")[:, :C]


def surroundings(x):
    """What lies in the storage of x besides x."""
    s = torch.empty(0, dtype=x.dtype, device=x.device).set_(x.untyped_storage())
    m = torch.ones(s.numel(), dtype=torch.bool, device=x.device)
    m.as_strided(x.shape, x.stride(), x.storage_offset()).fill_(False)
    return s[m]


class Case:
    def __init__(self, B, N, K, F, dtype="bf16", act="none", bias=False, gate="none", residual=False, heads=(1, 1), glu=False, pad=0, major=False,
                 scale=1.0, dscale=1.0, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + 7 * K + F)
        self.__dict__.update(B=B, N=N, K=K, F=F, dtype=dtype, act=act, glu=glu, heads=heads, pad=pad, major=major)
        hx, hy = heads
        assert K % hx == 0 and F % hy == 0
        R = 2 * F if glu else F
        self.X = fill(rows(B, hx, N, K // hx, dtype, major, pad), g)
        self.W = fill(matrix(R, K, dtype, pad), g, scale * K ** -0.5)
        self.dY = fill(rows(B, hy, N, F // hy, dtype, not major, pad), g, dscale)
        self.R = fill(rows(B, hy, N, F // hy, dtype, major, 0), g) if residual else None
        self.bias = (0.5 * torch.randn(R, generator=g, device="cuda")).to(T[dtype]) if bias else None
        self.gate = None if gate == "none" else torch.randn((B, F) if gate == "adaptive" else (F,), generator=g, device="cuda").to(T[dtype])

    def outputs(self):
        hx, hy = self.heads
        self.Y = rows(self.B, hy, self.N, self.F // hy, self.dtype, self.major, self.pad)
        self.dX = rows(self.B, hx, self.N, self.K // hx, self.dtype, not self.major, self.pad)
        self.dW = matrix(self.W.shape[0], self.K, self.dtype, self.pad)
        self.dbias, self.dgate = (None if x is None else torch.full_like(x, NAN) for x in (self.bias, self.gate))
        self.Z = (api.da2_glu_z if self.glu else api.da2_linear_z)(self.X, self.Y).fill_(NAN)

    def run(self, train=True, ws=None):
        s = self
        if ws is None:
            ws = torch.full(((api.da2_glu_ws_bytes if s.glu else api.da2_linear_ws_bytes)(s.X, s.W, s.Y, train),), 0xFF, dtype=torch.uint8, device="cuda")
        Z = s.Z if train else None
        if s.glu:
            api.da2_glu(s.X, s.W, s.Y, s.bias, act=s.act, Z=Z, ws=ws)
            if train:
                api.da2_glu_bwd(s.dY, s.X, s.W, Z, dX=s.dX, dW=s.dW, dbias=s.dbias, act=s.act, ws=ws)
        else:
            api.da2_linear(s.X, s.W, s.Y, s.bias, act=s.act, gate=s.gate, residual=s.R, Z=Z, ws=ws)
            if train:
                api.da2_linear_bwd(s.dY, s.X, s.W, Z, dX=s.dX, dW=s.dW, dbias=s.dbias, act=s.act, gate=s.gate, dgate=s.dgate, ws=ws)

    def check(self, train=True):
        s = self
        t, F, M = T[s.dtype], s.F, s.B * s.N
        x, w = f64(s.X), f64(s.W)
        S = np.abs(layer.flat(x)) @ np.abs(w).T
        ez = (s.K / 16 + 16) * 2.0 ** -23 * S
        flat_y = lambda y: torch.from_numpy(np.ascontiguousarray(y))  # noqa: E731
        back = lambda m, like: layer.unflat(m, *like.shape)  # noqa: E731
        if s.glu:
            y, z = layer.glu(x, w, f64(s.bias), s.act)
            ez = ez + 2.0 ** -23 * (S + np.abs(z))
            a, u = np.abs(layer.act(z[:, :F], s.act)[0]), np.abs(z[:, F:])
            e = 1.2 * ez[:, :F] * (u + ez[:, F:]) + a * ez[:, F:] + 2.0 ** -16 * a * u
        else:
            y, z = layer.linear(x, w, f64(s.bias), s.act, f64(s.gate), f64(s.R))
            ez = ez + 2.0 ** -23 * (S + np.abs(z))
            gate = 1.0 if s.gate is None else np.abs(layer.rows_gate(f64(s.gate), s.B, s.N))
            a = np.abs(layer.act(z, s.act)[0])
            e = (1.2 * ez + 2.0 ** -16 * a) * gate + 2.0 ** -23 * (np.abs(y) if s.R is None else np.abs(y) + np.abs(layer.flat(f64(s.R))))
        close(s.Y, back(y, s.Y), back(e, s.Y), "Y")
        assert surroundings(s.Y).isnan().all()
        if not train:
            return
        Z = f64(s.Z).reshape(M, 2 if s.glu else 1, -1)
        assert np.isnan(Z[:, :, F:]).all()
        zg = Z[:, :, :F].reshape(M, -1)
        assert (np.abs(zg - z) <= ez + 2.0 ** -24 * np.abs(z)).all()
        dy = np.abs(layer.flat(f64(s.dY)))
        if s.glu:
            g = layer.glu_bwd(f64(s.dY), x, w, zg, s.act)
            a = np.abs(layer.act(zg[:, :F], s.act)[0])
            ed = np.concatenate([2.0 ** -15 * dy * np.abs(zg[:, F:]), dy * (2.0 ** -16 * a)], 1)
        else:
            g = layer.linear_bwd(f64(s.dY), x, w, zg, s.act, f64(s.gate))
            ed = 2.0 ** -15 * dy * gate if s.act != "none" else 2.0 ** -23 * dy * gate
        rounded = s.glu or s.act != "none" or s.gate is not None
        # up to 16 tokens a second number has what the rounding left over
        er = ed + (half(t) ** (2 if M <= 16 else 1) * (np.abs(g["dz"]) + ed) + tiny(t) if rounded else 0)
        mag = np.abs(g["dz"]) + er
        close(s.dX, back(g["dx"], s.dX), back(er @ np.abs(w) + (w.shape[0] / 16 + 24) * 2.0 ** -23 * (mag @ np.abs(w)), s.dX), "dX")
        X = np.abs(layer.flat(x))
        close(s.dW, g["dw"], er.T @ X + (M / 16 + s.B + 40) * 2.0 ** -23 * (mag.T @ X), "dW")
        assert surroundings(s.dX).isnan().all() and surroundings(s.dW).isnan().all()
        if s.bias is not None:
            close(s.dbias, g["dbias"], ed.sum(0) + (M + 16) * 2.0 ** -24 * mag.sum(0), "dbias")
        if s.gate is not None:
            t1 = dy * np.abs(layer.act(zg, s.act)[0])
            per = lambda v: v.reshape(s.B, s.N, F).sum(1) if s.gate.dim() == 2 else v.sum(0)  # noqa: E731
            close(s.dgate, g["dgate"], (2.0 ** -16 + (M + 16) * 2.0 ** -24) * per(t1), "dgate")


def run(*a, train=True, **kw):
    c = Case(*a, **kw)
    c.outputs()
    c.run(train)
    c.check(train)
    return c


SIZES = [(1, 1, 1, 1), (1, 1, 8, 8), (1, 2, 7, 3), (3, 1, 64, 64), (1, 5, 65, 33), (2, 31, 63, 127), (1, 127, 128, 129), (1, 129, 200, 256), (3, 43, 40, 257),
         (1, 257, 136, 100), (2, 300, 1000, 17), (1, 16, 2048, 300), (17, 1, 520, 96), (1, 64, 1283, 40), (33, 2, 72, 1000), (1, 65, 4097, 65)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("B,N,K,F", SIZES)
def test_linear_sizes(B, N, K, F, dtype):
    run(B, N, K, F, dtype, "gelu", bias=True, gate="adaptive", residual=True)
    run(B, N, K, F, dtype, pad=1)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("B,N,K,F", SIZES)
def test_glu_sizes(B, N, K, F, dtype):
    run(B, N, K, F, dtype, "silu", bias=True, glu=True)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu", "sigmoid"])
@pytest.mark.parametrize("glu", [False, True])
def test_activations(act, glu):
    """Sums of up to 30, where tails and saturation count."""
    for dtype in ("bf16", "fp16"):
        run(2, 50, 96, 80, dtype, act, bias=True, glu=glu, scale=8.0)
        run(2, 50, 96, 80, dtype, act, glu=glu)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("B,N", [(1, 1), (2, 1), (1, 16), (16, 1), (3, 5), (1, 17)])
@pytest.mark.parametrize("F", [3, 16, 17, 300])
def test_gradients_of_few_tokens(B, N, F, dtype):
    """As many rows of dW as fit one launch and more; the gradients of the sums in two numbers."""
    for K in (24, 130, 640):
        run(B, N, K, F, dtype, "gelu", bias=True, gate="shared")
        run(B, N, K, F, dtype, "silu", glu=True)


@pytest.mark.parametrize("B,N,K,F", [(2, 9001, 24, 40), (1, 20, 17000, 130), (3, 2500, 130, 300)])
def test_long_sums(B, N, K, F):
    """Few tiles over a long axis, cut into many parts: of the tokens in dW, of K in the forward pass."""
    run(B, N, K, F, "bf16", "silu", glu=True)
    run(B, N, K, F, "fp16", "gelu", bias=True, gate="adaptive", residual=True)


@pytest.mark.parametrize("gate", ["none", "shared", "adaptive"])
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("bias,residual", [(False, False), (True, True)])
def test_gates_and_residuals(gate, act, bias, residual):
    run(3, 70, 136, 90, "bf16", act, bias=bias, gate=gate, residual=residual)


@pytest.mark.parametrize("heads", [(3, 1), (1, 5), (2, 4)])
@pytest.mark.parametrize("major", [False, True])
def test_heads_and_orders(heads, major):
    run(2, 75, 64 * heads[0], 8 * heads[1], "bf16", "none", heads=heads, major=major, pad=1)
    run(2, 75, 128 * heads[0], 64 * heads[1], "fp16", "gelu_tanh", bias=True, gate="adaptive", residual=True, heads=heads, major=major)
    run(2, 75, 64 * heads[0], 24 * heads[1], "bf16", "silu", glu=True, heads=heads, major=major)


@pytest.mark.parametrize("M,K,F", [(4096, 72, 4096), (4000, 64, 4200), (256 * 20, 200, 256 * 13)])
def test_large_tiles(M, K, F):
    run(1, M, K, F, "bf16", "gelu", bias=True, train=False)
    run(2, M // 2, K, F // 2, "fp16", "silu", glu=True, train=False)


def test_long_products_and_gradients():
    """Products over many tokens (weights' gradients), features and channels, which are cut into parts."""
    run(3, 1500, 200, 136, "bf16", "gelu", bias=True, gate="shared")
    run(1, 100, 6000, 60, "fp16", "none")
    run(1, 60, 96, 5000, "bf16", "silu", glu=True)


@pytest.mark.parametrize("glu", [False, True])
def test_extents_of_one_and_samples_far_apart(glu):
    """Strides of extents of one are not looked at; samples may lie anywhere."""
    c = Case(3, 2, 72, 40, glu=glu, act="silu")
    big = torch.zeros(3, 1, 5000, 72, dtype=torch.bfloat16, device="cuda")
    big[:, :, -2:] = c.X
    c.X = big[:, :, -2:]
    c.outputs()
    c.run()
    c.check()
    c = Case(1, 1, 72, 40, glu=glu, act="silu")
    c.X = torch.as_strided(c.X, c.X.shape, (3, 5, 7, 1), c.X.storage_offset())
    c.outputs()
    c.run()
    c.check()


def test_in_place_residual():
    c = Case(2, 60, 128, 72, residual=True, bias=True, gate="shared")
    c.outputs()
    c.run(False)
    want = c.Y.clone()
    r = c.R
    api.da2_linear(c.X, c.W, r, c.bias, gate=c.gate, residual=r, ws=torch.empty(max(api.da2_linear_ws_bytes(c.X, c.W, r), 1), dtype=torch.uint8, device="cuda"))
    assert torch.equal(r, want)


@pytest.mark.parametrize("glu", [False, True])
def test_single_gradients(glu):
    """Each output alone is what all together are."""
    c = Case(2, 90, 200, 130, act="gelu", bias=True, gate="none" if glu else "adaptive", glu=glu)
    c.outputs()
    c.run()
    want = {n: getattr(c, n).clone() for n in ("dX", "dW", "dbias", "dgate") if getattr(c, n) is not None}
    for name, w in want.items():
        c2 = {n: None for n in ("dX", "dW", "dbias")}
        out = torch.full_like(w, NAN) if name in ("dbias", "dgate") else getattr(c, name).fill_(NAN)
        ws = torch.empty((api.da2_glu_ws_bytes if glu else api.da2_linear_ws_bytes)(c.X, c.W, c.Y, True), dtype=torch.uint8, device="cuda")
        if glu:
            api.da2_glu_bwd(c.dY, c.X, c.W, c.Z, act=c.act, ws=ws, **{**c2, name: out})
        else:
            api.da2_linear_bwd(c.dY, c.X, c.W, c.Z, act=c.act, gate=c.gate, ws=ws, **{**c2, name: out})
        assert torch.equal(out, w), name


def test_not_a_number_stays_in_its_rows_and_columns():
    c = Case(1, 200, 100, 150, act="silu", glu=True)
    c.X[0, 0, 7, 3] = NAN
    c.W[20, 5] = float("inf")
    c.outputs()
    c.run(False)
    bad = c.Y[0, 0].float().cpu()
    ok = torch.ones(200, dtype=torch.bool)
    ok[7] = False
    cols = torch.ones(150, dtype=torch.bool)
    cols[20] = False
    assert bad[7].isnan().all() and bad[ok][:, cols].isfinite().all()


def test_small_gradients_in_half_precision():
    """fp16 gradients whose values are subnormal there (2^-24 apart) are off by what their own rounding and that of the gradients of
    the sums are off by."""
    run(2, 300, 136, 200, "fp16", "silu", bias=True, glu=True, dscale=1e-5)
    run(2, 300, 136, 200, "fp16", "gelu", bias=True, gate="shared", dscale=1e-5)


@pytest.mark.parametrize("glu", [False, True])
def test_captured_and_replayed_on_another_stream(glu):
    """A training step captured once and replayed with new inputs gives the eager results bit for bit."""
    c = Case(2, 150, 136, 264, act="gelu", bias=True, gate="none" if glu else "adaptive", residual=not glu, glu=glu)
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
        for seed in (1, 2, 3):
            g = torch.Generator(device="cuda")
            g.manual_seed(seed)
            fill(c.X, g)
            fill(c.dY, g)
            for n in names:
                getattr(c, n).fill_(NAN)
            graph.replay()
            got = {n: getattr(c, n).clone() for n in names}
            c.run(ws=ws)
            side.synchronize()
            for n in names:
                assert torch.equal(got[n].nan_to_num(7.0), getattr(c, n).nan_to_num(7.0)), n
    c.check()


def test_two_calls_at_once():
    """Calls on two streams with workspaces of their own."""
    cases = [Case(1, 64, 2048, 300, act="silu", seed=i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for c, s in zip(cases, streams):
        with torch.cuda.stream(s):
            c.outputs()
            for _ in range(10):
                c.run()
    torch.cuda.synchronize()
    for c in cases:
        c.check()


@pytest.mark.parametrize("glu", [False, True])
def test_offsets_that_pass_32_bits(glu):
    """Samples 4 GB apart, which no tile's 32-bit offsets span, of many tokens and of few."""
    for N in (130, 3):
        c = Case(2, N, 72, 40, act="silu", gate="none" if glu else "adaptive", residual=not glu, glu=glu)
        apart = 1 << 31
        for name in ("X", "dY"):
            t = getattr(c, name)
            big = torch.empty(apart + t.shape[2] * 80, dtype=t.dtype, device="cuda")
            far = torch.as_strided(big, t.shape, (apart, 0, 80, 1))
            far.copy_(t)
            setattr(c, name, far)
        c.outputs()
        y = torch.empty(apart + N * 48, dtype=torch.bfloat16, device="cuda")
        plain, c.Y = c.Y, torch.as_strided(y, c.Y.shape, (apart, 0, 48, 1))
        c.run()
        plain.copy_(c.Y)
        c.Y = plain
        c.check()
