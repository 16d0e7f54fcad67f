"""Differential attention on the GPU against the float64 oracle: forward, split
keys, single tokens over caches, masks, and the gradients.

Tolerances, with u = finfo(type).eps / 2 (half a step of the 16-bit type):
  - a score is a float32 sum of d/2 exact products, off by (d/2) 2^-24 of the sum of their magnitudes; scaled, with the
    rounding of the exponent (2^-24 of its size) and of the exponential (2^-22), a weight is off by e = 2^-22 +
    scale (d/2) 2^-24 |q|.|k| + 2^-23 (1 + max |score|) of itself. E is its largest value over a head.
  - a weight is rounded to the type for its product with V (u of itself), the sums over keys have at most M / 16 + 40
    additions in a chain (2^-24 each), and so have l and U, so O is off by (u + 2 E + 2 (M/16 + 40) 2^-24) of
    sum_j (P1 + lam P2) |V_j|, and by u of itself when it is stored.
  - dS_i = P_i (dP - del_i): dP is a float32 sum, off by d 2^-24 |dO|.|V|; del_i, the float32 sum of P_i dP, by
    t = sum P_i ((E + (M/16 + 40) 2^-24) |dP| + d 2^-24 |dO|.|V|). dS is rounded by u. So dS_i is off by
    P_i ((u + E) |dP - del_i| + d 2^-24 |dO|.|V| + t) and dK by the sums of that times |Q|; dV as O.
  - dQ is sum_j r_j K_j - (sum_j r_j) m from rounded r_j, with m the mean of some of the keys. That is
    sum_j r_j (K_j - m), and sum_j dS_j (K_j - m) = sum_j dS_j K_j since the dS_j sum to zero: so dQ is off by the sums of
    what dS is off times |K_j - m|, at most the distance w_j of K_j to the further end of the keys' range, channel by
    channel (the float32 sums of r_j K_j and r_j keep their error relative to |K_j| <= w_j + |m|).
  - dlam is the sum of del2, off by its t.
  - below the smallest normal number a rounding is off by half the spacing there, z = smallest_normal eps / 2 (2^-25 in
    fp16), not by u of the value: each rounded weight or dS adds z to its product, so z sum |V_j| (1 + lam) to O,
    z sum |dO| to dV, and z scale times sum w or |Q| to dQ (lam times that for the second map, whose lambda comes
    after the rounding) and dK. (A running maximum is at most the row's, so a row's sum is at least 1.)"""
import math

import numpy as np
import pytest
import torch

from oracle import token
from paper_2609_32628_amd import api

pytestmark = pytest.mark.gpu
T = {"bf16": torch.bfloat16, "fp16": torch.float16}


def f64(x):
    return x.double().cpu().numpy()


def make(B, H, N, d, dtype, seed, major=False, scale=1.0, shift=0.3):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((B, N, H, d) if major else (B, H, N, d), generator=g, device="cuda") * scale
    x = (x + shift * torch.randn(d, generator=g, device="cuda")).to(T[dtype])
    return x.transpose(1, 2) if major else x


class Case:
    def __init__(self, B, H, Hk, N, M, d, dtype="bf16", causal=False, lens=None, start=None, scale=None, seed=0, major=False,
                 q_scale=1.5):
        self.B, self.H, self.Hk, self.N, self.M, self.d, self.causal, self.scale = B, H, Hk, N, M, d, causal, scale
        self.Q = make(B, H, N, d, dtype, seed + 1, major, q_scale)
        self.K, self.V = (make(B, Hk, M, d, dtype, seed + i, major) for i in (2, 3))
        self.dO = make(B, H, N, d, dtype, seed + 4, not major)
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.lam = 0.2 + 0.6 * torch.rand(H, generator=g, device="cuda")
        ints = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        self.kv_lens, self.q_start = ints(lens), ints(start)
        self.n_keys = [M] * B if lens is None else [min(max(n, 0), M) for n in lens]
        self.start = [n - N for n in self.n_keys] if start is None else start
        for b, n in enumerate(self.n_keys):   # what lies behind a sample's keys is anything
            self.K[b, :, n:] = float("nan")
            self.V[b, :, n:] = float("inf")

    def how(self):
        return dict(kv_lens=self.kv_lens, q_start=self.q_start, causal=self.causal, scale=self.scale)

    def oracle(self, grads):
        return token.diff_attn(f64(self.Q), f64(self.K), f64(self.V), f64(self.lam), self.n_keys, self.start, self.causal,
                               self.scale, f64(self.dO) if grads else None)

    def bounds(self, want, grads):
        """Largest errors of O, lse and the gradients, as in the module's text."""
        B, H, Hk, N, M, d = self.B, self.H, self.Hk, self.N, self.M, self.d
        h, u, eps = d // 2, torch.finfo(self.Q.dtype).eps / 2, 2.0 ** -24
        scale = 1 / math.sqrt(h) if self.scale is None else self.scale
        out = {n: np.zeros(want[n].shape) for n in want}
        chain = (M / 16 + 40) * eps
        z = torch.finfo(self.Q.dtype).smallest_normal * torch.finfo(self.Q.dtype).eps / 2
        for b in range(B):
            n = self.n_keys[b]
            see = token.diff_visible(N, M, n, self.start[b], self.causal)[:, :n]
            for hq in range(H):
                kh, lam = hq // (H // Hk), float(self.lam[hq])
                q, k, v = f64(self.Q[b, hq]), f64(self.K[b, kh, :n]), f64(self.V[b, kh, :n])
                P, lse = token._maps(q, k, see, scale) if n else (np.zeros((2, N, 0)), want["lse"][b, hq])
                E = np.zeros(2)
                for m in (0, 1):
                    c = slice(m * h, (m + 1) * h)
                    dots = np.where(see, np.abs(q[:, c]) @ np.abs(k[:, c]).T, 0).max(initial=0.0)
                    E[m] = 2.0 ** -22 + scale * h * eps * dots + 2 * eps * (1 + scale * dots)
                    out["lse"][b, hq, m] = E[m] + chain + 4 * eps * np.abs(np.where(np.isfinite(lse[m]), lse[m], 0))
                ab = np.abs(v)
                o1, o2 = ((u + 2 * E[m] + 2 * chain) * (P[m] @ ab) for m in (0, 1))
                out["O"][b, hq] = o1 + lam * o2 + z * (1 + lam) * (see @ ab) + 4 * eps * (np.abs(P[0] @ v) + lam * np.abs(P[1] @ v))
                if not grads:
                    continue
                g = f64(self.dO[b, hq])
                dP, gv = g @ v.T, np.abs(g) @ ab.T
                out["dV"][b, kh, :n] += (u * np.abs(P[0] - lam * P[1]) + (E[0] + 4 * eps) * P[0] + lam * (E[1] + 4 * eps) * P[1]).T @ np.abs(g)
                out["dV"][b, kh, :n] += z * (see.T @ np.abs(g))
                out["dV"][b, kh, :n] += (N * H / Hk / 16 + 40) * eps * ((P[0] + lam * P[1]).T @ np.abs(g))
                t = [(P[m] * ((E[m] + chain) * np.abs(dP) + d * eps * gv)).sum(-1, keepdims=True) for m in (0, 1)]
                out["dlam"][hq] += t[1].sum()
                for m, f in ((0, 1.0), (1, lam)):
                    c = slice(m * h, (m + 1) * h)
                    delta = (P[m] * dP).sum(-1, keepdims=True)
                    mag = f * P[m] * np.abs(dP - delta)
                    off = (u + E[m] + 8 * eps) * mag + f * P[m] * (d * eps * gv + t[m] + 4 * eps * np.abs(delta))
                    w = np.maximum(k[:, c] - k[:, c].min(0), k[:, c].max(0) - k[:, c]) if n else k[:, c]
                    out["dQ"][b, hq, :, c] = scale * ((off + z * f * see) @ w + (chain * mag) @ (w + np.abs(k[:, c]).max(0, initial=0.0)))
                    out["dK"][b, kh, :n, c] += scale * ((off + z * see + (N * H / Hk / 16 + 40) * eps * mag).T @ np.abs(q[:, c]))
        return out


def close(got, want, bound, name):
    t = got.dtype
    got = f64(got)
    rounded = t != torch.float32
    tol = bound + (torch.finfo(t).eps / 2 * (np.abs(want) + bound) + torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2 if rounded else
                   2.0 ** -23 * np.abs(want))
    same = np.isneginf(want) & np.isneginf(got)
    with np.errstate(invalid="ignore"):
        bad = ~(np.abs(got - want) <= tol) & ~same
    assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:3].tolist(), float(np.abs(got - want)[bad].max()), float(np.nanmax(tol)))


def check(case, grads=True):
    out = {"O": torch.full_like(case.Q, float("nan"))}
    out["lse"] = torch.full((case.B, case.H, 2, case.N), float("nan"), device="cuda")
    ws = torch.full((api.da2_diff_ws_bytes(case.Q, case.K, True),), 0xFF, dtype=torch.uint8, device="cuda")
    api.da2_diff_attn(case.Q, case.K, case.V, case.lam, out["O"], ws, out["lse"], **case.how())
    want = case.oracle(grads)
    bound = case.bounds(want, grads)
    for n in ("O", "lse"):
        close(out[n], want[n], bound[n], n)
    alone = torch.full_like(case.Q, float("nan"))
    api.da2_diff_attn(case.Q, case.K, case.V, case.lam, alone, ws, **case.how())
    assert torch.equal(alone, out["O"])
    if not grads:
        return out
    for n, like in (("dQ", case.Q), ("dK", case.K), ("dV", case.V), ("dlam", case.lam)):
        out[n] = torch.full_like(like, float("nan"))
    ws.fill_(0xFF)
    api.da2_diff_attn_bwd(case.Q, case.K, case.V, case.lam, out["lse"], case.dO, out["dQ"], out["dK"], out["dV"],
                          out["dlam"], ws, **case.how())
    for n in ("dQ", "dK", "dV", "dlam"):
        close(out[n], want[n], bound[n], n)
    for b, n in enumerate(case.n_keys):
        assert (out["dK"][b, :, n:] == 0).all() and (out["dV"][b, :, n:] == 0).all()
    return out


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N,M", [(1, 1), (1, 2), (2, 31), (3, 32), (5, 33), (17, 64), (64, 65), (65, 63), (33, 128), (128, 129), (200, 257)])
def test_lengths(N, M, d, dtype):
    check(Case(2, 2, 2, N, M, d, dtype, seed=N + M))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N", [1, 31, 32, 33, 64, 65, 127, 129, 190, 300])
def test_causal(N, d):
    check(Case(1, 2, 1, N, N, d, "bf16", causal=True, seed=N))


@pytest.mark.parametrize("H,Hk", [(1, 1), (6, 2), (8, 1), (12, 4), (40, 1)])
@pytest.mark.parametrize("N", [1, 2, 9, 70])
def test_shared_heads(N, H, Hk):
    check(Case(2, H, Hk, N, 150, 64, "fp16", causal=True, seed=H, major=True))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_padded_batches_and_empty_rows(d, causal):
    """Lengths of zero, one, within and beyond the tensors; first queries that see nothing; starts far outside."""
    lens = [0, 1, 37, 200, 1000, -5]
    check(Case(6, 2, 1, 130, 200, d, "bf16", causal, lens, seed=1))
    check(Case(6, 2, 1, 130, 200, d, "bf16", causal, lens, [0] * 6, seed=2))
    check(Case(6, 4, 2, 3, 200, d, "fp16", causal, lens, [-2, 0, 35, -1000, 2 ** 31 - 1, -2 ** 31], seed=3))
    check(Case(2, 1, 1, 200, 130, d, "bf16", causal, None, [-150, 100], seed=4))


@pytest.mark.parametrize("d,dtype", [(64, "fp16"), (128, "bf16")])
@pytest.mark.parametrize("H,causal", [(64, False), (65, False), (128, False), (129, False), (65, True), (256, True), (257, True)])
def test_many_tiles(H, causal, d, dtype):
    """Two tiles of 128 rows a head: on both sides of the counts of tiles at which other workgroups take the rows."""
    check(Case(1, H, H, 150, 170, d, dtype, causal, seed=H))


@pytest.mark.parametrize("N,M,start", [(1, 300, [40, 0, -5]), (70, 300, [3, -50, -100]), (200, 500, [100, 0, 250]), (33, 3000, [1500, 7, 2900])])
@pytest.mark.parametrize("d", [64, 128])
def test_keys_that_no_query_sees(d, N, M, start):
    """A cache whose room behind the last query's position was never written: it may hold anything."""
    case = Case(3, 4, 2, N, M, d, "bf16", True, None, start, seed=25)
    want = check(case)
    for b, s in enumerate(start):
        case.K[b, :, max(s + N, 0):] = float("nan")
        case.V[b, :, max(s + N, 0):] = float("inf")
    out = {n: torch.full_like(x, float("nan")) for n, x in want.items()}
    ws = torch.empty(api.da2_diff_ws_bytes(case.Q, case.K, True), dtype=torch.uint8, device="cuda")
    api.da2_diff_attn(case.Q, case.K, case.V, case.lam, out["O"], ws, out["lse"], **case.how())
    api.da2_diff_attn_bwd(case.Q, case.K, case.V, case.lam, out["lse"], case.dO, out["dQ"], out["dK"], out["dV"], out["dlam"],
                          ws, **case.how())
    assert all(torch.equal(out[n], want[n]) for n in want)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("B,H,Hk,N,M,d", [(1, 12, 4, 1, 1000, 64), (3, 8, 2, 1, 4097, 128), (1, 1, 1, 5, 2500, 128), (2, 4, 4, 16, 3000, 64),
                                          (1, 2, 2, 100, 2000, 128), (1, 40, 20, 33, 1100, 64)])
def test_split_keys(B, H, Hk, N, M, d, dtype):
    """Few rows over long caches, whose keys are split over workgroups and joined."""
    lens = [M - 700 * b for b in range(B)]
    out = check(Case(B, H, Hk, N, M, d, dtype, True, lens, seed=5), grads=False)
    assert out["O"].isfinite().all()


@pytest.mark.parametrize("N,H,Hk,d", [(1, 8, 2, 128), (100, 2, 2, 64)])
def test_split_keys_of_short_and_empty_samples(N, H, Hk, d):
    """Parts that hold no key, and a sample without keys."""
    check(Case(4, H, Hk, N, 5000, d, "bf16", True, [5000, 0, 1, 300], seed=6), grads=False)
    check(Case(4, H, Hk, N, 5000, d, "bf16", False, [0, 0, 0, 2], seed=7), grads=False)


def test_large_and_peaked_scores():
    """Scores far apart: the maximum moves by much more than 2^8 on the way, upwards and downwards, and a row's weight
    lies on one key."""
    for dtype in ("bf16", "fp16"):
        case = Case(1, 2, 1, 40, 300, 64, dtype, seed=9, q_scale=6.0)
        order = torch.arange(300, device="cuda").float()[None, None, :, None] / 300
        for flip in (False, True):
            ramp = order.flip(2) if flip else order
            case.K.copy_((case.K.float() * 0.2 + 4 * ramp).to(case.K.dtype))
            check(case)


def test_strides_scale_and_sharing():
    """Rows inside larger storage, a scale of the caller's, and V given as K's memory."""
    case = Case(2, 4, 2, 50, 90, 128, "bf16", True, [90, 60], [40, 10], 0.05, seed=3)
    room = torch.zeros(2, 120, 3, 4, 128, dtype=torch.bfloat16, device="cuda")
    k = room[:, 10:100, 1, :2].transpose(1, 2)
    k.copy_(case.K)
    k[1, :, 60:] = 0
    case.K = case.V = k
    check(case)


def test_gradient_against_differences():
    """Directional derivatives of the oracle's forward pass against the kernel's gradients."""
    case = Case(1, 4, 2, 20, 70, 64, "fp16", True, seed=11)
    out = check(case)
    q, k, v, lam, g = (f64(x) for x in (case.Q, case.K, case.V, case.lam, case.dO))
    at = {"dQ": q, "dK": k, "dV": v, "dlam": lam}
    want = case.oracle(True)
    bound = case.bounds(want, True)
    rng = np.random.default_rng(0)
    h = 1e-5
    for name in at:
        x = dict(at)
        vec = rng.normal(size=at[name].shape)

        def f(s):
            x[name] = at[name] + s * vec
            return (g * token.diff_attn(x["dQ"], x["dK"], x["dV"], x["dlam"], case.n_keys, case.start, True)["O"]).sum()

        diff = (f(h) - f(-h)) / (2 * h)
        got = f64(out[name])
        step = 2.0 ** -11 if name != "dlam" else 2.0 ** -23
        slack = ((bound[name] + step * np.abs(got) + 2.0 ** -25) * np.abs(vec)).sum()
        assert abs((got * vec).sum() - diff) <= slack + 1e-5, name


def test_runs_give_the_same_bits():
    case = Case(3, 4, 2, 140, 260, 128, "bf16", True, [260, 100, 170], seed=13)
    first, again = check(case), check(case)
    for n in first:
        assert torch.equal(first[n], again[n]), n


def test_offsets_beyond_32_bits():
    """A cache whose heads and samples lie more than 2^32 bytes apart."""
    far = (1 << 31) + 512
    room = torch.empty(far + 300 * 128 * 4, dtype=torch.bfloat16, device="cuda")
    case = Case(2, 4, 2, 3, 300, 128, "bf16", True, [300, 150], seed=15)
    for name, offset in (("K", 0), ("V", 300 * 128 * 2)):
        view = room.as_strided((2, 2, 300, 128), (far, 300 * 128, 128, 1), offset)
        view.copy_(getattr(case, name))
        setattr(case, name, view)
    out = torch.empty_like(case.Q)
    ws = torch.empty(max(api.da2_diff_ws_bytes(case.Q, case.K), 16), dtype=torch.uint8, device="cuda")
    api.da2_diff_attn(case.Q, case.K, case.V, case.lam, out, ws, **case.how())
    want = case.oracle(False)
    close(out, want["O"], case.bounds(want, False)["O"], "O")


def test_streams_and_graph_replays():
    """Both passes on a stream of their own, and captured: replays with new inputs, eager work in between, and two graphs
    that share a workspace, one after the other."""
    case = Case(2, 4, 2, 150, 150, 64, "bf16", True, seed=17)
    small = Case(2, 4, 2, 1, 3000, 64, "bf16", True, [3000, 1700], seed=18)
    ws = torch.empty(max(api.da2_diff_ws_bytes(case.Q, case.K, True), api.da2_diff_ws_bytes(small.Q, small.K)), dtype=torch.uint8, device="cuda")

    def bufs():
        like = {"O": case.Q, "dQ": case.Q, "dK": case.K, "dV": case.V, "dlam": case.lam}
        return {**{n: torch.full_like(x, float("nan")) for n, x in like.items()}, "lse": torch.empty(2, 4, 2, 150, device="cuda"),
                "small": torch.full_like(small.Q, float("nan"))}

    def train(o, w, stream=None):
        api.da2_diff_attn(case.Q, case.K, case.V, case.lam, o["O"], w, o["lse"], stream=stream, **case.how())
        api.da2_diff_attn_bwd(case.Q, case.K, case.V, case.lam, o["lse"], case.dO, o["dQ"], o["dK"], o["dV"], o["dlam"], w,
                              stream=stream, **case.how())

    def serve(o, w, stream=None):
        api.da2_diff_attn(small.Q, small.K, small.V, small.lam, o["small"], w, stream=stream, **small.how())

    eager, out = bufs(), bufs()
    train(eager, torch.empty_like(ws))
    serve(eager, torch.empty_like(ws))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    train(out, ws, side)
    serve(out, ws, side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(out[n], eager[n]) for n in out)
    graphs = []
    for f in (train, serve):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            f(out, ws)
        graphs.append(graph)
    for seed in (21, 22, 23):
        case.Q.copy_(make(2, 4, 150, 64, "bf16", seed))
        small.Q.copy_(make(2, 4, 1, 64, "bf16", seed))
        for x in out.values():
            x.fill_(float("nan"))
        for graph in graphs:
            graph.replay()
        train(eager, torch.empty_like(ws))
        serve(eager, torch.empty_like(ws))
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], eager[n]) for n in out)
