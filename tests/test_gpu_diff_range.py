"""Differential attention on the GPU at the edges of its types' range: gradients of small and large size, keys of which one
is far from the others, rows of very many small weights.

Tolerance of the gradients' size: the 2-norm of the error over a whole gradient. Every rounded weight and score gradient is
off by at most u = finfo(type).eps / 2 of itself, and over the step around it evenly, so by u^2 / 3 of its square in the
mean; the roundings of different pairs do not depend on each other, so the mean squares add up: for dQ,
scale^2 u^2 / 3 sum_j dS_j^2 ((K_j - mean K)^2 + var K), as dQ takes each key's distance to a middle of the keys, which is
within a deviation of their mean; for dK the same with Q^2; for dV u^2 / 3 sum_i (P1 - lam P2)^2 dO^2. With more than 10^4
elements the sum is near its mean. The result is rounded to the type, subnormal numbers among them, by what rounding the
exact gradient gives. The error is at most 1.5 times both together; the float32 sums are finer by 2^-10 and more."""
import math

import numpy as np
import pytest
import torch

from oracle import token
from paper_2609_32628_amd import api
from test_gpu_diff import Case, T, check, f64

pytestmark = pytest.mark.gpu


def gradients(case):
    """Outputs of both passes."""
    out = {n: torch.full_like(x, float("nan")) for n, x in (("O", case.Q), ("dQ", case.Q), ("dK", case.K), ("dV", case.V), ("dlam", case.lam))}
    out["lse"] = torch.full((case.B, case.H, 2, case.N), float("nan"), device="cuda")
    ws = torch.full((api.da2_diff_ws_bytes(case.Q, case.K, True),), 0xFF, dtype=torch.uint8, device="cuda")
    api.da2_diff_attn(case.Q, case.K, case.V, case.lam, out["O"], ws, out["lse"], **case.how())
    ws.fill_(0xFF)
    api.da2_diff_attn_bwd(case.Q, case.K, case.V, case.lam, out["lse"], case.dO, out["dQ"], out["dK"], out["dV"], out["dlam"], ws,
                          **case.how())
    return out


def spread(case, first=0):
    """Mean square error of every element of dQ, dK and dV from the roundings of the weights and score gradients; the keys
    before ``first`` are not counted among those whose middle dQ takes."""
    h, u = case.d // 2, torch.finfo(case.Q.dtype).eps / 2
    scale = 1 / math.sqrt(h) if case.scale is None else case.scale
    var = {"dQ": np.zeros(case.Q.shape), "dK": np.zeros(case.K.shape), "dV": np.zeros(case.V.shape)}
    for b, n in enumerate(case.n_keys):
        see = token.diff_visible(case.N, case.M, n, case.start[b], case.causal)[:, :n]
        for hq in range(case.H):
            kh, lam = hq // (case.H // case.Hk), float(case.lam[hq])
            q, k, v, g = f64(case.Q[b, hq]), f64(case.K[b, kh, :n]), f64(case.V[b, kh, :n]), f64(case.dO[b, hq])
            P, _ = token._maps(q, k, see, scale)
            dP = g @ v.T
            var["dV"][b, kh, :n] += u * u / 3 * ((P[0] - lam * P[1]) ** 2).T @ g ** 2
            for m, f in ((0, 1.0), (1, lam)):
                c = slice(m * h, (m + 1) * h)
                dS2 = (u * scale * f * P[m] * (dP - (P[m] * dP).sum(-1, keepdims=True))) ** 2 / 3
                var["dQ"][b, hq, :, c] = dS2 @ ((k[:, c] - k[first:, c].mean(0)) ** 2 + k[first:, c].var(0))
                var["dK"][b, kh, :n, c] += dS2.T @ q[:, c] ** 2
    return var


def rounded(x, t):
    return f64(torch.from_numpy(x).to(t))


@pytest.mark.parametrize("size", [1e-5, 1e-4, 1e-3, 1.0, 1e3])
@pytest.mark.parametrize("B,H,Hk,N,M,d,causal,dtype", [
    (1, 2, 1, 200, 4096, 128, False, "fp16"), (1, 1, 1, 700, 4096, 64, False, "fp16"), (1, 4, 2, 600, 4500, 64, True, "fp16"),
    (2, 4, 2, 3000, 3000, 128, True, "fp16"), (1, 2, 2, 9000, 300, 64, False, "fp16"), (1, 2, 1, 200, 4096, 128, False, "bf16")])
def test_size_of_gradients(B, H, Hk, N, M, d, causal, dtype, size):
    """What comes back of a dO of any size: over thousands of keys the weights are small, and dS falls with dO below fp16's
    normal numbers. Q, K and V are taken smaller with a large one, so that the gradients stay numbers of the type."""
    case = Case(B, H, Hk, N, M, d, dtype, causal, seed=31)
    if size > 1:
        case.K *= 2.0 ** -6
        case.Q *= 2.0 ** -4
        case.V *= 0.25
    case.dO = (case.dO.float() * size).to(T[dtype])
    want, var, out = case.oracle(True), spread(case), gradients(case)
    for n in ("dQ", "dK", "dV"):
        off = np.linalg.norm(f64(out[n]) - want[n])
        own = np.linalg.norm(rounded(want[n], out[n].dtype) - want[n])
        assert np.abs(want[n]).max() < torch.finfo(out[n].dtype).max, n
        assert off <= 1.5 * (math.sqrt(var[n].sum()) + own), (n, off, math.sqrt(var[n].sum()), own)


@pytest.mark.parametrize("M", [2, 40])
@pytest.mark.parametrize("d,dtype", [(64, "fp16"), (128, "fp16"), (128, "bf16")])
def test_score_gradients_beyond_the_type(d, dtype, M):
    """dO V' of about 5 10^5, over few keys: dS passes fp16's largest number, dQ, dK and dV do not."""
    case = Case(1, 2, 2, 8, M, d, dtype, seed=33)
    case.Q *= 2.0 ** -6
    case.K *= 2.0 ** -6
    case.V *= 8
    case.dO = (case.dO.float() * 8e3).to(T[dtype])
    check(case)


@pytest.mark.parametrize("H,N,M,d,dtype", [(2, 130, 2048, 128, "bf16"), (2, 130, 2048, 64, "fp16"), (2, 9000, 400, 128, "bf16"), (40, 900, 300, 64, "bf16"),
                                           (36, 1000, 300, 128, "fp16")])
def test_a_large_first_key(H, N, M, d, dtype):
    """A first key 400 times as large as the others, which no query attends to: its weight, and with it what its dS is off,
    is zero, so dQ is as exact as without it."""
    case = Case(1, H, H, N, M, d, dtype, seed=35)
    case.Q += 1.5                # its distance from the other keys is along minus the queries' mean
    case.K[:, :, 0] = -400
    want, var, out = case.oracle(True), spread(case, 1), gradients(case)
    for n in ("dQ", "dK", "dV"):
        off = np.linalg.norm(f64(out[n]) - want[n])
        own = np.linalg.norm(rounded(want[n], out[n].dtype) - want[n])
        assert off <= 1.5 * (math.sqrt(var[n].sum()) + own), (n, off, math.sqrt(var[n].sum()), own)


def many_keys(N, dtype, bits):
    """O and lse of one key with a value of zero before 2^17 others with one, each of 2^-bits of its weight. There are heads
    enough that none of them is split; they share the keys' memory."""
    M, d = 2 ** 17, 64
    Q = torch.zeros(1, 256, N, d, dtype=T[dtype], device="cuda")
    K, V = (torch.zeros(1, 1, M, d, dtype=T[dtype], device="cuda") for _ in range(2))
    Q[..., 0], K[:, :, 0, 0], V[:, :, 1:] = 1, 1, 1
    out, lse = torch.full_like(Q, float("nan")), torch.full((1, 256, 2, N), float("nan"), device="cuda")
    K, V = K.expand(1, 256, M, d), V.expand(1, 256, M, d)
    ws = torch.empty(max(api.da2_diff_ws_bytes(Q, K), 1), dtype=torch.uint8, device="cuda")
    api.da2_diff_attn(Q, K, V, torch.zeros(256, device="cuda"), out, ws, lse, scale=bits * math.log(2))
    return out.double(), lse[0, :, 0].double(), M


@pytest.mark.parametrize("N", [1, 128, 600])
@pytest.mark.parametrize("bits,dtype", [(8.5, "fp16"), (20.5, "fp16"), (20.5, "bf16"), (25.5, "bf16")])
def test_a_sum_of_many_small_weights(bits, dtype, N):
    """A sum of M weights has M/16 + 40 additions in a chain, each off by 2^-24 of the sum; the logarithm adds the weights'
    own errors and a few steps of its size."""
    _, lse, M = many_keys(N, dtype, bits)
    want = bits * math.log(2) + math.log1p((M - 1) * 2.0 ** -bits)
    assert (lse - want).abs().max() <= (M / 16 + 40) * 2.0 ** -24 + 2.0 ** -20 + 4 * 2.0 ** -24 * want


@pytest.mark.parametrize("N", [1, 128, 600])
@pytest.mark.parametrize("bits,dtype", [(8.5, "fp16"), (20.5, "fp16"), (25.5, "fp16"), (30.5, "fp16"), (25.5, "bf16")])
def test_many_small_weights(bits, dtype, N):
    """The output is what the small weights come to together. Float32 sums of M weights are off by (M/16 + 40) 2^-24 of
    themselves, twice (weights and values), weights and outputs by u each, and fp16's smallest weights by 2^-25 of 2^-11 of
    the first key's each."""
    out, _, M = many_keys(N, dtype, bits)
    u = torch.finfo(T[dtype]).eps / 2
    rest = (M - 1) * 2.0 ** -bits
    want = rest / (1 + rest)
    tol = (2 * u + 2 * (M / 16 + 40) * 2.0 ** -24) * want + (M * 2.0 ** -36 if dtype == "fp16" else 0)
    assert (out - want).abs().max() <= tol


@pytest.mark.parametrize("H,N,M,d,causal", [(2, 9000, 300, 64, False), (4, 333, 333, 128, True), (2, 40, 40, 64, False)])
def test_scales_in_a_captured_pass(H, N, M, d, causal):
    """The powers of two are taken from the data at every replay: gradients of other sizes through one graph, bit for bit as
    outside of it."""
    case = Case(1, H, H, N, M, d, "fp16", causal, seed=37)
    gradients(case)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = gradients(case)
    for i, size in enumerate((1e-4, 30.0, 1e-2, 1.0)):
        g = torch.Generator(device="cuda")
        g.manual_seed(i)
        case.dO.copy_(torch.randn(case.dO.shape, generator=g, device="cuda") * size)
        case.lam.copy_(torch.randn(H, generator=g, device="cuda") * 3)
        for x in out.values():
            x.fill_(float("nan"))
        graph.replay()
        want = gradients(case)
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], want[n]) for n in out)


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "fp16")])
def test_lambda_gradient_of_values_far_from_zero(d, dtype):
    """dlam = -sum over the rows of del2, where values of one sign leave del2 much larger than what it changes by. A weight's
    own errors (2^-21, exponent and score) do not depend on another's and count with dP - del2; what a row's weights are off
    together, as by the float32 log sum, does not count at all. Roundings of del2's size: two sums of at most 12 terms in a
    chain (each addition off by 2^-24 of the sum so far, evenly: sqrt(12 / 3) 2^-24 / sqrt 3) and four more: 2^-23 of del2
    in the mean square. Over 64 heads the mean square is near its mean: the error is at most 1.5 times that."""
    case = Case(1, 64, 64, 100, 700, d, dtype, seed=39, q_scale=2.5)
    case.V += 16
    got, want = f64(gradients(case)["dlam"]), case.oracle(True)["dlam"]
    square = np.zeros(case.H)
    for h in range(case.H):
        P, _ = token._maps(f64(case.Q[0, h]), f64(case.K[0, h]), np.ones((case.N, case.M), bool), 1 / math.sqrt(d // 2))
        dP = f64(case.dO[0, h]) @ f64(case.V[0, h]).T
        delta = (P[1] * dP).sum(-1, keepdims=True)
        square[h] = (2.0 ** -46 * delta ** 2).sum() + (2.0 ** -42 * P[1] ** 2 * (dP - delta) ** 2).sum()
    assert math.sqrt(((got - want) ** 2 / square).mean()) <= 1.5
