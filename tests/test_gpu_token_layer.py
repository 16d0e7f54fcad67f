"""The token operators together, as a layer uses them: norm and rotary positions in front of the mixed-precision attention,
and a differential-attention layer forward and backward against the float64 oracle's chain."""
import numpy as np
import pytest
import torch

from gpu_harness import SMALL, inputs, problem_of, to_device
from oracle import token
from paper_2609_32628_amd import api

pytestmark = pytest.mark.gpu


def f64(x):
    return x.double().cpu().numpy()


@pytest.mark.parametrize("axes", [(128,), (44, 42, 42)])
def test_norm_and_rope_in_front_of_the_mixed_attention(axes):
    """attention(qk_norm, rope) is the norms, the rotation and the four calls; without them nothing changes."""
    p = problem_of(SMALL)
    Q, K, V = (to_device(x, SMALL) for x in inputs(SMALL))
    rope = api.da2_rope_plan(128, axes)
    w = [torch.rand(128, device="cuda").to(torch.bfloat16) + 0.5 for _ in range(2)]
    buf = api.alloc(p, SMALL.scope)
    q, k = Q.clone(), K.clone()
    for x, wx in ((q, w[0]), (k, w[1])):
        api.da2_norm(x, x, wx, kind="rms")
    grid = None if len(axes) == 1 else (SMALL.Hg, SMALL.Wg)
    api.da2_rope(rope, q, q, k, k, grid=grid)
    want = api.attention(q, k, V, buf, SMALL.lam, SMALL.budgets, torch.empty_like(Q)).clone()
    classes = buf.cls.clone()
    plain = api.attention(Q, K, V, buf, SMALL.lam, SMALL.budgets, torch.empty_like(Q)).clone()
    q2, k2 = Q.clone(), K.clone()
    got = api.attention(q2, k2, V, buf, SMALL.lam, SMALL.budgets, torch.empty_like(Q), qk_norm=w, rope=rope)
    assert torch.equal(got, want) and torch.equal(buf.cls, classes) and torch.equal(q2, q) and torch.equal(k2, k)
    assert not torch.equal(plain, want)


class Layer:
    """x -> layer norm -> (as Q, K, V with shared key heads) -> rotary positions of both halves -> differential attention
    -> RMS norm of the heads."""

    def __init__(self, dtype=torch.float16):
        g = torch.Generator(device="cuda")
        g.manual_seed(5)
        new = lambda *n: torch.randn(n, generator=g, device="cuda").to(dtype)  # noqa: E731
        self.B, self.H, self.Hk, self.N, self.d = 2, 4, 2, 50, 64
        self.lens = torch.tensor([50, 31], dtype=torch.int32, device="cuda")
        self.start = torch.zeros(2, dtype=torch.int32, device="cuda")
        self.q, self.k, self.v = new(2, 4, 50, 64), new(2, 2, 50, 64), new(2, 2, 50, 64)
        self.w = [1 + 0.2 * new(64) for _ in range(3)]
        self.lam = torch.tensor([0.2, 0.4, 0.5, 0.7], device="cuda")
        self.rope = api.da2_rope_plan(32, (32,), "half")
        self.dy = new(2, 4, 50, 64)
        self.how = dict(kv_lens=self.lens, q_start=self.start, causal=True)

    def gpu(self):
        s = self
        e = torch.empty_like
        st = [torch.empty(2, h, 50, 2, device="cuda") for h in (4, 2, 4)]
        q, k, o, y = e(s.q), e(s.k), e(s.q), e(s.q)
        api.da2_norm(s.q, q, s.w[0], eps=1e-5, stats=st[0])
        api.da2_norm(s.k, k, s.w[1], eps=1e-5, stats=st[1])
        api.da2_rope(s.rope, q, q, k, k)
        lse = torch.empty(2, 4, 2, 50, device="cuda")
        ws = torch.empty(max(api.da2_diff_ws_bytes(q, k, True), *(api.da2_norm_ws_bytes(x, s.w[0]) for x in (s.q, s.k))),
                         dtype=torch.uint8, device="cuda")
        api.da2_diff_attn(q, k, s.v, s.lam, o, ws, lse=lse, **s.how)
        api.da2_norm(o, y, s.w[2], kind="rms", eps=1e-5, stats=st[2])
        out = {"y": y}
        do, dq, dk = e(o), e(q), e(k)
        out.update(dv=e(s.v), dlam=e(s.lam), dw0=e(s.w[0]), dw1=e(s.w[1]), dw2=e(s.w[2]), dq=e(s.q), dk=e(s.k))
        api.da2_norm_bwd(s.dy, o, st[2], do, s.w[2], out["dw2"], kind="rms", ws=ws)
        api.da2_diff_attn_bwd(q, k, s.v, s.lam, lse, do, dq, dk, out["dv"], out["dlam"], ws, **s.how)
        api.da2_rope(s.rope, dq, dq, dk, dk, inverse=True)
        api.da2_norm_bwd(dq, s.q, st[0], out["dq"], s.w[0], out["dw0"], ws=ws)
        api.da2_norm_bwd(dk, s.k, st[1], out["dk"], s.w[1], out["dw1"], ws=ws)
        return out

    def forward64(self, t):
        s = self
        pos = np.broadcast_to(np.arange(50)[None, :, None], (2, 50, 1))
        turn = lambda x: token.rope(x, pos, f64(s.rope.turns), (32,), 1.0, "half", 32)  # noqa: E731
        q = turn(token.norm(t["dq"], t["dw0"], eps=1e-5)[0])
        k = turn(token.norm(t["dk"], t["dw1"], eps=1e-5)[0])
        o = token.diff_attn(q, k, t["dv"], t["dlam"], [50, 31], [0, 0], True)["O"]
        return token.norm(o, t["dw2"], kind="rms", eps=1e-5)[0]


def test_a_differential_layer_forward_and_backward():
    """End to end in fp16 (u = 2^-11). Two roundings of each of q and k move a score by at most 4 u scale |q|.|k| <= 4 u
    sqrt(32) max |q| max |k| / 1 (norm rows: |q|.|k| <= |q| |k| ~ 32 for a half), about 0.011, and so a weight by 1.1% at
    most and in root mean square over a row's channels and keys by less than u sqrt(8) ~ 0.14%; the other stages round
    three more times. A relative error of 2% in the 2-norm is more than ten times that, and a stage missing, a factor or an
    order that is wrong is an error of order one. Gradients are compared along random directions with central differences
    of the float64 chain, whose sums of about 10^4 random-signed terms lose a factor of a few to cancellation: 10%."""
    layer = Layer()
    out = layer.gpu()
    at = {"dq": f64(layer.q), "dk": f64(layer.k), "dv": f64(layer.v), "dlam": f64(layer.lam),
          "dw0": f64(layer.w[0]), "dw1": f64(layer.w[1]), "dw2": f64(layer.w[2])}
    want = layer.forward64(at)
    assert np.linalg.norm(f64(out["y"]) - want) <= 0.02 * np.linalg.norm(want)
    dy = f64(layer.dy)
    rng = np.random.default_rng(1)
    for name in at:
        # the direction of the gradient itself, so that nothing cancels, with some noise
        g = f64(out[name])
        v = g / np.linalg.norm(g) + 0.1 * rng.normal(size=g.shape) / np.sqrt(g.size)
        h = 1e-5
        diff = ((layer.forward64({**at, name: at[name] + h * v}) - layer.forward64({**at, name: at[name] - h * v})) * dy).sum() / (2 * h)
        assert abs((g * v).sum() - diff) <= 0.1 * abs(diff), (name, (g * v).sum(), diff)


def test_a_captured_layer():
    """The chain of a training step captured once and replayed with new inputs gives the eager results bit for bit."""
    layer = Layer(torch.bfloat16)
    layer.gpu()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer.gpu()
    for seed in (1, 2, 3):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        layer.q.copy_(torch.randn(layer.q.shape, generator=g, device="cuda"))
        for x in out.values():
            x.fill_(float("nan"))
        graph.replay()
        eager = layer.gpu()
        torch.cuda.synchronize()
        for n in out:
            assert torch.equal(out[n], eager[n]), n


def test_unlike_devices_are_refused_before_the_call():
    x = torch.zeros(1, 1, 2, 64, device="cuda")
    with pytest.raises(ValueError):
        api.da2_norm(x, x, torch.ones(64))
    with pytest.raises(ValueError):
        api.da2_norm(x, torch.zeros(1, 1, 2, 64))
