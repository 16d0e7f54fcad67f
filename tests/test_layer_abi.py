"""Host-only checks of the projections, gated blocks and the norm and rotation of Q and K: every refusal before the GPU is
touched, through the C entry points and the Python binding."""
import ctypes

import pytest
import torch

from paper_2609_32628_amd import _lib, api

FAKE = 0x1000   # never dereferenced: validation fails first
E, U, W = _lib.DA2_ERR_INVALID_ARG, _lib.DA2_ERR_UNSUPPORTED, _lib.DA2_ERR_WORKSPACE
GOOD = dict(B=2, N=5, Hx=1, Cx=64, Hy=1, Cy=128, act=0, dtype=_lib.DA2_BF16)


def proj(**kw):
    return _lib.Proj(*dict(GOOD, **kw).values())


def desc(B, H, N, C, dtype=_lib.DA2_BF16):
    return _lib.Tensor(H * N * C, N * C, C, dtype, 0)


X, Y = desc(2, 1, 5, 64), desc(2, 1, 5, 128)
BAD_PROJ = [dict(B=0), dict(N=0), dict(Hx=-1), dict(Cx=0), dict(Hy=0), dict(Cy=-5), dict(B=65536), dict(act=6), dict(act=-1), dict(dtype=3),
            dict(Cx=(1 << 20) + 8), dict(Cy=(1 << 20) + 8), dict(Hx=2, Cx=32), dict(Hy=2, Cy=4), dict(B=1024, N=1 << 21),
            dict(B=1, N=1 << 30, Cy=8192)]


def needs(call, p, train):
    b = ctypes.c_int64()
    assert getattr(_lib.lib(), call)(p, train, b) == 0
    return b.value


@pytest.mark.parametrize("call", ["da2_linear_ws_bytes", "da2_glu_ws_bytes"])
def test_workspace_sizes(call):
    f = getattr(_lib.lib(), call)
    b = ctypes.c_int64()
    assert f(proj(), 0, b) == 0 and b.value >= 0
    assert f(proj(), 1, b) == 0 and b.value >= 2 * 10 * 128 + 2 * 64 * 128
    assert f(None, 0, b) == E and f(proj(), 0, None) == E and f(proj(), 2, b) == E and f(proj(), -1, b) == E
    assert f(proj(dtype=_lib.DA2_FP32), 0, b) == U
    for bad in BAD_PROJ:
        assert f(proj(**bad), 0, b) == E, bad
    for N in (1, 16, 17, 100, 5000, 1 << 20):
        for K in (1, 63, 64, 5120):
            for F in (1, 1000, 13824):
                assert f(proj(B=1, N=N, Cx=K, Cy=F), 1, b) == 0 and b.value >= 2 * N * F


def forward_calls():
    """(call, arguments that only the workspace keeps from running) of da2_linear and da2_glu, with a workspace needed."""
    p = proj(N=100, Cx=8192)
    x, y = desc(2, 1, 100, 8192), desc(2, 1, 100, 128)
    assert needs("da2_linear_ws_bytes", p, 0) > 0 and needs("da2_glu_ws_bytes", p, 0) > 0
    return [("da2_linear", [p, FAKE, x, 2 * FAKE, 8192, None, None, 0, None, None, 3 * FAKE, y, None, 4 * FAKE, 0, None],
             dict(X=1, x=2, W=3, stride=4, gate=6, gate_sb=7, R=8, r=9, Y=10, y=11, Z=12, ws=13)),
            ("da2_glu", [p, FAKE, x, 2 * FAKE, 8192, None, 3 * FAKE, y, None, 4 * FAKE, 0, None],
             dict(X=1, x=2, W=3, stride=4, Y=6, y=7, Z=8, ws=9))]


@pytest.mark.parametrize("which", [0, 1])
def test_forward_refusals(which):
    call, ok, at = forward_calls()[which]
    f = getattr(_lib.lib(), call)
    x, y = ok[at["x"]], ok[at["y"]]

    def refused(status, **kw):
        a = list(ok)
        for k, v in kw.items():
            a[at[k] if k in at else 0] = v
        assert f(*a) == status, kw

    refused(W)
    refused(E, p=None)
    for n in ("X", "x", "W", "Y", "y", "ws"):
        refused(E, **{n: None})
    for n in ("X", "W", "Y", "ws"):
        refused(E, **{n: FAKE + 8})                                       # not on 16 bytes
    for s in (8191, 8190, 8196, -8, 0, (1 << 22) + 8):
        refused(E, stride=s)
    refused(E, x=desc(2, 1, 100, 8192, _lib.DA2_FP16))
    refused(E, y=desc(2, 1, 100, 128, _lib.DA2_FP32))
    refused(E, x=_lib.Tensor(100 * 8192, 0, 8196, 0, 0))                  # a stride that is no whole number of 16 bytes
    refused(E, x=_lib.Tensor(100 * 8192, 0, (1 << 22) + 8, 0, 0))
    refused(E, x=_lib.Tensor(-8, 0, 8192, 0, 0))
    refused(E, y=_lib.Tensor(100 * 128, 0, 120, 0, 0))                    # rows overlap
    refused(E, Y=FAKE)
    refused(E, Y=2 * FAKE)
    for z in (FAKE, 2 * FAKE, 3 * FAKE, 5 * FAKE + 4):
        refused(E, Z=z)
    for bad in BAD_PROJ:
        refused(E, p=proj(**{**dict(N=100, Cx=8192), **bad}))
    refused(U, p=proj(N=100, Cx=8192, dtype=_lib.DA2_FP32), x=desc(2, 1, 100, 8192, 1), y=desc(2, 1, 100, 128, 1))
    if call == "da2_linear":
        refused(E, gate=FAKE, gate_sb=127)
        refused(E, gate=FAKE, gate_sb=-128)
        refused(E, R=5 * FAKE)                                            # no descriptor
        refused(E, R=5 * FAKE, r=desc(2, 1, 100, 128, _lib.DA2_FP16))
        refused(E, R=3 * FAKE, r=_lib.Tensor(200 * 128, 0, 256, 0, 0))    # in place, other strides
        refused(W, R=3 * FAKE, r=y)
        refused(E, R=5 * FAKE, r=y, Z=5 * FAKE)
    else:
        # both halves of a tile of weights within 32 bits
        big = proj(N=100, Cx=8192, Cy=1 << 19)
        refused(E, p=big, stride=8192, y=desc(2, 1, 100, 1 << 19))
    assert x is not None


@pytest.mark.parametrize("glu", [False, True])
def test_backward_refusals(glu):
    L = _lib.lib()
    p = proj(act=4)
    x, y = X, Y
    if glu:
        f, names = L.da2_glu_bwd, ("p", "dY", "dy", "X", "x", "W", "stride", "Z", "dX", "dx", "dW", "dstride", "dbias", "ws", "ws_bytes", "stream")
        ok = [p, FAKE, y, 2 * FAKE, x, 3 * FAKE, 64, 4 * FAKE, 5 * FAKE, x, 6 * FAKE, 64, 7 * FAKE, 9 * FAKE, 0, None]
    else:
        f, names = L.da2_linear_bwd, ("p", "dY", "dy", "X", "x", "W", "stride", "gate", "gate_sb", "Z", "dX", "dx", "dW", "dstride", "dbias", "dgate", "ws",
                                      "ws_bytes", "stream")
        ok = [p, FAKE, y, 2 * FAKE, x, 3 * FAKE, 64, 10 * FAKE, 0, 4 * FAKE, 5 * FAKE, x, 6 * FAKE, 64, 7 * FAKE, 8 * FAKE, 9 * FAKE, 0, None]

    def refused(status, **kw):
        a = list(ok)
        for k, v in kw.items():
            a[names.index(k)] = v
        assert f(*a) == status, kw

    refused(W)
    need = needs("da2_glu_ws_bytes" if glu else "da2_linear_ws_bytes", p, 1)
    refused(W, ws_bytes=need - 1)
    for n in ("p", "dY", "dy", "X", "x", "W", "Z", "dx", "ws"):
        refused(E, **{n: None})
    for n in ("dY", "X", "W", "Z", "dX", "dW", "ws"):
        refused(E, **{n: 16 * FAKE + 8})
    refused(E, dX=None, dW=None, dbias=None, **({} if glu else dict(dgate=None)))
    for n in ("stride", "dstride"):
        for s in (56, 63, 65, -64, (1 << 22) + 8):
            refused(E, **{n: s})
    refused(E, dx=_lib.Tensor(5 * 64, 0, 56, 0, 0))
    outs = ["dX", "dW", "dbias"] + ([] if glu else ["dgate"])
    for i, n in enumerate(outs):
        for m in ["dY", "X", "W", "Z"] + outs[:i]:
            refused(E, **{n: ok[names.index(m)]})
    refused(U, p=proj(act=4, dtype=1), dy=desc(2, 1, 5, 128, 1), x=desc(2, 1, 5, 64, 1), dx=desc(2, 1, 5, 64, 1))
    refused(E, p=proj(B=512, N=8193, act=4))          # more tokens than a row of the transposed copies holds
    if not glu:
        refused(E, gate=None)                         # dgate without a gate
        refused(E, gate_sb=100)
        refused(E, p=proj(), Z=None)                  # dgate needs the sums, whatever the activation
        refused(W, p=proj(), Z=None, dgate=None)
    else:
        refused(E, p=proj(), Z=None)


def rope_args(**kw):
    r = _lib.RopeDesc(0, 64, 1, (ctypes.c_int32 * 3)(64, 0, 0))
    rows = dict(B=2, Hq=3, Hk=3, N=5, d=64, grid_h=0, grid_w=0, inverse=0)
    rows.update({k: v for k, v in kw.items() if k in rows})
    norm = dict(kind=1, wdtype=0, plus_one=0, reserved=0, stride_b=0, eps=1e-6)
    norm.update({k: v for k, v in kw.items() if k in norm})
    return r, _lib.RopeRows(*rows.values()), _lib.NormDesc(*norm.values())


BAD_QK = [(dict(B=0), E), (dict(Hq=0), E), (dict(Hk=-1), E), (dict(N=0), E), (dict(d=0), E), (dict(d=96), E), (dict(inverse=1), E), (dict(grid_h=2, grid_w=2), E),
          (dict(B=65536), E), (dict(Hq=65535), E), (dict(B=64, N=1 << 20), E), (dict(d=1024), U), (dict(kind=2), E), (dict(wdtype=3), E), (dict(plus_one=2), E),
          (dict(stride_b=64), E), (dict(eps=-1.0), E), (dict(eps=float("nan")), E)]


def test_qk_refusals():
    L = _lib.lib()
    t = desc(2, 3, 5, 64)
    r, s, n = rope_args()
    base = [r, FAKE, 1.0, FAKE, 5, s, n, None, None, FAKE, t, 2 * FAKE, t, 3 * FAKE, t, 4 * FAKE, t, None]

    def refused(status, **kw):
        a = list(base)
        for k, v in kw.items():
            if k[0] == "a" and k[1:].isdigit():
                a[int(k[1:])] = v
        a[5], a[6] = rope_args(**kw)[1:] if 5 not in [int(k[1:]) for k in kw if k[1:].isdigit()] else (None, n)
        assert L.da2_qk_norm_rope(*a) == status, kw

    for i in (0, 1, 5, 9, 10, 11, 12, 13, 14, 15, 16):
        refused(E, **{f"a{i}": None})
    for kw, status in BAD_QK:
        refused(status, **kw)
    refused(E, a2=float("inf"))
    refused(E, a4=4)
    refused(E, a12=_lib.Tensor(15 * 64, 5 * 64, 63, 0, 0))
    refused(E, a11=FAKE, a12=_lib.Tensor(15 * 64, 64, 3 * 64, 0, 0))     # in place, other strides
    refused(E, a15=2 * FAKE)                                             # Ko is Qo
    refused(E, a15=FAKE)                                                 # Ko is Q
    refused(E, a14=desc(2, 3, 5, 64, 1))
    b = ctypes.c_int64()
    assert L.da2_qk_norm_rope_ws_bytes(s, b) == 0 and b.value >= 8 * 64
    assert L.da2_qk_norm_rope_ws_bytes(None, b) == E and L.da2_qk_norm_rope_ws_bytes(s, None) == E
    assert L.da2_qk_norm_rope_ws_bytes(rope_args(d=1024)[1], b) == U


def test_qk_bwd_refusals():
    L = _lib.lib()
    t = desc(2, 3, 5, 64)
    r, s, n = rope_args()
    need = ctypes.c_int64()
    assert L.da2_qk_norm_rope_ws_bytes(s, need) == 0
    ok = [r, FAKE, 1.0, FAKE, 5, s, n, None, None, FAKE, t, 2 * FAKE, t, 3 * FAKE, t, 4 * FAKE, t, 5 * FAKE, t, 6 * FAKE, t, 7 * FAKE, 8 * FAKE, 9 * FAKE, 0, None]

    def refused(status, **kw):
        a = list(ok)
        for k, v in kw.items():
            a[int(k[1:])] = v
        assert L.da2_qk_norm_rope_bwd(*a) == status, kw

    refused(W)
    refused(W, a24=need.value - 1)
    for i in (0, 1, 5, 6, 9, 10, 11, 12, 13, 14, 15, 16, 17, 18, 19, 20, 23):
        refused(E, **{f"a{i}": None})
    refused(E, a23=9 * FAKE + 4)
    refused(E, a22=7 * FAKE)                    # dw_q is dw_k
    refused(E, a19=3 * FAKE)                    # dK is dQ
    refused(E, a13=4 * FAKE)                    # dQ is dKo
    refused(E, a13=FAKE, a14=_lib.Tensor(15 * 64, 64, 3 * 64, 0, 0))
    refused(E, a5=rope_args(Hk=0)[1])           # dw_k without K
    refused(U, a5=rope_args(d=576)[1])


def test_binding_refusals():
    X, Y = torch.zeros(2, 1, 5, 64, dtype=torch.float16), torch.zeros(2, 1, 5, 128, dtype=torch.float16)
    W = torch.zeros(128, 64, dtype=torch.float16)
    z = torch.zeros(2, 5, 128)
    b = torch.zeros(128, dtype=torch.float16)
    rope = api.da2_rope_plan(64, (64,), device="cpu")
    Q = torch.zeros(2, 3, 5, 64)
    for call in (lambda: api.da2_linear(X, W, Y),                              # not on a GPU
                 lambda: api.da2_linear(X[0], W, Y),
                 lambda: api.da2_linear(X, W.t(), Y),
                 lambda: api.da2_linear(X, W.bfloat16(), Y),
                 lambda: api.da2_linear(X, W[:, :32], Y),
                 lambda: api.da2_linear(X, W, Y[:, :, :3]),
                 lambda: api.da2_linear(X, W, Y.bfloat16()),
                 lambda: api.da2_linear(X, W, Y, b[:64]),
                 lambda: api.da2_linear(X, W, Y, b.float()),
                 lambda: api.da2_linear(X, W, Y, gate=torch.zeros(3, 128, dtype=torch.float16)),
                 lambda: api.da2_linear(X, W, Y, gate=b.expand(2, 128)),
                 lambda: api.da2_linear(X, W, Y, residual=X),
                 lambda: api.da2_linear(X, W, Y, Z=z.half()),
                 lambda: api.da2_linear(X, W, Y, Z=z[..., :64]),
                 lambda: api.da2_linear(X, W, Y, ws=torch.zeros(4, 4, dtype=torch.uint8).t()),
                 lambda: api.da2_linear_bwd(Y, X, W, z, dX=Y),
                 lambda: api.da2_linear_bwd(Y, X, W, z, dW=W.t()),
                 lambda: api.da2_linear_bwd(Y, X, W, z, gate=b, dgate=torch.zeros(2, 128, dtype=torch.float16)),
                 lambda: api.da2_glu(X, W, Y),                                 # half of the weights
                 lambda: api.da2_glu(X, torch.cat([W, W]), Y, b),
                 lambda: api.da2_glu_bwd(Y, X, torch.cat([W, W]), z),
                 lambda: api.da2_qk_norm_rope(rope, Q, Q),
                 lambda: api.da2_qk_norm_rope(rope, Q, Q, w_q=torch.ones(32)),
                 lambda: api.da2_qk_norm_rope(rope, Q, Q, Q, Q, torch.ones(64), torch.ones(64).half()),
                 lambda: api.da2_qk_norm_rope(rope, Q, Q, w_q=torch.ones(128)[::2]),
                 lambda: api.da2_qk_norm_rope(rope, Q, Q, Q),
                 lambda: api.da2_qk_norm_rope_bwd(rope, Q, Q[:, :2], Q),
                 lambda: api.da2_qk_norm_rope_bwd(rope, Q, Q, Q, Q, None, Q)):
        with pytest.raises((ValueError, _lib.Da2Error)):
            call()
    with pytest.raises(KeyError):
        api.da2_linear(X, W, Y, act="swish")
