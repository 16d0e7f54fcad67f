"""Host-only checks of the token operators: every refusal before the GPU is
touched, through the C entry points and the Python binding."""
import ctypes

import pytest
import torch

from paper_2609_32628_amd import _lib, api

FAKE = 0x1000   # never dereferenced: validation fails first
E, U, W = _lib.DA2_ERR_INVALID_ARG, _lib.DA2_ERR_UNSUPPORTED, _lib.DA2_ERR_WORKSPACE


def _desc(B, H, N, C, dtype=_lib.DA2_BF16):
    return _lib.Tensor(H * N * C, N * C, C, dtype, 0)


def _norm_desc(**kw):
    d = dict(kind=0, wdtype=_lib.DA2_FP32, plus_one=0, reserved=0, stride_b=0, eps=1e-6)
    d.update(kw)
    return _lib.NormDesc(*d.values())


def test_norm_refusals():
    L = _lib.lib()
    t, r, n = _desc(2, 3, 5, 64), _lib.Rows(2, 3, 5, 64), _norm_desc()
    far = _lib.Tensor(3 * 5 * 64, 5 * 64, 63, _lib.DA2_BF16, 0)   # rows overlap by an element
    f = L.da2_norm
    assert f(None, t, r, n, None, None, FAKE, t, None, None) == E
    assert f(FAKE, t, r, n, None, None, None, t, None, None) == E
    assert f(FAKE, None, r, n, None, None, FAKE, t, None, None) == E
    assert f(FAKE, t, None, n, None, None, FAKE, t, None, None) == E
    assert f(FAKE, t, r, None, None, None, FAKE, t, None, None) == E
    assert f(FAKE, t, r, n, None, None, 2 * FAKE, far, None, None) == E
    assert f(FAKE, t, r, n, None, None, FAKE, _lib.Tensor(15 * 64, 64, 3 * 64, 0, 0), None, None) == E   # in place, other strides
    assert f(FAKE, t, r, n, None, None, 2 * FAKE, _desc(2, 3, 5, 64, _lib.DA2_FP32), None, None) == E     # types differ
    assert f(FAKE, _desc(2, 3, 5, 64, 3), r, n, None, None, FAKE, t, None, None) == E
    for bad in [(0, 3, 5, 64), (2, 0, 5, 64), (2, 3, -1, 64), (2, 3, 5, 0), (65536, 1, 1, 8), (1, 65536, 65536, 8),
                (2, 32768, 32768, 8), (1, 1, 1, (1 << 24) + 1)]:
        assert f(FAKE, _desc(*bad), _lib.Rows(*bad), n, None, None, FAKE, _desc(*bad), None, None) == E, bad
    for bad in [dict(kind=2), dict(wdtype=3), dict(plus_one=2), dict(stride_b=63), dict(stride_b=-1), dict(eps=-1.0),
                dict(eps=float("nan")), dict(eps=float("inf"))]:
        assert f(FAKE, t, r, _norm_desc(**bad), FAKE, FAKE, FAKE, t, None, None) == E, bad
    neg = _lib.Tensor(-1, 5 * 64, 64, 0, 0)
    assert f(FAKE, neg, r, n, None, None, FAKE, t, None, None) == E


def test_norm_bwd_refusals():
    L = _lib.lib()
    t, r, n = _desc(2, 3, 5, 64), _lib.Rows(2, 3, 5, 64), _norm_desc()
    b = ctypes.c_int64()
    assert L.da2_norm_ws_bytes(r, 0, 0, b) == 0 and b.value >= 8 * 64
    need = b.value
    f = L.da2_norm_bwd
    ok = [FAKE, t, FAKE, t, r, n, None, FAKE, FAKE, t, None, None, None, 0, None]

    def refused(status, **kw):
        a = list(ok)
        for i, v in kw.items():
            a[int(i[1:])] = v
        assert f(*a) == status, kw

    refused(E, a0=None)
    refused(E, a2=None)
    refused(E, a7=None)
    refused(E, a8=None)                                    # nothing asked for
    refused(E, a9=None)
    refused(E, a1=_desc(2, 3, 5, 64, 1))
    refused(E, a9=_lib.Tensor(15 * 64, 64, 3 * 64, 0, 0))  # dX is X with other strides
    refused(E, a10=FAKE)                                   # dw without a workspace
    refused(W, a10=FAKE, a12=FAKE, a13=need - 1)
    refused(W, a11=FAKE, a12=FAKE, a13=0)
    assert L.da2_norm_ws_bytes(r, 0, 2, b) == E and L.da2_norm_ws_bytes(r, 5, 0, b) == E
    assert L.da2_norm_ws_bytes(r, 0, 0, None) == E and L.da2_norm_ws_bytes(None, 0, 0, b) == E
    assert L.da2_norm_ws_bytes(r, 0, 1, b) == 0 and b.value >= 2 * 8 * 64


def test_norm_binding_refusals():
    X = torch.zeros(2, 3, 5, 8)
    w = torch.ones(8)
    for call in (lambda: api.da2_norm(X, X),                                     # not on a GPU
                 lambda: api.da2_norm(X[0], X[0]),
                 lambda: api.da2_norm(X.transpose(2, 3), X.transpose(2, 3)),
                 lambda: api.da2_norm(X, X[:, :, :4]),
                 lambda: api.da2_norm(X, X.half()),
                 lambda: api.da2_norm(X.double(), X.double()),
                 lambda: api.da2_norm(X, X, w[:4]),
                 lambda: api.da2_norm(X, X, torch.ones(3, 8)),
                 lambda: api.da2_norm(X, X, torch.ones(1, 8).expand(2, 8)),
                 lambda: api.da2_norm(X, X, w, w.half()),
                 lambda: api.da2_norm(X, X, w, torch.ones(2, 8)),
                 lambda: api.da2_norm(X, X, w, w, stats=torch.zeros(2, 3, 5, 3)),
                 lambda: api.da2_norm_bwd(X, X, torch.zeros(2, 3, 5, 2), X, w, torch.ones(2, 8)),
                 lambda: api.da2_norm_bwd(X, X, torch.zeros(2, 3, 5, 2), X, w, w, w.half()),
                 lambda: api.da2_norm_bwd(X, X, None, X)):
        with pytest.raises((ValueError, _lib.Da2Error)):
            call()


def _rope_desc(layout=0, block=64, axes=1, rot=(64, 0, 0)):
    return _lib.RopeDesc(layout, block, axes, (ctypes.c_int32 * 3)(*rot))


BAD_ROPES = [dict(layout=2), dict(block=1, rot=(2, 0, 0)), dict(axes=0), dict(axes=4), dict(rot=(0, 0, 0)), dict(rot=(3, 0, 0)),
             dict(rot=(66, 0, 0)), dict(rot=(32, 32, 0)), dict(axes=2, rot=(64, 0, 0)), dict(axes=2, rot=(32, 34, 0)),
             dict(axes=3, rot=(20, 20, -2)), dict(block=65538, rot=(2, 0, 0))]


def test_rope_plan_refusals_and_values():
    L = _lib.lib()
    turns, scale = (ctypes.c_double * 32)(), ctypes.c_double()
    good = dict(scaling=0, orig_len=4096, base=1e4, factor=1.0, beta_fast=32.0, beta_slow=1.0)
    plan = lambda r, **kw: L.da2_rope_plan(r, _lib.RopeFreq(*dict(good, **kw).values()), turns, scale)  # noqa: E731
    assert plan(_rope_desc()) == 0 and turns[0] == pytest.approx(0.15915494309189535) and scale.value == 1.0
    for bad in BAD_ROPES:
        assert plan(_rope_desc(**bad)) == E, bad
    for bad in [dict(scaling=4), dict(scaling=-1), dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")),
                dict(factor=2.0), dict(scaling=1, factor=0.5), dict(scaling=1, factor=float("inf")),
                dict(scaling=3, factor=2.0, orig_len=0), dict(scaling=3, factor=2.0, beta_slow=0.0),
                dict(scaling=3, factor=2.0, beta_fast=0.5), dict(scaling=3, factor=2.0, beta_fast=float("inf"))]:
        assert plan(_rope_desc(), **bad) == E, bad
    f = _lib.RopeFreq(*good.values())
    assert L.da2_rope_plan(_rope_desc(), None, turns, scale) == E and L.da2_rope_plan(None, f, turns, scale) == E
    assert L.da2_rope_plan(_rope_desc(), f, None, scale) == E and L.da2_rope_plan(_rope_desc(), f, turns, None) == E


def test_rope_refusals():
    L = _lib.lib()
    t, r = _desc(2, 3, 5, 64), _rope_desc()
    rows = dict(B=2, Hq=3, Hk=3, N=5, d=64, grid_h=0, grid_w=0, inverse=0)
    base = [r, FAKE, 1.0, FAKE, 5, _lib.RopeRows(*rows.values()), FAKE, t, 2 * FAKE, t, FAKE, t, 3 * FAKE, t, None]

    def refused(**kw):
        a = list(base)
        for i, v in kw.items():
            if i[0] == "a":
                a[int(i[1:])] = v
        a[5] = _lib.RopeRows(*dict(rows, **{k: v for k, v in kw.items() if k in rows}).values())
        assert L.da2_rope(*a) == E, kw

    for i in (0, 1, 6, 7, 8, 9, 10, 11, 12, 13):
        refused(**{f"a{i}": None})
    for bad in BAD_ROPES:
        refused(a0=_rope_desc(**bad))
    for bad in [dict(B=0), dict(Hq=0), dict(Hk=-1), dict(N=0), dict(d=0), dict(d=96), dict(inverse=2), dict(grid_h=2, grid_w=2),
                dict(B=65536), dict(Hq=65535), dict(B=4096, N=1 << 20)]:
        refused(**bad)
    refused(a2=float("nan"))
    refused(a4=4)
    refused(a4=-1)
    refused(a7=_desc(2, 3, 5, 64, 1))
    refused(a13=_desc(2, 3, 5, 64, 1))
    refused(a9=_lib.Tensor(15 * 64, 5 * 64, 32, 0, 0))                      # rows of the output overlap
    refused(a8=FAKE, a9=_lib.Tensor(15 * 64, 64, 3 * 64, 0, 0))             # in place with other strides
    refused(a3=None, a4=0, a0=_rope_desc(axes=2, rot=(32, 32, 0)))          # a grid of no width
    refused(a3=None, a4=0, a0=_rope_desc(axes=3, rot=(32, 16, 16)), grid_w=4)


def test_rope_binding_refusals():
    X = torch.zeros(2, 3, 5, 64)
    rope = api.da2_rope_plan(64, (64,), device="cpu")
    pos = torch.zeros(2, 5, 1, dtype=torch.int32)
    for call in (lambda: api.da2_rope(rope, X, X, pos=pos),                  # not on a GPU
                 lambda: api.da2_rope(rope, X, X.half(), pos=pos),
                 lambda: api.da2_rope(rope, X, X, X, None, pos=pos),
                 lambda: api.da2_rope(rope, X, X, X[:1], X[:1], pos=pos),
                 lambda: api.da2_rope(rope, X, X, X[:, :, :4], X[:, :, :4], pos=pos),
                 lambda: api.da2_rope(rope, X, X, pos=pos.long()),
                 lambda: api.da2_rope(rope, X, X, pos=pos[:, :4]),
                 lambda: api.da2_rope(rope, X, X, pos=pos[..., 0]),
                 lambda: api.da2_rope(rope, X, X, pos=torch.zeros(2, 10, 1, dtype=torch.int32)[:, ::2]),
                 lambda: api.da2_rope(api.Rope("half", 64, (64,), rope.turns[:31]), X, X, pos=pos),
                 lambda: api.da2_rope(api.Rope("half", 64, (64,), rope.turns.float()), X, X, pos=pos),
                 lambda: api.da2_rope(api.Rope("half", 64, (16,) * 4, rope.turns), X, X, pos=pos),
                 lambda: api.da2_rope_plan(64, (64, 2), device="cpu"),
                 lambda: api.da2_rope_plan(64, (), device="cpu")):
        with pytest.raises((ValueError, _lib.Da2Error)):
            call()
