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
