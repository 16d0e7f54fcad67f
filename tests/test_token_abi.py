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


DIFF = dict(B=2, Hq=4, Hk=2, N=5, M=7, d=64, causal=0, reserved=0, scale=0.1)


def _diff_problem(**kw):
    return _lib.DiffProblem(*dict(DIFF, **kw).values())


BAD_DIFFS = [dict(B=0), dict(Hq=0), dict(Hk=0), dict(N=0), dict(M=-1), dict(d=0), dict(Hq=5), dict(Hk=3), dict(causal=2),
             dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=2.0 ** 65),
             dict(scale=2.0 ** -65), dict(B=65536), dict(N=(1 << 30) + 1), dict(M=(1 << 30) + 1), dict(B=60000, Hq=600, Hk=600)]


def test_diff_problem_refusals():
    L = _lib.lib()
    b = ctypes.c_int64()
    assert L.da2_diff_ws_bytes(_diff_problem(), 0, b) == 0 and b.value >= 0
    assert L.da2_diff_ws_bytes(_diff_problem(), 1, b) == 0 and b.value >= 2 * 4 * 5 * 20
    for bad in BAD_DIFFS:
        assert L.da2_diff_ws_bytes(_diff_problem(**bad), 1, b) == E, bad
    assert L.da2_diff_ws_bytes(_diff_problem(d=96), 0, b) == U
    assert L.da2_diff_ws_bytes(_diff_problem(), 2, b) == E
    assert L.da2_diff_ws_bytes(None, 0, b) == E and L.da2_diff_ws_bytes(_diff_problem(), 0, None) == E


def _refusals(call, base, cases):
    for status, change in cases:
        a = list(base)
        for i, v in change.items():
            a[i] = v
        assert call(*a) == status, change


def test_diff_refusals():
    L = _lib.lib()
    q, k = _desc(2, 4, 5, 64), _desc(2, 2, 7, 64)
    A = [FAKE * (i + 1) for i in range(8)]
    #       0                1     2  3     4  5     6  7     8     9     10    11 12    13    14       15
    base = [_diff_problem(), A[0], q, A[1], k, A[2], k, FAKE, None, None, A[3], q, None, FAKE, 1 << 30, None]
    odd = _lib.Tensor(4 * 5 * 64, 5 * 64, 68, 0, 0)
    wide = _lib.Tensor(4 * 5 << 25, 5 << 25, (1 << 24) + 8, 0, 0)
    over = _lib.Tensor(4 * 5 * 64, 5 * 64, 56, 0, 0)
    f32, f16 = _desc(2, 4, 5, 64, _lib.DA2_FP32), _desc(2, 4, 5, 64, _lib.DA2_FP16)
    need = [(E, {i: None}) for i in (0, 1, 2, 3, 4, 5, 6, 7, 10, 11)]
    _refusals(L.da2_diff_attn, base, need + [
        (E, {1: FAKE + 2}), (E, {3: FAKE + 8}), (E, {10: 3 * FAKE + 2}), (E, {2: odd}), (E, {2: wide}), (E, {11: over}),
        (U, {2: f32, 4: _desc(2, 2, 7, 64, 1), 6: _desc(2, 2, 7, 64, 1), 11: f32}), (E, {2: f16}), (E, {2: _desc(2, 4, 5, 64, 3)}),
        (E, {10: A[0]}), (E, {10: A[1]}), (E, {10: A[2]}),
        (U, {0: _diff_problem(d=32)})] + [(E, {0: _diff_problem(**bad)}) for bad in BAD_DIFFS])
    # a problem whose keys are split: a workspace that is missing, too small or not aligned
    p = _diff_problem(N=1, M=4000)
    b = ctypes.c_int64()
    assert L.da2_diff_ws_bytes(p, 0, b) == 0 and b.value > 0
    split = dict(zip((0, 2, 4, 6, 11), (p, _desc(2, 4, 1, 64), _desc(2, 2, 4000, 64), _desc(2, 2, 4000, 64), _desc(2, 4, 1, 64))))
    _refusals(L.da2_diff_attn, base, [(E, {**split, 13: None}), (E, {**split, 13: FAKE + 4}), (W, {**split, 14: b.value - 1})])


def test_diff_bwd_refusals():
    L = _lib.lib()
    q, k = _desc(2, 4, 5, 64), _desc(2, 2, 7, 64)
    A = [FAKE * (i + 1) for i in range(12)]
    b = ctypes.c_int64()
    assert L.da2_diff_ws_bytes(_diff_problem(), 1, b) == 0
    #       0                1     2  3     4  5     6  7     8     9     10    11    12 13   14 15   16 17   18 19    20    21       22
    base = [_diff_problem(), A[0], q, A[1], k, A[2], k, FAKE, None, None, FAKE, A[5], q, A[6], q, A[7], k, A[8], k, FAKE, FAKE, b.value, None]
    over = _lib.Tensor(4 * 5 * 64, 5 * 64, 56, 0, 0)
    cases = [(E, {i: None}) for i in (0, 1, 2, 3, 4, 5, 6, 7, 10, 11, 12, 13, 14, 15, 16, 17, 18, 19, 20)]
    cases += [(W, {21: b.value - 1}), (E, {20: FAKE + 4}), (E, {13: A[0]}), (E, {15: A[2]}), (E, {17: A[7]}), (E, {13: A[5]}),
              (E, {14: over}), (E, {11: A[5] + 2}), (E, {12: _desc(2, 4, 5, 64, 2)})]
    cases += [(E, {0: _diff_problem(**bad)}) for bad in BAD_DIFFS]
    _refusals(L.da2_diff_attn_bwd, base, cases)


def test_diff_binding_refusals():
    Q, K = torch.zeros(2, 4, 5, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 7, 64, dtype=torch.bfloat16)
    lam, O = torch.zeros(4), torch.zeros_like(Q)
    ok = dict(kv_lens=torch.zeros(2, dtype=torch.int32), q_start=torch.zeros(2, dtype=torch.int32))
    call = api.da2_diff_attn
    for f in (lambda: call(Q, K, K, lam, O, **ok),                                         # not on a GPU
              lambda: call(Q, K[:, :, :, :32], K, lam, O),
              lambda: call(Q, K[:1], K, lam, O),
              lambda: call(Q[:, :3], K, K, lam[:3], O[:, :3]),
              lambda: call(Q, K, K[:, :1], lam, O),
              lambda: call(Q, K.half(), K, lam, O),
              lambda: call(Q, K, K, None, O),
              lambda: call(Q, K, K, lam[:3], O),
              lambda: call(Q, K, K, lam.double(), O),
              lambda: call(Q, K, K, lam, O[:1]),
              lambda: call(Q, K, K, lam, O.float()),
              lambda: call(Q, K, K, lam, O, lse=torch.zeros(2, 4, 5, 2)),
              lambda: call(Q, K, K, lam, O, kv_lens=torch.zeros(2)),
              lambda: call(Q, K, K, lam, O, q_start=torch.zeros(3, dtype=torch.int32)),
              lambda: call(Q[0], K, K, lam, O),
              lambda: api.da2_diff_ws_bytes(Q[:, :, :, :32], K[:, :, :, :32]),
              lambda: api.da2_diff_attn_bwd(Q, K, K, lam, torch.zeros(2, 4, 2, 5), O, O, K, K, lam, None),
              lambda: api.da2_diff_attn_bwd(Q, K, K, lam, None, O, O, K, K[:, :1], lam, O)):
        with pytest.raises((ValueError, _lib.Da2Error)):
            f()


def test_outputs_that_share_memory_are_refused():
    """Q and K rotated into one tensor or into each other, and dw written where db is."""
    L = _lib.lib()
    t, A = _desc(2, 3, 5, 64), FAKE
    rows = _lib.RopeRows(2, 3, 3, 5, 64, 0, 0, 0)
    for q, qo, k, ko in ((A, 2 * A, 3 * A, 2 * A), (A, A, 2 * A, A), (A, 2 * A, 3 * A, A), (A, 3 * A, 3 * A, 2 * A)):
        assert L.da2_rope(_rope_desc(), 5 * A, 1.0, None, 0, rows, q, t, qo, t, k, t, ko, t, None) == E
    n = _lib.NormDesc(0, 1, 0, 0, 0, 1e-6)
    assert L.da2_norm_bwd(A, t, 2 * A, t, _lib.Rows(2, 3, 5, 64), n, None, 3 * A, None, None, 4 * A, 4 * A, 5 * A, 1 << 30, None) == E


def test_attention_refuses_what_it_would_rotate_wrongly():
    from types import SimpleNamespace
    buf = SimpleNamespace(p=None, fmt4="nvfp4", with16=False)
    Q, K = torch.ones(1, 1, 4, 64), torch.ones(1, 1, 4, 64)
    rope = api.Rope("half", 64, (32, 32), torch.zeros(32, dtype=torch.float64))
    with pytest.raises(ValueError, match="axes"):
        api.attention(Q, K, K, buf, 0, (1, 1, 2), Q, rope=rope)
    with pytest.raises(ValueError, match="one tensor"):
        api.attention(Q, Q, K, buf, 0, (1, 1, 2), Q, qk_norm=(None, None))
