"""Host-only checks of the token operators at the ends of what they take: sizes and strides that add up beyond 64 bits,
limits that a launch has and those that none has, workspaces and weights as torch lays them out."""
import ctypes

import pytest
import torch

from paper_2609_32628_amd import _lib, api

FAKE = 0x1000   # never dereferenced: validation fails first
E, U, W = _lib.DA2_ERR_INVALID_ARG, _lib.DA2_ERR_UNSUPPORTED, _lib.DA2_ERR_WORKSPACE


def test_outputs_whose_spans_pass_64_bits_are_refused():
    """Strides and extents whose product wraps: rows of sample 1 are rows of sample 0."""
    L = _lib.lib()
    for N in ((1 << 25) + 1, (1 << 24) + 1, 3, (1 << 31) - 1):
        for stride in (1 << 39, 1 << 40):
            out = _lib.Tensor(1 << 40, 0, stride, _lib.DA2_BF16, 0)
            x = _lib.Tensor(0, 0, 0, _lib.DA2_BF16, 0)
            n = _lib.NormDesc(0, _lib.DA2_FP32, 0, 0, 0, 1e-6)
            assert L.da2_norm(FAKE, x, _lib.Rows(2, 1, N, 64), n, None, None, 2 * FAKE, out, None, None) == E, (N, stride)


def test_long_prompts_have_no_limit_but_the_launches():
    L, b = _lib.lib(), ctypes.c_int64()
    size = lambda **kw: L.da2_diff_ws_bytes(_lib.DiffProblem(*{**dict(B=1, Hq=1, Hk=1, N=1, M=1, d=128, causal=0, reserved=0, scale=0.1),  # noqa: E731
                                                               **kw}.values()), 1, b)
    for ok in (dict(N=(1 << 28) - 64), dict(N=(1 << 28) + 64), dict(N=(1 << 29) - 256, d=64), dict(Hq=1 << 22, N=100), dict(M=1 << 30),
               dict(Hq=(1 << 23) - 600)):
        assert size(**ok) == 0 and b.value >= 4 * 4 * ok.get("N", 1) * ok.get("Hq", 1), ok
    for bad in (dict(N=1 << 29), dict(N=1 << 30), dict(N=(1 << 30) + 1), dict(M=(1 << 30) + 1), dict(Hq=1 << 23), dict(Hq=1 << 23, N=256), dict(Hq=2, N=1 << 30),
                dict(Hq=2048, Hk=2048, M=1 << 30)):
        assert size(**bad) == E, bad


def test_outputs_may_lie_apart():
    """Rows more than 2^24 elements apart are refused where a tile is copied from them, not where results are stored. (A CPU
    has no device to launch on: what passes the checks is UNSUPPORTED.)"""
    if torch.cuda.is_available():
        pytest.skip("would launch")
    L = _lib.lib()
    p = _lib.DiffProblem(1, 1, 1, 5, 7, 64, 0, 0, 0.1)
    q, k, far = (_lib.Tensor(0, 0, s, _lib.DA2_BF16, 0) for s in (64, 64, (1 << 24) + 8))
    A = [FAKE * (i + 1) for i in range(8)]
    call = lambda q, k, o: L.da2_diff_attn(p, A[0], q, A[1], k, A[2], k, FAKE, None, None, A[3], o, None, FAKE, 1 << 30, None)  # noqa: E731
    assert call(q, k, far) == U and call(far, k, q) == E and call(q, far, q) == E
    back = lambda q, do, dq, dk: L.da2_diff_attn_bwd(p, A[0], q, A[1], k, A[2], k, FAKE, None, None, FAKE, A[3], do, A[4], dq, A[5], dk, A[6],  # noqa: E731
                                                     dk, FAKE, FAKE, 1 << 30, None)
    assert back(q, q, far, far) == U and back(far, q, q, k) == E and back(q, far, q, k) == E


def test_workspaces_hold_what_their_elements_count():
    """A byte repeated, or every second one, counts more elements than it has memory behind its address."""
    Q = torch.zeros(1, 2, 1, 64, dtype=torch.bfloat16)
    K = torch.zeros(1, 2, 4000, 64, dtype=torch.bfloat16)
    X, w, stats = torch.zeros(1, 1, 5, 8), torch.ones(8), torch.zeros(1, 1, 5, 2)
    for ws in (torch.zeros(1, dtype=torch.uint8).expand(1 << 22), torch.zeros(1 << 23, dtype=torch.uint8)[::2]):
        for call in (lambda: api.da2_diff_attn(Q, K, K, torch.zeros(2), torch.zeros_like(Q), ws),
                     lambda: api.da2_diff_attn_bwd(Q, K, K, torch.zeros(2), torch.zeros(1, 2, 2, 1), Q, Q, K, K, torch.zeros(2), ws),
                     lambda: api.da2_norm_bwd(X, X, stats, X, w, w, ws=ws)):
            with pytest.raises(ValueError, match="contiguous"):
                call()


def test_strides_of_one_sample_are_not_looked_at():
    """A slice of one sample's modulation beside a packed tensor for its gradient: the distance to a next sample is nobody's.
    (The call gets as far as to see that nothing is on a GPU.)"""
    X, stats = torch.zeros(1, 1, 5, 8), torch.zeros(1, 1, 5, 2)
    w, b = torch.ones(1, 48).chunk(6, 1)[:2]
    packed = torch.empty(1, 8)
    one, narrow = torch.ones(4)[::4], torch.ones(1, 1, 5, 1)
    for call in (lambda: api.da2_norm(X, X, w, packed), lambda: api.da2_norm_bwd(X, X, stats, X, w, packed, torch.empty(1, 8), ws=torch.empty(64)),
                 lambda: api.da2_norm(narrow, narrow, one, torch.ones(1))):
        with pytest.raises(ValueError, match="GPU"):
            call()
    X, w = torch.zeros(2, 1, 5, 8), torch.ones(2, 48).chunk(6, 1)[0]
    for bad in (torch.empty(2, 8), torch.ones(2, 96).chunk(6, 1)[0][:, :8]):
        with pytest.raises(ValueError, match="strides"):
            api.da2_norm(X, X, w, bad)
