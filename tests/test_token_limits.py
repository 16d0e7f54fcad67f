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
