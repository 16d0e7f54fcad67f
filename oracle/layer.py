"""Projections, gated blocks and the norm and rotation of Q and K in float64 (numpy), with their gradients, written from the
formulas. Arrays are [B, H, N, C]; a row's features are its heads' channels one after the other."""
import math

import numpy as np
from scipy.special import ndtr

from oracle import token


# ---- norm and rotation of Q and K ------------------------------------------------------
def qk_norm_rope(x, pos, turns, rot_axis, w=None, kind="rms", eps=1e-6, plus_one=False, scale=1.0, layout="interleaved", block=None):
    y, _, _ = token.norm(x, w, None, kind, eps, plus_one)
    return token.rope(y, pos, turns, rot_axis, scale, layout, block)


def qk_norm_rope_bwd(dy, x, pos, turns, rot_axis, w=None, kind="rms", eps=1e-6, plus_one=False, scale=1.0, layout="interleaved", block=None):
    """(dx, dw)"""
    g = token.rope(dy, pos, turns, rot_axis, scale, layout, block, inverse=True)
    _, mean, rstd = token.norm(x, None, None, kind, eps)
    dx, dw, _ = token.norm_bwd(g, x, mean, rstd, w, kind, plus_one)
    return dx, dw


# ---- projections -------------------------------------------------------------------
def act(z, kind):
    """The activation and its derivative."""
    sig = lambda v: np.where(v >= 0, 1 / (1 + np.exp(-np.abs(v))), np.exp(-np.abs(v)) / (1 + np.exp(-np.abs(v))))  # noqa: E731
    if kind == "relu":
        return np.maximum(z, 0), (z > 0).astype(np.float64)
    if kind == "gelu":
        return z * ndtr(z), ndtr(z) + z * np.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        a = math.sqrt(2 / math.pi)
        p = sig(2 * a * (z + 0.044715 * z ** 3))
        return z * p, p + z * p * (1 - p) * 2 * a * (1 + 3 * 0.044715 * z * z)
    if kind == "silu":
        return z * sig(z), sig(z) * (1 + z * (1 - sig(z)))
    if kind == "sigmoid":
        return sig(z), sig(z) * sig(-z)
    return z, np.ones_like(z)


def flat(x):
    """[B, H, N, C] as a matrix [B N, H C]."""
    B, H, N, C = x.shape
    return x.astype(np.float64).transpose(0, 2, 1, 3).reshape(B * N, H * C)


def unflat(m, B, H, N, C):
    return m.reshape(B, N, H, C).transpose(0, 2, 1, 3)


def rows_gate(gate, B, N):
    """[F] or [B, F] gates for every row [B N, F]."""
    g = gate.astype(np.float64)
    return np.broadcast_to(g, (B * N, g.shape[-1])) if g.ndim == 1 else np.repeat(g, N, 0)


def linear(x, w, bias=None, kind="none", gate=None, r=None):
    """(y, z) as matrices; x, r: [B, H, N, C]."""
    B, _, N, _ = x.shape
    z = flat(x) @ w.astype(np.float64).T
    if bias is not None:
        z = z + bias.astype(np.float64)
    y = act(z, kind)[0]
    if gate is not None:
        y = y * rows_gate(gate, B, N)
    return (y if r is None else y + flat(r)), z


def linear_bwd(dy, x, w, z, kind="none", gate=None):
    """Dict of dz, dx, dw, dbias and dgate (matrices) for the sums z."""
    B, _, N, _ = x.shape
    dy, x, w = flat(dy), flat(x), w.astype(np.float64)
    a, da = act(z, kind)
    out = {}
    if gate is not None:
        per = (dy * a).reshape(B, N, -1).sum(1)
        out["dgate"] = per.sum(0) if gate.ndim == 1 else per
        dy = dy * rows_gate(gate, B, N)
    dz = dy * da
    out.update(dz=dz, dx=dz @ w, dw=dz.T @ x, dbias=dz.sum(0))
    return out


def glu(x, w, bias=None, kind="silu"):
    """(y, z) as matrices; z holds both halves."""
    z = flat(x) @ w.astype(np.float64).T
    if bias is not None:
        z = z + bias.astype(np.float64)
    F = w.shape[0] // 2
    return act(z[:, :F], kind)[0] * z[:, F:], z


def glu_bwd(dy, x, w, z, kind="silu"):
    dy, x, w = flat(dy), flat(x), w.astype(np.float64)
    F = w.shape[0] // 2
    a, da = act(z[:, :F], kind)
    dz = np.concatenate([dy * z[:, F:] * da, dy * a], 1)
    return dict(dz=dz, dx=dz @ w, dw=dz.T @ x, dbias=dz.sum(0))
