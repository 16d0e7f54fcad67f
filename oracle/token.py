"""Token operators around the attention in float64 (numpy): row norms, rotary
positions and differential attention, with their gradients, written from the
formulas. Arrays are [B, H, N, C]."""
import math

import numpy as np


# ---- row norms -------------------------------------------------------------------
def norm(x, w=None, b=None, kind="layer", eps=1e-6, plus_one=False):
    """(y, mean, rstd); w and b: [C] or [B, C] or None."""
    x = x.astype(np.float64)
    mean = x.mean(-1, keepdims=True) if kind == "layer" else np.zeros(x.shape[:-1] + (1,))
    rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + eps)
    y = (x - mean) * rstd * norm_factor(x, w, plus_one)
    if b is not None:
        y = y + per_row(b)
    return y, mean, rstd


def per_row(w):
    """[C] or [B, C] weights against [B, H, N, C] rows."""
    w = w.astype(np.float64)
    return w if w.ndim == 1 else w[:, None, None, :]


def norm_factor(x, w, plus_one):
    return np.ones(x.shape[-1]) if w is None else per_row(w) + (1.0 if plus_one else 0.0)


def norm_bwd(dy, x, mean, rstd, w=None, kind="layer", plus_one=False, adaptive=False):
    """(dx, dw, db); dw and db are [B, C] when adaptive, else [C]."""
    dy, x = dy.astype(np.float64), x.astype(np.float64)
    xh = (x - mean) * rstd
    g = dy * norm_factor(x, w, plus_one)
    dx = g - xh * (g * xh).mean(-1, keepdims=True)
    if kind == "layer":
        dx = dx - g.mean(-1, keepdims=True)
    over = (1, 2) if adaptive else (0, 1, 2)
    return rstd * dx, (dy * xh).sum(over), dy.sum(over)


# ---- rotary positions ------------------------------------------------------------
def rope_turns(rot_axis, base=10000.0, scaling="none", factor=1.0, orig_len=4096, beta_fast=32.0, beta_slow=1.0):
    """(turns per position of every pair [rot/2], factor of cosine and sine)."""
    out = []
    for D in rot_axis:
        for i in range(D // 2):
            b = base
            if scaling == "ntk" and D > 2:
                b = base * factor ** (D / (D - 2))
            f = b ** (-2.0 * i / D)
            if scaling == "linear":
                f /= factor
            if scaling == "yarn":
                # pairs that turn more than beta_fast times over the original length keep their frequency, those
                # below beta_slow are stretched, and a ramp lies between
                lo = max(math.floor(D * math.log(orig_len / (beta_fast * 2 * math.pi)) / (2 * math.log(base))), 0)
                hi = min(math.ceil(D * math.log(orig_len / (beta_slow * 2 * math.pi)) / (2 * math.log(base))), D - 1)
                r = min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0)
                f = f / factor * r + f * (1.0 - r)
            out.append(f / (2 * math.pi))
    return np.array(out), (0.1 * math.log(factor) + 1.0 if scaling == "yarn" else 1.0)


def rope(x, pos, turns, rot_axis, scale=1.0, layout="interleaved", block=None, inverse=False):
    """x [B, H, N, d] rotated at pos [B, N, axes]."""
    d = x.shape[-1]
    block = block or d
    rot = sum(rot_axis)
    y = x.astype(np.float64).copy()
    axis = [a for a, D in enumerate(rot_axis) for _ in range(D // 2)]
    for p in range(rot // 2):
        # the product of an integer and a double, reduced by whole turns before the factor 2 pi
        t = pos[:, :, axis[p]].astype(np.longdouble) * np.longdouble(turns[p])
        a = (2 * math.pi) * (t - np.rint(t)).astype(np.float64)[:, None]
        c, s = np.cos(a) * scale, np.sin(a) * scale * (-1.0 if inverse else 1.0)
        for o in range(0, d, block):
            i, j = (o + 2 * p, o + 2 * p + 1) if layout == "interleaved" else (o + p, o + rot // 2 + p)
            u, v = x[..., i].astype(np.float64), x[..., j].astype(np.float64)
            y[..., i], y[..., j] = u * c - v * s, u * s + v * c
    return y


# ---- differential attention --------------------------------------------------------
def diff_visible(N, M, n_keys, start, causal):
    """Which of M keys each of N queries sees: [N, M]."""
    j = np.arange(M)[None]
    see = np.broadcast_to(j < n_keys, (N, M))
    return see & (j <= start + np.arange(N)[:, None]) if causal else see


def _maps(q, k, see, scale):
    """Both softmax maps [2, N, M] of one head and their log sums [2, N]; rows that see nothing are zero."""
    h = q.shape[-1] // 2
    P, lse = [], []
    for m in (0, 1):
        s = np.where(see, (q[:, m * h:(m + 1) * h] @ k[:, m * h:(m + 1) * h].T) * scale, -np.inf)
        top = s.max(-1, keepdims=True)
        top = np.where(np.isneginf(top), 0.0, top)
        e = np.exp(s - top)
        t = e.sum(-1, keepdims=True)
        P.append(e / np.where(t == 0, 1.0, t))
        with np.errstate(divide="ignore"):
            lse.append((top + np.log(t))[:, 0])
    return np.stack(P), np.stack(lse)


def _clean(x, see_any):
    """Rows no query sees hold nothing (their memory may be anything)."""
    return np.where(see_any[:, None], x.astype(np.float64), 0.0)


def diff_attn(Q, K, V, lam, n_keys, start, causal, scale=None, dO=None):
    """Dict of O, lse and, with dO, of dQ, dK, dV and dlam. n_keys and start: one per sample."""
    B, H, N, d = Q.shape
    Hk, M = K.shape[1], K.shape[2]
    scale = 1.0 / math.sqrt(d // 2) if scale is None else scale
    h = d // 2
    out = {"O": np.zeros((B, H, N, d)), "lse": np.zeros((B, H, 2, N))}
    if dO is not None:
        out.update(dQ=np.zeros((B, H, N, d)), dK=np.zeros((B, Hk, M, d)), dV=np.zeros((B, Hk, M, d)), dlam=np.zeros(H))
    for b in range(B):
        see = diff_visible(N, M, n_keys[b], start[b], causal)
        for hq in range(H):
            kh = hq // (H // Hk)
            q = Q[b, hq].astype(np.float64)
            k, v = (_clean(x[b, kh], np.arange(M) < n_keys[b]) for x in (K, V))
            P, out["lse"][b, hq] = _maps(q, k, see, scale)
            out["O"][b, hq] = (P[0] - lam[hq] * P[1]) @ v
            if dO is None:
                continue
            g = dO[b, hq].astype(np.float64)
            dP = g @ v.T
            out["dV"][b, kh] += (P[0] - lam[hq] * P[1]).T @ g
            out["dlam"][hq] -= (P[1] * dP).sum()
            for m, f in ((0, 1.0), (1, -lam[hq])):
                dS = f * P[m] * (dP - (P[m] * dP).sum(-1, keepdims=True)) * scale
                out["dQ"][b, hq, :, m * h:(m + 1) * h] = dS @ k[:, m * h:(m + 1) * h]
                out["dK"][b, kh, :, m * h:(m + 1) * h] += dS.T @ q[:, m * h:(m + 1) * h]
    return out
