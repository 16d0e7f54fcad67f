"""Python binding of libda2: the C entry points under the same names.

Argument marshalling only: tensors are torch tensors on the GPU (device
memory and streams come from PyTorch); every step of the path runs in the
library's HIP kernels. Each call is enqueued on ``stream`` (default: torch's
current stream) and returns without synchronizing.

The token operators (norm, rotary positions, differential attention) check
that their tensors' shapes and types belong together and that all of them are
on one GPU, and raise ValueError before the call otherwise. They run on the
tensors' GPU, whichever device is current.
"""
import ctypes
import math
from dataclasses import dataclass

import numpy as np
import torch

from . import _lib
from ._lib import (DA2_ACT_GELU, DA2_ACT_GELU_TANH, DA2_ACT_NONE, DA2_ACT_RELU, DA2_ACT_SIGMOID, DA2_ACT_SILU, DA2_BF16, DA2_ERR_WORKSPACE, DA2_FMT4_MXFP4, DA2_FMT4_NVFP4, DA2_FP16, DA2_FP32, DA2_NORM_LAYER, DA2_NORM_RMS,
                   DA2_PART_RAGGED, DA2_PART_TILES8, DA2_ROPE_HALF, DA2_ROPE_INTERLEAVED, DA2_ROPE_LINEAR,
                   DA2_ROPE_NTK, DA2_ROPE_PLAIN, DA2_ROPE_YARN, DA2_SCOPE_HEAD, DA2_SCOPE_ROW, DiffProblem, NormDesc, Problem,
                   RopeDesc, RopeFreq, RopeRows, Rows, Tensor, check, lib)

SCOPES = {"head": DA2_SCOPE_HEAD, "row": DA2_SCOPE_ROW}
PARTITIONS = {"tiles8": DA2_PART_TILES8, "ragged": DA2_PART_RAGGED}
FMT4 = {"nvfp4": DA2_FMT4_NVFP4, "mxfp4": DA2_FMT4_MXFP4}


def problem(B, H, d, T, Hg, Wg, partition="tiles8"):
    return Problem(B, H, d, T, Hg, Wg, PARTITIONS[partition])


def _tensor_desc(x):
    if x.dim() != 4 or x.stride(3) != 1:
        raise ValueError("expected a [B, H, N, d] tensor with d contiguous")
    dt = {torch.bfloat16: DA2_BF16, torch.float32: DA2_FP32}.get(x.dtype)
    if dt is None:
        raise ValueError(f"unsupported dtype {x.dtype}")
    return Tensor(x.stride(0), x.stride(1), x.stride(2), dt, 0)


def _stream(stream):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr())


def da2_sizes(p, scope="head", fmt4="nvfp4", with16=False):
    s = _lib.Sizes()
    check("da2_sizes", lib().da2_sizes(ctypes.byref(p), SCOPES[scope], FMT4[fmt4], int(with16), ctypes.byref(s)))
    return {f: getattr(s, f) for f, _ in _lib.Sizes._fields_}


def da2_ops_layout_version():
    return lib().da2_ops_layout_version()


def da2_layout_build(p):
    """Host-side region layout (int32 numpy array: n_a, slot2tok, tok2slot)."""
    n = da2_sizes(p)["layout_bytes"] // 4
    out = np.empty(n, dtype=np.int32)
    check("da2_layout_build", lib().da2_layout_build(
        ctypes.byref(p), out.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), n))
    return out


def _offsets(fn, p, n, *extra):
    arr = (ctypes.c_int64 * n)()
    check(fn, getattr(lib(), fn)(ctypes.byref(p), *extra, arr))
    return list(arr)


def da2_ws_draft_offsets(p):
    return _offsets("da2_ws_draft_offsets", p, 7)


def da2_lists_offsets(p):
    return _offsets("da2_lists_offsets", p, 4)


def da2_ops_offsets(p, fmt4="nvfp4", with16=False):
    """Byte offsets of the 16 ops sections for a run with (fmt4, with16); -1
    for a section such a run does not use."""
    return _offsets("da2_ops_offsets", p, 16, FMT4[fmt4], int(with16))


def da2_draft_map(Q, K, layout, p, lam, A, stats, ws, stream=None):
    check("da2_draft_map", lib().da2_draft_map(
        _ptr(Q), _ptr(K), ctypes.byref(_tensor_desc(Q)), _ptr(layout), ctypes.byref(p), float(lam),
        _ptr(A), _ptr(stats), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def da2_rank_assign(A, p, num16, num8, num4, den, scope, cls, lists, ws, stream=None):
    check("da2_rank_assign", lib().da2_rank_assign(
        _ptr(A), ctypes.byref(p), num16, num8, num4, den, SCOPES[scope], _ptr(cls), _ptr(lists), _ptr(ws),
        ws.numel() * ws.element_size(), _stream(stream)))


def da2_rank_assign_noalloc(A, p, num16, num8, num4, den, scope, cls, lists, stream=None):
    check("da2_rank_assign_noalloc", lib().da2_rank_assign_noalloc(
        _ptr(A), ctypes.byref(p), num16, num8, num4, den, SCOPES[scope], _ptr(cls), _ptr(lists), _stream(stream)))


def da2_prep_operands(Q, K, V, layout, p, with16, fmt4, stats, ops, ws, stream=None):
    if not (Q.shape == K.shape == V.shape and Q.stride() == K.stride() == V.stride() and Q.dtype == K.dtype == V.dtype):
        raise ValueError("Q, K and V must share shape, strides and dtype")
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    check("da2_prep_operands", lib().da2_prep_operands(
        _ptr(Q), _ptr(K), _ptr(V), ctypes.byref(_tensor_desc(Q)), _ptr(layout), ctypes.byref(p), int(with16),
        FMT4[fmt4], _ptr(stats), _ptr(ops), ops.numel() * ops.element_size(), None if ws is None else _ptr(ws),
        ws_bytes, _stream(stream)))


def da2_mixed_attn(ops, lists, layout, p, O, stream=None, fmt4="nvfp4"):
    check("da2_mixed_attn", lib().da2_mixed_attn(
        _ptr(ops), ops.numel() * ops.element_size(), _ptr(lists), _ptr(layout), ctypes.byref(p), FMT4[fmt4],
        ctypes.byref(_tensor_desc(O)), _ptr(O), _stream(stream)))


@dataclass
class Buffers:
    """Device buffers of one problem, sized by da2_sizes (allocation only).
    ``fmt4`` and ``with16`` are the 4-bit encoding and 16-bit option the ops
    buffer is sized for."""
    p: Problem
    scope: str
    fmt4: str
    with16: bool
    sizes: dict
    layout: torch.Tensor
    A: torch.Tensor
    cls: torch.Tensor
    stats: torch.Tensor
    lists: torch.Tensor
    ops: torch.Tensor
    ws_draft: torch.Tensor
    ws_rank: torch.Tensor


def alloc(p, scope="head", device="cuda", fmt4="nvfp4", with16=False):
    s = da2_sizes(p, scope, fmt4, with16)
    R = s["R"]
    B, H = p.B, p.H

    def raw(n):
        return torch.empty(max(int(n), 1), dtype=torch.uint8, device=device)

    layout = torch.from_numpy(da2_layout_build(p)).to(device)
    return Buffers(p, scope, fmt4, bool(with16), s, layout,
                   A=torch.empty((B, H, R, R), dtype=torch.float32, device=device),
                   cls=torch.empty((B, H, R, R), dtype=torch.uint8, device=device),
                   stats=raw(s["stats_bytes"]), lists=raw(s["lists_bytes"]), ops=raw(s["ops_bytes"]),
                   ws_draft=raw(s["ws_draft_bytes"]), ws_rank=raw(s["ws_rank_bytes"]))


def attention(Q, K, V, buf, lam, budgets, O, stream=None, num16=0, fmt4=None, qk_norm=None, rope=None, one_pass=False):
    """The four calls in order: draft map, ranking, operand preparation,
    attention. budgets = (num8, num4, den); num16/den go to the 16-bit path;
    fmt4 ("nvfp4" or "mxfp4", default: the buffers' encoding) is the encoding
    of the 4-bit path. qk_norm = (w_q, w_k), weights [d] or None each: the heads
    of Q and K are RMS-normalised first; rope, a Rope over one axis (the token
    numbers) or three (the problem's grid): they are rotated next. Both work in
    place, on Q and K themselves: a second call with them would do so again, and
    who needs them as they were calls da2_norm and da2_rope into tensors of
    their own and then this without. one_pass: both in one call, da2_qk_norm_rope,
    which reads and writes Q and K once and rounds once. All arguments of all
    calls are checked before Q and K are touched."""
    p = buf.p
    fmt4 = buf.fmt4 if fmt4 is None else fmt4
    if fmt4 != buf.fmt4 or (num16 > 0 and not buf.with16):
        raise ValueError(f"buffers sized for fmt4={buf.fmt4}, with16={buf.with16}; asked for fmt4={fmt4}, "
                         f"num16={num16}")
    if rope is not None and len(rope.rot_axis) not in (1, 3):
        raise ValueError(f"rope: expected 1 or 3 axes, got {len(rope.rot_axis)}")
    if one_pass and (qk_norm is None or rope is None):
        raise ValueError("one_pass: expected qk_norm and rope")
    if (qk_norm is not None or rope is not None) and Q.data_ptr() == K.data_ptr():
        raise ValueError("Q and K are one tensor: the norm and rotation in place would meet it twice")
    if qk_norm is not None or rope is not None:
        turn = _check_in_place(Q, K, V, buf, lam, budgets, O, num16, qk_norm, rope)
    if one_pass:
        da2_qk_norm_rope(rope, Q, Q, K, K, *qk_norm, grid=None if len(rope.rot_axis) == 1 else (p.Hg, p.Wg), stream=stream)
    elif qk_norm is not None:
        da2_norm(Q, Q, qk_norm[0], kind="rms", stream=stream)
        da2_norm(K, K, qk_norm[1], kind="rms", stream=stream)
    if rope is not None and not one_pass:
        _run("da2_rope", stream, *turn)
    da2_draft_map(Q, K, buf.layout, p, lam, buf.A, buf.stats, buf.ws_draft, stream)
    da2_rank_assign(buf.A, p, num16, *budgets, buf.scope, buf.cls, buf.lists, buf.ws_rank, stream)
    da2_prep_operands(Q, K, V, buf.layout, p, int(num16 > 0), fmt4, buf.stats, buf.ops, None, stream)
    da2_mixed_attn(buf.ops, buf.lists, buf.layout, p, O, stream, fmt4)
    return O


def _in_order(call, *args):
    """Raises what the call says of its arguments, which it is given without a workspace: it looks at that last, and so
    launches nothing."""
    status = getattr(lib(), call)(*args)
    if status != DA2_ERR_WORKSPACE:
        check(call, status)
        raise AssertionError(f"{call} ran without a workspace")


def _check_in_place(Q, K, V, buf, lam, budgets, O, num16, qk_norm, rope):
    """Everything that attention's calls refuse, before the first of them writes to Q and K. Returns what da2_rope takes."""
    p = buf.p
    size = da2_sizes(p, buf.scope, buf.fmt4, buf.with16)
    shape = (p.B, p.H, p.T * p.Hg * p.Wg, p.d)
    for name, t in (("Q", Q), ("K", K), ("V", V), ("O", O)):
        _tensor_desc(t)
        if t.shape != shape:
            raise ValueError(f"{name}: expected shape {shape}, got {tuple(t.shape)}")
    if not (Q.stride() == K.stride() == V.stride() and Q.dtype == K.dtype == V.dtype):
        raise ValueError("Q, K and V must share shape, strides and dtype")
    if V.data_ptr() in (Q.data_ptr(), K.data_ptr()):
        raise ValueError("V is Q's or K's memory: the norm and rotation in place would meet it too")
    if min(O.stride()) <= 0 or O.stride(2) < p.d:
        raise ValueError("O: rows overlap")
    for name in ("layout", "A", "cls", "stats", "lists", "ops", "ws_draft", "ws_rank"):
        t = getattr(buf, name)
        if not t.is_contiguous() or t.numel() * t.element_size() < size[name + "_bytes"]:
            raise ValueError(f"buf.{name}: expected {size[name + '_bytes']} contiguous bytes")
    desc = ctypes.byref(_tensor_desc(Q))
    P = ctypes.byref(p)
    _in_order("da2_draft_map", _ptr(Q), _ptr(K), desc, _ptr(buf.layout), P, float(lam), _ptr(buf.A), _ptr(buf.stats),
              _ptr(buf.ws_draft), 0, None)
    _in_order("da2_rank_assign", _ptr(buf.A), P, num16, *budgets, SCOPES[buf.scope], _ptr(buf.cls), _ptr(buf.lists), _ptr(buf.ws_rank), 0,
              None)
    _in_order("da2_prep_operands", _ptr(Q), _ptr(K), _ptr(V), desc, _ptr(buf.layout), P, int(num16 > 0), FMT4[buf.fmt4],
              _ptr(buf.stats), _ptr(buf.ops), 0, None, -1, None)
    tensors, turn = [Q, K, V, O, buf.layout, buf.A, buf.cls, buf.stats, buf.lists, buf.ops, buf.ws_draft, buf.ws_rank], None
    if qk_norm is not None:
        w_q, w_k = qk_norm
        _norm_desc(Q, (("w_q", w_q),), "rms", 0.0, False)
        _norm_desc(K, (("w_k", w_k),), "rms", 0.0, False)
        tensors += [w_q, w_k]
    if rope is not None:
        turn = _rope_args(rope, Q, Q, K, K, None, None if len(rope.rot_axis) == 1 else (p.Hg, p.Wg), False)
        # what da2_rope itself asks
        if (any(D < 2 or D % 2 for D in rope.rot_axis) or sum(rope.rot_axis) > rope.block or p.d % rope.block
                or not math.isfinite(rope.scale) or p.B * shape[2] * rope.block > (1 << 32) - 256):
            raise ValueError(f"rope: {rope.rot_axis} of {rope.block} channels, scale {rope.scale}, for heads of {p.d}")
        tensors.append(rope.turns)
    _one_gpu(tensors)
    return turn


# ---- token operators ---------------------------------------------------------------
DTYPES = {torch.bfloat16: DA2_BF16, torch.float32: DA2_FP32, torch.float16: DA2_FP16}
ROPE_LAYOUTS = {"interleaved": DA2_ROPE_INTERLEAVED, "half": DA2_ROPE_HALF}
ROPE_SCALINGS = {"none": DA2_ROPE_PLAIN, "linear": DA2_ROPE_LINEAR, "ntk": DA2_ROPE_NTK, "yarn": DA2_ROPE_YARN}
NORM_KINDS = {"layer": DA2_NORM_LAYER, "rms": DA2_NORM_RMS}


def _rows(name, x, shape=None, dtype=None):
    """Descriptor of a [B, H, N, C] tensor, checked against the shape and type it must have."""
    st = x.stride()
    if len(st) != 4 or (st[3] != 1 and x.shape[3] > 1):
        raise ValueError(f"{name}: expected a [B, H, N, C] tensor with its last dimension contiguous")
    dt = DTYPES.get(x.dtype)
    if dt is None or (dtype is not None and x.dtype != dtype):
        raise ValueError(f"{name}: unsupported dtype {x.dtype}" + (f", expected {dtype}" if dtype else ""))
    if shape is not None and x.shape != shape:
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(x.shape)}")
    return Tensor(st[0], st[1], st[2], dt, 0)


def _plain(name, x, shape, dtype):
    """Address of a contiguous tensor of the given shape and type (None: a null pointer)."""
    if x is None:
        return None
    if x.shape != shape or x.dtype != dtype or not x.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)}")
    return x.data_ptr()


def _addr(x):
    return None if x is None else x.data_ptr()


def _bytes(ws):
    """Bytes of a workspace; one that has gaps or repeats itself does not hold as many as its elements count."""
    if ws is None:
        return 0
    if not ws.is_contiguous():
        raise ValueError("ws: expected a contiguous tensor")
    return ws.numel() * ws.element_size()


def _one_gpu(tensors):
    dev = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError("expected all tensors on one GPU")
    if dev < 0:
        raise ValueError("expected tensors on a GPU")
    return dev


def _run(call, stream, tensors, *args):
    """Makes the call on the GPU that holds all the tensors and on its current stream (or the given one)."""
    dev = _one_gpu(tensors)
    if stream is None:
        s = torch._C._cuda_getCurrentRawStream(dev)
    elif stream.device.index == dev:
        s = stream.cuda_stream
    else:
        raise ValueError(f"the stream belongs to {stream.device}, the tensors to cuda:{dev}")
    f = getattr(lib(), call)
    if torch._C._cuda_getDevice() == dev:
        check(call, f(*args, s))
    else:
        with torch.cuda.device(dev):
            check(call, f(*args, s))


def _norm_desc(X, given, kind, eps, plus_one):
    """Rows and NormDesc of a norm over X's last dimension with weights [C] or [B, C] (``given``: by name)."""
    B, H, N, C = X.shape
    stride, wdtype, first = 0, X.dtype, None
    for name, t in given:
        if t is None:
            continue
        st = t.stride()
        if t.dtype not in DTYPES or t.shape not in ((C,), (B, C)) or (C > 1 and st[-1] != 1):
            raise ValueError(f"{name}: expected [C] or [B, C] weights with C contiguous")
        # one sample's weights serve all its rows whatever their stride
        per = st[0] if len(st) == 2 and B > 1 else 0
        if first is None:
            first, wdtype, stride = t, t.dtype, per
            if len(st) == 2 and B > 1 and per < C:
                raise ValueError(f"{name}: the samples' weights overlap")
        elif t.shape != first.shape or t.dtype != wdtype or per != stride:
            raise ValueError("weights and bias (and their gradients) must share shape, strides and dtype")
    return Rows(B, H, N, C), NormDesc(NORM_KINDS[kind], DTYPES[wdtype], int(plus_one), 0, stride, float(eps))


def da2_norm(X, Y, w=None, b=None, kind="layer", eps=1e-6, plus_one=False, stats=None, stream=None):
    """Y = norm of X's rows (the last dimension of [B, H, N, C]) times w (or 1 + w) plus b; w, b: [C], or [B, C] per
    sample. ``stats``: float32 [B, H, N, 2] for da2_norm_bwd. Y may be X."""
    x = _rows("X", X)
    y = _rows("Y", Y, X.shape, X.dtype)
    r, n = _norm_desc(X, (("w", w), ("b", b)), kind, eps, plus_one)
    st = _plain("stats", stats, X.shape[:3] + (2,), torch.float32)
    _run("da2_norm", stream, (X, Y, w, b, stats), X.data_ptr(), x, r, n, _addr(w), _addr(b), Y.data_ptr(), y, st)
    return Y


def da2_norm_ws_bytes(X, w=None):
    """Workspace bytes of da2_norm_bwd for the gradients of weights like ``w`` ([C] or [B, C])."""
    _rows("X", X)
    B, H, N, C = X.shape
    out = ctypes.c_int64()
    check("da2_norm_ws_bytes", lib().da2_norm_ws_bytes(Rows(B, H, N, C), DTYPES[X.dtype],
                                                       int(w is not None and w.dim() == 2 and B > 1), out))
    return out.value


def da2_norm_bwd(dY, X, stats, dX=None, w=None, dw=None, db=None, kind="layer", plus_one=False, ws=None, stream=None):
    """Gradients of da2_norm; dX, dw and db are written where given. ``ws``: da2_norm_ws_bytes(X, w) bytes, for dw and db."""
    x = _rows("X", X)
    dy = _rows("dY", dY, X.shape, X.dtype)
    dx = None if dX is None else _rows("dX", dX, X.shape, X.dtype)
    r, n = _norm_desc(X, (("w", w), ("dw", dw), ("db", db)), kind, 0.0, plus_one)
    st = _plain("stats", stats, X.shape[:3] + (2,), torch.float32)
    _run("da2_norm_bwd", stream, (X, dY, stats, dX, w, dw, db, ws), dY.data_ptr(), dy, X.data_ptr(), x, r, n, _addr(w),
         st, _addr(dX), dx, _addr(dw), _addr(db), _addr(ws), _bytes(ws))


_I32x3 = ctypes.c_int32 * 3


@dataclass
class Rope:
    """Plan of the rotary positions: layout ("interleaved" or "half"), channels of a rotated block, rotated channels of
    each position axis, and the turns per position of every pair (float64 [rot / 2] on the GPU) with the factor of
    cosine and sine, from da2_rope_plan or the caller's own."""
    layout: str
    block: int
    rot_axis: tuple
    turns: torch.Tensor
    scale: float = 1.0

    def desc(self):
        n = len(self.rot_axis)
        if not 1 <= n <= 3:
            raise ValueError("rot_axis: expected 1 to 3 axes")
        return RopeDesc(ROPE_LAYOUTS[self.layout], self.block, n, _I32x3(*self.rot_axis))


def da2_rope_plan(block, rot_axis, layout="interleaved", base=10000.0, scaling="none", factor=1.0, orig_len=4096,
                  beta_fast=32.0, beta_slow=1.0, device="cuda"):
    """Rope of blocks of ``block`` channels with rot_axis[i] of them turning with position axis i. scaling: "none",
    "linear", "ntk" or "yarn", for contexts ``factor`` times longer than trained on (orig_len: for yarn)."""
    rope = Rope(layout, block, tuple(rot_axis), torch.empty(max(sum(rot_axis) // 2, 1), dtype=torch.float64))
    scale = ctypes.c_double()
    check("da2_rope_plan", lib().da2_rope_plan(
        rope.desc(), RopeFreq(ROPE_SCALINGS[scaling], orig_len, base, factor, beta_fast, beta_slow),
        ctypes.cast(rope.turns.data_ptr(), ctypes.POINTER(ctypes.c_double)), scale))
    rope.turns, rope.scale = rope.turns.to(device), scale.value
    return rope


def _rope_args(rope, Q, Qo, K, Ko, pos, grid, inverse):
    """The tensors of a da2_rope call and its arguments."""
    q = _rows("Q", Q)
    qo = _rows("Qo", Qo, Q.shape, Q.dtype)
    B, Hq, N, d = Q.shape
    Hk, k, ko = 0, None, None
    if (K is None) != (Ko is None):
        raise ValueError("K and Ko are given together")
    if K is not None:
        Hk = K.shape[1] if K.dim() == 4 else 0
        k = _rows("K", K, (B, Hk, N, d), Q.dtype)
        ko = _rows("Ko", Ko, K.shape, Q.dtype)
    axes, stride = len(rope.rot_axis), 0
    if pos is not None:
        if pos.shape not in ((B, N, axes), (1, N, axes)) or pos.dtype != torch.int32:
            raise ValueError(f"pos: expected int32 [{B} or 1, {N}, {axes}]")
        if not pos[0].is_contiguous():
            raise ValueError("pos: expected each sample's positions contiguous")
        stride = pos.stride(0) if pos.shape[0] > 1 else 0
    t = _plain("turns", rope.turns, (sum(rope.rot_axis) // 2,), torch.float64)
    gh, gw = grid if grid is not None else (0, 0)
    return ((Q, Qo, K, Ko, pos, rope.turns), rope.desc(), t, rope.scale, _addr(pos), stride,
            RopeRows(B, Hq, Hk, N, d, gh, gw, int(inverse)), Q.data_ptr(), q, Qo.data_ptr(), qo, _addr(K), k, _addr(Ko), ko)


def da2_rope(rope, Q, Qo, K=None, Ko=None, pos=None, grid=None, inverse=False, stream=None):
    """Rotates Q (and K) into Qo (and Ko), which may be the inputs. pos: int32 [B or 1, N, axes] positions; without it
    the tokens are numbered, on 2 and 3 axes over a ``grid`` of (height, width) per frame. inverse: the gradient."""
    _run("da2_rope", stream, *_rope_args(rope, Q, Qo, K, Ko, pos, grid, inverse))


def _diff_problem(Q, K, causal=False, scale=None):
    if Q.dim() != 4 or K.dim() != 4:
        raise ValueError("expected [B, H, N, d] tensors")
    B, Hq, N, d = Q.shape
    Hk, M = K.shape[1:3]
    if K.shape[0] != B or K.shape[3] != d or Hk == 0 or Hq % Hk:
        raise ValueError(f"Q {tuple(Q.shape)} and K {tuple(K.shape)} do not belong together")
    return DiffProblem(B, Hq, Hk, N, M, d, int(causal), 0, (d / 2) ** -0.5 if scale is None else float(scale))


def da2_diff_ws_bytes(Q, K, train=False):
    """Workspace bytes of da2_diff_attn (train: and of da2_diff_attn_bwd) for tensors of these shapes."""
    out = ctypes.c_int64()
    check("da2_diff_ws_bytes", lib().da2_diff_ws_bytes(_diff_problem(Q, K), int(train), out))
    return out.value


def _diff_inputs(Q, K, V, lam, kv_lens, q_start, causal, scale):
    """Problem, descriptors of Q, K, V and addresses of lam, kv_lens, q_start."""
    q, k = _rows("Q", Q), _rows("K", K, dtype=Q.dtype)
    p = _diff_problem(Q, K, causal, scale)
    v = _rows("V", V, K.shape, Q.dtype)
    if lam is None:
        raise ValueError("lam: expected float32 weights of the query heads")
    return p, q, k, v, (_plain("lam", lam, (p.Hq,), torch.float32), _plain("kv_lens", kv_lens, (p.B,), torch.int32),
                        _plain("q_start", q_start, (p.B,), torch.int32))


def da2_diff_attn(Q, K, V, lam, O, ws=None, lse=None, kv_lens=None, q_start=None, causal=False, scale=None, stream=None):
    """O = (softmax(scale Q1 K1') - lam softmax(scale Q2 K2')) V, with Q1 and Q2 (K1, K2) the halves of a head's channels
    and the heads of K and V shared by Hq / Hk heads of Q. lam: float32 [Hq]. kv_lens, q_start: int32 [B], the valid keys
    of each sample and the position of its first query (default: all keys, and the queries are the last of them). lse
    (float32 [B, Hq, 2, N]) is for da2_diff_attn_bwd. ws: da2_diff_ws_bytes(Q, K)."""
    p, q, k, v, (l, kl, qs) = _diff_inputs(Q, K, V, lam, kv_lens, q_start, causal, scale)
    o = _rows("O", O, Q.shape, Q.dtype)
    ls = _plain("lse", lse, (p.B, p.Hq, 2, p.N), torch.float32)
    _run("da2_diff_attn", stream, (Q, K, V, lam, O, ws, lse, kv_lens, q_start), p, Q.data_ptr(), q, K.data_ptr(), k,
         V.data_ptr(), v, l, kl, qs, O.data_ptr(), o, ls, _addr(ws), _bytes(ws))
    return O


def da2_diff_attn_bwd(Q, K, V, lam, lse, dO, dQ, dK, dV, dlam, ws, kv_lens=None, q_start=None, causal=False, scale=None,
                      stream=None):
    """Gradients of da2_diff_attn from its inputs and what it wrote to lse. ws: da2_diff_ws_bytes(Q, K, True)."""
    p, q, k, v, (l, kl, qs) = _diff_inputs(Q, K, V, lam, kv_lens, q_start, causal, scale)
    do, dq = (_rows(n, t, Q.shape, Q.dtype) for n, t in (("dO", dO), ("dQ", dQ)))
    dk, dv = (_rows(n, t, K.shape, Q.dtype) for n, t in (("dK", dK), ("dV", dV)))
    ls = _plain("lse", lse, (p.B, p.Hq, 2, p.N), torch.float32)
    dl = _plain("dlam", dlam, (p.Hq,), torch.float32)
    _run("da2_diff_attn_bwd", stream, (Q, K, V, lam, lse, dO, dQ, dK, dV, dlam, ws, kv_lens, q_start), p, Q.data_ptr(), q,
         K.data_ptr(), k, V.data_ptr(), v, l, kl, qs, ls, dO.data_ptr(), do, dQ.data_ptr(), dq, dK.data_ptr(), dk,
         dV.data_ptr(), dv, dl, _addr(ws), _bytes(ws))


# ---- the rest of a layer: norm and rotation of Q and K, projections, gated blocks -------
ACTS = {"none": DA2_ACT_NONE, "relu": DA2_ACT_RELU, "gelu": DA2_ACT_GELU, "gelu_tanh": DA2_ACT_GELU_TANH, "silu": DA2_ACT_SILU,
        "sigmoid": DA2_ACT_SIGMOID}


def _head_weights(d, given, kind, eps, plus_one, dtype):
    """NormDesc of a norm over heads of d channels with weights [d] (``given``: by name)."""
    wdtype = None
    for name, t in given:
        if t is None:
            continue
        if t.dtype not in DTYPES or t.shape != (d,) or not t.is_contiguous():
            raise ValueError(f"{name}: expected contiguous weights [{d}]")
        if wdtype is not None and t.dtype != wdtype:
            raise ValueError("the weights (and their gradients) must share a dtype")
        wdtype = t.dtype
    return NormDesc(NORM_KINDS[kind], DTYPES[wdtype or dtype], int(plus_one), 0, 0, float(eps))


def da2_qk_norm_rope(rope, Q, Qo, K=None, Ko=None, w_q=None, w_k=None, kind="rms", eps=1e-6, plus_one=False, pos=None, grid=None,
                     stream=None):
    """Qo (and Ko) = rotation of the normalised heads of Q (and K) times w_q (w_k), or 1 + w: da2_norm over the heads and da2_rope
    in one pass. w_q, w_k: [d]. pos and grid as in da2_rope. Qo and Ko may be Q and K."""
    tensors, desc, turns, scale, p, stride, rows, *io = _rope_args(rope, Q, Qo, K, Ko, pos, grid, False)
    n = _head_weights(Q.shape[3], (("w_q", w_q), ("w_k", w_k)), kind, eps, plus_one, Q.dtype)
    _run("da2_qk_norm_rope", stream, tensors + (w_q, w_k), desc, turns, scale, p, stride, rows, n, _addr(w_q), _addr(w_k), *io)


def da2_qk_norm_rope_ws_bytes(Q, K=None):
    """Workspace bytes of da2_qk_norm_rope_bwd for the gradients of the weights."""
    _rows("Q", Q)
    B, Hq, N, d = Q.shape
    out = ctypes.c_int64()
    check("da2_qk_norm_rope_ws_bytes", lib().da2_qk_norm_rope_ws_bytes(
        RopeRows(B, Hq, 0 if K is None else K.shape[1], N, d, 0, 0, 0), out))
    return out.value


def da2_qk_norm_rope_bwd(rope, dQo, Q, dQ, dKo=None, K=None, dK=None, w_q=None, w_k=None, dw_q=None, dw_k=None, kind="rms", eps=1e-6,
                         plus_one=False, pos=None, grid=None, ws=None, stream=None):
    """Gradients of da2_qk_norm_rope from its inputs Q and K; dw_q and dw_k are written where given. dQ and dK may be dQo and dKo, or
    Q and K. ws: da2_qk_norm_rope_ws_bytes(Q, K), for dw_q and dw_k."""
    if (K is None) != (dK is None):
        raise ValueError("K, dKo and dK are given together")
    tensors, desc, turns, scale, p, stride, rows, dqo, dqo_t, dq, dq_t, dko, dko_t, dk, dk_t = _rope_args(rope, dQo, dQ, dKo, dK, pos, grid, False)
    q = _rows("Q", Q, dQo.shape, dQo.dtype)
    k = None if K is None else _rows("K", K, dKo.shape if dKo is not None else None, dQo.dtype)
    n = _head_weights(Q.shape[3], (("w_q", w_q), ("w_k", w_k), ("dw_q", dw_q), ("dw_k", dw_k)), kind, eps, plus_one, Q.dtype)
    _run("da2_qk_norm_rope_bwd", stream, tensors + (Q, K, w_q, w_k, dw_q, dw_k, ws), desc, turns, scale, p, stride, rows, n, _addr(w_q),
         _addr(w_k), dqo, dqo_t, Q.data_ptr(), q, dq, dq_t, dko, dko_t, _addr(K), k, dk, dk_t, _addr(dw_q), _addr(dw_k), _addr(ws), _bytes(ws))


def _proj(X, Y, act="none"):
    """Proj of rows X -> Y, and the input and output features."""
    _rows("X", X)
    _rows("Y", Y, dtype=X.dtype)
    B, Hx, N, Cx = X.shape
    if Y.shape[0] != B or Y.shape[2] != N:
        raise ValueError(f"X {tuple(X.shape)} and Y {tuple(Y.shape)} do not belong together")
    return _lib.Proj(B, N, Hx, Cx, Y.shape[1], Y.shape[3], ACTS[act], DTYPES[X.dtype]), Hx * Cx, Y.shape[1] * Y.shape[3]


def _matrix(name, W, shape, dtype):
    """Address and row stride of a matrix of the given shape and type whose rows are contiguous."""
    if W.shape != shape or W.dtype != dtype or (shape[1] > 1 and W.stride(1) != 1):
        raise ValueError(f"{name}: expected {dtype} [{shape[0]}, {shape[1]}] with contiguous rows")
    return W.data_ptr(), W.stride(0) if shape[0] > 1 else -(-shape[1] // 8) * 8


def _gate(gate, like, B, F, dtype):
    """Distance between the samples' gates; ``like``: a gradient, laid out alike."""
    for name, t in (("gate", gate), ("dgate", like)):
        if t is not None and (t.dtype != dtype or t.shape not in ((F,), (B, F)) or (F > 1 and t.stride(-1) != 1)):
            raise ValueError(f"{name}: expected {dtype} [{F}] or [{B}, {F}] with contiguous rows")
    if gate is None:
        return 0
    per = gate.stride(0) if gate.dim() == 2 and B > 1 else 0
    if gate.dim() == 2 and B > 1 and per < F:
        raise ValueError("gate: the samples' gates overlap")
    if like is not None and (like.shape != gate.shape or (per and like.stride(0) != per)):
        raise ValueError("gate and dgate must share shape and strides")
    return per


def _z(X, Y, parts):
    p, _, F = _proj(X, Y)
    wide = -(-F // 8) * 8
    return (p.B, p.N, wide) if parts == 1 else (p.B, p.N, 2, wide)


def da2_linear_z(X, Y):
    """An empty Z (float32) for da2_linear and da2_linear_bwd."""
    return torch.empty(_z(X, Y, 1), device=X.device)


def da2_glu_z(X, Y):
    """An empty Z (float32) for da2_glu and da2_glu_bwd."""
    return torch.empty(_z(X, Y, 2), device=X.device)


def _ws_bytes(call, X, W, Y, train):
    p, _, _ = _proj(X, Y)
    out = ctypes.c_int64()
    check(call, getattr(lib(), call)(p, int(train), out))
    return out.value


def da2_linear_ws_bytes(X, W, Y, train=False):
    """Workspace bytes of da2_linear (train: and of da2_linear_bwd) for tensors of these shapes."""
    return _ws_bytes("da2_linear_ws_bytes", X, W, Y, train)


def da2_glu_ws_bytes(X, W, Y, train=False):
    """Workspace bytes of da2_glu (train: and of da2_glu_bwd) for tensors of these shapes."""
    return _ws_bytes("da2_glu_ws_bytes", X, W, Y, train)


def da2_linear(X, W, Y, bias=None, act="none", gate=None, residual=None, Z=None, ws=None, stream=None):
    """Y = residual + gate * act(X W' + bias). X [B, Hx, N, Cx] and Y [B, Hy, N, Cy]: rows of Hx Cx and Hy Cy features (hidden rows are
    one block; heads as the attention has them). W: [Hy Cy, Hx Cx]; bias [Hy Cy]; gate [Hy Cy] or [B, Hy Cy]; residual like Y, or Y
    itself. act: "none", "relu", "gelu", "gelu_tanh", "silu" or "sigmoid". Z: da2_linear_z(X, Y), for da2_linear_bwd. ws:
    da2_linear_ws_bytes(X, W, Y)."""
    p, K, F = _proj(X, Y, act)
    x, y = _rows("X", X), _rows("Y", Y)
    w, stride = _matrix("W", W, (F, K), X.dtype)
    r = None if residual is None else _rows("residual", residual, Y.shape, X.dtype)
    b = _plain("bias", bias, (F,), X.dtype)
    z = _plain("Z", Z, _z(X, Y, 1), torch.float32)
    _run("da2_linear", stream, (X, W, Y, bias, gate, residual, Z, ws), p, X.data_ptr(), x, w, stride, b, _addr(gate),
         _gate(gate, None, p.B, F, X.dtype), _addr(residual), r, Y.data_ptr(), y, z, _addr(ws), _bytes(ws))
    return Y


def da2_linear_bwd(dY, X, W, Z=None, dX=None, dW=None, dbias=None, act="none", gate=None, dgate=None, ws=None, stream=None):
    """Gradients of da2_linear (that of the residual is dY), written where given. Z: what da2_linear wrote, needed with an activation or
    for dgate. ws: da2_linear_ws_bytes(X, W, Y, True)."""
    p, K, F = _proj(X, dY, act)
    x, dy = _rows("X", X), _rows("dY", dY)
    w, stride = _matrix("W", W, (F, K), X.dtype)
    dx = None if dX is None else _rows("dX", dX, X.shape, X.dtype)
    dw, dstride = (None, 0) if dW is None else _matrix("dW", dW, (F, K), X.dtype)
    db = _plain("dbias", dbias, (F,), X.dtype)
    z = _plain("Z", Z, _z(X, dY, 1), torch.float32)
    _run("da2_linear_bwd", stream, (X, W, dY, gate, Z, dX, dW, dbias, dgate, ws), p, dY.data_ptr(), dy, X.data_ptr(), x, w, stride,
         _addr(gate), _gate(gate, dgate, p.B, F, X.dtype), z, _addr(dX), dx, dw, dstride, db, _addr(dgate), _addr(ws), _bytes(ws))


def da2_glu(X, W, Y, bias=None, act="silu", Z=None, ws=None, stream=None):
    """Y = act(X Wg' + bg) * (X Wu' + bu): W [2 F, K] holds the rows of Wg, then those of Wu, and bias [2 F] alike. Z: da2_glu_z(X, Y), for
    da2_glu_bwd. ws: da2_glu_ws_bytes(X, W, Y). The rest as in da2_linear."""
    p, K, F = _proj(X, Y, act)
    x, y = _rows("X", X), _rows("Y", Y)
    w, stride = _matrix("W", W, (2 * F, K), X.dtype)
    b = _plain("bias", bias, (2 * F,), X.dtype)
    z = _plain("Z", Z, _z(X, Y, 2), torch.float32)
    _run("da2_glu", stream, (X, W, Y, bias, Z, ws), p, X.data_ptr(), x, w, stride, b, Y.data_ptr(), y, z, _addr(ws), _bytes(ws))
    return Y


def da2_glu_bwd(dY, X, W, Z, dX=None, dW=None, dbias=None, act="silu", ws=None, stream=None):
    """Gradients of da2_glu, written where given. Z: what da2_glu wrote. ws: da2_glu_ws_bytes(X, W, Y, True)."""
    p, K, F = _proj(X, dY, act)
    x, dy = _rows("X", X), _rows("dY", dY)
    w, stride = _matrix("W", W, (2 * F, K), X.dtype)
    dx = None if dX is None else _rows("dX", dX, X.shape, X.dtype)
    dw, dstride = (None, 0) if dW is None else _matrix("dW", dW, (2 * F, K), X.dtype)
    db = _plain("dbias", dbias, (2 * F,), X.dtype)
    z = _plain("Z", Z, _z(X, dY, 2), torch.float32)
    _run("da2_glu_bwd", stream, (X, W, dY, Z, dX, dW, dbias, ws), p, dY.data_ptr(), dy, X.data_ptr(), x, w, stride, z, _addr(dX), dx, dw,
         dstride, db, _addr(ws), _bytes(ws))
