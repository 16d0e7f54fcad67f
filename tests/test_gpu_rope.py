"""Rotary positions on the GPU against the float64 oracle.

Tolerance. The angle in turns is a float64 product (off by 2^-53 of itself), whose fraction is rounded to float32 (2^-26
of a turn) before a sine and cosine of 2 ulp (2^-22 at values up to one). Each result is a sum of two products with three
roundings, so it is off by (2^-22 + 2 pi 2^-26 + 3 * 2^-24 + 2 pi 2^-53 |turns|) <= 2^-20.4 + 2^-50 |turns| of
scale (|a| + |b|), and by the rounding to the result's type."""
import numpy as np
import pytest
import torch

from oracle import token
from paper_2609_32628_amd import api

pytestmark = pytest.mark.gpu
T = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def make(B, H, N, d, dtype, seed, major=False, offset=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((B, N, H, d + 2 * offset) if major else (B, H, N, d + 2 * offset), generator=g, device="cuda").to(T[dtype])
    x = x.transpose(1, 2) if major else x
    return x[..., offset:offset + d] if offset else x


def partner(x, rot, block, layout):
    """|a| + |b| of each channel's pair (channels that only move: 0)."""
    a = np.abs(x)
    out = np.zeros_like(a)
    for o in range(0, x.shape[-1], block):
        for p in range(rot // 2):
            i, j = (o + 2 * p, o + 2 * p + 1) if layout == "interleaved" else (o + p, o + rot // 2 + p)
            out[..., i] = out[..., j] = a[..., i] + a[..., j]
    return out


def compare(got, x, pos, rope, inverse):
    x = x.double().cpu().numpy()
    turns = rope.turns.cpu().numpy()
    rot = sum(rope.rot_axis)
    want = token.rope(x, pos, turns, rope.rot_axis, rope.scale, rope.layout, rope.block, inverse)
    far = float(np.abs(pos).max()) * float(turns.max())
    bound = (2.0 ** -20.4 + 2.0 ** -50 * far) * rope.scale * partner(x, rot, rope.block, rope.layout)
    t = got.dtype
    tol = bound + torch.finfo(t).eps / 2 * (np.abs(want) + bound) + torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2
    got = got.double().cpu().numpy()
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) - tol).max())
    # channels beyond the rotated ones are copies
    for o in range(0, x.shape[-1], rope.block):
        np.testing.assert_array_equal(got[..., o + rot:o + rope.block], x[..., o + rot:o + rope.block])


def check(rope, Q, K, pos=None, grid=None, inverse=False, Qo=None, Ko=None):
    B, _, N, _ = Q.shape
    if pos is not None:
        at = np.broadcast_to(pos.cpu().numpy().astype(np.int64), (B, N, len(rope.rot_axis)))
    else:
        n = np.arange(N)
        gh, gw = grid or (1, 1)
        at = {1: [n], 2: [n // gw, n % gw], 3: [n // (gh * gw), n // gw % gh, n % gw]}[len(rope.rot_axis)]
        at = np.broadcast_to(np.stack(at, -1)[None], (B, N, len(at)))
    Qo = torch.empty_like(Q) if Qo is None else Qo
    if K is not None:
        Ko = torch.empty_like(K) if Ko is None else Ko
    api.da2_rope(rope, Q, Qo, K, Ko, pos=pos, grid=grid, inverse=inverse)
    compare(Qo, Q, at, rope, inverse)
    if K is not None:
        compare(Ko, K, at, rope, inverse)


def positions(B, N, axes, seed, top=1 << 20):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randint(-top, top, (B, N, axes), generator=g).to(torch.int32).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("d,block,rot_axis", [(128, 128, (44, 42, 42)), (128, 64, (24, 20, 20)), (64, 64, (64,)), (64, 32, (16,)),
                                              (128, 128, (64,)), (128, 128, (10, 2, 4)), (96, 48, (20, 6)), (40, 20, (14,)),
                                              (6, 3, (2,)), (2, 2, (2,)), (256, 256, (128, 128))])
def test_layouts_widths_and_axes(d, block, rot_axis, layout, dtype):
    rope = api.da2_rope_plan(block, rot_axis, layout)
    for inverse, major in ((False, True), (True, False)):
        Q, K = make(2, 4, 7, d, dtype, 1, major), make(2, 2, 7, d, dtype, 2, not major)
        check(rope, Q, K, positions(2, 7, len(rot_axis), 3), inverse=inverse)


@pytest.mark.parametrize("rot_axis,grid", [((64,), None), ((32, 32), (5, 6)), ((24, 20, 20), (5, 6))])
def test_grid_positions(rot_axis, grid):
    rope = api.da2_rope_plan(64, rot_axis)
    check(rope, make(2, 3, 90, 64, "fp32", 1), make(2, 3, 90, 64, "fp32", 2), grid=grid)


@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "yarn"])
@pytest.mark.parametrize("base", [10000.0, 5e6])
def test_plans_and_far_positions(scaling, base):
    """The plan's turns against the formulas, and positions of up to 31 bits."""
    factor = 1.0 if scaling == "none" else 8.0
    rope = api.da2_rope_plan(128, (96,), "half", base, scaling, factor, 2048)
    turns, scale = token.rope_turns((96,), base, scaling, factor, 2048)
    np.testing.assert_allclose(rope.turns.cpu().numpy(), turns, rtol=1e-14)
    assert rope.scale == pytest.approx(scale, rel=1e-15)
    check(rope, make(3, 2, 5, 128, "fp32", 1), make(3, 1, 5, 128, "fp32", 2), positions(3, 5, 1, 3, (1 << 31) - 1))
    check(rope, make(3, 2, 5, 128, "bf16", 1), None, positions(1, 5, 1, 4))


@pytest.mark.parametrize("B,H,Hk,N", [(1, 1, 1, 1), (32, 32, 8, 1), (1, 40, 40, 700), (3, 1, 1, 3001), (1, 500, 3, 2)])
def test_heads_and_lengths(B, H, Hk, N):
    rope = api.da2_rope_plan(64, (64,), "half")
    check(rope, make(B, H, N, 64, "bf16", 1), make(B, Hk, N, 64, "bf16", 2, True), positions(B, N, 1, 3, 100000))


@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("offset", [1, 3])
def test_alignment_in_place_and_gaps(layout, offset):
    rope = api.da2_rope_plan(64, (48,), layout)
    pos = positions(2, 5, 1, 3)
    for dtype in ("bf16", "fp32"):
        Q, K = make(2, 3, 5, 64, dtype, 1, False, offset), make(2, 3, 5, 64, dtype, 2, True, offset)
        room = torch.full((2, 3, 5, 64 + 2 * offset), 7.0, dtype=T[dtype], device="cuda")
        check(rope, Q, K, pos, Qo=room[..., offset:offset + 64])
        assert (room[..., :offset] == 7).all() and (room[..., offset + 64:] == 7).all()
        want = [torch.empty_like(Q), torch.empty_like(K)]
        api.da2_rope(rope, Q, want[0], K, want[1], pos=pos)
        api.da2_rope(rope, Q, Q, K, K, pos=pos)
        assert torch.equal(Q, want[0]) and torch.equal(K, want[1])


def test_channels_that_move_keep_any_value():
    """Infinities and NaN beyond the rotated channels, and in other pairs, reach nothing else."""
    for layout in ("interleaved", "half"):
        rope = api.da2_rope_plan(64, (20,), layout)
        Q = make(1, 1, 3, 64, "bf16", 1)
        bad = Q.clone()
        bad[..., 20], bad[..., 21], bad[..., 0] = float("inf"), float("nan"), float("nan")
        pos = positions(1, 3, 1, 3)
        a, b = api_out(rope, Q, pos), api_out(rope, bad, pos)
        hit = [0, 1 if layout == "interleaved" else 10]
        keep = [i for i in range(64) if i not in hit + [20, 21]]
        assert torch.equal(a[..., keep], b[..., keep])
        assert b[..., hit].isnan().all() and b[..., 20].isinf().all() and b[..., 21].isnan().all()


def api_out(rope, Q, pos, **kw):
    out = torch.empty_like(Q)
    api.da2_rope(rope, Q, out, pos=pos, **kw)
    return out


def test_gradient_is_the_transpose():
    """<R x, y> = <x, R' y> in float32, with the scale of a long context; and a difference of the oracle's rotation,
    which is linear, along y."""
    rope = api.da2_rope_plan(64, (32, 32), "half", scaling="yarn", factor=4.0, orig_len=64)
    x, y = make(2, 2, 6, 64, "fp32", 1), make(2, 2, 6, 64, "fp32", 2)
    pos = positions(2, 6, 2, 3, 5000)
    rx, ry = api_out(rope, x, pos), api_out(rope, y, pos, inverse=True)
    lhs, rhs = (rx.double() * y.double()).sum(), (x.double() * ry.double()).sum()
    # each product is off by 2^-20 of its pair's magnitudes, twice
    assert abs(lhs - rhs) <= 2.0 ** -19 * 2 * rope.scale * (x.double().norm() * y.double().norm())
    f = lambda t: (token.rope(t, pos.cpu().numpy(), rope.turns.cpu().numpy(), rope.rot_axis, rope.scale, "half", 64)  # noqa: E731
                   * y.double().cpu().numpy()).sum()
    v = np.random.default_rng(0).normal(size=x.shape)
    x0 = x.double().cpu().numpy()
    want = (f(x0 + v) - f(x0 - v)) / 2
    assert abs((ry.double().cpu().numpy() * v).sum() - want) <= 2.0 ** -19 * 2 * rope.scale * np.linalg.norm(v) * float(y.double().norm())


def test_offsets_beyond_32_bits():
    far = (1 << 31) + 64
    room = torch.empty(far + 8192, dtype=torch.bfloat16, device="cuda")
    rope = api.da2_rope_plan(128, (44, 42, 42))
    Q = room.as_strided((2, 2, 6, 128), (far, 6 * 128, 128, 1))
    Q.copy_(make(2, 2, 6, 128, "bf16", 1))
    check(rope, Q, None, grid=(2, 3), Qo=room.as_strided((2, 2, 6, 128), (far, 6 * 128, 128, 1), 4096))


def test_streams_and_graph_replays():
    rope = api.da2_rope_plan(128, (44, 42, 42))
    Q, K = make(1, 12, 300, 128, "bf16", 1), make(1, 12, 300, 128, "bf16", 2)
    out, eager = [torch.empty_like(Q), torch.empty_like(K)], [torch.empty_like(Q), torch.empty_like(K)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    api.da2_rope(rope, Q, out[0], K, out[1], grid=(10, 10), stream=side)
    torch.cuda.current_stream().wait_stream(side)
    api.da2_rope(rope, Q, eager[0], K, eager[1], grid=(10, 10))
    assert all(torch.equal(a, e) for a, e in zip(out, eager))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.da2_rope(rope, Q, out[0], K, out[1], grid=(10, 10))
    for seed in (11, 12, 13):
        Q.copy_(make(1, 12, 300, 128, "bf16", seed))
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        api.da2_rope(rope, Q, eager[0], K, eager[1], grid=(10, 10))
        torch.cuda.synchronize()
        assert all(torch.equal(a, e) for a, e in zip(out, eager))
