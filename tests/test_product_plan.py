"""How products are cut (few rows at once, tiles of two sizes, parts of a long sum), from the library's own rule compiled for the CPU:
long sums are not left to a few workgroups, workspaces follow, and the shapes that the GPU tests run reach every kernel."""
import os
import subprocess

import pytest

from paper_2609_32628_amd import _lib

PROBE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "probes", "plan_probe.cpp")


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """For (rows, features, K, parts) each, or with a fifth, whether the rows are in two numbers: (kernel, parts of K, K ends inside a step, several units a workgroup, bytes)."""
    exe = str(tmp_path_factory.mktemp("plan") / "plan_probe")
    subprocess.run(["g++", "-O1", "-std=c++20", "-o", exe, PROBE], check=True, timeout=120)

    def ask(shapes):
        r = subprocess.run([exe], input="".join("%d %d %d %d %d\n" % (*s, 0)[:5] for s in shapes), capture_output=True, text=True, check=True, timeout=60)
        out = [line.split() for line in r.stdout.splitlines()]
        assert len(out) == len(shapes)
        return [(o[0], int(o[1]), o[2] == "1", o[3] == "1", int(o[4])) for o in out]

    return ask


def ws_bytes(call, train, B, N, K, F):
    out = _lib.ctypes.c_int64()
    assert getattr(_lib.lib(), call)(_lib.Proj(B, N, 1, K, 1, F, 0, _lib.DA2_BF16), train, out) == 0
    return out.value


@pytest.mark.parametrize("rows", [1, 5, 16])
def test_long_sums_of_few_rows_are_cut(plans, rows):
    """The kernel for few rows has a workgroup for 16 features and does not cut K: 4 workgroups for 64 features, however long K is."""
    for F in (1, 16, 64, 1000):
        for K in (20000, 200000, 1 << 22):
            kernel, cut, _, _, _ = plans([(rows, F, K, 1)])[0]
            assert kernel != "few" and cut >= 8, (F, K)
    long = plans([(rows, F, K, parts) for F, K, parts in ((5120, 13824, 1), (4096, 32768, 1), (5120, 6200, 2))])
    assert all((p[0] == "few") == (rows <= 4) for p in long)
    short = plans([(rows, F, K, parts) for F in (16, 1000, 8192) for K in (64, 2048, 4096) for parts in (1, 2)])
    assert all(p[0] == "few" for p in short)


def test_few_rows_in_two_numbers(plans):
    """They read long weight rows twice on tiles, and stay with the kernel for few rows for longer."""
    assert [p[0] for p in plans([(1, 1536, 11500, 1), (1, 1536, 16000, 1, 1), (16, 1536, 8000, 1), (16, 1536, 8000, 1, 1)])] == ["few", "few", "small", "few"]
    # what is cut is not taken for few rows when its sum is twice as long
    shapes = [(M, F, K, 1, lo) for M in range(1, 17) for F in (100, 5000) for K in range(64, 40000, 320) for lo in (0, 1)]
    few = {s: p[0] == "few" for s, p in zip(shapes, plans(shapes))}
    twice = plans([(M, F, 2 * K, 1, 0) for M, F, K, _, lo in shapes if lo])
    assert all(few[s] or p[0] != "few" for s, p in zip([s for s in shapes if s[4]], twice))


def test_workspaces_of_few_rows(plans):
    """Calls of few tokens with a long sum need room for its parts, forward, and backward for the gradients of few weight rows and for
    those of few tokens of many features, whose two numbers count twice."""
    for call, parts in (("da2_linear_ws_bytes", 1), ("da2_glu_ws_bytes", 2)):
        for N, K, F in ((1, 131072, 64), (16, 20000, 100), (6, 6000, 40), (1, 64, 64)):
            (kernel, _, _, _, need), = plans([(N, F, K, parts)])
            assert ws_bytes(call, 0, 1, N, K, F) == need and (need > 0) == (K > 64 and (kernel != "few"))
        for N, K, F in ((200000, 64, 16 // parts), (5, 24, 20000), (16, 100, 10000)):
            rows, wide, up = F * parts, -(-F // 64) * 64 * parts, -(-(-(-N // 8) * 8) // 64) * 64
            both = 2 if N <= 16 else 1
            products = [(N, K, wide, 1, n) for n in range(both)] + [(rows, K, up, 1, n) for n in range(both)]
            need = max(p[4] for p in plans(products))
            assert need > 0 and ws_bytes(call, 1, 1, N, K, F) >= need + 2 * both * (N + up) * wide


# (tokens, K, F, gated) of forward products
PATHS = [(700, 64, 12800, False), (700, 40, 12800, False), (2000, 64, 9000, False), (2000, 40, 9000, False), (300, 64, 12800, True), (300, 40, 12800, True),
         (700, 64, 12800, True), (700, 40, 12800, True), (3000, 8192, 257, False), (6000, 4100, 257, False), (4154, 6016, 67, True), (4154, 5932, 67, True),
         (640, 64, 12800, True), (640, 40, 12800, True), (1025, 64, 13120, False), (2101, 40, 7426, False), (17, 6720, 8538, False), (17, 7625, 8386, False),
         (19, 7616, 4108, True), (21, 8333, 4314, True), (40, 64, 72, False), (40, 40, 72, False), (40, 64, 72, True), (40, 40, 72, True),
         (20, 1024, 40, False), (20, 1000, 40, False), (20, 1024, 40, True), (20, 1000, 40, True), (5, 64, 40, False), (5, 40, 40, True)]
# (tokens, K, F, gated) of gradients: of weights on large tiles in parts, of few weight rows over many tokens, of few tokens of many features
GRADIENTS = [(8192, 257, 3000, False), (8150, 257, 1500, True), (18002, 24, 16, False), (20000, 130, 3, False), (18002, 72, 8, True),
             (5, 24, 20000, False), (16, 100, 5000, True), (1, 40, 20000, False)]


def test_shapes_reach_every_kernel(plans):
    """Each tile, with whole steps and without, plain, gated and in parts, with one unit of work a workgroup and with several. (Large
    tiles in parts are only taken where they are too few for the card, so no workgroup has several.)"""
    seen = set()
    for (M, K, F, glu), (kernel, cut, end, several, _) in zip(PATHS, plans([(M, F, K, 1 + glu) for M, K, F, glu in PATHS])):
        seen.add((kernel, "gated" if glu else "plain", cut > 1, end, several) if kernel != "few" else (kernel, glu))
    want = {("few", False), ("few", True)}
    for tile in ("big", "small"):
        for kind in ("plain", "gated"):
            for end in (False, True):
                want |= {(tile, kind, False, end, False), (tile, kind, False, end, True), (tile, kind, True, end, False)}
                if tile == "small":
                    want.add((tile, kind, True, end, True))
    assert seen == want, (sorted(want - seen, key=str), sorted(seen - want, key=str))


def test_gradients_reach_the_cut_products(plans):
    up = lambda n: -(-n // 64) * 64  # noqa: E731
    dw = plans([(F * (1 + glu), K, up(M), 1, M <= 16) for M, K, F, glu in GRADIENTS])
    dx = plans([(M, K, up(F) * (1 + glu), 1, M <= 16) for M, K, F, glu in GRADIENTS])
    assert all(p[0] == "big" and p[1] > 1 for p in dw[:2])
    assert all(p[0] == "small" and p[1] > 1 for p in dw[2:5])
    assert all(p[0] == "small" and p[1] > 1 for p in dx[5:])
