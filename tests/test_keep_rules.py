"""The rules by which trees of drafted tokens, weights and eviction choose their kernels (csrc/attn_win_rules.hpp), on the CPU: the shapes of the GPU tests
take every one, and what the rules promise holds over many sizes."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest

from tests.test_gpu_evict import EVICT, WEIGH
from tests.test_gpu_tree import CASES

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_09397_amd", "csrc")
SOURCE = """
#include "attn_win_rules.hpp"
using namespace attn;
extern "C" void tree_of(int bf16, int fp8, int b, int h, int k, int d, int total, int max_q, int max_len, int window, int sinks, long long* out) {
    const WinReach r = win_reach(window, sinks, max_len);
    const bool wide = win_is_wide(bf16 != 0, d, fp8 != 0);
    const TreeShares p = tree_shares(wide, b, h, k, d, total, max_q, max_len, r.window, r.sinks);
    const int rows = tree_rows(wide, b, h, k, total, max_q);
    out[0] = rows, out[1] = p.row_blocks, out[2] = p.blocks, out[3] = p.places, out[4] = p.least, out[5] = p.grid, out[6] = join_rows((int64_t)p.blocks * k, rows), out[7] = p.fold;
}
extern "C" void weigh_of(int bf16, int fp8, int b, int h, int k, int d, int max_q, int max_len, long long n, long long s, int* out) {
    const WeighPlan p = weigh_plan(win_is_wide(bf16 != 0, d, fp8 != 0), b, h, k, max_q, max_len, n, s);
    out[0] = p.kind, out[1] = p.blocks, out[2] = p.chunk, out[3] = p.parts;
}
extern "C" int blocks_of(long long bk, long long cap, long long rows) { return evict_blocks(bk, cap, rows); }
extern "C" int here() { return kEvictHere; }
"""
pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
ONE, FEW, MANY, ANY = range(4)


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    folder = tmp_path_factory.mktemp("rules")
    (folder / "rules.cpp").write_text(SOURCE)
    out = str(folder / "rules.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(folder / "rules.cpp"), "-o", out])
    return ctypes.CDLL(out)


def _tree(lib, *args):
    out = (ctypes.c_longlong * 8)()
    lib.tree_of(*args, out)
    return tuple(out)


def _weigh(lib, *args):
    out = (ctypes.c_int * 4)()
    lib.weigh_of(*args[:-2], ctypes.c_longlong(args[-2]), ctypes.c_longlong(args[-1]), out)
    return tuple(out)


def test_the_shapes_of_the_gpu_tests_reach_every_kernel_of_trees(lib):
    met, joined, folded = set(), set(), set()
    for dtype, kind, lens, new, h, k, d, page, window, sinks, _ in CASES:
        width = max(-(-x // page) for x in lens) * page
        rows, _, _, places, _, _, many, fold = _tree(lib, int(dtype == "bf16"), int(kind == "fp8"), len(lens), h, k, d, sum(new), max([1] + new), width, window, sinks)
        met.add((rows, places > 0))
        folded.add((rows, fold > 0)) if places > 0 else None
        joined.add((places > 0, many > 8))
    assert met == {(rows, shared) for rows in (16, 32, 128) for shared in (False, True)}
    assert joined >= {(True, False), (True, True)}, joined
    assert folded >= {(128, False), (128, True), (32, False), (16, False)}, folded


def test_every_part_of_a_tree_has_a_workgroup_and_a_lane(lib):
    """The device's own sharing out (TreeItems), with its division in 32-bit floating point, against the workgroups of the launch and the 64 lanes of a row's sums."""
    import numpy
    rng = random.Random(2)
    shared = 0
    for _ in range(3000):
        batch, k, group, d = rng.choice([1, 2, 5, 16, 64, 200]), rng.choice([1, 2, 8]), rng.choice([1, 2, 4, 8, 16]), rng.choice([64, 72, 128, 256])
        bf16, fp8 = rng.choice([(1, 0), (1, 1), (0, 0), (0, 1)])
        max_q, max_len = rng.choice([1, 3, 8, 15, 40, 64, 200, 1000]), rng.choice([100, 1000, 10000, 70000, 1 << 20])
        new = [rng.randint(0, max_q) for _ in range(batch)]
        lens = [min(max_len, rng.randint(0, max_len) + q) for q in new]
        window = rng.choice([0, 0, 100, 5000])
        sinks = rng.choice([0, 4, 70]) if window else 0
        total = sum(new)
        rows, _, blocks, places, least, grid, many, fold = _tree(lib, bf16, fp8, batch, k * group, k, d, total, max_q, max_len, window, sinks)
        assert rows % many == 0 and grid % k == 0 and 0 < grid < 1 << 31
        tile, items, tiles_of = 64 if rows >= 64 else 32, grid // k, []
        for length, q in zip(lens, new):
            context = max(0, length - q)
            first = max(0, context - window) if window else 0
            front = -(-min(sinks, context) // tile)
            seen = front + max(0, -(-context // tile) - max(first // tile, front))
            tiles_of.append((-(-q * group // rows), seen + -(-q // tile)))
        assert sum(b for b, _ in tiles_of) <= blocks
        chunk = 0x7fffffff
        if places:
            shared += 1
            work = sum(b * t for b, t in tiles_of)
            chunk = max(least, int(min(numpy.ceil(numpy.float32(work) / numpy.float32(places)), numpy.float32(1e9))))
        parts = [max(1, -(-t // chunk)) for _, t in tiles_of]
        assert max(parts) <= 64
        assert sum(b * x for (b, _), x in zip(tiles_of, parts)) <= items
        if fold:  # every item is some workgroup's: the order of find_folded
            assert rows == 128 and 1 < batch <= 64 and blocks * k <= 512
            order = sorted(range(batch), key=lambda x: (-(-(-tiles_of[x][1] // parts[x])), x))
            runs, every = [tiles_of[x][0] * parts[x] for x in order], sum(b * x for (b, _), x in zip(tiles_of, parts))
            assert sorted(x if x < fold else every - 1 - (x - fold) for x in range(every)) == list(range(every)) and sum(runs) == every
    assert shared > 500


def test_the_shapes_of_the_gpu_tests_reach_every_kernel_of_weights(lib):
    met = set()
    for dtype, kind, lens, new, h, k, d, page, *_ in WEIGH:
        width = max(-(-x // page) for x in lens) * page
        got, _, chunk, parts = _weigh(lib, int(dtype == "bf16"), int(kind == "fp8"), len(lens), h, k, d, max([1] + new), width, h * d, d)
        met.add((got, parts > 1) if got == MANY else (got, chunk))
    assert {x for x, _ in met} == {ONE, FEW, MANY, ANY}, met
    assert met >= {(MANY, False), (MANY, True), (ANY, 32), (ONE, 128)}, met


def test_every_key_of_a_weight_belongs_to_a_workgroup(lib):
    rng = random.Random(3)
    for _ in range(4000):
        bf16, fp8 = rng.choice([(1, 0), (1, 1), (0, 0), (0, 1)])
        batch, k, group, d = rng.choice([1, 2, 7, 64, 300]), rng.choice([1, 2, 8]), rng.choice([1, 2, 3, 8, 100, 129, 200]), rng.choice([24, 64, 80, 128, 256])
        max_q, max_len = rng.choice([1, 2, 16, 17, 32, 100, 4096]), rng.choice([1, 31, 32, 33, 127, 129, 1000, 5000, 70000])
        stride = rng.choice([k * group * d, 1 << 22, 1 << 30])
        kind, blocks, chunk, parts = _weigh(lib, bf16, fp8, batch, k * group, k, d, max_q, max_len, stride, d)
        rows = max_q * group
        assert blocks == -(-max_len // chunk) and chunk in (32, 128, 256, 512, 1024) and 1 <= parts <= 64
        assert kind == ONE if rows <= 16 else kind != ONE
        if kind in (FEW, MANY):
            assert group <= 128 and stride < 1 << 22 and (rows <= 128) == (kind == FEW)
        if kind == MANY:
            assert chunk == 256 and (parts == 1 or parts * 2 <= -(-max_q // (128 // group)))
        else:
            assert parts == 1


def test_moves_of_an_eviction(lib):
    for cap, bk, rows in ((1, 1, 64), (65, 8, 64), (2048, 64, 32), (1 << 20, 1, 16), (1 << 20, (1 << 24) - 1, 4)):
        blocks = lib.blocks_of(ctypes.c_longlong(bk), ctypes.c_longlong(cap), ctypes.c_longlong(rows))
        assert 1 <= blocks <= 1024 and (blocks - 1) * rows < cap and blocks * bk < 1 << 31
    moved = {min(c[5], max(c[2]) - c[5]) > lib.here() for c in EVICT if max(c[2]) > c[5]}
    assert moved == {False, True}
