"""The rules by which windowed attention and the paged cache choose their kernels (csrc/attn_win_rules.hpp), on the CPU: the shapes of the GPU
tests take what they are there for, and what the rules promise holds over many sizes."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest

from tests.window_shapes import CACHE, CACHE_LINE, PAGED, TRAIN

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_09397_amd", "csrc")
SOURCE = """
#include "attn_win_rules.hpp"
using namespace attn;
extern "C" int rows_of(int b, int h, int k, int n) { return win_rows(b, h, k, n); }
extern "C" void parts_of(int bf16, int b, int h, int k, int n, int d, int window, int sinks, int* out) {
    const WinReach r = win_reach(window, sinks, n);
    const WinParts p = win_parts(win_is_wide(bf16 != 0, d), b, h, k, n, d, r.window, r.sinks);
    out[0] = p.sink_tiles, out[1] = p.parts, out[2] = p.rest_parts, out[3] = p.slots;
}
extern "C" void splits_of(int bf16, int fp8, int b, int h, int k, int d, int total, int max_q, int max_len, int window, int sinks, int* out) {
    const WinReach r = win_reach(window, sinks, max_len);
    const bool wide = win_is_wide(bf16 != 0, d, fp8 != 0);
    const PagedSplits p = paged_splits(wide, b, h, k, d, total, max_q, max_len, r.window, r.sinks);
    out[0] = paged_rows(wide, b, h, k, total, max_q), out[1] = p.row_blocks, out[2] = p.blocks, out[3] = p.splits, out[4] = p.chunk;
}
extern "C" int cache_rows(int k, int total, int d) { return cache_rows_per_thread(k, total, d); }
"""
pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    folder = tmp_path_factory.mktemp("rules")
    (folder / "rules.cpp").write_text(SOURCE)
    out = str(folder / "rules.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(folder / "rules.cpp"), "-o", out])
    return ctypes.CDLL(out)


def _parts(lib, *args):
    out = (ctypes.c_int * 4)()
    lib.parts_of(*args, out)
    return tuple(out)


def _splits(lib, *args):
    out = (ctypes.c_int * 5)()
    lib.splits_of(*args, out)
    return tuple(out)


@pytest.mark.parametrize("case,want", TRAIN)
def test_training_shapes_take_their_kernels(lib, case, want):
    dtype, b, h, k, n, d, window, sinks, _ = case
    _, parts, rest, _ = _parts(lib, int(dtype == "bf16"), b, h, k, n, d, window, sinks)
    assert (lib.rows_of(b, h, k, n), parts, rest) == want


@pytest.mark.parametrize("case,want", PAGED)
def test_serving_shapes_take_their_kernels(lib, case, want):
    dtype, kind, lens, new, h, k, d, page, window, sinks = case
    width = max(-(-x // page) for x in lens) * page
    rows, _, _, splits, _ = _splits(lib, int(dtype == "bf16"), int(kind == "fp8"), len(lens), h, k, d, sum(new), max(new), width, window, sinks)
    assert (rows, splits > 1) == want


def test_cache_shapes_take_their_kernels(lib):
    for _, _, new, k, d, _ in CACHE:
        assert lib.cache_rows(k, sum(new), d) == 2
    for total, k, d, rows in CACHE_LINE:
        assert lib.cache_rows(k, total, d) == rows


def test_every_tile_of_keys_that_a_block_sees_belongs_to_a_split(lib):
    """Splits of `chunk` tiles each cover what WinTiles counts: the tiles of the sinks and those that the windows of a block's tokens touch."""
    rng = random.Random(1)
    for _ in range(4000):
        k = rng.choice([1, 2, 8])
        h, b, d = k * rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 5, 64]), rng.choice([64, 128, 256, 80])
        max_len, max_q = rng.randint(1, 20000), rng.choice([1, 1, 2, 9, 64, 200])
        window, sinks = rng.choice([0, rng.randint(1, 9000)]), rng.choice([0, 1, 4, 70, 300])
        bf16 = rng.randint(0, 1)
        rows, row_blocks, blocks, splits, chunk = _splits(lib, bf16, 0, b, h, k, d, b * max_q, max_q, max_len, window, sinks)
        assert row_blocks * rows >= max_q * (h // k) and blocks == row_blocks * b and 1 <= splits <= 64
        limits = 0 < window < max_len and sinks < max_len
        tile = 64 if rows >= 64 else 32
        for length in (max_len, rng.randint(1, max_len)):
            first = length - max_q
            t0 = rng.randrange(max_q)
            t1 = min(max_q - 1, t0 + rows // (h // k))
            i_min, i_max = first + t0, first + t1
            end = min(i_max, length - 1) + 1
            lo = max(0, i_min - window + 1) if limits else 0
            ns = -(-min(sinks if limits else 0, max(end, 0)) // tile)
            count = ns + max(0, -(-end // tile) - max(lo // tile, ns)) if end > 0 else 0
            assert count <= splits * chunk, (max_len, max_q, window, sinks, splits, chunk, count)


def test_shares_of_the_key_owners_fit_their_workspace(lib):
    rng = random.Random(2)
    for _ in range(4000):
        k = rng.choice([1, 2, 3, 8])
        h, b, n, d = k * rng.choice([1, 2, 4, 8, 16]), rng.choice([1, 2, 5, 64]), rng.randint(1, 9000), rng.choice([64, 128, 256, 80, 200])
        window, sinks, bf16 = rng.choice([0, rng.randint(1, n)]), rng.choice([0, 1, 4, 70, 300]), rng.randint(0, 1)
        tile = 64 if bf16 else 32
        sink_tiles, parts, rest, slots = _parts(lib, bf16, b, h, k, n, d, window, sinks)
        tiles = -(-n // tile)
        assert 0 <= sink_tiles <= tiles and 1 <= parts <= 64 and rest >= 1
        assert (sink_tiles == 0) == (parts == 1 or not (0 < window < n and 0 < sinks < n))
        assert slots == (sink_tiles * parts if parts > 1 else 0) + ((tiles - sink_tiles) * rest if rest > 1 else 0)
