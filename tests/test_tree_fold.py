"""The order in which trees' parts share the chip (TreeFold of csrc/attn_win_rules.hpp, the code that the kernels run), on the CPU: every part of every row block is some
workgroup's, its sums lie where the joining launch looks for them, and parts with most tiles share a CU with those that have fewest."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_09397_amd", "csrc")
SOURCE = """
#include "attn_win_rules.hpp"
// blocks, parts, tiles of `batch` sequences; out: of every workgroup its sequence and its item in the order of the sums, sizes: tiles of its part
extern "C" int fold(int batch, int fold_at, const int* blocks, const int* parts, const int* tiles, int* sequence, int* item, int* sizes) {
    int all = 0;
    for (int b = 0; b < batch; ++b) all += blocks[b] * parts[b];
    for (int idx = 0; idx < all; ++idx) {
        int found = 0;
        for (int lane = 0; lane < batch; ++lane) {  // as the lanes of a wave do, each for one sequence
            const int own = blocks[lane] * parts[lane], size = (tiles[lane] + parts[lane] - 1) / parts[lane];
            attn::TreeFold at;
            for (int x = 0; x < batch; ++x) at.count(lane, size, x, blocks[x] * parts[x], (tiles[x] + parts[x] - 1) / parts[x]);
            if (at.all != all) return -1;
            const int place = attn::TreeFold::place(idx, at.all, fold_at);
            if (!at.has(place, own)) continue;
            ++found;
            sequence[idx] = lane;
            item[idx] = at.before + place - at.first;
            sizes[idx] = size;
        }
        if (found != 1) return -2;
    }
    return all;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    folder = tmp_path_factory.mktemp("fold")
    (folder / "fold.cpp").write_text(SOURCE)
    out = str(folder / "fold.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(folder / "fold.cpp"), "-o", out])
    return ctypes.CDLL(out)


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_the_folded_order_has_every_part_once_and_long_ones_beside_short_ones(lib):
    rng, folded = random.Random(4), 0
    for _ in range(1500):
        batch = rng.choice([2, 3, 16, 63, 64])
        blocks = [rng.choice([0, 1, 1, 2, 5]) for _ in range(batch)]
        tiles = [rng.choice([0, 1, 7, 7, rng.randint(1, 300)]) for _ in range(batch)]
        chunk = rng.choice([4, 7, 22, 400])
        parts = [max(1, -(-t // chunk)) for t in tiles]
        every = sum(b * x for b, x in zip(blocks, parts))
        fold = rng.choice([32, 64, 256])
        if not 0 < every <= 2 * fold:  # (the rule folds launches that are on the chip at once)
            continue
        array = lambda x: (ctypes.c_int * len(x))(*x)
        sequence, item, sizes = ((ctypes.c_int * every)() for _ in range(3))
        assert lib.fold(batch, fold, array(blocks), array(parts), array(tiles), sequence, item, sizes) == every
        # a sequence's items stand together, part by part, in the order of the sequences: where part k of row block blk is looked for, start + k * blocks + blk
        start = 0
        for b in range(batch):
            mine = sorted(item[i] for i in range(every) if sequence[i] == b)
            assert mine == [start + k * blocks[b] + blk for k in range(parts[b]) for blk in range(blocks[b])]
            start += blocks[b] * parts[b]
        assert sorted(item) == list(range(every))
        front, back = list(sizes)[:fold], list(sizes)[fold:]
        assert front == sorted(front, reverse=True) and back == sorted(back) and (not back or max(back) <= min(front))
        folded += bool(back)
    assert folded > 100
