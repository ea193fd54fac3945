"""Row blocks of trees have 16, 32 or 128 rows (csrc/attn_win_rules.hpp): a launch for any other number is turned down, and not run on a grid and a
workspace that are made for another one.  CPU only: the calls are refused before anything is launched."""
import os
import random
import shutil
import subprocess

import pytest

from tests.test_keep_rules import _tree, lib  # noqa: F401 (the fixture)

SOURCE = """
#include <cstdio>
#include <cstring>
#include "attn_internal.hpp"
#include "attn_win_rules.hpp"
#include "attn_window.hpp"

int main() {
    attn::WinParams p;
    std::memset(&p, 0, sizeof(p));
    p.d = 128;
    p.group = p.heads = p.kv_heads = p.blocks = p.batch = p.row_blocks = 1;
    p.table = reinterpret_cast<const int32_t*>(0x1000);
    p.tree = reinterpret_cast<const uint32_t*>(0x1000);
    for (int rows : {0, 8, 33, 48, 64, 96, 127, 256})
        for (int fp8 = 0; fp8 < 2; ++fp8) {
            const hipError_t fwd = attn::launch_tree_fwd(fp8 != 0, rows, 1, p, nullptr), join = attn::launch_tree_join(true, rows, p, nullptr);
            std::printf("%d %d %d\\n", rows, fwd == hipErrorInvalidValue, join == hipErrorInvalidValue);
        }
    for (int rows : {16, 64, 128})  // 32-bit arithmetic has blocks of 32
        std::printf("%d 1 %d\\n", rows, attn::launch_tree_join(false, rows, p, nullptr) == hipErrorInvalidValue);
}
"""


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_other_row_blocks_are_refused(tmp_path):
    from paper_2410_09397_amd import build
    objects = [os.path.join(build.OBJ, s.replace(".hip", ".o")) for s in build.SOURCES]
    if not all(os.path.exists(o) for o in objects):
        build.build()
    (tmp_path / "launches.hip").write_text(SOURCE)
    obj, exe = str(tmp_path / "launches.o"), str(tmp_path / "launches")
    for command in (["hipcc", *build.FLAGS, "-I", build.CSRC, "-c", str(tmp_path / "launches.hip"), "-o", obj],
                    ["hipcc", "--offload-arch=gfx950", "--hip-link", obj, *objects, "-o", exe]):
        r = subprocess.run(command, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
    lines = [x.split() for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.splitlines()]
    assert len(lines) == 19 and all(line[1:] == ["1", "1"] for line in lines), lines


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_the_rule_gives_no_other_row_blocks(lib):  # noqa: F811
    rng, met = random.Random(5), set()
    for _ in range(5000):
        bf16, fp8 = rng.choice([(1, 0), (1, 1), (0, 0), (0, 1)])
        k, group, batch, max_q = rng.choice([1, 2, 8]), rng.choice([1, 2, 3, 4, 8, 16, 64, 65]), rng.choice([1, 3, 64, 500]), rng.randint(1, 1024)
        d = rng.choice([64, 72, 128, 256])
        rows = _tree(lib, bf16, fp8, batch, k * group, k, d, batch * max_q, max_q, 5000, 0, 0)[0]
        wide = bf16 and (not fp8 or d != 72)
        assert rows == (32 if not wide or 16 < max_q * group <= 64 else 16 if max_q * group <= 16 else 128)
        met.add(rows)
    assert met == {16, 32, 128}
