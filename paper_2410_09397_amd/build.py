"""Builds libattn_mi355x.so (HIP kernels + C ABI) for gfx950 with hipcc, in-tree.

Run as `python -m paper_2410_09397_amd.build`.  hipcc cross-compiles without a GPU.
"""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libattn_mi355x.so")
SOURCES = ["attn_api.hip", "attn_fwd.hip", "attn_bwd.hip", "attn_bwd_onepass.hip", "attn_generic.hip", "attn_stream.hip", "attn_larged.hip", "attn_splitd.hip", "attn_wgrad.hip",
           "attn_win_api.hip", "attn_win_plain.hip", "attn_win_fwd.hip", "attn_win_bwd.hip", "attn_cache.hip", "attn_probe.hip"]
# -packed-fp32-ops is switched off: packed fp32 VALU forms are not trusted on this target.
# -Wno-inline-asm: the tile copies write M0 in inline assembly and say so in their clobber lists; clang notes that
# M0 is a reserved register (it never keeps a value of its own there across a statement that clobbers it).
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-Wall", "-Wno-unused-function",
         "-Wno-inline-asm",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def _compile(src):
    obj = os.path.join(OBJ, src.replace(".hip", ".o"))
    cmd = ["hipcc", *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s" % (src, err))
    return obj, err


def build(verbose=False):
    os.makedirs(OBJ, exist_ok=True)
    srcs = [s for s in SOURCES if os.path.exists(os.path.join(CSRC, s))]
    with ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        results = list(ex.map(_compile, srcs))
    if verbose:
        for _, err in results:
            if err.strip():
                print(err, file=sys.stderr)
    subprocess.check_call(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB]
                          + [o for o, _ in results])
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
