"""The host-side validation of windowed attention and the paged cache (csrc/attn_win_api.hip) under AddressSanitizer and UBSan on the CPU, over
descriptors whose fields reach the ends of their types; and sizes whose products leave 64 bits."""
import ctypes
import os
import shutil

import pytest

from paper_2410_09397_amd import attn
from tests.test_sanitizers import ROOT, SAN, _clean, _run
from tests.test_window_abi import paged


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_window_validation_under_asan_ubsan(tmp_path):
    from paper_2410_09397_amd import build as hip_build
    others = [os.path.join(hip_build.OBJ, s.replace(".hip", ".o")) for s in hip_build.SOURCES if s != "attn_win_api.hip"]  # uninstrumented
    if not all(os.path.exists(o) for o in others):
        hip_build.build()
    obj, drv, exe = (str(tmp_path / x) for x in ("attn_win_api_san.o", "window_api_driver.o", "window_api_san"))
    host_san = [a for f in SAN for a in ("-Xarch_host", f)]
    r = _run(["hipcc", *[f for f in hip_build.FLAGS if f != "-fvisibility=hidden"], *host_san, "-g", "-c",
              os.path.join(hip_build.CSRC, "attn_win_api.hip"), "-o", obj])
    assert r.returncode == 0, r.stderr[-2000:]
    r = _run(["g++", "-O1", "-g", "-std=c++17", *SAN, "-c", os.path.join(ROOT, "tests", "sanitize", "window_api_driver.cpp"), "-o", drv])
    assert r.returncode == 0, r.stderr[-2000:]
    r = _run(["hipcc", "--offload-arch=gfx950", "--hip-link", "-fsanitize=address", "-fsanitize=undefined", "-fno-gpu-sanitize", "-g", "-o", exe, drv, obj,
              *others])
    assert r.returncode == 0, r.stderr[-2000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:verify_asan_link_order=0:protect_shadow_gap=0")
    env.pop("LD_PRELOAD", None)
    r = _run([exe], env=env)
    assert r.returncode == 0 and _clean(r.stderr), (r.stdout[-2000:], r.stderr[-2000:])
    assert " 0 failed" in r.stdout


@pytest.mark.parametrize("kw", [
    dict(batch=65535, heads=1 << 30, kv_heads=1 << 30, max_q=1 << 22),  # row blocks of all sequences and heads: 2^18 2^16 2^30
    dict(batch=65535, heads=1 << 30, kv_heads=1 << 30, max_q=1 << 10),
    dict(batch=1 << 15, heads=1 << 30, kv_heads=2, max_q=1),
    dict(batch=1 << 12, heads=1 << 20, kv_heads=1 << 20, max_q=1),
])
def test_sizes_whose_products_leave_the_range_of_a_launch(kw):
    d = paged(total_q=1 << 22, q_stride_n=1 << 40, kv_stride_n=1 << 40, **kw)
    assert attn.lib().attn_paged_workspace_bytes(ctypes.byref(d)) == 0


@pytest.mark.parametrize("kw", [dict(batch=65535, heads=512, kv_heads=64, max_q=1, total_q=65535), dict(batch=4096, heads=64, kv_heads=8, max_q=1, total_q=4096)])
def test_the_largest_batches_are_taken(kw):
    d = paged(q_stride_n=1 << 20, kv_stride_n=1 << 20, **kw)
    assert attn.lib().attn_paged_workspace_bytes(ctypes.byref(d)) >= 256
