"""The host-side validation of trees, weights and eviction (csrc/attn_win_api.hip) under AddressSanitizer and UBSan on the CPU, over descriptors whose
fields reach the ends of their types."""
import os
import shutil

import pytest

from tests.test_sanitizers import ROOT, SAN, _clean, _run


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_keep_validation_under_asan_ubsan(tmp_path):
    from paper_2410_09397_amd import build as hip_build
    others = [os.path.join(hip_build.OBJ, s.replace(".hip", ".o")) for s in hip_build.SOURCES if s != "attn_win_api.hip"]  # uninstrumented
    if not all(os.path.exists(o) for o in others):
        hip_build.build()
    obj, drv, exe = (str(tmp_path / x) for x in ("attn_keep_api_san.o", "keep_api_driver.o", "keep_api_san"))
    host_san = [a for f in SAN for a in ("-Xarch_host", f)]
    r = _run(["hipcc", *[f for f in hip_build.FLAGS if f != "-fvisibility=hidden"], *host_san, "-g", "-c",
              os.path.join(hip_build.CSRC, "attn_win_api.hip"), "-o", obj])
    assert r.returncode == 0, r.stderr[-2000:]
    r = _run(["g++", "-O1", "-g", "-std=c++17", *SAN, "-c", os.path.join(ROOT, "tests", "sanitize", "keep_api_driver.cpp"), "-o", drv])
    assert r.returncode == 0, r.stderr[-2000:]
    r = _run(["hipcc", "--offload-arch=gfx950", "--hip-link", "-fsanitize=address", "-fsanitize=undefined", "-fno-gpu-sanitize", "-g", "-o", exe, drv, obj,
              *others])
    assert r.returncode == 0, r.stderr[-2000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:verify_asan_link_order=0:protect_shadow_gap=0")
    env.pop("LD_PRELOAD", None)
    r = _run([exe], env=env)
    assert r.returncode == 0 and _clean(r.stderr), (r.stdout[-2000:], r.stderr[-2000:])
    assert " 0 failed" in r.stdout
