"""AddressSanitizer + UndefinedBehaviorSanitizer build of the 4-bit cache's host code, driven by tests/sanitize/kv4_driver.cpp.  No GPU is
used: the GPU code objects are compiled without sanitizers and never run here."""
import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from .test_sanitizers import ROOT, SAN, _run


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not on PATH")
def test_the_calls_of_the_4_bit_cache_under_address_and_ub_sanitizers(tmp_path):
    flags = ["--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-Xarch_host", "-fsanitize=address,undefined", "-fno-gpu-sanitize",
             "-fno-sanitize-recover=all", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
    csrc = os.path.join(ROOT, "paper_2504_12329_amd", "csrc")
    srcs = [os.path.join(csrc, f) for f in ("kv4.hip", "kv4_attend.hip", "kv4_evict.hip")] + [os.path.join(SAN, "kv4_driver.cpp")]

    def compile_one(src):
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        subprocess.run(["hipcc", *flags, "-x", "hip", "-c", src, "-o", obj], check=True, capture_output=True)
        return obj

    with ThreadPoolExecutor(max_workers=4) as ex:
        objs = list(ex.map(compile_one, srcs))
    exe = str(tmp_path / "kv4_san")
    subprocess.run(["hipcc", "--offload-arch=gfx950", "-Xarch_host", "-fsanitize=address,undefined", "-fno-gpu-sanitize", "-o", exe, *objs],
                   check=True, capture_output=True)
    assert "ok" in _run(exe)
