"""What the paged cache's calls and the verdict over drafts ask of the HIP runtime, on the CPU: the host pass of their sources with the runtime's functions replaced
(tests/sanitize/paged_launch_driver.cpp), under AddressSanitizer and UndefinedBehaviorSanitizer.  GPU code is not compiled and never runs here."""
import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from .test_sanitizers import ENV, ROOT, SAN

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not on PATH")


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("paged_launches")
    flags = ["--offload-arch=gfx950", "--cuda-host-only", "-O1", "-g", "-std=c++17", "-Xarch_host", "-fsanitize=address,undefined",
             "-fno-gpu-sanitize", "-fno-sanitize-recover=all"]
    csrc = os.path.join(ROOT, "paper_2504_12329_amd", "csrc")
    srcs = [os.path.join(csrc, f) for f in ("paged.hip", "paged_attend.hip", "verify.hip")] + [os.path.join(SAN, "paged_launch_driver.cpp")]

    def compile_one(src):
        obj = str(tmp / (os.path.basename(src) + ".o"))
        subprocess.run(["hipcc", *flags, "-x", "hip", "-c", src, "-o", obj], check=True, capture_output=True)
        return obj

    with ThreadPoolExecutor(max_workers=4) as ex:
        objs = list(ex.map(compile_one, srcs))
    exe = str(tmp / "paged_launches")
    # (the GPU code that the objects refer to does not exist: its registration is replaced too)
    subprocess.run(["hipcc", "-no-hip-rt", "-Xarch_host", "-fsanitize=address,undefined", "-Wl,--unresolved-symbols=ignore-all", "-o", exe, *objs],
                   check=True, capture_output=True)
    return exe


@pytest.mark.parametrize("name", ["grids", "lds", "verify"])
def test_launches(driver, name):
    r = subprocess.run([driver, name], env=ENV, capture_output=True, text=True, timeout=200)
    assert r.returncode == 0 and "ok" in r.stdout, f"{name}: {r.returncode}\n{r.stdout}\n{r.stderr}"
