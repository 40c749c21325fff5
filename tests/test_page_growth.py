"""Steps of a paged cache while host memory runs out, on the CPU: refused with nothing
changed, and nothing throws across the C interface."""

import os
import subprocess

import pytest

from paper_2609_03430_amd import binding as B
from test_slot_order import ATTENTION, CLANG, CSRC, FUZZ, HIPCC, ROOT

pytestmark = pytest.mark.skipif(
    not (os.path.exists(HIPCC) and os.path.exists(CLANG) and os.path.isdir(FUZZ)),
    reason="hipcc / clang++ or the stand-ins missing")


@pytest.fixture(scope="module")
def page_growth(tmp_path_factory):
    d = tmp_path_factory.mktemp("pages")
    hip = [HIPCC, "-x", "hip", "--cuda-host-only", "-O1", "-g", "-std=c++17",
           "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-fno-sanitize-recover=all"]
    objs = []
    for src in (os.path.join(CSRC, "api.cpp"), os.path.join(CSRC, "api_blocks.cpp"),
                os.path.join(FUZZ, "stub_launchers.cpp"), os.path.join(FUZZ, "page_growth.cpp")):
        objs.append(str(d / (os.path.basename(src) + ".o")))
        subprocess.run(hip + ["-c", src, "-o", objs[-1]], check=True, capture_output=True)
    exe = str(d / "page_growth")
    subprocess.run([CLANG, "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-Wl,--wrap=" + ATTENTION] + objs + ["-o", exe], check=True, capture_output=True)
    return exe


@pytest.mark.parametrize("sparse", [0, 1])
@pytest.mark.parametrize("dtype", [B.RA_BF16, B.RA_E4M3])
def test_a_step_without_host_memory_is_refused(page_growth, dtype, sparse):
    r = subprocess.run([page_growth, str(dtype), str(sparse)], capture_output=True, text=True,
                       timeout=120)
    assert r.returncode == 0, r.stderr
    assert int(r.stdout) > 5          # (pages were needed while there was no memory)
