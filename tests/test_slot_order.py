"""The order in which attention over blocks takes the slots, on the CPU: random calls
on the host library, whose steps mix dense and sparse layers while sequences come
and go, under AddressSanitizer and UndefinedBehaviorSanitizer."""

import json
import os
import subprocess

import pytest

from paper_2609_03430_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_03430_amd", "csrc")
FUZZ = os.path.join(ROOT, "tests", "host_fuzz")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CLANG = "/opt/rocm/llvm/bin/clang++"
CHRON, PAGED = B.RA_LAYOUT_CHRONOLOGICAL, B.RA_LAYOUT_PAGED
ATTENTION = "_ZN2ra16launch_attentionERKNS_5ShapeERKNS_10AttnLaunchEP12ihipStream_t"

pytestmark = pytest.mark.skipif(
    not (os.path.exists(HIPCC) and os.path.exists(CLANG) and os.path.isdir(FUZZ)),
    reason="hipcc / clang++ or the stand-ins missing")


@pytest.fixture(scope="module")
def slot_order(tmp_path_factory):
    d = tmp_path_factory.mktemp("order")
    hip = [HIPCC, "-x", "hip", "--cuda-host-only", "-O1", "-g", "-std=c++17",
           "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-fno-sanitize-recover=all"]
    objs = []
    for src in (os.path.join(CSRC, "api.cpp"), os.path.join(CSRC, "api_blocks.cpp"),
                os.path.join(FUZZ, "stub_launchers.cpp"), os.path.join(FUZZ, "slot_order.cpp")):
        objs.append(str(d / (os.path.basename(src) + ".o")))
        subprocess.run(hip + ["-c", src, "-o", objs[-1]], check=True, capture_output=True)
    exe = str(d / "slot_order")
    subprocess.run([CLANG, "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-Wl,--wrap=" + ATTENTION] + objs + ["-o", exe], check=True, capture_output=True)
    return exe


# 300 slots: more active ones than an order holds, and fewer
@pytest.mark.parametrize("slots,seeds,ops", [(4, 12, 400), (300, 2, 2000)])
@pytest.mark.parametrize("dtype,layout", [(B.RA_BF16, CHRON), (B.RA_BF16, PAGED),
                                          (B.RA_E4M3, CHRON), (B.RA_E4M3, PAGED)])
def test_an_order_holds_every_active_slot(slot_order, dtype, layout, slots, seeds, ops):
    total = {"steps": 0, "ordered": 0, "after_dense": 0}
    for seed in range(1, seeds + 1):
        r = subprocess.run([slot_order] + [str(x) for x in (seed, dtype, layout, slots, ops)],
                           capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, (seed, r.stderr)
        for k, v in json.loads(r.stdout).items():
            total[k] += v
    # the runs did what they are there for
    assert total["steps"] > 500 and total["ordered"] > 200 and total["after_dense"] > 50, total
