"""The host side of biased steps and accumulated weights on the CPU, under AddressSanitizer
and UndefinedBehaviorSanitizer: random calls, whose launches' plans, workspaces, weights and
row moves the stand-ins check (tests/host_fuzz/biased_protocol.cpp)."""

import json
import os
import subprocess

import pytest

from paper_2609_03430_amd import binding as B
from test_blocks_host import CLANG, CSRC, FUZZ, HIPCC, _build

CHRON, HOLE, PAGED = B.RA_LAYOUT_CHRONOLOGICAL, B.RA_LAYOUT_HOLE_FILL, B.RA_LAYOUT_PAGED

pytestmark = pytest.mark.skipif(
    not (os.path.exists(HIPCC) and os.path.exists(CLANG) and os.path.isdir(FUZZ)),
    reason="hipcc / clang++ or the stand-ins missing")


@pytest.fixture(scope="module")
def protocol(tmp_path_factory):
    return _build(tmp_path_factory.mktemp("biased"), "biased_protocol",
                  [os.path.join(CSRC, "api.cpp"), os.path.join(CSRC, "api_biased.cpp"),
                   os.path.join(FUZZ, "stub_launchers.cpp"),
                   os.path.join(FUZZ, "biased_protocol.cpp")], True)


@pytest.mark.parametrize("dtype,layout,weighed", [
    (B.RA_BF16, CHRON, 0), (B.RA_BF16, CHRON, 1), (B.RA_BF16, PAGED, 1), (B.RA_E4M3, CHRON, 1),
    (B.RA_E4M3, PAGED, 0), (B.RA_F32, CHRON, 1), (B.RA_F32, PAGED, 1), (B.RA_F32, HOLE, 0),
    (B.RA_BF16, HOLE, 0)])
def test_launches_of_random_calls(protocol, dtype, layout, weighed):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1")
    total = {}
    for seed in range(1, 13):
        r = subprocess.run([protocol, str(seed), str(dtype), str(layout), str(weighed), "400"],
                           env=env, capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, (seed, r.stderr[-2000:])
        for k, v in json.loads(r.stdout).items():
            total[k] = total.get(k, 0) + v
    assert total["steps"] > 300 and total["attends"] > 500, total
    assert (total["events"] > 20) == bool(weighed), total
    if (dtype, layout, weighed) == (B.RA_BF16, CHRON, 0):
        assert total["flushed"] > 0 and total["mixed"] > 50, total
