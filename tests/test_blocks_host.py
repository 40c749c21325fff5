"""The host side of block-sparse steps and 8-bit caches on the CPU: which bounds are
computed when, under AddressSanitizer and UndefinedBehaviorSanitizer, and the launch
plan's rules on both sides of each line."""

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

pytestmark = pytest.mark.skipif(
    not (os.path.exists(HIPCC) and os.path.exists(CLANG) and os.path.isdir(FUZZ)),
    reason="hipcc / clang++ or the stand-ins missing")


def _build(d, name, sources, sanitize):
    """Host-only objects of HIP sources, linked with the host compiler."""
    hip = [HIPCC, "-x", "hip", "--cuda-host-only", "-O1", "-g", "-std=c++17",
           "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]
    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all"] if sanitize else []
    if sanitize:
        hip += ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                "-fno-sanitize-recover=all"]
    objs = []
    for src in sources:
        objs.append(str(d / (os.path.basename(src) + ".o")))
        subprocess.run(hip + ["-c", src, "-o", objs[-1]], check=True, capture_output=True)
    exe = str(d / name)
    link = [CLANG] + san if sanitize else ["g++", "-no-pie"]
    subprocess.run(link + objs + ["-o", exe], check=True, capture_output=True)
    return exe


@pytest.fixture(scope="module")
def protocol(tmp_path_factory):
    return _build(tmp_path_factory.mktemp("blocks"), "blocks_protocol",
                  [os.path.join(CSRC, "api.cpp"), os.path.join(CSRC, "api_blocks.cpp"),
                   os.path.join(FUZZ, "stub_launchers.cpp"),
                   os.path.join(FUZZ, "blocks_protocol.cpp")], True)


@pytest.mark.parametrize("dtype,layout", [(B.RA_BF16, CHRON), (B.RA_BF16, PAGED),
                                          (B.RA_E4M3, CHRON), (B.RA_E4M3, PAGED)])
def test_bounds_follow_the_rows(protocol, dtype, layout):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1")
    total = {"sparse": 0, "built": 0, "checked": 0, "refused": 0}
    for seed in range(1, 13):
        r = subprocess.run([protocol, str(seed), str(dtype), str(layout), "400"], env=env,
                           capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, (seed, r.stderr)
        for k, v in json.loads(r.stdout).items():
            total[k] += v
    # the runs did what they are there for
    assert total["sparse"] > 500 and total["built"] > 1000 and total["checked"] > 5000, total
    assert total["refused"] > 50, total


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    exe = _build(tmp_path_factory.mktemp("plans"), "plan_rules",
                 [os.path.join(CSRC, "api.cpp"), os.path.join(FUZZ, "stub_launchers.cpp"),
                  os.path.join(FUZZ, "plan_rules.cpp")], False)

    def launches(lens, layout=CHRON, q_heads=40, kv_heads=8, budget=64, recent=64, every=64,
                 forward=0, steps=1):
        args = [B.RA_E4M3, layout, q_heads, kv_heads, budget, recent, every, forward, steps] + lens
        r = subprocess.run([exe] + [str(a) for a in args], capture_output=True, text=True,
                           timeout=60)
        assert r.returncode == 0, r.stderr
        return [json.loads(line) for line in r.stdout.splitlines()]
    return launches


@pytest.mark.parametrize("n,kv_heads,keys,splits", [
    (1, 8, 384, 1), (1, 8, 385, 2), (1, 8, 600, 3), (1, 8, 2200, 9), (1, 8, 9000, 12),
    (1, 8, 30000, 30), (1, 8, 120000, 32), (1, 2, 120000, 64), (2, 8, 9000, 12),
    (4, 8, 9000, 8), (8, 8, 9000, 4), (12, 8, 9000, 2), (16, 8, 768, 1), (16, 8, 769, 2),
    (17, 8, 9000, 1), (32, 8, 9000, 1), (33, 8, 9000, 3), (33, 8, 4095, 1), (44, 8, 9000, 3),
    (45, 8, 9000, 2), (56, 8, 9000, 2), (57, 8, 9000, 1), (72, 8, 9000, 1), (73, 8, 9000, 2),
    (95, 8, 9000, 2), (96, 8, 9000, 1),
])
def test_splits_of_8_bit_heads(plans, n, kv_heads, keys, splits):
    a = plans([keys - 1] * n, kv_heads=kv_heads, q_heads=5 * kv_heads)[0]
    assert (a["waves"], a["splits"]) == (4, splits)
    assert a["keys"] % 32 == 0 and a["keys"] * a["splits"] >= keys


def test_partials_past_256_heads_fit_the_fixed_array(plans):
    """Three splits of 264 heads of 16 queries need 6.6 MB, of 352 heads 8.8 MB."""
    assert plans([9000] * 33, q_heads=128)[0]["splits"] == 3
    assert plans([9000] * 44, q_heads=128)[0]["splits"] == 1


@pytest.mark.parametrize("n,moved,chunks", [
    # (moved: the candidates and recent rows of the event)
    (1, 505, 0), (1, 506, 2), (4, 9000, 18), (1, 10745, 21), (1, 10746, 0),
    (32, 2041, 4), (32, 2042, 0), (33, 2000, 0),
])
def test_moves_of_8_bit_events_split_past_a_chunk(plans, n, moved, chunks):
    """Several workgroups per head while they are at most four to a CU; events of more
    sequences than a launch lists (32) are never split."""
    a = plans([40] * n, budget=moved - 17, recent=16, every=1, forward=moved - 1)[0]
    assert a["evicted"] == n and a["len"] == 40 + moved - 1
    assert a["chunks"] == chunks
