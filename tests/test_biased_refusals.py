"""Sizes and refusals of rotary positions, score rules and accumulated weights, on the CPU."""

import ctypes

import numpy as np
import pytest

from oracle import rotary, rule
from paper_2609_03430_amd import binding as B

INVALID, UNSUPPORTED = B.RA_ERR_INVALID_ARG, B.RA_ERR_UNSUPPORTED


def _cfg(**kw):
    return B.make_config(2, 8, 2, 64, max_seqs=2, **kw)


def test_weight_sizes():
    c = _cfg()
    assert B.ra_weights_bytes(c, 3200) == 4 * 3200
    assert B.ra_weights_bytes(c, 0) == B.ra_weights_bytes(c, 33) == 0
    # the split partials (to 256 bytes), two floats per query (to 64 of them), a float per row
    rows = B.ra_region_rows(c, 100)
    part = -(-B.ra_workspace_bytes(c) // 256) * 256
    assert B.ra_weights_workspace_bytes(c, 100) == part + 4 * (64 + 2 * 8 * rows)
    assert B.ra_weights_workspace_bytes(c, -1) == 0
    total = _cfg(budget_mode=B.RA_BUDGET_TOTAL)
    assert B.ra_weights_workspace_bytes(total, 65) == 0        # no such prompt
    paged = _cfg(layout=B.RA_LAYOUT_PAGED, page_rows=128, max_prompt_len=70)
    held = -(-(70 + 64 + 64 + 64) // 128) * 128
    for lp in (0, 70, 10 ** 6):
        assert B.ra_weights_workspace_bytes(paged, lp) == part + 4 * (64 + 2 * 8 * held)
    hole = _cfg(layout=B.RA_LAYOUT_HOLE_FILL)
    assert B.ra_weights_bytes(hole, 3200) == B.ra_weights_workspace_bytes(hole, 3) == 0
    # an attachment, not a policy: the caches' own sizes are what they were
    assert B.ra_config_check(_cfg(policy=5)) == INVALID


def test_null_handles_are_refused():
    lib = B._lib()
    r, s = B.make_rotary(10000.0), B.make_score_rule()
    assert lib.ra_rotate_step(None, ctypes.byref(r), 16, 16, 16, 16, None) == INVALID
    assert lib.ra_biased_attention(None, 0, ctypes.byref(s), 16, 16, 16, 16, 16, 0, None) == INVALID
    assert lib.ra_biased_attention(None, 0, None, 16, 16, 16, 16, 16, 0, None) == INVALID
    assert lib.ra_weights_attach(None, None, 0) == INVALID
    assert lib.ra_write_weights(None, 0, None, None) == INVALID
    assert lib.ra_export_weights(None, 0, None, 0, None) == INVALID
    assert lib.ra_write_positions(None, 0, None, None) == INVALID


@pytest.mark.parametrize("kw", [
    dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")), dict(base=-5.0), dict(dims=0),
    dict(dims=3), dict(dims=130), dict(dims=-2), dict(pairs=2), dict(pairs=-1), dict(scaling=4),
    dict(scaling=-1), dict(magnitude=-1.0), dict(magnitude=float("nan")),
    dict(scaling=1, factor=0.5), dict(scaling=1, factor=float("inf")),
    dict(scaling=2, low=4.0, high=4.0), dict(scaling=2, low=0.0), dict(scaling=2, original_len=0),
    dict(scaling=3, high=float("inf")), dict(scaling=3, low=float("nan")),
    dict(scaling=3, original_len=-1),
])
def test_rotary_arguments(kw):
    kw = dict(dict(base=10000.0), **kw)
    r = B.make_rotary(**kw)
    # (addresses that nothing may touch: every call ends before a launch)
    assert B._lib().ra_rotate_rows(ctypes.byref(r), B.RA_BF16, 16, 16, 1, 1, 0, None, None) == INVALID


def test_rotated_rows_arguments():
    f, r = B._lib().ra_rotate_rows, B.make_rotary(10000.0)
    p = ctypes.byref(r)
    assert f(None, B.RA_BF16, 16, 16, 1, 1, 0, None, None) == INVALID
    for dtype in (B.RA_E4M3, 3, -1):
        assert f(p, dtype, 16, 16, 1, 1, 0, None, None) == INVALID
    assert f(p, B.RA_BF16, 16, 16, -1, 1, 0, None, None) == INVALID
    assert f(p, B.RA_BF16, 16, 16, 1, -1, 0, None, None) == INVALID
    assert f(p, B.RA_BF16, 8, 16, 1, 1, 0, None, None) == INVALID        # not 16-byte aligned
    assert f(p, B.RA_BF16, 16, 24, 1, 1, 0, None, None) == INVALID
    assert f(p, B.RA_BF16, None, 16, 1, 1, 0, None, None) == INVALID
    assert f(p, B.RA_BF16, 16, 16, 1, 1, -1, None, None) == INVALID
    assert f(p, B.RA_BF16, 16, 16, 1, 3, 2 ** 31 - 2, None, None) == INVALID
    assert f(p, B.RA_BF16, None, None, 0, 5, 0, None, None) == B.RA_OK   # nothing to do
    assert f(p, B.RA_BF16, None, None, 5, 0, 0, None, None) == B.RA_OK


def test_oracle_rule():
    """The oracle: a window of one attends to the new row (and the prefix), a cap bounds the
    scores, slopes favour the nearest, drops go to the earliest of equals."""
    rng = np.random.default_rng(1)
    q, K, pos = rng.normal(size=8), rng.normal(size=(5, 8)), np.array([0, 1, 5, 9, 12])
    p = rule.rule_weights(q, K, pos, 12, window=1)
    assert np.array_equal(p, [0, 0, 0, 0, 1])
    assert (rule.rule_weights(q, K, pos, 12, window=1, prefix=2) > 0).tolist() == [1, 1, 0, 0, 1]
    flat = rule.rule_weights(1e6 * q, K, pos, 12, cap=1e-9)
    assert np.allclose(flat, 0.2)
    near = rule.rule_weights(0 * q, K, pos, 12, slope=1.0)
    assert np.allclose(near[1:] / near[:-1], np.exp(np.diff(pos)))
    w = np.array([9, 1, 0, 1, np.nan, 1, 5])
    assert rule.weight_drops(w, 1, 1, 3).tolist() == [1, 2, 4]
    assert rule.weight_drops(w, 1, 0, 0).tolist() == []


def test_oracle_rotary():
    """Rotations keep lengths, and products of rows turned by p and p' depend on p - p'."""
    rng = np.random.default_rng(2)
    f = rotary.frequencies(10000.0, 96, "channels", 16.0, 1.0, 32.0, 4096)
    plain = rotary.frequencies(10000.0, 96)
    assert f[0] == plain[0] and np.isclose(f[-1], plain[-1] / 16)
    assert ((f <= plain) & (f >= plain / 16 * (1 - 1e-12))).all()
    for adjacent in (False, True):
        a, b = rng.normal(size=(2, 128))
        x = [rotary.rotate(a, p, f, adjacent) @ rotary.rotate(b, p + 7, f, adjacent)
             for p in (0, 5, 1000)]
        assert np.allclose(x, x[0])
        assert np.isclose(np.linalg.norm(rotary.rotate(a, 77, f, adjacent)), np.linalg.norm(a))
