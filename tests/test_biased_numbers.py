"""Integers that do not fit the C interface's 32 bits are refused by the Python calls, not
wrapped to others (CPU only)."""

import pytest
import torch

from paper_2609_03430_amd import binding as B

WRAPS = [2 ** 32, 2 ** 32 + 3, -2 ** 32 + 7, 2 ** 31, -2 ** 31 - 1, 2 ** 63, 1.5]
CFG = B.make_config(2, 8, 2, 100)


@pytest.mark.parametrize("x", WRAPS)
def test_refused(x):
    rotary, rule = B.make_rotary(1e4), B.make_score_rule()
    calls = [
        lambda: B.make_score_rule(window=x),
        lambda: B.make_score_rule(prefix=x),
        lambda: B.make_rotary(1e4, dims=x),
        lambda: B.make_rotary(1e4, pairs=x),
        lambda: B.make_rotary(1e4, scaling=x),
        lambda: B.make_rotary(1e4, original_len=x),
        lambda: B.ra_rotate_rows(rotary, torch.zeros(1, 1, 128), None, first=x),
        lambda: B.ra_biased_attention(None, x if x != 1.5 else 2 ** 31, rule, None, None, None, None,
                                      None),
        lambda: B.ra_weights_workspace_bytes(CFG, x),
        lambda: B.ra_write_weights(None, x, None, 0),
        lambda: B.ra_export_weights(None, x, None, 0),
        lambda: B.ra_write_positions(None, x, None, 0),
    ]
    for call in calls:
        with pytest.raises(B.RandAttnError, match="not an integer of 32 bits") as e:
            call()
        assert e.value.status == B.RA_ERR_INVALID_ARG


def test_the_limits_are_taken():
    rule = B.make_score_rule(window=2 ** 31 - 1, prefix=0)
    assert rule.window == 2 ** 31 - 1
    assert B.make_rotary(1e4, original_len=2 ** 31 - 1).original_len == 2 ** 31 - 1
    assert B.ra_weights_workspace_bytes(CFG, -2 ** 31) == 0
