"""The largest selection by weight, 32 weights to a thread, holds 32-bit keys: what its 128
registers do not take stays small (CPU only)."""

import os
import shutil

import pytest

from test_kernel_resources import HIPCC, _spills

LARGEST = "weight_event_kernelILi1024ELi32E"


@pytest.mark.skipif(not os.path.exists(HIPCC) and shutil.which(HIPCC) is None,
                    reason="hipcc not available")
def test_the_largest_selection_spills_next_to_nothing():
    spills = {k: v for k, v in _spills("weights.hip").items() if LARGEST in k}
    assert len(spills) == 2                    # a region's rows, a block table's
    assert max(spills.values()) <= 4, spills
