"""The kernels of rotary positions, biased attention and accumulated weights keep their
working sets in registers (CPU only).  The selection of 32 weights per thread keeps its keys
in scratch memory, as the random events' largest build does."""

import os
import shutil

import pytest

from test_kernel_resources import HIPCC, _spills


@pytest.mark.skipif(not os.path.exists(HIPCC) and shutil.which(HIPCC) is None,
                    reason="hipcc not available")
@pytest.mark.parametrize("src", ["attn_biased.hip", "weights.hip", "rotary.hip"])
def test_no_register_spills(src):
    spills = _spills(src)
    assert spills, "no kernels found in " + src
    assert not {k: v for k, v in spills.items() if v and "weight_event_kernelILi1024ELi32E" not in k}
