"""The 8-bit and block-sparse kernels keep their working sets in registers (CPU only)."""

import os
import shutil

import pytest

from test_kernel_resources import HIPCC, _spills


@pytest.mark.skipif(not os.path.exists(HIPCC) and shutil.which(HIPCC) is None,
                    reason="hipcc not available")
@pytest.mark.parametrize("src", ["attn_blocks.hip", "blocks.hip"])
def test_no_register_spills(src):
    spills = _spills(src)
    assert spills, "no kernels found in " + src
    assert not {k: v for k, v in spills.items() if v}, spills
