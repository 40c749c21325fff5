"""The step's new pair in attention over blocks: attended and appended as it was given
(or as an 8-bit row holds it), by the wavefront that stages it, at every place of its block."""

import pytest
import torch

from blocks_harness import fill_stale, held
from gpu_harness import DEV
from oracle.attention import gqa_decode
from paper_2609_03430_amd import binding as B

pytestmark = pytest.mark.gpu
CHRON, PAGED = B.RA_LAYOUT_CHRONOLOGICAL, B.RA_LAYOUT_PAGED


@pytest.mark.parametrize("dtype", [B.RA_BF16, B.RA_E4M3])
@pytest.mark.parametrize("layout", [CHRON, PAGED])
@pytest.mark.parametrize("first", [0, 17])
def test_rows_grow_from_new_pairs_alone(first, layout, dtype):
    """Steps from a cache of `first` rows on, over two blocks: the rows read back are the
    pairs given, and the last step's output is the attention over them (within half a bf16
    step and the 2^-17 and fp32 roundings of weights and sums, under 1e-4)."""
    Hq, Hkv, steps = 6, 3, 70
    g = torch.Generator().manual_seed(first + 1)
    k, v = (torch.randn(Hkv, first + steps, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    cfg = B.make_config(1, Hq, Hkv, 200, 0, 64, dtype=dtype, max_seqs=2, layout=layout,
                        page_rows=32, max_prompt_len=32)
    c = B.Cache(cfg, 2 * B.ra_seq_rows(cfg, first))
    fill_stale(c)
    c.attach_sparse(64)
    for s in range(2):
        rows = [x[:, :first][None].contiguous().to(DEV) for x in (k, v)] if first else [None, None]
        B.ra_seq_begin(c.handle, s, first, 1, s, *rows)
    for t in range(first, first + steps):
        q = torch.randn(2, Hq, 128, generator=g).to(torch.bfloat16)
        new = [x[:, t][None].expand(2, -1, -1).contiguous().to(DEV) for x in (k, v)]
        out = torch.empty(2, Hq, 128, dtype=torch.bfloat16, device=DEV)
        c.decode_sparse(0, 64, 0, q.to(DEV), *new, out)
        B.ra_end_step(c.handle)
        if t == 0:                                  # one row: its value, whatever the query
            one = v[:, 0] if dtype == B.RA_BF16 else held(v[:, 0])
            assert torch.equal(out[0].cpu(), one.repeat_interleave(Hq // Hkv, 0))
    n = first + steps
    ko, vo = (torch.empty(1, Hkv, n, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    hk, hv = (k, v) if dtype == B.RA_BF16 else (held(k), held(v))
    for s in range(2):
        assert B.ra_get_seq_info(c.handle, s).len == n
        B.ra_export_rows(c.handle, s, ko, vo)
        assert torch.equal(ko[0].cpu(), hk) and torch.equal(vo[0].cpu(), hv)
        want = gqa_decode(q[s].double().numpy(), [x.double().numpy() for x in hk],
                          [x.double().numpy() for x in hv])
        err = (out[s].double().cpu() - torch.from_numpy(want)).abs()
        assert (err <= 2.0 ** -8 * torch.from_numpy(want).abs() + 1e-4).all(), err.max()
    c.close()
