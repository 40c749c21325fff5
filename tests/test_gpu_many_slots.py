"""Attention over blocks of more sequences and layers than one launch's arguments hold:
bounds of more than 64 slots or layers (several launches), and more active slots than an
order has room for (slots as they come)."""

import pytest
import torch

from blocks_harness import fill_stale, held
from gpu_harness import DEV, attn_err, log
from oracle import blocks
from oracle.attention import softmax_attention
from paper_2609_03430_amd import binding as B

pytestmark = pytest.mark.gpu
CHRON, PAGED = B.RA_LAYOUT_CHRONOLOGICAL, B.RA_LAYOUT_PAGED


@pytest.mark.parametrize("dtype", [B.RA_BF16, B.RA_E4M3])
@pytest.mark.parametrize("layout", [CHRON, PAGED])
@pytest.mark.parametrize("n_seqs,L", [(70, 2), (300, 1), (2, 67)])
def test_more_than_a_launch_holds(n_seqs, L, layout, dtype):
    log("many slots: %s" % ((n_seqs, L, layout, dtype),))
    n_blocks, recent, G = 2, 8, 2
    lens = [(37 * i) % 230 for i in range(n_seqs)]
    cfg = B.make_config(L, G, 1, 0, 0, 1, dtype=dtype, max_seqs=n_seqs, layout=layout, page_rows=32,
                        max_prompt_len=230)
    c = B.Cache(cfg, B.ra_required_slots(cfg, lens))
    fill_stale(c)
    c.attach_sparse(n_blocks)
    c.bounds.fill_(0x55)
    g = torch.Generator().manual_seed(n_seqs)
    keep = held if dtype == B.RA_E4M3 else (lambda x: x)
    rows = []
    for i, n in enumerate(lens):
        kv = [torch.randn(L, 1, n, 128, generator=g).to(torch.bfloat16) for _ in range(2)]
        B.ra_seq_begin(c.handle, i, n, 1, i, *[x.to(DEV) if n else None for x in kv])
        rows.append([keep(x) if n else x for x in kv])
    for sparse in (True, False):
        for layer in range(L):
            q = torch.randn(n_seqs, G, 128, generator=g).to(torch.bfloat16)
            kn, vn = (torch.randn(n_seqs, 1, 128, generator=g).to(torch.bfloat16) for _ in range(2))
            out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device=DEV)
            if sparse:
                c.decode_sparse(layer, n_blocks, recent, q.to(DEV), kn.to(DEV), vn.to(DEV), out)
            else:
                c.decode(layer, q.to(DEV), kn.to(DEV), vn.to(DEV), out)
            kn, vn = keep(kn), keep(vn)
            if layer not in (0, 1, 64, L - 1):
                continue
            for i, n in enumerate(lens):
                K, V = (torch.cat([rows[i][w][layer, 0], x[i]]).double().numpy()
                        for w, x in ((0, kn), (1, vn)))
                mine = q[i].double().numpy()
                if sparse:
                    at = blocks.attended(mine, K, n, n_blocks, recent)
                    K, V = K[at], V[at]
                for h in range(G):
                    attn_err(out[i, h], softmax_attention(mine[h], K, V), B.RA_BF16,
                             (sparse, layer, i, h))
        B.ra_end_step(c.handle)
    c.close()
