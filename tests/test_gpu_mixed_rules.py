"""Layers of a step through ra_sparse_attention, ra_biased_attention and ra_decode_attention, in
any mixture, through events: outputs under rules against float64, those over chosen blocks as
of a twin whose steps are all made that way, rows and positions exactly."""

import numpy as np
import pytest
import torch

from biased_harness import Sim, slopes
from gpu_harness import DEV
from paper_2609_03430_amd import binding as B

pytestmark = pytest.mark.gpu
CHRON, PAGED = B.RA_LAYOUT_CHRONOLOGICAL, B.RA_LAYOUT_PAGED
L, Hq, Hkv, BLOCKS, RECENT = 3, 4, 2, 3, 40


@pytest.mark.parametrize("layout", [CHRON, PAGED])
@pytest.mark.parametrize("dtype", [B.RA_BF16, B.RA_E4M3])
def test_mixed_layers(dtype, layout):
    """Slots of 5 to 430 rows (up to ten blocks to choose from), one inactive; one ends and
    another begins between steps."""
    sims = [Sim(L, Hq, Hkv, 60, [5, 300, 130], r=16, every=16, dtype=dtype, layout=layout,
                weights=False, max_seqs=4, extra_rows=L * Hkv * 512, seed=3) for _ in range(2)]
    mixed, twin = sims
    for sim in sims:
        sim.cache.attach_sparse(BLOCKS)
    kw = dict(cap=9.0, slopes=slopes(Hq), window=90, prefix=20)
    rule = mixed.rule(kw)
    rng = np.random.default_rng(int(dtype) * 7 + int(layout))
    seen = {}
    for t in range(75):
        if t in (30, 55):
            for sim in sims:
                B.ra_seq_end(sim.h, 1)
                sim.seq.pop(1)
                sim.begin(1, 250 if t == 30 else 77)
        last = None
        for l in range(L):
            q, k, v = mixed.inputs()
            assert all(torch.equal(a, b) for a, b in zip((q, k, v), twin.inputs()))
            dev = [x.to(DEV) for x in (q, k, v)]
            out, other = (torch.full((4, Hq, 128), 7.0, dtype=torch.bfloat16, device=DEV)
                          for _ in range(2))
            twin.cache.decode_sparse(l, BLOCKS, RECENT, *dev, other)
            call = "sparse rule plain".split()[rng.integers(3)]
            seen[last, call] = seen.get((last, call), 0) + 1
            last = call
            if call == "sparse":
                mixed.cache.decode_sparse(l, BLOCKS, RECENT, *dev, out)
                # (the splits follow the lengths, which are the twin's)
                assert torch.equal(out, other), (t, l)
            elif call == "rule":
                mixed.cache.decode_biased(l, rule, *dev, out)
            else:
                mixed.cache.decode(l, *dev, out)
            for s in mixed.seq:
                if call == "sparse":
                    _append(mixed, s, l, k, v)
                else:
                    mixed.follow(s, l, q, k, v, out, kw if call == "rule" else {}, (t, l, call))
        ends = [B.ra_end_step(sim.h) for sim in sims]
        torch.cuda.synchronize()
        assert ends[0] == ends[1]
        for s, seq in mixed.seq.items():
            seq["step"] += 1
            m = len(seq["heads"][0, 0]["P"]) - seq["lp"] - mixed.r - mixed.K
            if seq["step"] % mixed.every == 0 and m > 0:
                mixed.event(s, m)
    assert len(seen) == 12 and all(n >= 3 for n in seen.values()), seen
    mixed.check()
    for s in mixed.seq:
        for a, b in zip(mixed.export(s)[:3], twin.export(s)[:3]):
            assert torch.equal(a, b)
    for sim in sims:
        sim.close()


def _append(sim, s, l, k, v):
    """follow() without an output to check."""
    from biased_harness import held
    now = sim.seq[s]["lp"] + sim.seq[s]["step"]
    for g in range(Hkv):
        h = sim.seq[s]["heads"][l, g]
        h["P"] = np.append(h["P"], now)
        h["K"] = np.vstack([h["K"], held(k[s, g:g + 1], sim.dtype)])
        h["V"] = np.vstack([h["V"], held(v[s, g:g + 1], sim.dtype)])
        h["W"], h["E"] = np.append(h["W"], 0.0), np.append(h["E"], 0.0)
