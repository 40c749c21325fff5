"""Events by weight at the end of steps whose heads are long enough for a workgroup to a chunk of
rows: several listed slots, more slots than an event lists, and captured steps, where the
launch is made for the longest heads that a region holds.

Queries of zeros attend to every row alike, so a step adds the same to all weights and the
rows that an event drops are those of least given weight, which are whole numbers apart."""

import numpy as np
import pytest
import torch

from gpu_harness import DEV
from paper_2609_03430_amd import binding as B

pytestmark = pytest.mark.gpu
CHRON, PAGED = B.RA_LAYOUT_CHRONOLOGICAL, B.RA_LAYOUT_PAGED
DTYPES = [B.RA_BF16, B.RA_E4M3, B.RA_F32]
G, R, EVERY, STEPS = 2, 64, 64, 3


class Slots:
    """Slots whose first event comes at the end of step phases[s], their rows and weights as
    given and as the events leave them."""

    def __init__(self, dtype, layout, L, Hkv, K, phases, seed):
        self.L, self.Hkv, self.K, self.phases, self.dtype = L, Hkv, K, phases, dtype
        self.lps = [10 + 7 * (s % 30) for s in range(len(phases))]
        self.cfg = B.make_config(L, G * Hkv, Hkv, K, R, EVERY, dtype=dtype, max_seqs=len(phases),
                                 layout=layout, max_prompt_len=max(self.lps))
        self.cache = B.Cache(self.cfg, B.ra_required_slots(self.cfg, self.lps))
        self.cache.attach_weights(max(self.lps))
        self.h = self.cache.handle
        self.gen = torch.Generator().manual_seed(seed)
        self.tdtype = torch.float32 if dtype == B.RA_F32 else torch.bfloat16
        first = ((K + R) // EVERY + 1) * EVERY
        self.given = []
        for s, (lp, phase) in enumerate(zip(self.lps, phases)):
            B.ra_seq_begin(self.h, s, lp, 1, s)
            B.ra_seq_fast_forward(self.h, s, first - phase)
            n = lp + first - phase
            assert B.ra_get_seq_info(self.h, s).len == n
            rows = [torch.randn(L, Hkv, n, 128, generator=self.gen).to(self.tdtype).to(DEV)
                    for _ in range(2)]
            w = torch.stack([torch.randperm(n, generator=self.gen) for _ in range(L * Hkv)])
            w = w.view(L, Hkv, n).float().to(DEV)
            B.ra_write_rows(self.h, s, *rows)
            B.ra_write_weights(self.h, s, w)
            if dtype == B.RA_E4M3:
                B.ra_export_rows(self.h, s, *rows)     # the values the codes stand for
            self.given.append((rows, w))
        S = len(phases)
        self.q = torch.zeros(S, G * Hkv, 128, dtype=self.tdtype, device=DEV)
        self.new = [torch.randn(S, Hkv, 128, generator=self.gen).to(self.tdtype).to(DEV)
                    for _ in range(2)]
        self.out = torch.empty_like(self.q)
        self.rule = B.make_score_rule()

    def step(self):
        for l in range(self.L):
            self.cache.decode_biased(l, self.rule, self.q, *self.new, self.out)
        return B.ra_end_step(self.h)

    def check(self):
        for s, (phase, lp, (rows, w)) in enumerate(zip(self.phases, self.lps, self.given)):
            n0 = w.shape[2]
            m = n0 + phase - R - lp - self.K
            assert 0 < m <= EVERY
            n = n0 + STEPS - m
            assert B.ra_get_seq_info(self.h, s).len == n, s
            shape = (self.L, self.Hkv, n)
            pos = torch.empty(shape, dtype=torch.int32, device=DEV)
            got = [torch.empty(*shape, 128, dtype=self.tdtype, device=DEV) for _ in range(2)]
            weights = torch.empty(shape, device=DEV)
            B.ra_export_positions(self.h, s, pos)
            B.ra_export_rows(self.h, s, *got)
            B.ra_export_weights(self.h, s, weights)
            # what each step adds to the rows it attends to, and to its own
            adds = [G / (n0 + t + 1 - (m if t >= phase else 0)) for t in range(STEPS)]
            for l in range(self.L):
                for g in range(self.Hkv):
                    cand = w[l, g, lp:n0 + phase - R].cpu().numpy()
                    drop = lp + np.argsort(cand)[:m]
                    keep = np.setdiff1d(np.arange(n0), drop)
                    want = np.concatenate([keep, n0 + np.arange(STEPS)])
                    assert np.array_equal(pos[l, g].cpu().numpy(), want), (s, l, g)
                    at = torch.from_numpy(keep).to(DEV)
                    for x, y in zip(got, rows):
                        assert torch.equal(x[l, g, :len(keep)], y[l, g, at]), (s, l, g)
                    for x, y in zip(got, self.new):
                        new = x[l, g, len(keep):]
                        assert torch.equal(new[0], new[1]) and torch.equal(new[0], new[2])
                        if self.dtype != B.RA_E4M3:
                            assert torch.equal(new[0], y[s, g])
                    wants = np.concatenate([w[l, g].cpu().numpy()[keep] + sum(adds),
                                            [sum(adds[t:]) for t in range(STEPS)]])
                    # a rounding of a weight below n0 + 1 per step, and 2^-12 of what is added
                    # (a sum of n equal terms, its quotient, G of them)
                    bound = STEPS * (n0 + 1) * 2.0 ** -24 + 2.0 ** -12 * sum(adds)
                    assert np.abs(weights[l, g].cpu().numpy() - wants).max() <= bound, (s, l, g)


# K: at least three chunks of rows at an event (512 to a chunk, 256 of fp32)
KEEP = {B.RA_BF16: 1111, B.RA_E4M3: 1111, B.RA_F32: 540}


@pytest.mark.parametrize("layout", [CHRON, PAGED])
@pytest.mark.parametrize("dtype", DTYPES)
def test_listed_slots(dtype, layout):
    """Three slots, two due at once and one a step later; then heads of many chunks."""
    for K in (KEEP[dtype], 4 * KEEP[dtype] + 7):
        sim = Slots(dtype, layout, 2, 2, K, [1, 2, 1], K)
        assert [sim.step() for _ in range(STEPS)] == [2, 1, 0]
        sim.check()
        sim.cache.close()


@pytest.mark.parametrize("layout", [CHRON, PAGED])
@pytest.mark.parametrize("dtype", DTYPES)
def test_more_slots_than_an_event_lists(dtype, layout):
    phases = [2 if s in (0, 5, 39) else 3 if s == 17 else 1 for s in range(40)]
    sim = Slots(dtype, layout, 1, 1, KEEP[dtype], phases, 7)
    assert [sim.step() for _ in range(STEPS)] == [36, 3, 1]
    sim.check()
    sim.cache.close()


@pytest.mark.parametrize("dtype", DTYPES)
def test_captured_steps(dtype):
    """Captured once, replayed through the slots' events with eager work between."""
    for K in (KEEP[dtype], 4 * KEEP[dtype] + 7):
        sim = Slots(dtype, CHRON, 2, 2, K, [3, 2, 3], K + 1)
        B.ra_graph_mode(sim.h, True)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            sim.step()
            with torch.cuda.graph(graph, stream=side):
                sim.step()
        torch.cuda.current_stream().wait_stream(side)
        for _ in range(STEPS - 1):
            graph.replay()
            torch.cuda.synchronize()
            torch.full((1000,), 3.0, device=DEV).sum()
        del graph
        B.ra_graph_mode(sim.h, False)
        sim.check()
        sim.cache.close()
