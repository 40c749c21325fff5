"""Events by accumulated weight: the choice exactly, the moves, resuming, refusals."""

import numpy as np
import pytest
import torch

from biased_harness import Sim
from blocks_harness import status
from gpu_harness import DEV, _f64
from oracle.rule import weight_drops
from paper_2609_03430_amd import binding as B

pytestmark = pytest.mark.gpu
CHRON, PAGED = B.RA_LAYOUT_CHRONOLOGICAL, B.RA_LAYOUT_PAGED


def _event(dtype, layout, L, Hkv, lp, K, r, extra, make, seqs=1, page_rows=32,
           every=1024):
    """Requests restored with rows and weights of their own, evicted by one explicit event each,
    and read back; `make(shape)` gives the weights.  (No trigger comes before it: K + r + extra
    steps pass no multiple of the period above K + r.)"""
    t = torch.float32 if dtype == B.RA_F32 else torch.bfloat16
    cfg = B.make_config(L, Hkv, Hkv, K, r, every, dtype=dtype, max_seqs=seqs, layout=layout,
                        page_rows=page_rows, max_prompt_len=lp)
    c = B.Cache(cfg, seqs * B.ra_seq_rows(cfg, lp))
    c.attach_weights(lp)
    c.weights.fill_(float("nan"))
    n, kept = lp + K + r + extra, lp + K + r
    for s in range(seqs):
        # numbers that 8-bit rows hold exactly: a power of two per row, its index in the codes
        k = torch.randint(-7, 8, (L, Hkv, n, 128), device=DEV).to(t)
        v = torch.randint(-7, 8, (L, Hkv, n, 128), device=DEV).to(t)
        w = make((L, Hkv, n)).to(DEV)
        B.ra_seq_begin(c.handle, s, lp, 1, s)
        B.ra_seq_fast_forward(c.handle, s, K + r + extra)
        B.ra_write_rows(c.handle, s, k, v)
        B.ra_write_weights(c.handle, s, w)
        B.ra_evict_now(c.handle, s)
        assert B.ra_get_seq_info(c.handle, s).len == (kept if extra > 0 else n)
        m = max(0, extra)
        shape = (L, Hkv, n - m)
        pos = torch.empty(shape, dtype=torch.int32, device=DEV)
        ko, vo = (torch.empty(*shape, 128, dtype=t, device=DEV) for _ in range(2))
        wo = torch.empty(shape, device=DEV)
        B.ra_export_positions(c.handle, s, pos)
        B.ra_export_rows(c.handle, s, ko, vo)
        B.ra_export_weights(c.handle, s, wo)
        pos, wn = pos.cpu().numpy(), w.cpu().numpy()
        for l in range(L):
            for g in range(Hkv):
                gone = weight_drops(wn[l, g], lp, r, m)
                keep = np.setdiff1d(np.arange(n), gone)
                assert np.array_equal(pos[l, g], keep), (s, l, g)
                at = torch.from_numpy(keep).to(DEV)
                assert torch.equal(ko[l, g], k[l, g, at]) and torch.equal(vo[l, g], v[l, g, at])
                assert np.array_equal(wo[l, g].cpu().numpy().view(np.int32),
                                      wn[l, g][keep].view(np.int32))
    c.close()


def _plain(shape):
    return torch.rand(shape) * 4


def _ties(shape):
    return torch.randint(0, 3, shape).float() / 2


def _odd(shape):
    """NaN, infinities, negative weights, zeros of both signs, the smallest numbers."""
    x = torch.tensor([float("nan"), float("inf"), -float("inf"), 0.0, -0.0, 1e-45, -1e-45, 3.0, -3.0,
                      1e38, 2.0 ** -126])
    return x[torch.randint(0, len(x), shape)]


@pytest.mark.parametrize("dtype", [B.RA_BF16, B.RA_E4M3, B.RA_F32])
@pytest.mark.parametrize("layout", [CHRON, PAGED])
@pytest.mark.parametrize("make", [_plain, _ties, _odd])
def test_the_least_weights_go(make, layout, dtype):
    torch.manual_seed(1)
    for lp, K, r, extra in ((0, 0, 0, 5), (1, 1, 1, 1), (7, 50, 3, 64), (33, 1000, 64, 24),
                            (33, 1000, 64, 25), (64, 0, 40, 960), (5, 30, 0, -3)):
        _event(dtype, layout, 2, 3, lp, K, r, extra, make)


@pytest.mark.parametrize("K", [2000, 2900, 4900, 9000, 16000, 30000])
def test_every_selection_build(K):
    torch.manual_seed(K)
    for layout in (CHRON, PAGED):
        _event(B.RA_BF16, layout, 1, 2, 3, K, 70, 60, _plain if K % 2000 else _ties, page_rows=64)


@pytest.mark.parametrize("dtype", [B.RA_BF16, B.RA_E4M3, B.RA_F32])
def test_moves_in_chunks_and_by_head(dtype):
    """Few long heads (a workgroup to a chunk of rows) and many (one to a head); more recent
    rows than threads."""
    torch.manual_seed(2)
    for layout in (CHRON, PAGED):
        # (K + r a multiple of the period: the explicit event is the first)
        _event(dtype, layout, 2, 4, 100, 2944, 64, 63, _plain, every=64)
        _event(dtype, layout, 36, 8, 10, 620, 20, 33, _plain, every=64)
        _event(dtype, layout, 1, 2, 10, 332, 2100, 40, _plain, every=64)


def test_events_of_many_slots():
    """More due slots than an event lists, and a batch's event at the end of a step."""
    sim = Sim(1, 2, 1, 6, [(5 * i) % 40 for i in range(40)], r=2, every=4)
    rule = sim.rule({})
    for t in range(17):
        sim.step(rule, {}, (t,))
    sim.check()
    sim.close()


@pytest.mark.parametrize("dtype", [B.RA_BF16, B.RA_E4M3, B.RA_F32])
@pytest.mark.parametrize("layout", [CHRON, PAGED])
def test_fast_forward_and_resume(layout, dtype):
    """A request preempted after events by weight resumes in another slot as it was: the same
    outputs, kept rows and weights as one that went on."""
    kw = dict(cap=10.0)
    sim = Sim(2, 4, 2, 24, [20, 9], r=8, every=8, dtype=dtype, layout=layout, max_seqs=3,
              extra_rows=2 * 2 * 96)
    rule = sim.rule(kw)
    for t in range(43):
        sim.step(rule, kw, (t,))
    saved = sim.export(0)
    info = B.ra_get_seq_info(sim.h, 0)
    B.ra_seq_end(sim.h, 0)
    B.ra_seq_begin(sim.h, 2, 20, 5, 0)
    B.ra_seq_fast_forward(sim.h, 2, info.step)
    after = B.ra_get_seq_info(sim.h, 2)
    assert (after.len, after.step, after.event) == (info.len, info.step, info.event)
    B.ra_write_positions(sim.h, 2, saved[0])
    B.ra_write_rows(sim.h, 2, saved[1], saved[2])
    B.ra_write_weights(sim.h, 2, saved[3])
    sim.seq[2] = sim.seq.pop(0)
    sim.check()
    for t in range(20):
        sim.step(rule, kw, (t,))
    sim.check()
    sim.close()


def test_fast_forward_rows_weigh_nothing():
    """Rows of a fast forward start at 0, and its events drop the earliest among them."""
    cfg = B.make_config(1, 2, 2, 8, 4, 8, max_seqs=2)
    c = B.Cache(cfg, B.ra_required_slots(cfg, [3, 5]))
    c.attach_weights(5)
    c.weights.fill_(float("nan"))
    for s, lp in enumerate((3, 5)):
        B.ra_seq_begin(c.handle, s, lp, 1, s)
    B.ra_fast_forward(c.handle, 21)
    for s, lp in enumerate((3, 5)):
        n = B.ra_get_seq_info(c.handle, s).len
        w = torch.full((2, n), 7.0, device=DEV)
        B.ra_export_weights(c.handle, s, w)
        assert (w == 0).all()
        for g in range(2):
            got = B.ra_read_positions(c.handle, s, 0, g, 100)
            assert np.array_equal(got, np.r_[np.arange(lp), np.arange(lp + 21 - (n - lp), lp + 21)])
    c.close()


def test_states_and_refusals():
    cfg = B.make_config(1, 2, 2, 8, 4, 8, max_seqs=2)
    c = B.Cache(cfg, B.ra_required_slots(cfg, [3, 5]))
    h, S = c.handle, B.RA_ERR_STATE
    bf = dict(dtype=torch.bfloat16, device=DEV)
    q, k, out = torch.zeros(2, 2, 128, **bf), torch.zeros(2, 2, 128, **bf), torch.zeros(2, 2, 128, **bf)
    rule = B.make_score_rule()
    w = torch.zeros(2, 100, device=DEV)
    B.ra_seq_begin(h, 0, 3, 1, 0)
    # no weights attached; not while a request is active
    assert status(B.ra_write_weights, h, 0, w) == S
    assert status(B.ra_export_weights, h, 0, w) == S
    assert status(B.ra_write_positions, h, 0, w.int()) == S
    assert status(c.attach_weights, 5) == S
    B.ra_seq_end(h, 0)
    c.attach_weights(5)
    B.ra_seq_begin(h, 0, 3, 1, 0)
    assert status(B.ra_weights_attach, h, None) == S
    # the other attention calls and rounds
    assert status(c.decode, 0, q, k, k, out) == S
    assert status(c.decode_noalloc, 0, q, k, k, out) == S
    c.attach_sparse(4)
    assert status(c.decode_sparse, 0, 4, 4, q, k, k, out) == S
    # arguments
    A = B.RA_ERR_INVALID_ARG
    assert status(B.ra_export_weights, h, 0, w[:1, :5]) == B.RA_ERR_CAPACITY
    assert status(B.ra_write_weights, h, 0, w[:1, :5]) == A
    assert status(B.ra_write_weights, h, 2, w) == A
    assert status(B.ra_write_weights, h, 1, w) == S           # inactive
    for kw in (dict(scale=-1.0), dict(scale=float("nan")), dict(cap=-1.0), dict(cap=float("inf")),
               dict(scale=1e-20), dict(cap=1e20), dict(cap=float("nan")),
               dict(window=-1), dict(prefix=-1)):
        assert status(c.decode_biased, 0, B.make_score_rule(**kw), q, k, k, out) == A, kw
    short = B.make_score_rule(slopes=torch.zeros(1, device=DEV))
    assert status(c.decode_biased, 0, short, q, k, k, out) == A
    assert status(c.decode_biased, 1, rule, q, k, k, out) == A
    assert status(B.ra_biased_attention, h, 0, rule, q, k, k, out, c.workspace) == A   # too small
    c.decode_biased(0, rule, q, k, k, out)
    assert status(c.decode_biased, 0, rule, q, k, k, out) == S   # appended already
    assert status(B.ra_export_weights, h, 0, w) == S             # open step
    assert status(B.ra_write_positions, h, 0, w.int()) == S
    B.ra_end_step(h)
    B.ra_export_weights(h, 0, w)
    B.ra_seq_end(h, 0)
    B.ra_weights_attach(h, None)
    c.weights = None
    B.ra_seq_begin(h, 1, 5, 1, 0)
    c.decode(0, q, k, k, out)
    B.ra_end_step(h)
    assert np.isfinite(_f64(out[1])).all()
    c.close()
    hole = B.make_config(1, 2, 2, 8, 4, 8, layout=B.RA_LAYOUT_HOLE_FILL)
    c = B.Cache(hole, B.ra_seq_rows(hole, 3))
    assert status(c.attach_weights, 3) == B.RA_ERR_UNSUPPORTED
    assert B._lib().ra_weights_attach(c.handle, None, 0) == B.RA_ERR_UNSUPPORTED
    c.close()


def test_external_rounds_are_refused():
    cfg = B.make_config(1, 4, 2, 32, 8, 64, policy=B.RA_POLICY_EXTERNAL)
    c = B.Cache(cfg, B.ra_seq_rows(cfg, 10))
    c.attach_weights(10)
    B.ra_seq_begin(c.handle, 0, 10, 1, 0)
    B.ra_fast_forward(c.handle, 70)
    win = torch.zeros(1, 1, 4, 64, 128, dtype=torch.bfloat16, device=DEV)
    scratch = torch.empty(B.ra_scored_scratch_bytes(cfg, 10), dtype=torch.uint8, device=DEV)
    assert status(B.ra_scored_evict, c.handle, 0, 1, B.make_scorer(B.RA_SCORER_SNAPKV), win,
                  scratch) == B.RA_ERR_STATE
    w = torch.rand(1, 2, 80, device=DEV)
    B.ra_write_weights(c.handle, 0, w)
    B.ra_evict_now(c.handle, 0)
    for g in range(2):
        gone = weight_drops(w[0, g].cpu().numpy(), 10, 8, 30)
        assert np.array_equal(B.ra_read_positions(c.handle, 0, 0, g, 100),
                              np.setdiff1d(np.arange(80), gone))
    c.close()
