"""Decode attention under score rules, and the accumulated weights, against float64."""

import numpy as np
import pytest
import torch

from biased_harness import Sim, slopes
from blocks_harness import status
from gpu_harness import DEV, _f64
from oracle.rule import rule_attention
from paper_2609_03430_amd import binding as B

pytestmark = pytest.mark.gpu
CHRON, HOLE, PAGED = (B.RA_LAYOUT_CHRONOLOGICAL, B.RA_LAYOUT_HOLE_FILL, B.RA_LAYOUT_PAGED)
DTYPES = [B.RA_BF16, B.RA_E4M3, B.RA_F32]

RULES = {
    "zero": dict(),
    "scale-cap": dict(scale=0.2, cap=3.0),
    "slopes": dict(slopes=True),
    "window": dict(window=21, prefix=5),
    "all": dict(cap=5.0, slopes=True, window=40, prefix=33),
}


def _kw(name, Hq):
    kw = dict(RULES[name])
    if kw.get("slopes"):
        kw["slopes"] = slopes(Hq)
    return kw


@pytest.mark.parametrize("name", list(RULES))
@pytest.mark.parametrize("layout", [CHRON, PAGED])
@pytest.mark.parametrize("dtype", DTYPES)
def test_steps_weights_and_events(dtype, layout, name):
    """Ragged slots (one empty, one inactive) through three events by weight."""
    sim = Sim(2, 6, 2, 24, [0, 1, 37, 130], r=9, every=16, dtype=dtype, layout=layout, max_seqs=5)
    kw = _kw(name, 6)
    rule = sim.rule(kw)
    for t in range(70):
        sim.step(rule, kw, (t,))
        if t in (0, 31, 32, 47):
            sim.check((t,))
    sim.check()
    sim.close()


@pytest.mark.parametrize("dtype,layout", [
    (d, l) for d in DTYPES for l in (CHRON, HOLE, PAGED) if (d, l) != (B.RA_E4M3, HOLE)])
def test_steps_without_weights(dtype, layout):
    """The policy's events (deferred ones among them) and mixed rules and layers."""
    sim = Sim(1, 8, 2, 20, [3, 50], r=8, every=8, dtype=dtype, layout=layout, weights=False)
    if layout == HOLE:
        # rows in no order: the model's positions are read back, rows are not compared
        sim.event = lambda s, m: _reorder(sim, s, m)
    rules = [(kw, sim.rule(kw)) for kw in (_kw(n, 8) for n in ("all", "zero", "window", "slopes"))]
    for t in range(40):
        kw, rule = rules[t % 4]
        sim.step(rule, kw, (t,))
    if layout != HOLE:
        sim.check()
    sim.close()


def _reorder(sim, s, m):
    lp = sim.seq[s]["lp"]
    n = len(sim.seq[s]["heads"][0, 0]["P"]) - m
    pos, _, _, _ = sim.export(s)
    for (l, g), h in sim.seq[s]["heads"].items():
        got = pos[l, g].cpu().numpy()
        assert len(got) == n and (got[:lp] == np.arange(lp)).all()
        at = {int(p): i for i, p in enumerate(h["P"])}
        keep = np.array([at[int(p)] for p in got])
        for x in ("P", "K", "V", "W", "E"):
            h[x] = h[x][keep]


@pytest.mark.parametrize("dtype,G", [(B.RA_BF16, 1), (B.RA_BF16, 5), (B.RA_E4M3, 16), (B.RA_F32, 8)])
def test_long_heads_in_splits(dtype, G):
    """Heads of thousands of rows, in splits, among short ones; a window across pages."""
    for name, layout in (("all", PAGED), ("scale-cap", CHRON), ("window", PAGED)):
        sim = Sim(1, 2 * G, 2, 0, [4321, 1, 64], r=0, every=64, dtype=dtype, layout=layout)
        kw = _kw(name, 2 * G)
        if kw.get("window"):
            kw.update(window=2777, prefix=600)
        rule = sim.rule(kw)
        for t in range(2):
            sim.step(rule, kw, (t, name))
        sim.check((name,))
        sim.close()


@pytest.mark.parametrize("dtype,layout", [(B.RA_BF16, CHRON), (B.RA_E4M3, PAGED), (B.RA_F32, PAGED)])
def test_weights_of_many_whole_heads(dtype, layout):
    """132 heads, a workgroup each, whose scores stay in LDS and take two rounds of rows; ragged
    ones; a window's two runs of blocks."""
    for lens, kw in (([1300] * 33, {}), ([1 + 37 * i for i in range(33)], dict(window=700, prefix=40)),
                     ([1290 - i for i in range(33)], dict(window=1200, prefix=3, cap=9.0))):
        sim = Sim(1, 8, 4, 0, lens, r=0, every=64, dtype=dtype, layout=layout)
        rule = sim.rule(kw)
        for t in range(2):
            sim.step(rule, kw, (t,))
        sim.check()
        sim.close()


@pytest.mark.parametrize("dtype,layout", [(B.RA_BF16, PAGED), (B.RA_E4M3, CHRON), (B.RA_F32, CHRON)])
def test_weights_of_whole_heads_longer_than_lds(dtype, layout):
    """Scores of G = 16 and 2,000 rows (LDS holds 1,792), part of them in LDS and part in the
    workspace; shorter heads of the same launch, all of whose are in LDS."""
    lens = [2000] + [1999] * 4 + [1700, 1, 40, 1900] * 2
    # (attn_split keeps the few heads whole)
    sim = Sim(1, 16, 1, 0, lens, r=0, every=64, dtype=dtype, layout=layout, attn_split=4096)
    kw = dict(cap=9.0, window=1800, prefix=100)
    rule = sim.rule(kw)
    for t in range(2):
        sim.step(rule, kw, (t,))
    sim.check()
    sim.close()


@pytest.mark.parametrize("dtype", DTYPES)
def test_one_head_of_more_rows_than_its_splits_hold_at_512(dtype):
    """One head of 33,000 rows (65 splits of 512) and a short one beside it."""
    for n in ([33000], [33000, 100]):
        sim = Sim(1, 2, 1, 0, n, r=0, every=64, dtype=dtype)
        kw = dict(cap=30.0)
        sim.step(sim.rule(kw), kw)
        sim.check()
        sim.close()


@pytest.mark.parametrize("window,prefix", [(1, 0), (1, 40), (32, 0), (33, 32), (2 ** 31 - 1, 0),
                                           (97, 2 ** 31 - 1), (64, 1)])
def test_window_edges(window, prefix):
    for dtype in DTYPES:
        sim = Sim(1, 2, 1, 0, [0, 31, 32, 33, 95, 96, 97, 200], r=0, every=8, dtype=dtype)
        kw = dict(window=window, prefix=prefix)
        rule = sim.rule(kw)
        for t in range(3):
            sim.step(rule, kw, (t, dtype))
        sim.check()
        sim.close()


@pytest.mark.parametrize("dtype", DTYPES)
def test_hidden_rows_have_no_part(dtype):
    """Infinities and NaN in keys and values of rows that the window hides."""
    n, window = 150, 40
    t = torch.float32 if dtype == B.RA_F32 else torch.bfloat16
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(1, 2, n, 128, generator=g).to(t) for _ in range(2))
    for j, x in ((2, np.inf), (60, -np.inf), (100, np.nan), (110, np.inf)):   # 110: just hidden
        v[:, :, j, ::3] = x
        k[:, 1, j, 1::3] = x
    cfg = B.make_config(1, 4, 2, 16, 0, 16, dtype=dtype)
    c = B.Cache(cfg, B.ra_seq_rows(cfg, n))
    c.attach_weights(n)
    B.ra_seq_begin(c.handle, 0, n, 1, 0, k.to(DEV), v.to(DEV))
    q, kn, vn = (torch.randn(1, h, 128, generator=g).to(t) for h in (4, 2, 2))
    out = torch.empty(1, 4, 128, dtype=t, device=DEV)
    w = torch.empty(1, 2, n + 1, device=DEV)
    c.decode_biased(0, B.make_score_rule(window=window), q.to(DEV), kn.to(DEV), vn.to(DEV), out)
    B.ra_end_step(c.handle)
    B.ra_export_weights(c.handle, 0, w)
    out, w = _f64(out), _f64(w)
    assert (w[0, :, :n + 1 - window] == 0).all() and (w[0, :, n + 1 - window:] > 0).all()
    for h in range(4):
        assert np.isfinite(out[0, h]).all()
        if dtype != B.RA_E4M3:
            K = np.vstack([_f64(k[0, h // 2]), _f64(kn[0, h // 2])[None]])
            V = np.vstack([_f64(v[0, h // 2]), _f64(vn[0, h // 2])[None]])
            want, _ = rule_attention(_f64(q[0, h]), K, V, np.arange(n + 1), n, window=window)
            # half a bf16 step and 1e-4 of split weights and fp32 sums
            assert (np.abs(out[0, h] - want) <= 2.0 ** -8 * np.abs(want) + 1e-4).all()
    c.close()


def test_capped_infinite_scores():
    """With a cap an infinite score is one of the cap; without one a row of -inf weighs nothing."""
    cfg = B.make_config(1, 1, 1, 16, 0, 16)
    k = torch.ones(1, 1, 40, 128).to(torch.bfloat16)
    v = torch.arange(40.0).view(1, 1, 40, 1).expand(1, 1, 40, 128).to(torch.bfloat16).contiguous()
    k[0, 0, 7, 0] = float("-inf")
    for cap, want in ((2.0, None), (0.0, None)):
        c = B.Cache(cfg, B.ra_seq_rows(cfg, 40))
        B.ra_seq_begin(c.handle, 0, 40, 1, 0, k.to(DEV), v.to(DEV))
        q = torch.full((1, 1, 128), 0.01, dtype=torch.bfloat16)
        new = torch.ones(1, 1, 128, dtype=torch.bfloat16)
        out = torch.empty(1, 1, 128, dtype=torch.bfloat16, device=DEV)
        c.decode_biased(0, B.make_score_rule(cap=cap), q.to(DEV), new.to(DEV), new.to(DEV), out)
        s = np.full(41, 128 * float(q[0, 0, 0]) * 128 ** -0.5)
        s[7] = -np.inf
        if cap:
            s = cap * np.tanh(s / cap)
        p = np.exp(s - s.max())
        want = p @ np.append(np.arange(40.0), 1.0) / p.sum()
        assert np.abs(_f64(out) - want).max() <= 2.0 ** -8 * want + 1e-4
        B.ra_end_step(c.handle)
        c.close()


def test_a_rule_of_zeros_and_mixed_layers():
    """Layers of a step through either call; a rule of zeros gives the plain call's result."""
    for dtype in DTYPES:
        sims = [Sim(2, 4, 2, 12, [70, 5], r=4, every=8, dtype=dtype, weights=False, seed=9)
                for _ in range(2)]
        rule = B.make_score_rule()
        t = sims[0].tdtype
        for step in range(30):
            outs = []
            for j, sim in enumerate(sims):
                for l in range(2):
                    q, k, v = (x.to(DEV) for x in sim.inputs())
                    out = torch.empty(2, 4, 128, dtype=t, device=DEV)
                    if (step + j * l) % 2:
                        sim.cache.decode(l, q, k, v, out)
                    else:
                        sim.cache.decode_biased(l, rule, q, k, v, out)
                    outs.append(_f64(out))
                B.ra_end_step(sim.h)
            # the same attention of at most 100 rows: each within half a step and 1e-4 (fp32
            # 1e-5) of it
            half, floor = (2.0 ** -24, 1e-5) if dtype == B.RA_F32 else (2.0 ** -8, 1e-4)
            for l in range(2):
                a, b = outs[l], outs[2 + l]
                assert (np.abs(a - b) <= 2 * half * np.abs(a) + 3 * floor).all(), (dtype, step)
        for sim in sims:
            for s in range(2):
                pos, k, v, _ = sim.export(s)
                other = sims[0].export(s)
                assert torch.equal(pos, other[0])
                assert torch.equal(k, other[1]) and torch.equal(v, other[2])
        for sim in sims:
            sim.close()


@pytest.mark.parametrize("order", ["plain first", "biased first", "alternate"])
def test_layers_either_way_after_a_deferred_event(order):
    """An event whose row moves are deferred, then a step of which some layers carry their moves
    and others do not: every layer's rows move once."""
    # (a head to a work item: such events defer their moves)
    sim = Sim(4, 4, 2, 40, [30, 12], r=8, every=16, weights=False, attn_split=4096)
    rule = B.make_score_rule()
    calls = dict(zip(("plain first", "biased first", "alternate"),
                     ([0, 0, 1, 1], [1, 1, 0, 0], [0, 1, 0, 1])))[order]
    deferred = 0
    for t in range(100):
        pending = B.ra_get_seq_info(sim.h, 0).move_pending
        deferred += pending
        for l in range(4):
            q, k, v = sim.inputs()
            out = torch.empty(2, 4, 128, dtype=torch.bfloat16, device=DEV)
            biased = pending and calls[l]
            call = (lambda *a: sim.cache.decode_biased(l, rule, *a)) if biased else \
                (lambda *a: sim.cache.decode(l, *a))
            call(q.to(DEV), k.to(DEV), v.to(DEV), out)
            for s in range(2):
                sim.follow(s, l, q, k, v, out, {}, (t, order))
        B.ra_end_step(sim.h)
        for s, seq in sim.seq.items():
            seq["step"] += 1
            m = len(seq["heads"][0, 0]["P"]) - seq["lp"] - sim.r - sim.K
            if seq["step"] % sim.every == 0 and m > 0:
                pos = torch.empty(4, 2, B.ra_get_seq_info(sim.h, s).len, dtype=torch.int32, device=DEV)
                B.ra_export_positions(sim.h, s, pos)      # (leaves the moves pending)
                for (l, g), h in seq["heads"].items():
                    keep = np.isin(h["P"], pos[l, g].cpu().numpy())
                    for x in ("P", "K", "V", "W", "E"):
                        h[x] = h[x][keep]
    assert deferred >= 3
    sim.check()
    sim.close()


def test_every_run_is_the_same():
    """Outputs and weights of two runs of the same steps, in splits, bit for bit."""
    got = []
    for _ in range(2):
        sim = Sim(1, 10, 2, 0, [9000, 700], r=0, every=64, seed=4)
        kw = dict(cap=20.0)
        rule = sim.rule(kw)
        ins = [x.to(DEV) for x in sim.inputs()]
        outs = []
        for _ in range(3):
            out = torch.empty(2, 10, 128, dtype=torch.bfloat16, device=DEV)
            sim.cache.decode_biased(0, rule, *ins, out)
            B.ra_end_step(sim.h)
            outs.append(out)
        got.append(outs + [sim.export(s)[3] for s in range(2)])
        sim.close()
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_rows_past_32_bits_of_elements():
    """A request of 17 million rows, and one whose rows lie behind them: offsets past 2^31
    elements of the pools, a window of the long one, its weights' sum."""
    long, n = 17_000_000, 300
    cfg = B.make_config(1, 2, 1, 8, 0, 8, max_seqs=2)
    c = B.Cache(cfg, B.ra_required_slots(cfg, [long, n]))
    c.attach_weights(long)
    g = torch.Generator().manual_seed(8)
    k, v = (torch.randn(1, 1, n, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    B.ra_seq_begin(c.handle, 0, long, 1, 0)              # (its rows are the pool's zeros)
    B.ra_seq_begin(c.handle, 1, n, 1, 1, k.to(DEV), v.to(DEV))
    assert B.ra_get_seq_info(c.handle, 1).base * 128 > 2 ** 31
    K, V, W = _f64(k[0, 0]), _f64(v[0, 0]), np.zeros(n + 2)
    for t, kw in enumerate((dict(), dict(window=100, prefix=7))):
        q, kn, vn = (torch.randn(2, h, 128, generator=g).to(torch.bfloat16) for h in (2, 1, 1))
        q[0], vn[0] = 0.0, 1.0                           # equal scores: 1 / rows in sight
        out = torch.empty(2, 2, 128, dtype=torch.bfloat16, device=DEV)
        c.decode_biased(0, B.make_score_rule(**kw), q.to(DEV), kn.to(DEV), vn.to(DEV), out)
        B.ra_end_step(c.handle)
        seen = 107 if kw else long + 1
        # one row (the first step's pair is in sight of the second, too) of value 1
        want = (2 if kw else 1) / seen
        assert np.abs(_f64(out[0]) - want).max() <= 2.0 ** -8 * want + 2.0 ** -14 * want
        K, V = np.vstack([K, _f64(kn[1])]), np.vstack([V, _f64(vn[1])])
        for h in range(2):
            want, p = rule_attention(_f64(q[1, h]), K, V, np.arange(len(K)), n + t, **kw)
            assert (np.abs(_f64(out[1, h]) - want) <= 2.0 ** -8 * np.abs(want) + 1e-4).all()
            W[:len(p)] += p
    w = torch.empty(1, 1, n + 2, device=DEV)
    B.ra_export_weights(c.handle, 1, w)
    # (scores of about 10 from 131 roundings each: 10^-4 of a weight of at most 1)
    assert np.abs(_f64(w[0, 0]) - W).max() <= 1e-4
    w = torch.empty(1, 1, long + 2, device=DEV)
    B.ra_export_weights(c.handle, 0, w)
    # each weight is 1 / (17 million + 1) and two of 1 / 107 in sight, to a few fp32 roundings
    w = w[0, 0].double()
    assert abs(float(w.sum()) - 4.0) <= 4 * 2.0 ** -18
    assert abs(float(w[5_000_000]) * (long + 1) / 2 - 1) <= 2.0 ** -18
    assert abs(float(w[3]) * 107 / 2 - 1) <= 2.0 ** -12
    c.close()


def test_more_slots_than_an_order_holds_and_other_streams():
    """300 ragged slots, steps on two streams in turn."""
    n = 300
    cfg = B.make_config(1, 2, 1, 16, 0, 16, max_seqs=n)
    lps = [1 + (37 * i) % 101 for i in range(n)]
    c = B.Cache(cfg, B.ra_required_slots(cfg, lps))
    c.attach_weights(max(lps))
    g = torch.Generator().manual_seed(2)
    rows = [torch.randn(2, 1, 1, lp, 128, generator=g).to(torch.bfloat16) for lp in lps]
    for i, x in enumerate(rows):
        B.ra_seq_begin(c.handle, i, lps[i], 1, i, *(y.to(DEV) for y in x))
    rule = B.make_score_rule(window=50, prefix=3)
    side = torch.cuda.Stream()
    steps = [[torch.randn(n, h, 128, generator=g).to(torch.bfloat16) for h in (2, 1, 1)]
             for _ in range(2)]
    outs = []
    for t, ins in enumerate(steps):
        dev = [x.to(DEV) for x in ins]
        out = torch.empty(n, 2, 128, dtype=torch.bfloat16, device=DEV)
        torch.cuda.synchronize()
        c.decode_biased(0, rule, *dev, out, stream=side if t else None)
        B.ra_end_step(c.handle, stream=side if t else None)
        torch.cuda.synchronize()
        outs.append(_f64(out))
    for i in (0, 7, 255, 256, 299):
        K, V = (_f64(x[0, 0]) for x in rows[i])
        for t, ins in enumerate(steps):
            K, V = np.vstack([K, _f64(ins[1][i])]), np.vstack([V, _f64(ins[2][i])])
            m = len(K)
            for h in range(2):
                want, _ = rule_attention(_f64(ins[0][i, h]), K, V, np.arange(m), m - 1, window=50,
                                         prefix=3)
                assert (np.abs(outs[t][i, h] - want) <= 2.0 ** -8 * np.abs(want) + 1e-4).all()
    c.close()


@pytest.mark.parametrize("lps,window", [([30, 3], 60), ([900, 90], 0)])
def test_captured_steps(lps, window):
    """Steps captured once and replayed through events, weights added at once or (heads in
    splits) after: outputs, kept sets and weights are an eager twin's."""
    kw = dict(cap=8.0, slopes=slopes(6), window=window, prefix=4)
    for dtype in DTYPES:
        sims = [Sim(2, 6, 2, 40, lps, r=8, every=8, dtype=dtype, seed=6) for _ in range(2)]
        rules = [sim.rule(kw) for sim in sims]
        ins = [[x.to(DEV) for x in sims[0].inputs()] for _ in range(2)]
        outs = [torch.empty(2, 2, 6, 128, dtype=sims[0].tdtype, device=DEV) for _ in range(2)]

        def step(j):
            for l in range(2):
                sims[j].cache.decode_biased(l, rules[j], *ins[l], outs[j][l])
            B.ra_end_step(sims[j].h)

        B.ra_graph_mode(sims[1].h, True)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            step(1)
            with torch.cuda.graph(graph, stream=side):
                step(1)
        torch.cuda.current_stream().wait_stream(side)
        step(0)
        for t in range(75):
            for l in range(2):
                for x in ins[l]:
                    x.copy_(torch.randn(x.shape, generator=sims[0].gen))
            step(0)
            graph.replay()
            torch.cuda.synchronize()
            # (the splits differ: a graph's plan is for the largest cache)
            a, b = _f64(outs[0]), _f64(outs[1])
            half, floor = (2.0 ** -24, 1e-5) if dtype == B.RA_F32 else (2.0 ** -8, 1e-4)
            assert (np.abs(a - b) <= 2 * half * np.abs(a) + 2 * floor).all(), t
        assert status(B.ra_export_weights, sims[1].h, 0, torch.empty(10000, device=DEV)) \
            == B.RA_ERR_STATE
        del graph
        B.ra_graph_mode(sims[1].h, False)
        for s in range(2):
            x, y = sims[0].export(s), sims[1].export(s)
            assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1]) and torch.equal(x[2], y[2])
            assert torch.allclose(x[3], y[3], rtol=1e-4, atol=1e-6)
        for sim in sims:
            sim.close()
