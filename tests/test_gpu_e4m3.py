"""The 8-bit cache on the GPU: rows held exactly as the oracle holds them, through
writes, reads, events and resumes, and attention over the values they stand for."""

import numpy as np
import pytest
import torch

from blocks_harness import Run8, OracleSeq8, check_step, fill_stale, held, status
from gpu_harness import DEV, attn_err, check_heads, log
from oracle.attention import gqa_decode
from paper_2609_03430_amd import binding as B

pytestmark = pytest.mark.gpu
CHRON, PAGED = B.RA_LAYOUT_CHRONOLOGICAL, B.RA_LAYOUT_PAGED


def _cache(L, Hq, Hkv, lens, layout=CHRON, page_rows=32, budget=0, r=0, every=1, **kw):
    cfg = B.make_config(L, Hq, Hkv, budget, r, every, dtype=B.RA_E4M3, max_seqs=len(lens),
                        layout=layout, page_rows=page_rows, max_prompt_len=max(lens), **kw)
    cache = B.Cache(cfg, B.ra_required_slots(cfg, lens))
    fill_stale(cache)
    return cache


def _rows(seed, *shape):
    """Rows of mixed magnitude: ordinary ones, and every kind of edge."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(*shape, 128, generator=g)
    x = x * torch.pow(2.0, torch.randint(-30, 30, shape + (1,), generator=g).float())
    x = x.to(torch.bfloat16)
    flat = x.view(-1, 128)
    top = torch.finfo(torch.bfloat16).max
    edges = [
        torch.zeros(128), torch.full((128,), top), torch.full((128,), -2.0 ** -133),
        torch.linspace(-1.75, 1.75, 128), torch.linspace(-1.7578125, 1.7578125, 128),
        # every tie between neighbouring codes of a row whose scale is 1
        torch.cat([torch.tensor([448.0]), torch.arange(127) * 2.0 ** -10]),
        torch.cat([torch.tensor([256.0]), 17.0 + 2 * torch.arange(127)]),
        torch.randn(128, generator=g) * 2.0 ** -120, torch.linspace(2.0 ** -132, 2.0 ** -126, 128),
        torch.cat([torch.tensor([top, -top * 0.75]), torch.randn(126, generator=g)]),
    ]
    for i, e in enumerate(edges):
        if 3 * i + 1 < len(flat):
            flat[3 * i + 1] = e.to(torch.bfloat16)
    return x


def _same(a, b):
    a, b = a.float().cpu(), b.float().cpu()
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(
        torch.nan_to_num(a), torch.nan_to_num(b))


@pytest.mark.parametrize("layout,page_rows", [(CHRON, 32), (PAGED, 32), (PAGED, 128)])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 31, 32, 33, 127, 128, 129, 300])
def test_rows_are_held_as_the_oracle_holds_them(n, layout, page_rows):
    L, Hkv = 2, 3
    c = _cache(L, 6, Hkv, [n, 45], layout, page_rows)
    k, v = _rows(n, L, Hkv, n).to(DEV), _rows(n + 1, L, Hkv, n).to(DEV)
    other = [_rows(s, L, Hkv, 45).to(DEV) for s in (901, 902)]
    B.ra_seq_begin(c.handle, 1, 45, 5, 6, *other)
    B.ra_seq_begin(c.handle, 0, n, 1, 2, k, v)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    B.ra_export_rows(c.handle, 0, ko, vo)
    wk, wv = held(k), held(v)
    assert _same(ko, wk) and _same(vo, wv)
    # one head at a time, and either output alone
    kh, vh = torch.empty(n, 128, dtype=torch.bfloat16, device=DEV), torch.empty(
        n, 128, dtype=torch.bfloat16, device=DEV)
    B.ra_read_rows(c.handle, 0, 1, 2, kh, None)
    B.ra_read_rows(c.handle, 0, 1, 2, None, vh)
    assert _same(kh, wk[1, 2]) and _same(vh, wv[1, 2])
    # what was read is held as it is
    B.ra_write_rows(c.handle, 0, ko, vo)
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    B.ra_export_rows(c.handle, 0, k2)
    B.ra_export_rows(c.handle, 0, None, v2)
    assert _same(k2, wk) and _same(v2, wv)
    # the other sequence's rows are as they were
    got = [torch.empty_like(x) for x in other]
    B.ra_export_rows(c.handle, 1, *got)
    assert _same(got[0], held(other[0])) and _same(got[1], held(other[1]))
    c.close()


def test_values_that_are_not_finite():
    n = 40
    c = _cache(1, 2, 1, [n])
    x = _rows(3, 1, 1, n)
    x[0, 0, 3, 7] = float("inf")
    x[0, 0, 4, :] = float("-inf")
    x[0, 0, 5, 100] = float("nan")
    x[0, 0, 6, :] = float("nan")
    x = x.to(DEV)
    B.ra_seq_begin(c.handle, 0, n, 1, 2, x, x)
    k, v = torch.empty_like(x), torch.empty_like(x)
    B.ra_export_rows(c.handle, 0, k, v)
    assert _same(k, held(x)) and _same(v, held(x))
    c.close()


@pytest.mark.parametrize("dtype", [B.RA_F32, B.RA_BF16])
@pytest.mark.parametrize("layout", [CHRON, B.RA_LAYOUT_HOLE_FILL, PAGED])
def test_export_rows_of_the_other_caches(dtype, layout):
    tdtype = torch.bfloat16 if dtype == B.RA_BF16 else torch.float32
    cfg = B.make_config(3, 4, 2, 0, 0, 1, dtype=dtype, max_seqs=1, layout=layout, page_rows=32,
                        max_prompt_len=77)
    c = B.Cache(cfg, B.ra_required_slots(cfg, [77]))
    k, v = (torch.randn(3, 2, 77, 128, device=DEV).to(tdtype) for _ in range(2))
    B.ra_seq_begin(c.handle, 0, 77, 1, 2, k, v)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    B.ra_export_rows(c.handle, 0, ko, vo)
    assert torch.equal(k, ko) and torch.equal(v, vo)
    short = torch.empty(k.numel() - 1, dtype=tdtype, device=DEV)
    assert status(B.ra_export_rows, c.handle, 0, short, None) == B.RA_ERR_CAPACITY
    c.close()


# lengths about the block, the work items and the splits; groups of every padding
@pytest.mark.parametrize("layout", [CHRON, PAGED])
@pytest.mark.parametrize("lens,Hq,Hkv", [
    ([0, 1, 31], 4, 2), ([32, 33, 63, 64, 65], 5, 1), ([127, 128, 129, 96], 8, 1),
    ([255, 256, 257], 16, 1), ([511, 512, 1023, 1024, 1025], 6, 3), ([2047, 5000], 10, 2),
    ([9001], 2, 2), ([700, 3, 20000], 8, 8),
])
def test_attention_over_every_length(lens, Hq, Hkv, layout):
    c = _cache(1, Hq, Hkv, lens, layout, 64)
    g = torch.Generator().manual_seed(sum(lens))
    rows = []
    for i, n in enumerate(lens):
        k, v = (torch.randn(1, Hkv, n, 128, generator=g).mul(1.5).to(torch.bfloat16)
                for _ in range(2))
        rows.append((held(k)[0], held(v)[0]) if n else (k[0], v[0]))
        B.ra_seq_begin(c.handle, i, n, 1, i, k.to(DEV) if n else None, v.to(DEV) if n else None)
    for noalloc in (False, True):
        q = torch.randn(len(lens), Hq, 128, generator=g).to(torch.bfloat16)
        k, v = (torch.randn(len(lens), Hkv, 128, generator=g).to(torch.bfloat16) for _ in range(2))
        out = torch.empty_like(q, device=DEV)
        (c.decode_noalloc if noalloc else c.decode)(0, q.to(DEV), k.to(DEV), v.to(DEV), out)
        hk, hv = held(k), held(v)
        for i, n in enumerate(lens):
            want = gqa_decode(q[i].double().numpy(),
                              [torch.cat([rows[i][0][h], hk[i, h][None]]).double().numpy()
                               for h in range(Hkv)],
                              [torch.cat([rows[i][1][h], hv[i, h][None]]).double().numpy()
                               for h in range(Hkv)])
            attn_err(out[i], want, B.RA_BF16, (lens, i, noalloc))
        B.ra_end_step(c.handle)          # drops the new row again (K = 0, r = 0)
    c.close()


@pytest.mark.parametrize("kw", [
    dict(L=2, Hq=8, Hkv=2, K=48, lps=[12, 5, 0, 33], r=16, every=16),
    dict(L=1, Hq=10, Hkv=2, K=70, lps=[9, 100], r=8, every=24, layout=PAGED, page_rows=32),
    dict(L=2, Hq=4, Hkv=4, K=33, lps=[3], r=0, every=1),
    dict(L=1, Hq=6, Hkv=2, K=20, lps=[17, 40], r=33, every=7, policy=B.RA_POLICY_RECENCY),
    dict(L=2, Hq=4, Hkv=2, K=50, lps=[30, 20], r=10, every=10, policy=B.RA_POLICY_BLOCK, block=4,
         layout=PAGED, page_rows=64),
    dict(L=1, Hq=4, Hkv=1, K=64, lps=[40, 40], r=16, every=16, mode=B.RA_BUDGET_TOTAL),
])
def test_decoding_with_events(kw):
    """Outputs of every step, and after every event the kept positions, keys and
    values, whose scales move with them."""
    log("8-bit decoding %s" % (kw,))
    run = Run8(**kw)
    oracles = [OracleSeq8(run, s) for s in range(run.n)]
    events = 0
    for t in range(3 * max(run.every, 24) + kw["K"]):
        outs, evicted = run.step(noalloc=t % 3 == 2)
        check_step(run, oracles, outs, (t,))
        events += evicted
        if evicted:
            check_heads(run, oracles)
    assert events >= 2 * run.n
    check_heads(run, oracles)
    run.close()


@pytest.mark.parametrize("layout", [CHRON, PAGED])
@pytest.mark.parametrize("n,Hkv,K,every", [
    (1, 2, 2100, 300),     # few heads: several workgroups share a head's rows
    (1, 1, 40, 1000),      # more drops than rows kept
    (40, 2, 600, 64),      # more sequences than an event lists
])
def test_long_moves(n, Hkv, K, every, layout):
    run = Run8(L=1, Hq=2 * Hkv, Hkv=Hkv, K=K, lps=[13] * n, r=20, every=every, layout=layout,
               page_rows=32)
    steps = ((K + 20) // every + 1) * every - 1
    run.fast_forward(steps)
    for s in range(n):
        run.materialise(s)
    oracles = [OracleSeq8(run, s) for s in range(min(n, 3))]
    for o in oracles:
        o.advance(steps)
    check_heads(run, oracles)
    outs, evicted = run.step()
    assert evicted == n
    check_step(run, oracles, outs)
    check_heads(run, oracles)
    outs, _ = run.step()
    check_step(run, oracles, outs)
    B.ra_evict_now(run.h, 0)             # the new row puts the head over its budget
    oracles[0].rep.evict_now()
    check_heads(run, oracles[:1])
    run.close()


def test_preempted_request_resumes_exactly():
    """Rows exported, the slot ended, another one begun, forwarded and given the rows:
    the same values, so the same outputs to the bit."""
    kw = dict(L=2, Hq=8, Hkv=2, K=60, lps=[21, 21], r=12, every=12, max_seqs=3)
    a, b = Run8(**kw), Run8(**kw)
    for _ in range(100):
        a.step()
        b.step()
    n = B.ra_get_seq_info(b.h, 0).len
    k, v = (torch.empty(2, 2, n, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    B.ra_export_rows(b.h, 0, k, v)
    B.ra_seq_end(b.h, 0)
    B.ra_seq_begin(b.h, 0, 21, b.seeds[0], b.rids[0])
    B.ra_seq_fast_forward(b.h, 0, 100)
    B.ra_write_rows(b.h, 0, k, v)
    for _ in range(30):
        oa, ob = a.step()[0], b.step()[0]
        assert torch.equal(oa[:, :2], ob[:, :2])
    a.close()
    b.close()


def test_captured_steps():
    """A captured step replays as the eager one, events included."""
    kw = dict(L=2, Hq=8, Hkv=2, K=40, lps=[5, 0, 17], r=8, every=8)
    eager, graph = Run8(**kw), Run8(**kw)
    oracles = [OracleSeq8(graph, s) for s in range(graph.n)]
    for run in (eager, graph):
        B.ra_graph_mode(run.h, 1)
    shape = (graph.L, graph.max_seqs)
    bufs = {}
    for run in (eager, graph):
        q = torch.zeros(*shape, run.Hq, 128, dtype=torch.bfloat16, device=DEV)
        k = torch.zeros(*shape, run.Hkv, 128, dtype=torch.bfloat16, device=DEV)
        bufs[run] = (q, k, torch.zeros_like(k), torch.zeros_like(q))

    def load(run):
        for layer in range(run.L):
            for dst, src in zip(bufs[run], run.step_inputs(layer)):
                dst[layer].copy_(src)

    def issue(run):
        q, k, v, out = bufs[run]
        for layer in range(run.L):
            run.cache.decode(layer, q[layer], k[layer], v[layer], out[layer])
        B.ra_end_step(run.h)

    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        issue(graph)
    for t in range(70):
        for run in (eager, graph):
            load(run)
        issue(eager)
        g.replay()
        torch.cuda.synchronize()
        for run in (eager, graph):
            run.steps = [s + 1 for s in run.steps]
        assert torch.equal(bufs[eager][3], bufs[graph][3]), t
        check_step(graph, oracles, bufs[graph][3], (t,))
    B.ra_graph_mode(graph.h, 0)
    check_heads(graph, oracles)
    outs, _ = graph.step()
    check_step(graph, oracles, outs)
    eager.close()
    graph.close()


def test_the_new_pair_is_attended_as_it_is_held():
    """An empty cache: the output is the new value as the row stands for it."""
    c = _cache(1, 4, 2, [0, 0])
    for i in range(2):
        B.ra_seq_begin(c.handle, i, 0, 1, i)
    q, k = torch.randn(2, 4, 128).to(torch.bfloat16), _rows(4, 2, 2)
    v = _rows(5, 2, 2)
    v[1, 1] = torch.linspace(-1.7578125, 1.7578125, 128).to(torch.bfloat16)
    out = torch.empty(2, 4, 128, dtype=torch.bfloat16, device=DEV)
    c.decode(0, q.to(DEV), k.to(DEV), v.to(DEV), out)
    assert torch.equal(out.cpu(), held(v).repeat_interleave(2, 1))
    c.close()


def test_on_another_stream():
    """Every call on a stream that is not the current one."""
    run = Run8(L=1, Hq=8, Hkv=2, K=30, lps=[20, 40], r=8, every=8)
    oracles = [OracleSeq8(run, s) for s in range(run.n)]
    side = torch.cuda.Stream()
    for t in range(60):
        q, k, v = run.step_inputs(0)
        out = torch.empty_like(q)
        side.wait_stream(torch.cuda.current_stream())
        run.cache.decode(0, q, k, v, out, stream=side)
        B.ra_end_step(run.h, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        run.steps = [s + 1 for s in run.steps]
        check_step(run, oracles, out[None], (t,))
    n = B.ra_get_seq_info(run.h, 0).len
    k = torch.empty(1, 2, n, 128, dtype=torch.bfloat16, device=DEV)
    B.ra_export_rows(run.h, 0, k, None, stream=side)
    side.synchronize()
    for g in range(2):
        assert torch.equal(k[0, g].cpu(), oracles[0].rows(0, g, oracles[0].rep.P[(0, g)])[0])
    run.close()


def test_random_configurations():
    rng = np.random.default_rng(77)
    for trial in range(8):
        Hkv = int(rng.integers(1, 4))
        kw = dict(L=int(rng.integers(1, 3)), Hq=Hkv * int(rng.integers(1, 17)), Hkv=Hkv,
                  K=int(rng.integers(0, 150)), lps=[int(x) for x in rng.integers(0, 200, 3)],
                  r=int(rng.integers(0, 70)), every=int(rng.integers(1, 50)),
                  layout=int(rng.choice([CHRON, PAGED])), page_rows=int(rng.choice([32, 64])),
                  attn_split=int(rng.choice([0, 32, 96, 256])))
        log("8-bit trial %d: %s" % (trial, kw))
        run = Run8(**kw)
        oracles = [OracleSeq8(run, s) for s in range(run.n)]
        skip = int(rng.integers(0, 200))
        run.fast_forward(skip)
        for s in range(run.n):
            run.materialise(s)
        for o in oracles:
            o.advance(skip)
        for t in range(int(rng.integers(5, 60))):
            outs, _ = run.step()
            check_step(run, oracles, outs, (trial, t))
        check_heads(run, oracles)
        run.close()


@pytest.mark.parametrize("ratio", [1, 2.0 ** 10, 2.0 ** 14])
def test_a_channel_that_dwarfs_the_query(ratio):
    """One channel of the query, 4 * `ratio`, dwarfs the others, of size 1, and no key has
    it: the scores come from the others alone.  The query's parts hold every channel to
    2^-26 of the largest, so a score is off by at most 127 * 2 * 2^-26 * 4 ratio /
    sqrt(128) (|k| <= 2), a weight by e to the power of twice that, an output (|v| <= 2)
    by 4 times its distance from 1."""
    n = 700
    c = _cache(1, 4, 1, [n])
    g = torch.Generator().manual_seed(int(ratio))
    k, v = (torch.randn(1, 1, n, 128, generator=g).clamp(-2, 2).to(torch.bfloat16) for _ in range(2))
    k[..., 5] = 0
    B.ra_seq_begin(c.handle, 0, n, 1, 0, k.to(DEV), v.to(DEV))
    q = torch.randn(1, 4, 128, generator=g).to(torch.bfloat16)
    q[..., 5] = ratio * 4
    kn, vn = (torch.randn(1, 1, 128, generator=g).clamp(-2, 2).to(torch.bfloat16) for _ in range(2))
    kn[..., 5] = 0
    out = torch.empty_like(q, device=DEV)
    c.decode(0, q.to(DEV), kn.to(DEV), vn.to(DEV), out)
    K = torch.cat([held(k)[0, 0], held(kn)[0]]).double().numpy()
    V = torch.cat([held(v)[0, 0], held(vn)[0]]).double().numpy()
    want = gqa_decode(q[0].double().numpy(), [K], [V])
    slack = 2 * 2 * np.expm1(2 * 127 * 2 * 2.0 ** -26 * 4 * ratio / np.sqrt(128))
    err = np.abs(out[0].double().cpu().numpy() - want)
    assert (err <= 2.0 ** -8 * np.abs(want) + 1e-4 + slack).all(), (ratio, err.max(), slack)
    c.close()


@pytest.mark.parametrize("top", ["largest", "infinite"])
def test_the_largest_queries(top):
    """A query channel of the largest bf16 number, 255 * 2^120, which the codes of a cached
    row would not reach, or infinite, which counts as that: against keys of 2^-126 to 2^-122 the
    scores are up to 64 / sqrt(128), and as exact as others."""
    n = 500
    largest = 255 * 2.0 ** 120
    c = _cache(1, 2, 1, [n])
    g = torch.Generator().manual_seed(12)
    k = torch.zeros(1, 1, n + 1, 128)
    k[..., 7] = (torch.rand(1, 1, n + 1, generator=g) * 32 - 16).round() * 2.0 ** -126
    k = k.to(torch.bfloat16)
    v = torch.randn(1, 1, n + 1, 128, generator=g).clamp(-2, 2).to(torch.bfloat16)
    q = torch.zeros(1, 2, 128)
    q[0, 0, 7], q[0, 1, 7] = largest, -largest
    want = gqa_decode(q[0].double().numpy(), [held(k)[0, 0].double().numpy()],
                      [held(v)[0, 0].double().numpy()])
    if top == "infinite":
        q *= float("inf")
        q[q.isnan()] = 0
    B.ra_seq_begin(c.handle, 0, n, 1, 0, k[:, :, :n].contiguous().to(DEV),
                   v[:, :, :n].contiguous().to(DEV))
    out = torch.empty(1, 2, 128, dtype=torch.bfloat16, device=DEV)
    c.decode(0, q.to(torch.bfloat16).to(DEV), k[:, :, n].contiguous().to(DEV),
             v[:, :, n].contiguous().to(DEV), out)
    err = np.abs(out[0].double().cpu().numpy() - want)
    assert (err <= 2.0 ** -8 * np.abs(want) + 1e-4).all(), err.max()
    c.close()
