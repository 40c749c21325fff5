"""Block-sparse decode steps on the GPU: the chosen blocks equal the oracle's, and the
outputs are the attention over the rows they name."""

import numpy as np
import pytest
import torch

from blocks_harness import (OracleSeq8, Run8, check_step, fill_stale, held, oracle_of, sparse_step,
                            status)
from gpu_harness import DEV, Run, attn_err, check_heads, log
from oracle import blocks
from oracle.attention import softmax_attention
from paper_2609_03430_amd import binding as B

pytestmark = pytest.mark.gpu
CHRON, PAGED = B.RA_LAYOUT_CHRONOLOGICAL, B.RA_LAYOUT_PAGED
BF16, E4M3 = B.RA_BF16, B.RA_E4M3


def _run(dtype, **kw):
    run = Run8(**kw) if dtype == E4M3 else Run(dtype=dtype, **kw)
    run.cache.attach_sparse(64)
    run.cache.bounds.fill_(0x55)
    return run


class Fixed:
    """Prompt-only caches over given rows: a step's new row is dropped at its end."""

    def __init__(self, dtype, Hq, Hkv, keys, values, layout=CHRON, page_rows=32, blocks_max=64,
                 L=1):
        self.lens = [k.shape[1] for k in keys]
        self.dtype, self.Hq, self.Hkv, self.G = dtype, Hq, Hkv, Hq // Hkv
        cfg = B.make_config(L, Hq, Hkv, 0, 0, 1, dtype=dtype, max_seqs=len(keys), layout=layout,
                            page_rows=page_rows, max_prompt_len=max(self.lens))
        self.c = B.Cache(cfg, B.ra_required_slots(cfg, self.lens))
        fill_stale(self.c)
        self.c.attach_sparse(blocks_max)
        self.c.bounds.fill_(0x55)
        keep = held if dtype == E4M3 else (lambda x: x)
        self.k, self.v = [keep(k) for k in keys], [keep(v) for v in values]
        self.keep = keep
        for i, (k, v) in enumerate(zip(keys, values)):
            k, v = (x.expand(L, -1, -1, -1).contiguous().to(DEV) for x in (k, v))
            B.ra_seq_begin(self.c.handle, i, self.lens[i], 1, i, k, v)

    def step(self, n_blocks, recent, q, kn, vn, layer=0, end=True):
        out = torch.full(q.shape, float("nan"), dtype=q.dtype, device=DEV)
        self.c.sparse_workspace.fill_(0xEE)
        self.c.decode_sparse(layer, n_blocks, recent, q.to(DEV), kn.to(DEV), vn.to(DEV), out)
        lists = self.c.sparse_workspace[:4 * len(self.lens) * self.Hkv * n_blocks].view(
            torch.int32).view(len(self.lens), self.Hkv, n_blocks).cpu().numpy()
        if end:
            B.ra_end_step(self.c.handle)
        return out.cpu(), lists

    def check(self, n_blocks, recent, q, kn, vn, ctx=()):
        out, lists = self.step(n_blocks, recent, q, kn, vn)
        kn, vn = self.keep(kn), self.keep(vn)
        for i, n in enumerate(self.lens):
            for g in range(self.Hkv):
                k = torch.cat([self.k[i][g], kn[i, g][None]]).double().numpy()
                v = torch.cat([self.v[i][g], vn[i, g][None]]).double().numpy()
                mine = q[i, g * self.G:(g + 1) * self.G].double().numpy()
                pick = blocks.chosen(mine, k, n, n_blocks, recent)
                if pick is not None:
                    assert np.array_equal(lists[i, g], pick), (i, g, n_blocks, recent) + tuple(ctx)
                rows = blocks.attended(mine, k, n, n_blocks, recent)
                want = np.stack([softmax_attention(x, k[rows], v[rows]) for x in mine])
                attn_err(out[i, g * self.G:(g + 1) * self.G], want, B.RA_BF16,
                         (i, g, n_blocks, recent) + tuple(ctx))

    def close(self):
        self.c.close()


def _inputs(seed, lens, Hq, Hkv, scale=1.0):
    g = torch.Generator().manual_seed(seed)

    def rows(n, h):
        x = torch.randn(h, n, 128, generator=g) * scale
        runs = torch.randn(h, n // 40 + 1, 128, generator=g).repeat_interleave(40, 1)[:, :n]
        return (x + runs).to(torch.bfloat16)
    keys, values = [rows(n, Hkv) for n in lens], [rows(n, Hkv) for n in lens]
    q = torch.randn(len(lens), Hq, 128, generator=g).to(torch.bfloat16)
    kn, vn = (torch.randn(len(lens), Hkv, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    return keys, values, q, kn, vn


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("layout,page_rows", [(CHRON, 32), (PAGED, 32), (PAGED, 256)])
@pytest.mark.parametrize("lens,Hq,Hkv", [
    ([0, 31, 32, 33], 4, 2), ([64, 65, 95, 96, 97], 16, 1), ([515, 1000, 2049], 10, 2),
    ([5000, 40], 6, 6),
])
def test_choice_and_output(lens, Hq, Hkv, layout, page_rows, dtype):
    keys, values, q, kn, vn = _inputs(sum(lens), lens, Hq, Hkv)
    f = Fixed(dtype, Hq, Hkv, keys, values, layout, page_rows)
    for n_blocks, recent in [(1, 0), (0, 0), (2, 1), (3, 31), (5, 32), (17, 64), (0, 40),
                             (64, 100), (2, 10 ** 9), (1, 0)]:
        f.check(n_blocks, recent, q, kn, vn)
    f.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_equal_scores_take_the_lowest_blocks(dtype):
    keys, values, q, kn, vn = _inputs(5, [700, 1500], 4, 2)
    for k in keys:
        k[:, 32:] = k[:, :32].repeat(1, 50, 1)[:, :k.shape[1] - 32]
    f = Fixed(dtype, 4, 2, keys, values)
    f.check(7, 20, q, kn, vn)
    q[:] = 0                                   # every score 0
    f.check(7, 20, q, kn, vn)
    f.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_keys_below_the_smallest_normal(dtype):
    """Bounds of magnitudes under 2^-126: any positive one rounds up to 2^-60, any
    negative one down to -2^-60, and zeros stay."""
    keys, values, q, kn, vn = _inputs(9, [900, 1300], 4, 2)
    for i, k in enumerate(keys):
        g = torch.Generator().manual_seed(90 + i)
        k *= (torch.rand(k.shape, generator=g) < 0.02) * 2.0 ** -128
        k[0] = k[0].abs()
    f = Fixed(dtype, 4, 2, keys, values)
    for n_blocks in (1, 7):
        _, lists = f.step(n_blocks, 20, q, kn, vn)
        for i, n in enumerate((900, 1300)):
            for g in range(2):
                want = blocks.chosen(q[i, 2 * g:2 * g + 2].double().numpy(),
                                     f.k[i][g].double().numpy(), n, n_blocks, 20)
                assert np.array_equal(lists[i, g], want), (i, g, n_blocks)
    f.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_equal_scores_of_long_heads(dtype):
    """Heads that a launch of its own chooses from: every score the same, every score 0,
    two scores, and scores of both signs."""
    lens = [17000, 36000]
    keys, values, q, kn, vn = _inputs(7, lens, 4, 2)
    for k in keys:
        k[:, 32:] = k[:, :32].repeat(1, k.shape[1] // 32 + 1, 1)[:, :k.shape[1] - 32]
    f = Fixed(dtype, 4, 2, keys, values)
    f.check(7, 20, q, kn, vn)
    q[:] = 0
    f.check(7, 20, q, kn, vn)
    f.close()
    keys, values, q, kn, vn = _inputs(8, lens, 4, 2)
    for k in keys:
        k[:, 32:] = k[:, :32].repeat(1, k.shape[1] // 32 + 1, 1)[:, :k.shape[1] - 32]
        k[:, 320:] *= -1
    f = Fixed(dtype, 4, 2, keys, values)
    f.check(13, 20, q, kn, vn)
    f.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_extreme_scales(dtype):
    """Exponents outside the scores' range, signs of one kind, zero keys."""
    keys, values, q, kn, vn = _inputs(6, [600, 600, 600], 6, 2)
    keys[0] = (keys[0].float() * 2.0 ** torch.arange(-75, 75).repeat_interleave(4)[:, None]).to(
        torch.bfloat16)
    keys[1] = -keys[1].abs()
    keys[2][0] = 0
    q[0] = (q[0].float() * 2.0 ** -70).to(torch.bfloat16)
    q[2, 1] = 0
    f = Fixed(dtype, 6, 2, keys, values)
    for n_blocks in (1, 6, 11):
        _, lists = f.step(n_blocks, 16, q, kn, vn)
        for i in range(3):
            for g in range(2):
                want = blocks.chosen(q[i, 3 * g:3 * g + 3].double().numpy(),
                                     f.k[i][g].double().numpy(), 600, n_blocks, 16)
                assert np.array_equal(lists[i, g], want), (i, g, n_blocks)
    f.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_keys_that_are_not_finite_stay_in_their_block(dtype):
    """A NaN or an infinity in a block that is not chosen leaves the others' choice and
    output as they are."""
    keys, values, q, kn, vn = _inputs(7, [640], 4, 1)
    keys[0][0, 200:204] = 0
    clean = Fixed(dtype, 4, 1, keys, values)
    out0, lists0 = clean.step(4, 32, q, kn, vn)
    assert 6 not in lists0[0, 0]
    keys[0][0, 200, :] = float("nan")
    values[0][0, 201, 3] = float("nan")
    f = Fixed(dtype, 4, 1, keys, values)
    out1, lists1 = f.step(4, 32, q, kn, vn)
    assert np.array_equal(lists0, lists1) and torch.equal(out0, out1)
    keys[0][0, 200, :] = 0
    keys[0][0, 200, 5] = float("inf")          # its block's other bounds vanish beside it
    g = Fixed(dtype, 4, 1, keys, values)
    _, lists2 = g.step(4, 32, q, kn, vn)
    kd = g.k[0][0].double().numpy()
    assert np.array_equal(lists2[0, 0], blocks.chosen(q[0].double().numpy(), kd, 640, 4, 32))
    q[0, 0, 0] = float("inf")
    q[0, 1, 1] = float("nan")
    _, lists3 = g.step(4, 32, q, kn, vn)
    assert np.array_equal(lists3[0, 0], blocks.chosen(q[0].double().numpy(), kd, 640, 4, 32))
    for x in (clean, f, g):
        x.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_all_blocks_give_the_dense_result(dtype):
    """2,100 rows have 65 candidates: 65 chosen are all of them.  The two calls' outputs
    are each within half a bf16 step and the fp32 sums' 1e-4 of the exact one."""
    keys, values, q, kn, vn = _inputs(8, [1, 300, 2100], 8, 2)
    f = Fixed(dtype, 8, 2, keys, values, blocks_max=65)
    sparse, _ = f.step(65, 0, q, kn, vn)
    dense = torch.empty_like(sparse, device=DEV)
    f.c.decode(0, q.to(DEV), kn.to(DEV), vn.to(DEV), dense)
    B.ra_end_step(f.c.handle)
    a, b = sparse.double(), dense.cpu().double()
    assert ((a - b).abs() <= 2 * (2.0 ** -8 * torch.maximum(a.abs(), b.abs()) + 1e-4)).all()
    f.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("kw", [
    dict(L=2, Hq=8, Hkv=2, K=200, lps=[100, 33, 250], r=16, every=16),
    dict(L=2, Hq=6, Hkv=2, K=150, lps=[70, 10], r=20, every=25, layout=PAGED, page_rows=32,
         max_seqs=4),
    dict(L=1, Hq=4, Hkv=1, K=90, lps=[0, 200], r=8, every=8, layout=PAGED, page_rows=64),
])
def test_decoding_with_events(kw, dtype):
    """Sparse steps across events: bounds follow the rows that move."""
    log("sparse decoding dtype=%d %s" % (dtype, kw))
    run = _run(dtype, **kw)
    run.fast_forward(150)
    for s in range(run.n):
        run.materialise(s)
    oracles = [oracle_of(run, s) for s in range(run.n)]
    for o in oracles:
        o.advance(150)
    events = 0
    for t in range(90):
        layers = None if t % 3 else {t % run.L}         # the others attend to every row
        n_blocks, recent = [(3, 16), (1, 0), (5, 40)][t % 3]
        outs, evicted = sparse_step(run, n_blocks, recent, layers)
        check_step(run, oracles, outs, (t,), (n_blocks, recent, layers))
        events += evicted
    assert events >= 2
    check_heads(run, oracles)
    run.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_rows_written_and_slots_reused(dtype):
    """ra_write_rows, explicit events, another sequence in the slot and leaving graph
    mode all make bounds anew."""
    run = _run(dtype, L=2, Hq=4, Hkv=2, K=100, lps=[130, 64, 90], r=8, every=8, max_seqs=3)
    oracles = [oracle_of(run, s) for s in range(3)]

    def step():
        outs, _ = sparse_step(run, 2, 8)
        check_step(run, oracles, outs, sparse=(2, 8, None))
    run.fast_forward(120)
    for s in range(3):
        run.materialise(s)
        oracles[s].advance(120)
    for _ in range(9):
        step()
    # rows of another workload, and back
    n = B.ra_get_seq_info(run.h, 1).len
    k, v = (torch.empty(2, 2, n, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    B.ra_export_rows(run.h, 1, k, v)
    B.ra_write_rows(run.h, 1, -k, v)
    q, kn, vn = run.step_inputs(0)
    scratch = torch.empty_like(q)
    for layer in range(2):
        run.cache.decode_sparse(layer, 2, 8, q, kn, vn, scratch)
    B.ra_end_step(run.h)
    run.steps = [s + 1 for s in run.steps]
    for o in oracles:
        o.rep.append()
        o.rep.end_step()
    # every row as its position's again (that step's pair was layer 0's in both layers)
    for s in range(3):
        run.materialise(s)
    step()
    B.ra_evict_now(run.h, 0)
    oracles[0].rep.evict_now()
    step()
    run.end(0)
    run.lps[0], run.rids[0] = 125, 17
    run.begin(0)
    oracles[0] = oracle_of(run, 0)
    for _ in range(12):
        step()
    B.ra_graph_mode(run.h, 1)
    assert status(sparse_step, run, 2, 8) == B.RA_ERR_STATE
    for _ in range(10):
        outs, _ = run.step()
        check_step(run, oracles, outs)
    B.ra_graph_mode(run.h, 0)
    for _ in range(10):
        step()
    check_heads(run, oracles)
    run.close()


def test_bounds_attached_while_moves_are_pending():
    """A deferred event's rows move when bounds are attached, and later events move
    theirs themselves; detached, events defer again."""
    run = Run(L=2, Hq=4, Hkv=2, K=24, lps=[20, 20], r=8, every=8)   # one work item per head
    oracles = [oracle_of(run, s) for s in range(2)]
    while True:
        outs, evicted = run.step()
        check_step(run, oracles, outs)
        if evicted:
            break
    assert B.ra_get_seq_info(run.h, 0).move_pending == 1
    run.cache.attach_sparse(8)
    assert B.ra_get_seq_info(run.h, 0).move_pending == 0
    for t in range(20):
        outs, _ = sparse_step(run, 0, 4, {t % 2})
        assert B.ra_get_seq_info(run.h, 0).move_pending == 0
        check_step(run, oracles, outs, (t,), (0, 4, {t % 2}))
    B.ra_sparse_attach(run.h, None)
    assert status(sparse_step, run, 0, 4) == B.RA_ERR_STATE
    pending = 0
    for _ in range(10):
        outs, _ = run.step()
        pending += B.ra_get_seq_info(run.h, 0).move_pending
        check_step(run, oracles, outs)
    assert pending == 1
    check_heads(run, oracles)
    run.close()


def test_two_caches_and_streams():
    """Two caches stepped on streams of their own, at once."""
    runs = [_run(d, L=1, Hq=8, Hkv=2, K=300, lps=[200, 90], r=16, every=16, wl_seed=50 + d)
            for d in (BF16, E4M3)]
    oracles = [[oracle_of(r, s) for s in range(2)] for r in runs]
    for r, os_ in zip(runs, oracles):
        r.fast_forward(180)
        for s in range(2):
            r.materialise(s)
            os_[s].advance(180)
    streams = [torch.cuda.Stream() for _ in runs]
    for t in range(20):
        inputs = [r.step_inputs(0) for r in runs]
        outs = [torch.empty_like(i[0]) for i in inputs]
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        for r, i, o, s in zip(runs, inputs, outs, streams):
            r.cache.decode_sparse(0, 4, 16, *i, o, stream=s)
            B.ra_end_step(r.h, stream=s)
        for s in streams:
            torch.cuda.current_stream().wait_stream(s)
        for r, os_, o in zip(runs, oracles, outs):
            r.steps = [s + 1 for s in r.steps]
            check_step(r, os_, o[None], (t,), (4, 16, None))
    for r in runs:
        r.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_long_heads(dtype):
    """Every build of the selection, to the most candidates there may be."""
    for n, n_blocks in [(32 * 257, 9), (32 * 1025, 40), (32 * 4097, 64), (32 * 16384 + 5, 64)]:
        log("long head of %d rows, dtype %d" % (n, dtype))
        g = torch.Generator().manual_seed(n)
        x = torch.randn(1, 4096, 128, generator=g)
        keys = (x.repeat(1, n // 4096 + 1, 1)[:, :n] *
                torch.linspace(0.5, 1.5, n)[None, :, None]).to(torch.bfloat16)
        f = Fixed(dtype, 4, 1, [keys], [keys], blocks_max=64)
        _, _, q, kn, vn = _inputs(n, [32], 4, 1)
        f.check(n_blocks, 0, q, kn, vn)
        f.close()
    f = Fixed(dtype, 2, 1, [torch.zeros(1, 32 * 16385, 128, dtype=torch.bfloat16)] * 1,
              [torch.zeros(1, 32 * 16385, 128, dtype=torch.bfloat16)])
    q, kn = torch.zeros(1, 2, 128).to(torch.bfloat16), torch.zeros(1, 1, 128).to(torch.bfloat16)
    assert status(f.step, 8, 0, q, kn, kn) == B.RA_ERR_UNSUPPORTED
    out, _ = f.step(8, 32, q, kn, kn)          # one block fewer to choose from
    assert torch.equal(out, torch.zeros_like(out))
    f.close()


def test_refusals():
    lens = [100]
    keys, values, q, kn, vn = _inputs(1, lens, 4, 2)
    f = Fixed(BF16, 4, 2, keys, values, L=2)
    h, ws, out = f.c.handle, f.c.sparse_workspace, torch.empty_like(q, device=DEV)
    args = (q.to(DEV), kn.to(DEV), vn.to(DEV), out)
    call = B.ra_sparse_attention
    assert status(call, h, 0, -1, 0, *args, ws) == B.RA_ERR_INVALID_ARG
    assert status(call, h, 0, 1, -1, *args, ws) == B.RA_ERR_INVALID_ARG
    assert status(call, h, 2, 1, 0, *args, ws) == B.RA_ERR_INVALID_ARG
    assert status(call, h, 0, 1, 0, *args, ws[:256]) == B.RA_ERR_INVALID_ARG
    assert status(call, h, 0, 65, 0, *args, ws[:-256]) == B.RA_ERR_INVALID_ARG
    assert status(call, h, 0, 1, 0, args[0][:, :3], *args[1:], ws) == B.RA_ERR_INVALID_ARG
    small = torch.empty(B.ra_sparse_bytes(f.c.cfg, f.c.pool_rows) - 1, dtype=torch.uint8, device=DEV)
    assert status(B.ra_sparse_attach, h, small) == B.RA_ERR_INVALID_ARG
    call(h, 0, 1, 0, *args, ws)
    assert status(call, h, 0, 1, 0, *args, ws) == B.RA_ERR_STATE        # the layer is appended
    assert status(B.ra_sparse_attach, h, f.c.bounds) == B.RA_ERR_STATE  # inside a step
    assert status(B.ra_export_rows, h, 0) == B.RA_ERR_STATE
    call(h, 1, 1, 0, *args, ws)
    B.ra_end_step(h)
    assert status(B.ra_export_rows, h, 0, torch.empty(5, dtype=torch.bfloat16, device=DEV)) \
        == B.RA_ERR_CAPACITY
    assert status(B.ra_export_rows, h, 1) == B.RA_ERR_INVALID_ARG
    f.close()
    for kw in (dict(dtype=B.RA_F32), dict(layout=B.RA_LAYOUT_HOLE_FILL)):
        cfg = B.make_config(1, 4, 2, 64, max_seqs=1, **kw)
        c = B.Cache(cfg, B.ra_seq_rows(cfg, 8))
        assert status(c.attach_sparse, 4) == B.RA_ERR_UNSUPPORTED
        assert status(B.ra_sparse_attach, c.handle, c.meta) == B.RA_ERR_UNSUPPORTED
        c.close()
    cfg = B.make_config(1, 4, 2, 64, dtype=E4M3, max_seqs=1)
    c = B.Cache(cfg, B.ra_seq_rows(cfg, 80))
    B.ra_seq_begin(c.handle, 0, 80, 1, 1)
    B.ra_fast_forward(c.handle, 70)
    w = torch.empty(2 * 4 * 64 * 128 * 8, dtype=torch.bfloat16, device=DEV)
    assert status(B.ra_window_select, c.handle, 0, 1, w) == B.RA_ERR_UNSUPPORTED
    assert status(B.ra_scored_evict, c.handle, 0, 1, B.make_scorer(0), w, w) \
        == B.RA_ERR_UNSUPPORTED
    c.close()


def test_a_captured_step_is_refused():
    """Nothing is launched into a capture, and the step goes on after it."""
    run = _run(BF16, L=1, Hq=4, Hkv=2, K=100, lps=[150], r=8, every=8)
    o = [oracle_of(run, 0)]
    q, k, v = run.step_inputs(0)
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        marker = torch.zeros(4, device=DEV)
        st = status(run.cache.decode_sparse, 0, 2, 8, q, k, v, out)
    assert st == B.RA_ERR_STATE
    g.replay()
    torch.cuda.synchronize()
    assert marker.eq(0).all()
    outs, _ = sparse_step(run, 2, 8)
    check_step(run, o, outs, sparse=(2, 8, None))
    run.close()


@pytest.mark.parametrize("scorer", [B.RA_SCORER_SNAPKV, B.RA_SCORER_VASE])
def test_after_a_scored_round(scorer):
    """A score-based round drops prompt rows too: bounds from the first row on are
    computed anew.  The rows are read back for the expected output."""
    Hq, Hkv, n_blocks, recent = 8, 2, 3, 20
    cfg = B.make_config(1, Hq, Hkv, 200, 16, 64, dtype=BF16, max_seqs=2,
                        policy=B.RA_POLICY_EXTERNAL)
    c = B.Cache(cfg, B.ra_required_slots(cfg, [150, 90]))
    c.attach_sparse(n_blocks)
    gen = torch.Generator(device=DEV).manual_seed(3)

    def rnd(*shape):
        return torch.randn(*shape, 128, device=DEV, generator=gen).to(torch.bfloat16)
    for i, lp in enumerate((150, 90)):
        B.ra_seq_begin(c.handle, i, lp, 1, i, rnd(1, Hkv, lp), rnd(1, Hkv, lp))

    def step(check):
        q, k, v = rnd(2, Hq), rnd(2, Hkv), rnd(2, Hkv)
        out = torch.empty_like(q)
        before = [[torch.empty(B.ra_get_seq_info(c.handle, i).len, 128, dtype=torch.bfloat16,
                               device=DEV) for _ in range(2 * Hkv)] for i in range(2)]
        for i in range(2):
            for h in range(Hkv):
                B.ra_read_rows(c.handle, i, 0, h, before[i][2 * h], before[i][2 * h + 1])
        c.decode_sparse(0, n_blocks, recent, q, k, v, out)
        B.ra_end_step(c.handle)
        if not check:
            return
        for i in range(2):
            for h in range(Hkv):
                K, V = (torch.cat([before[i][2 * h + j], x[i, h][None]]).double().cpu().numpy()
                        for j, x in enumerate((k, v)))
                mine = q[i, h * 4:h * 4 + 4].double().cpu().numpy()
                rows = blocks.attended(mine, K, len(K) - 1, n_blocks, recent)
                want = np.stack([softmax_attention(x, K[rows], V[rows]) for x in mine])
                attn_err(out[i, h * 4:h * 4 + 4], want, B.RA_BF16, (i, h))
    for round_ in range(2):
        for t in range(205 if round_ == 0 else 40):
            step(t % 40 == 0)
        qwin = torch.randn(2, 1, Hq, 64, 128, device=DEV, generator=gen).to(torch.bfloat16)
        scratch = torch.empty(B.ra_scored_scratch_bytes(cfg, 150), dtype=torch.uint8, device=DEV)
        was = [B.ra_get_seq_info(c.handle, i).len for i in range(2)]
        B.ra_scored_evict(c.handle, 0, 2, B.make_scorer(scorer), qwin, scratch)
        assert all(B.ra_get_seq_info(c.handle, i).len <= was[i] for i in range(2))
        for _ in range(3):
            step(True)
    assert all(B.ra_get_seq_info(c.handle, i).event >= 1 for i in range(2))
    c.close()


@pytest.mark.parametrize("layout", [CHRON, PAGED])
def test_a_serving_run(layout):
    """The operators together: an 8-bit cache whose first layer attends to every row
    and whose second to part of them, requests admitted, preempted (their rows exported),
    resumed in another slot and ended between steps."""
    run = _run(E4M3, L=2, Hq=6, Hkv=2, K=120, lps=[100, 40, 70, 0], r=16, every=16, max_seqs=4,
               layout=layout, page_rows=32, max_prompt_len=300, begin=False, pool_rows=6144)
    rng = np.random.default_rng(11)
    rep, saved, done, next_rid = {}, None, 0, 50

    def admit(slot):
        nonlocal next_rid
        run.lps[slot], run.rids[slot] = int(rng.integers(0, 101)), next_rid
        next_rid += 1
        run.begin(slot)
        rep[slot] = oracle_of(run, slot)
    run.active = set()
    for slot in (0, 1, 3):
        admit(slot)
    for t in range(220):
        outs, _ = sparse_step(run, 2, 16, {1})
        check_step(run, list(rep.values()), outs, (t,), (2, 16, {1}))
        if t % 23 == 22 and saved is None:                      # preempt one
            slot = int(rng.choice(sorted(rep)))
            o = rep.pop(slot)
            n = B.ra_get_seq_info(run.h, slot).len
            kv = [torch.empty(2, 2, n, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
            B.ra_export_rows(run.h, slot, *kv)
            run.end(slot)
            saved = (o, run.steps[slot], run.lps[slot], run.rids[slot], run.seeds[slot], kv)
        elif t % 23 == 10 and saved is not None:                # and resume it elsewhere
            slot = int(rng.choice([s for s in range(4) if s not in rep]))
            o, steps, lp, rid, seed, kv = saved
            run.lps[slot], run.rids[slot], run.seeds[slot] = lp, rid, seed
            B.ra_seq_begin(run.h, slot, lp, seed, rid)
            B.ra_seq_fast_forward(run.h, slot, steps)
            B.ra_write_rows(run.h, slot, *kv)
            run.steps[slot] = steps
            run.active.add(slot)
            o.slot = slot
            rep[slot], saved = o, None
        elif t % 37 == 36:                                      # end one, admit another
            slot = int(rng.choice(sorted(rep)))
            rep.pop(slot)
            run.end(slot)
            admit(slot)
            done += 1
    check_heads(run, list(rep.values()))
    assert done >= 3
    run.close()


def test_random_configurations():
    rng = np.random.default_rng(78)
    for trial in range(10):
        Hkv, n = int(rng.integers(1, 4)), int(rng.integers(1, 4))
        Hq = Hkv * int(rng.integers(1, 17))
        lens = [int(x) for x in np.exp(rng.uniform(0, np.log(6000), n))]
        layout, page_rows = int(rng.choice([CHRON, PAGED])), int(rng.choice([32, 64, 512]))
        dtype, n_blocks, recent = int(rng.choice([BF16, E4M3])), int(rng.integers(0, 40)), int(
            rng.integers(0, 200))
        log("sparse trial %d: %s" % (trial, (Hq, Hkv, lens, layout, page_rows, dtype, n_blocks,
                                             recent)))
        keys, values, q, kn, vn = _inputs(trial, lens, Hq, Hkv, scale=0.5)
        f = Fixed(dtype, Hq, Hkv, keys, values, layout, page_rows)
        f.check(n_blocks, recent, q, kn, vn, (trial,))
        f.check(n_blocks, recent, q, kn, vn, (trial, "again"))
        f.close()
