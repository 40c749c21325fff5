"""Rotary positions against float64: both pairings, every scaling, parts of the head, odd
row counts, far positions, in place, captured."""

import numpy as np
import pytest
import torch

from gpu_harness import DEV, _f64
from oracle import rotary
from paper_2609_03430_amd import binding as B

pytestmark = pytest.mark.gpu

SCALINGS = {
    "plain": dict(),
    "linear": dict(factor=4.0),
    "rotations": dict(factor=8.0, low=1.0, high=4.0, original_len=8192),
    "channels": dict(factor=16.0, low=1.0, high=32.0, original_len=4096),
}
CODES = dict(plain=B.RA_ROTARY_PLAIN, linear=B.RA_ROTARY_LINEAR,
             rotations=B.RA_ROTARY_ROTATIONS, channels=B.RA_ROTARY_CHANNELS)


def _rotary(base, dims, adjacent, scaling, magnitude):
    kw = SCALINGS[scaling]
    r = B.make_rotary(base, dims=dims, pairs=int(adjacent), scaling=CODES[scaling],
                      magnitude=magnitude, **kw)
    return r, rotary.frequencies(base, dims, scaling, **kw)


def _check(got, x, positions, freqs, adjacent, magnitude):
    """fp32: sine and cosine within 3 * 2^-23 of their own (the rounding of an angle of an
    eighth of a turn and the functions' error), times the magnitude (a rounding), two products
    and a sum (a rounding each): 8 * 2^-23 of |a| + |b|, then the output's half step.  The angle
    itself is off by fp64 roundings: here of two powers (half a step each, and their exponents'
    2^-53 |ln f|, 14 at most, halved for each), their product, the turns and the angle, there
    of one power, its angle and the remainder: under 2^-49 of it.  Channels that stay are equal."""
    dims = 2 * len(freqs)
    want = rotary.rotate(_f64(x), positions, freqs, adjacent, magnitude)
    got, x = _f64(got), _f64(x)
    assert np.array_equal(got[..., dims:], x[..., dims:])
    half = len(freqs)
    a = slice(0, dims, 2) if adjacent else slice(0, half)
    b = slice(1, dims, 2) if adjacent else slice(half, dims)
    size = magnitude * (np.abs(x[..., a]) + np.abs(x[..., b]))
    bound = np.zeros_like(x)
    angle = np.abs(np.asarray(positions, np.float64))[..., None] * freqs
    bound[..., a] = bound[..., b] = (8 * 2.0 ** -23 + 2.0 ** -49 * angle) * size
    return want[..., :dims], got[..., :dims], bound[..., :dims]


def _assert_close(parts, dtype):
    want, got, bound = parts
    half = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8
    bound = bound + half * (np.abs(want) + bound)
    assert (np.abs(got - want) <= bound).all(), np.max(np.abs(got - want) / (bound + 1e-30))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("dims", [128, 96, 80, 64, 18, 16, 2, 126])
def test_rows(dims, adjacent, dtype):
    g = torch.Generator().manual_seed(dims)
    cases = [("plain", 1, 1, 0, 0.0), ("linear", 3, 33, 7, 1.25), ("rotations", 17, 130, 100000, 1.0),
             ("channels", 9, 257, 2 ** 31 - 257, 1.2772588722239782)]
    for scaling, heads, rows, first, magnitude in cases:
        r, f = _rotary(500000.0, dims, adjacent, scaling, magnitude)
        m = magnitude or 1.0
        x = torch.randn(heads, rows, 128, generator=g).to(dtype).to(DEV)
        out = torch.full((heads * rows + 1, 128), 7.0, dtype=dtype, device=DEV)
        B.ra_rotate_rows(r, x, out, first=first)
        got = out[:-1].view_as(x)
        assert (out[-1] == 7.0).all()
        pos = first + np.arange(rows, dtype=np.int64)
        _assert_close(_check(got, x, pos, f, adjacent, m), dtype)
        # positions of their own, any order and sign, in place
        p = torch.randint(-1000, 200000, (heads, rows), generator=g, dtype=torch.int32)
        y = x.clone()
        B.ra_rotate_rows(r, y, y, positions=p.to(DEV))
        _assert_close(_check(y, x, p.numpy(), f, adjacent, m), dtype)


def test_more_heads_than_a_grid_has_rows():
    r, f = _rotary(10000.0, 128, False, "plain", 0.0)
    x = torch.randn(65535 * 8 + 9, 1, 128, device=DEV).to(torch.bfloat16)
    out = torch.empty_like(x)
    B.ra_rotate_rows(r, x, out, first=5)
    _assert_close(_check(out[-20:], x[-20:], np.array([5]), f, False, 1.0), torch.bfloat16)
    _assert_close(_check(out[:20], x[:20], np.array([5]), f, False, 1.0), torch.bfloat16)


@pytest.mark.parametrize("dtype", [B.RA_BF16, B.RA_E4M3, B.RA_F32])
@pytest.mark.parametrize("dims,adjacent", [(128, False), (64, True), (22, False)])
def test_steps(dims, adjacent, dtype):
    """Queries and keys of the active slots at their next positions; others are left."""
    cfg = B.make_config(1, 6, 2, 16, 0, 16, dtype=dtype, max_seqs=4)
    c = B.Cache(cfg, B.ra_required_slots(cfg, [3, 0, 40]))
    made = {0: 0, 1: 70, 3: 33}
    lps = {0: 3, 1: 0, 3: 40}
    for s, n in made.items():
        B.ra_seq_begin(c.handle, s, lps[s], 1, s)
        B.ra_seq_fast_forward(c.handle, s, n)
    r, f = _rotary(10000.0, dims, adjacent, "rotations", 1.5)
    t = torch.float32 if dtype == B.RA_F32 else torch.bfloat16
    q, k = torch.randn(4, 6, 128, device=DEV).to(t), torch.randn(4, 2, 128, device=DEV).to(t)
    qo, ko = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    B.ra_rotate_step(c.handle, r, q, k, qo, ko)
    for s in range(4):
        if s not in made:
            assert (qo[s] == 7.0).all() and (ko[s] == 7.0).all()
            continue
        at = np.array([lps[s] + made[s]])
        _assert_close(_check(qo[s], q[s], at, f, adjacent, 1.5), t)
        _assert_close(_check(ko[s], k[s], at, f, adjacent, 1.5), t)
    # one of the two, in place
    q2, k2 = q.clone(), k.clone()
    B.ra_rotate_step(c.handle, r, q2, None, q2, None)
    B.ra_rotate_step(c.handle, r, None, k2, None, k2)
    for s in made:
        assert torch.equal(q2[s], qo[s]) and torch.equal(k2[s], ko[s])
    assert torch.equal(q2[2], q[2]) and torch.equal(k2[2], k[2])
    c.close()


def test_captured_steps_turn_by_each_replays_position():
    """A captured call reads the slot's position at each replay."""
    cfg = B.make_config(1, 4, 2, 16, 0, 16, max_seqs=1)
    c = B.Cache(cfg, B.ra_seq_rows(cfg, 5))
    B.ra_seq_begin(c.handle, 0, 5, 1, 0)
    r, f = _rotary(10000.0, 128, False, "plain", 1.0)
    q, k, v = (torch.randn(1, h, 128, device=DEV).to(torch.bfloat16) for h in (4, 2, 2))
    qo, ko, out = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q)

    def step():
        B.ra_rotate_step(c.handle, r, q, k, qo, ko)
        c.decode(0, qo, ko, v, out)
        B.ra_end_step(c.handle)

    B.ra_graph_mode(c.handle, True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.current_stream().wait_stream(side)
    for t in range(1, 40):
        graph.replay()
        torch.cuda.synchronize()
        _assert_close(_check(qo[0], q[0], np.array([5 + t]), f, False, 1.0), torch.bfloat16)
        _assert_close(_check(ko[0], k[0], np.array([5 + t]), f, False, 1.0), torch.bfloat16)
    del graph
    B.ra_graph_mode(c.handle, False)
    assert B.ra_get_seq_info(c.handle, 0).step == 40
    c.close()


def test_refused_arrays():
    r = B.make_rotary(10000.0)
    x = torch.zeros(2, 3, 128, device=DEV)
    bad = [dict(x=x.half(), out=x), dict(x=x, out=x[:1]), dict(x=x, out=x.bfloat16()),
           dict(x=x.transpose(0, 1), out=x), dict(x=x[..., :64].contiguous(), out=x),
           dict(x=x, out=x.cpu()), dict(x=x, out=x, positions=torch.zeros(6, device=DEV)),
           dict(x=x, out=x, positions=torch.zeros(5, device=DEV, dtype=torch.int32)),
           dict(x=x, out=x, first=-1), dict(x=x, out=x, first=2 ** 31 - 2)]
    for kw in bad:
        with pytest.raises(B.RandAttnError):
            B.ra_rotate_rows(r, **kw)
    B.ra_rotate_rows(r, x[:0], x[:0])
    B.ra_rotate_rows(r, torch.zeros(2, 0, 128, device=DEV), x)
