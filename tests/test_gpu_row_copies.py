"""Rows into a cache's layout and back, bit for bit: lengths around value tiles, workgroups and
pages, every head or one, and exports larger than the last-level cache holds twice."""

import pytest
import torch

from gpu_harness import DEV
from paper_2609_03430_amd import binding as B

pytestmark = pytest.mark.gpu
CHRON, PAGED = B.RA_LAYOUT_CHRONOLOGICAL, B.RA_LAYOUT_PAGED
TYPES = {B.RA_BF16: torch.bfloat16, B.RA_F32: torch.float32}
STALE = 77.0


def _bits(shape, dtype, seed):
    """Any bits at all: NaN, infinities and subnormal numbers among them."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    width = torch.int16 if dtype == torch.bfloat16 else torch.int32
    info = torch.iinfo(width)
    return torch.randint(info.min, info.max + 1, shape, generator=g, device=DEV, dtype=torch.int64).to(width)


def _check(dtype, layout, page_rows, L, Hkv, n, seed):
    t = TYPES[dtype]
    cfg = B.make_config(L, 2 * Hkv, Hkv, 40, 8, 8, dtype=dtype, layout=layout, page_rows=page_rows,
                        max_prompt_len=n)
    c = B.Cache(cfg, B.ra_seq_rows(cfg, n))
    c.k_pool.fill_(STALE)
    c.v_pool.fill_(STALE)
    c.pos_pool.fill_(-5)
    k, v = (_bits((L, Hkv, n, 128), t, seed + i).view(t) for i in range(2))
    B.ra_seq_begin(c.handle, 0, n, 1, 0, k, v)
    ints = k.view(torch.int16 if t == torch.bfloat16 else torch.int32).dtype

    def same(a, b):
        return torch.equal(a.view(ints), b.view(ints))

    def outs(*shape):
        return [torch.full((*shape, n + 1, 128), STALE, dtype=t, device=DEV) for _ in range(2)]

    for which in ((1, 1), (1, 0), (0, 1)):
        got = [x.view(-1) if w else None for x, w in zip(outs(L, Hkv), which)]
        B.ra_export_rows(c.handle, 0, *got)
        for x, want in zip(got, (k, v)):
            if x is not None:
                assert same(x[:want.numel()].view(want.shape), want), which
                assert (x[want.numel():] == STALE).all()
    one = outs()
    B.ra_read_rows(c.handle, 0, L - 1, Hkv - 1, *one)
    for x, want in zip(one, (k, v)):
        assert same(x[:n], want[L - 1, Hkv - 1]) and (x[n:] == STALE).all()
    pos = torch.empty(L, Hkv, n, dtype=torch.int32, device=DEV)
    B.ra_export_positions(c.handle, 0, pos)
    assert (pos == torch.arange(n, device=DEV, dtype=torch.int32)).all()
    # nothing else was written: keys of n rows a head, values of whole tiles, zeros past the rows
    heads, tiles = L * Hkv, -(-n // 8)
    used = (c.pos_pool >= 0).sum().item()
    assert used == heads * n
    stale_k = (c.k_pool[c.pos_pool < 0] == STALE).all(dim=1).sum().item()
    assert stale_k == c.pool_rows - heads * n
    stale_v = (c.v_pool.view(-1, 8 * 128) == STALE).all(dim=1).sum().item()
    assert stale_v >= c.pool_rows // 8 - heads * tiles
    if n % 8 and layout == CHRON:
        cap = B.ra_region_rows(cfg, n)
        last = c.v_pool.view(-1, 128, 8)[:heads * cap // 8].view(heads, cap // 8, 128, 8)
        assert (last[:, tiles - 1, :, n % 8:].contiguous().view(ints) == 0).all()
    B.ra_write_rows(c.handle, 0, v, k)               # the other way round
    got = [x.view(-1) for x in outs(L, Hkv)]
    B.ra_export_rows(c.handle, 0, *got)
    assert same(got[0][:v.numel()].view(v.shape), v) and same(got[1][:k.numel()].view(k.shape), k)
    c.close()


@pytest.mark.parametrize("layout,page_rows", [(CHRON, 64), (PAGED, 32), (PAGED, 128)])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_lengths(dtype, layout, page_rows):
    for n in (1, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 1000):
        _check(dtype, layout, page_rows, 2, 3, n, n)


@pytest.mark.parametrize("dtype,L,Hkv,n", [(B.RA_BF16, 40, 8, 4093), (B.RA_F32, 20, 8, 4095)])
@pytest.mark.parametrize("layout", [CHRON, PAGED])
def test_exports_past_the_cache(dtype, L, Hkv, n, layout):
    assert L * Hkv * n * 2 * 128 * TYPES[dtype].itemsize > 2 * 256 << 20
    _check(dtype, layout, 64, L, Hkv, n, 3)
