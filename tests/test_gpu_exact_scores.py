"""Scores are fp32 sums of exact products, of 8-bit rows as of bf16 ones.

Queries and keys are whole numbers times a power of two, and the magnitudes of a score's
products add up to less than 2^24 of their unit, so every partial sum is an fp32
number: a sum in fp32 is exact in any order.  Keys come in neighbouring pairs whose
second holds the first's channels elsewhere, among channels of equal query values: the
scores of a pair are equal, and with values +1 and -1 the exact output is 0.

What a kernel may leave: the weights of a pair, taken from equal scores against the
same maximum, are equal, so only the sums of weights round.  A product with the values
adds 32 weights to an accumulator, in two parts of a weight each: at most 2 * 33
roundings of 2^-23 (were they truncations) of the weights that a block adds, so all of
them at most 66 * 2^-23 of the sum of all weights, by which the output is divided; the
rounding to bf16 adds 2^-8 of that.  A pair whose scores differ by d leaves
tanh(d / 2) of its share."""

import pytest
import torch

from blocks_harness import held
from gpu_harness import DEV, note
from oracle.attention import gqa_decode
from paper_2609_03430_amd import binding as B

pytestmark = pytest.mark.gpu
CHRON, PAGED = B.RA_LAYOUT_CHRONOLOGICAL, B.RA_LAYOUT_PAGED
BOUND = 66 * 2.0 ** -23 * (1 + 2.0 ** -8)

CODES = [m * 2 ** e for e in range(0, 6) for m in range(8, 16) if m * 2 ** e <= 448]


def _pairs(g, n, Hkv, G, kind):
    """(queries [Hkv G 128], keys [Hkv n 128]) of n (even) rows."""
    # eight query values, one magnitude in seven small: neighbours' products differ widely
    values = torch.randint(-127, 128, (Hkv, G, 8), generator=g).float()
    values[..., 3] = values[..., 3].sign()
    q = values.repeat(1, 1, 16)                     # channel c has value c % 8
    if kind == "small":                             # -15 .. 15 beside one pair of 256
        k = torch.randint(-15, 16, (Hkv, n // 2, 128), generator=g).float()
        shift = -7
    else:                                           # every E4M3 number that is whole, to 448
        table = torch.tensor([0] + list(range(1, 8)) + CODES).float()
        k = table[torch.randint(0, len(table), (Hkv, n // 2, 128), generator=g)]
        k = k * (2 * torch.randint(0, 2, k.shape, generator=g) - 1)
        shift = -12
    k[..., 5] = 256                                 # the scale of the row ..
    k[..., 13] = -256                               # .. and what takes it out of the score
    at = torch.rand(Hkv, n // 2, 16, 8, generator=g).argsort(-2)
    other = k.view(Hkv, n // 2, 16, 8).gather(-2, at).view_as(k)
    keys = torch.stack([k, other], 2).view(Hkv, n, 128)
    # a row's unit: 1, 1/2, 1/4 or 1/8, the same for a pair
    unit = torch.randint(-3, 1, (Hkv, n // 2, 1), generator=g).float()
    keys = keys * torch.exp2(unit.repeat_interleave(2, 1))
    most = (q.abs() @ keys.abs().transpose(1, 2)).max()
    assert most * 8 < 2 ** 24
    dots = q.double() @ keys.double().transpose(1, 2)
    assert torch.equal(dots[..., ::2], dots[..., 1::2])
    return (q * 2.0 ** shift).to(torch.bfloat16), keys.to(torch.bfloat16)


@pytest.mark.parametrize("kind", ["small", "wide"])
@pytest.mark.parametrize("dtype", [B.RA_BF16, B.RA_E4M3])
@pytest.mark.parametrize("layout", [CHRON, PAGED])
@pytest.mark.parametrize("n,Hkv,G", [(2, 1, 1), (30, 2, 5), (64, 1, 16), (600, 2, 8), (4096, 1, 4)])
def test_equal_scores_weigh_the_same(n, Hkv, G, layout, dtype, kind):
    g = torch.Generator().manual_seed(n + G)
    q, k = _pairs(g, n, Hkv, G, kind)
    if dtype == B.RA_E4M3:
        assert torch.equal(held(k).float(), k.float())
    v = torch.ones(Hkv, n, 128)
    v[:, 1::2] = -1
    cfg = B.make_config(1, Hkv * G, Hkv, 0, 0, 1, dtype=dtype, max_seqs=1, layout=layout,
                        page_rows=32, max_prompt_len=n)
    c = B.Cache(cfg, B.ra_required_slots(cfg, [n]))
    B.ra_seq_begin(c.handle, 0, n, 1, 0, k[None].contiguous().to(DEV),
                   v[None].to(torch.bfloat16).to(DEV))
    zero = torch.zeros(1, Hkv, 128, dtype=torch.bfloat16, device=DEV)
    out = torch.empty(1, Hkv * G, 128, dtype=torch.bfloat16, device=DEV)
    outs = []
    c.decode(0, q.view(1, -1, 128).to(DEV), zero, zero, out)
    outs.append(out.double().cpu())
    B.ra_end_step(c.handle)
    c.attach_sparse(4)                              # the block-sparse kernels, all rows attended
    c.decode_sparse(0, 4, n, q.view(1, -1, 128).to(DEV), zero, zero, out)
    outs.append(out.double().cpu())
    B.ra_end_step(c.handle)
    c.close()
    for x in outs:
        note("left", x.abs().max())
        assert x.abs().max() <= BOUND, (x.abs().max(), BOUND)


@pytest.mark.parametrize("dtype", [B.RA_BF16, B.RA_E4M3])
def test_keys_below_the_smallest_normal_number(dtype):
    """Keys of up to 16 * 2^-133, bf16 numbers below 2^-126, against queries of 2^127: the
    products are whole multiples of 2^-6 and their sums, at most 32, exact.  What is left
    is the rounding of the weights, in two bf16 parts (2^-17 of each), of fp32 sums, and of
    the output: under 1e-4 for values up to 2."""
    n = 300
    g = torch.Generator().manual_seed(3)
    k = (torch.randint(-16, 17, (1, 1, n + 1, 128), generator=g).float() * 2.0 ** -133).to(
        torch.bfloat16)
    v = torch.randn(1, 1, n + 1, 128, generator=g).clamp(-2, 2).to(torch.bfloat16)
    q = (2.0 ** 127 * (2 * torch.randint(0, 2, (1, 4, 128), generator=g) - 1)).to(torch.bfloat16)
    keep = held if dtype == B.RA_E4M3 else (lambda x: x)
    if dtype == B.RA_E4M3:
        assert torch.equal(held(k), k)
    want = gqa_decode(q[0].double().numpy(), [k[0, 0].double().numpy()],
                      [keep(v)[0, 0].double().numpy()])
    cfg = B.make_config(1, 4, 1, 0, 0, 1, dtype=dtype, max_seqs=1, max_prompt_len=n)
    c = B.Cache(cfg, B.ra_required_slots(cfg, [n]))
    B.ra_seq_begin(c.handle, 0, n, 1, 0, k[:, :, :n].contiguous().to(DEV),
                   v[:, :, :n].contiguous().to(DEV))
    out = torch.empty(1, 4, 128, dtype=torch.bfloat16, device=DEV)
    c.decode(0, q.to(DEV), k[:, :, n].contiguous().to(DEV), v[:, :, n].contiguous().to(DEV), out)
    err = (out[0].double().cpu() - torch.from_numpy(want)).abs()
    assert (err <= 2.0 ** -8 * torch.from_numpy(want).abs() + 1e-4).all(), err.max()
    c.close()
