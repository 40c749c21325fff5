"""fp32 rows under a rule lose no more to rounding than their sums must: errors of outputs and
weights in the mean square, against what independent roundings come to.

u^2 = 2^-48 / 3 is the variance of a rounding of 1, evenly spread over half a step either way.
  - A score is eight sums of 16 products, then seven sums of those.  Of products of variance v a
    sum of k has k v, so the roundings of products, sums and sums of sums come to
    u^2 v (128 + 8 * 136 + 4 * 32 + 2 * 64 + 128) = 12.5 u^2 (128 v): a score of magnitude S =
    scale sqrt(sum of (q k)^2) is off by 12.5 (u S)^2.  A cap's slope 1 - tanh^2 lowers it; tanh
    is right to about a step, two roundings of the score, and its argument to one: 5 (u s)^2.
    Slopes add the roundings of the score in natural units and of the lowered one.
  - The difference d from the head's maximum is rounded once, the exponential is right to a step
    (two roundings) and corrected with one more: (d^2 + 5) u^2 relative to the weight.
  - Values are added up in blocks of 32 keys (each rounding half the block's sum on the average:
    16, and one for the product), the blocks of a wavefront in turn (b of them), four wavefronts
    (a product and a sum each) and the splits (likewise, at least 64 keys each).
  - The sum of weights has 8 + 2 roundings in a block, one a block, as many joins, all at most
    its size; quotient, product and result three more.
A chain of 128 products instead of the eight sums would make 12.5 of it 65.5, and the
difference's product with a rounded unit 2.25 d^2 of d^2.
"""

import pytest
import torch

from gpu_harness import DEV
from paper_2609_03430_amd import binding as B

pytestmark = pytest.mark.gpu
U2 = 2.0 ** -48 / 3


def _case(S, G, Hkv, n, size, kw, weighed, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    Hq = G * Hkv
    k, v = (torch.randn(S, Hkv, n, 128, generator=g, device=DEV) for _ in range(2))
    q = size * torch.randn(S, Hq, 128, generator=g, device=DEV)
    new = [torch.randn(S, Hkv, 128, generator=g, device=DEV) for _ in range(2)]
    cfg = B.make_config(1, Hq, Hkv, 64, 0, 64, dtype=B.RA_F32, max_seqs=S)
    c = B.Cache(cfg, B.ra_required_slots(cfg, [n] * S))
    if weighed:
        c.attach_weights(n)
    for s in range(S):
        B.ra_seq_begin(c.handle, s, n, 1, s, k[s:s + 1].contiguous(), v[s:s + 1].contiguous())
    slopes = torch.tensor([2.0 ** -(1 + i % 8) for i in range(Hq)], device=DEV)
    rule = B.make_score_rule(cap=kw.get("cap", 0.0), slopes=slopes if kw.get("slopes") else None)
    out = torch.empty_like(q)
    c.decode_biased(0, rule, q, *new, out)
    B.ra_end_step(c.handle)
    got = torch.empty(S, Hkv, n + 1, device=DEV)
    if weighed:
        for s in range(S):
            B.ra_export_weights(c.handle, s, got[s])
    torch.cuda.synchronize()
    c.close()

    K, V = (torch.cat([x, y[:, :, None]], 2).double().repeat_interleave(G, 1)
            for x, y in ((k, new[0]), (v, new[1])))
    prod = K * q.double()[:, :, None] * 128 ** -0.5
    s, var = prod.sum(-1), 12.5 * prod.square().sum(-1)
    del prod
    if kw.get("cap"):
        t = torch.tanh(s / kw["cap"])
        s, var = kw["cap"] * t, var * (1 - t * t) ** 2
        var = var + 5 * s * s
    if kw.get("slopes"):
        dist = (n - torch.arange(n + 1, device=DEV)).double()
        var = var + s * s
        s = s - slopes.double()[None, :, None] * dist
        var = var + s * s
    d = s - s.amax(-1, keepdim=True)
    var = var + d * d + 5                                   # of a weight, relative, in u^2
    p = torch.exp(d)
    p = p / p.sum(-1, keepdim=True)
    want = (p[..., None] * V).sum(-2)
    blocks, splits = n // 128 + 2, n // 64 + 2
    pv2 = (p * p)[..., None] * V * V
    bound = ((p * p * var)[..., None] * (V - want[..., None, :]).square()).sum(-2)
    bound = bound + (17 + blocks + 8 + 2 * splits) * pv2.sum(-2)
    bound = U2 * (bound + (13 + blocks + 8 + 2 * splits) * want * want)
    err = (out.double() - want).square()
    ratios = [(err.mean() / bound.mean()).sqrt().item()]
    if weighed:
        total = 10 + blocks + 8 + 2 * splits + (p * p * var).sum(-1, keepdim=True)
        w = p.view(S, Hkv, G, n + 1).sum(2)
        wb = (p * p * (var + total + 2)).view(S, Hkv, G, n + 1).sum(2) + G * w * w
        # relative to each row's weight, however small
        ratios.append((((got.double() - w) / w).square().mean() / (U2 * wb / (w * w)).mean())
                      .sqrt().item())
    return ratios


@pytest.mark.parametrize("kw", [dict(), dict(cap=20.0), dict(slopes=True),
                                dict(cap=20.0, slopes=True)], ids=lambda kw: "-".join(kw) or "zero")
@pytest.mark.parametrize("size", [1.0, 4.0])
@pytest.mark.parametrize("S,G,Hkv,n", [(8, 2, 2, 200), (1, 8, 2, 2000), (8, 4, 8, 600),
                                       (32, 4, 8, 900)])
def test_errors_in_the_mean_square(S, G, Hkv, n, size, kw):
    for weighed in (False, True):
        ratios = _case(S, G, Hkv, n, size, kw, weighed, 11)
        print("ratios", ["%.2f" % r for r in ratios])
        assert max(ratios) <= 1.0, ratios
