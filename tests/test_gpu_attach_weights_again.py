"""Weights attached again while calls on other streams that use the former ones are still in
flight: their memory is not handed out before those calls have ended."""

import pytest
import torch

from gpu_harness import DEV
from paper_2609_03430_amd import binding as B

pytestmark = pytest.mark.gpu

LP, K, R, EVERY = 20, 1200, 100, 64
HEADS = (2, 2)                                   # layers, KV heads


def _cache():
    cfg = B.make_config(HEADS[0], 4, HEADS[1], K, R, EVERY, dtype=B.RA_BF16, max_seqs=1)
    c = B.Cache(cfg, B.ra_required_slots(cfg, [LP]))
    c.attach_weights(LP)
    return c


def _restore_evict_save(c, w, out, stream):
    """No biased step: a request restored, evicted by weight (moves by chunk) and saved."""
    B.ra_seq_begin(c.handle, 0, LP, 1, 1, stream=stream)
    B.ra_seq_fast_forward(c.handle, 0, K + R + 40, stream=stream)
    B.ra_write_weights(c.handle, 0, w, stream=stream)
    B.ra_evict_now(c.handle, 0, stream=stream)
    B.ra_export_weights(c.handle, 0, out, stream=stream)
    B.ra_seq_end(c.handle, 0, stream=stream)


def _end_of_step(c, rule, ins, out, side):
    """Biased attention on the current stream, its event at the end of the step on another."""
    B.ra_seq_begin(c.handle, 0, LP, 1, 1)
    B.ra_seq_fast_forward(c.handle, 0, K + R + 63 - (K + R) % EVERY)
    for layer in range(HEADS[0]):
        c.decode_biased(layer, rule, *ins, out)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
        assert B.ra_end_step(c.handle) == 1
        B.ra_seq_end(c.handle, 0)


@pytest.mark.parametrize("how", ["restored and saved", "the end of a step"])
def test_memory_in_use_is_not_handed_out(how):
    c = _cache()
    side = torch.cuda.Stream()
    n = LP + K + R
    w = torch.rand(*HEADS, n + 40, device=DEV)
    out = torch.empty(*HEADS, n, device=DEV)
    ins = [torch.randn(1, h, 128, device=DEV).to(torch.bfloat16) for h in (4, 2, 2)]
    attended = torch.empty_like(ins[0])
    rule = B.make_score_rule()
    torch.cuda.synchronize()
    old, size = c.weights.data_ptr(), c.weights.numel() * 4
    if how == "restored and saved":
        with torch.cuda.stream(side):
            torch.cuda._sleep(200_000_000)          # a tenth of a second or so
        _restore_evict_save(c, w, out, side)
    else:
        _end_of_step(c, rule, ins, attended, side)
    c.attach_weights(LP)
    taken = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(4)]
    busy = not side.query()
    got = {t.data_ptr() for t in taken} | {c.weights.data_ptr()}
    torch.cuda.synchronize()
    assert busy                                     # (or the test has shown nothing)
    assert old not in got
    if how == "restored and saved":                 # the 40 least of the candidates are gone
        rows = w.view(-1, n + 40).cpu()
        for row, kept in zip(rows, out.view(-1, n).cpu()):
            drop = set((row[LP:LP + K + 40].argsort()[:40] + LP).tolist())
            want = row[[j for j in range(n + 40) if j not in drop]]
            assert torch.equal(kept, want)
    _restore_evict_save(c, w, out, side)            # with the new ones, as before
    torch.cuda.synchronize()
    c.close()
