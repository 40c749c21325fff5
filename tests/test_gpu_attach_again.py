"""Bounds attached again while sparse steps on other streams are still in flight: their
memory, and the workspace's, is not handed out before those steps have ended."""

import pytest
import torch

from gpu_harness import DEV
from paper_2609_03430_amd import binding as B

pytestmark = pytest.mark.gpu


def _cache(n=400):
    cfg = B.make_config(1, 4, 2, 0, 0, 1, dtype=B.RA_BF16, max_seqs=1, max_prompt_len=n)
    c = B.Cache(cfg, B.ra_required_slots(cfg, [n]))
    k = torch.randn(1, 2, n, 128, device=DEV).to(torch.bfloat16)
    B.ra_seq_begin(c.handle, 0, n, 1, 1, k, k)
    q = torch.randn(1, 4, 128, device=DEV).to(torch.bfloat16)
    new = torch.randn(1, 2, 128, device=DEV).to(torch.bfloat16)
    return c, q, new, torch.empty_like(q)


@pytest.mark.parametrize("given", ["a stream", "its handle", "the current stream"])
def test_memory_in_use_is_not_handed_out(given):
    c, q, new, out = _cache()
    c.attach_sparse(2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    old = {c.bounds.data_ptr(): c.bounds.numel(),
           c.sparse_workspace.data_ptr(): c.sparse_workspace.numel()}
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)              # a tenth of a second or so
        if given == "the current stream":
            c.decode_sparse(0, 2, 0, q, new, new, out)
            B.ra_end_step(c.handle)
    if given != "the current stream":
        stream = side if given == "a stream" else side.cuda_stream
        c.decode_sparse(0, 2, 0, q, new, new, out, stream=stream)
        B.ra_end_step(c.handle, stream=stream)
    c.attach_sparse(2)
    taken = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in old.values() for _ in range(4)]
    busy = not side.query()
    got = {t.data_ptr() for t in taken}
    torch.cuda.synchronize()
    assert busy                                     # (or the test has shown nothing)
    assert not got & set(old), (got, old)
    c.decode_sparse(0, 2, 0, q, new, new, out)      # with the new ones, as before
    B.ra_end_step(c.handle)
    c.close()


def test_memory_for_a_stream_comes_from_that_stream():
    """The new bounds may not be memory that the current stream's work still uses: given a
    stream they are allocated for it."""
    c, q, new, out = _cache()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.attach_sparse(2)
    n = [c.bounds.numel(), c.sparse_workspace.numel()]
    torch.cuda.synchronize()
    mine = [torch.empty(x, dtype=torch.uint8, device=DEV) for x in n]
    torch.cuda._sleep(200_000_000)
    for x in mine:
        x.fill_(0x55)                               # still to come on the current stream ..
    where = {x.data_ptr() for x in mine}
    del mine, x                                     # .. which may have the memory again at once
    c.attach_sparse(2, stream=side)
    busy = not torch.cuda.current_stream().query()
    got = {c.bounds.data_ptr(), c.sparse_workspace.data_ptr()}
    c.decode_sparse(0, 2, 0, q, new, new, out, stream=side)
    B.ra_end_step(c.handle, stream=side)
    torch.cuda.synchronize()
    assert busy
    assert not got & where
    want = torch.empty_like(out)
    c.decode_sparse(0, 2, 0, q, new, new, want)
    B.ra_end_step(c.handle)
    assert torch.equal(out, want)
    c.close()
