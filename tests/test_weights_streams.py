"""Every wrapper whose call uses attached weights tells the allocator on which stream, so that
their memory is not handed out under its work (CPU only: the library and the tensors are
stand-ins that record what they are given)."""

import ctypes

import pytest
import torch

from paper_2609_03430_amd import binding as B


class Tensor:
    """Of the weights: which streams it was told of."""
    device, dtype = torch.device("cuda"), torch.float32

    def __init__(self):
        self.on = []

    def data_ptr(self):
        return 4096

    def numel(self):
        return 64

    def element_size(self):
        return 4

    def record_stream(self, stream):
        self.on.append(stream)


class Library:
    def __init__(self):
        self.streams = {}            # by entry point: integers and pointers it was given

    def __getattr__(self, name):
        def call(*args):
            self.streams[name] = args
            return B.RA_OK
        return call


CALLS = {
    "ra_seq_begin": lambda h, s: B.ra_seq_begin(h, 0, 4, 1, 1, stream=s),
    "ra_fast_forward": lambda h, s: B.ra_fast_forward(h, 3, s),
    "ra_seq_fast_forward": lambda h, s: B.ra_seq_fast_forward(h, 0, 3, s),
    "ra_end_step": lambda h, s: B.ra_end_step(h, s),
    "ra_evict_now": lambda h, s: B.ra_evict_now(h, 0, s),
    "ra_write_weights": lambda h, s: B.ra_write_weights(h, 0, None, s),
    "ra_export_weights": lambda h, s: B.ra_export_weights(h, 0, None, s),
    "ra_biased_attention": lambda h, s: B.ra_biased_attention(
        h, 0, B.make_score_rule(), None, None, None, None, None, s),
}


@pytest.fixture
def lib(monkeypatch):
    lib = Library()
    monkeypatch.setattr(B, "_lib", lambda: lib)
    monkeypatch.setattr(B, "_arg", lambda *a, **k: None)
    monkeypatch.setattr(B, "_torch_stream", lambda raw, device: raw)
    return lib


@pytest.mark.parametrize("name", list(CALLS))
def test_the_calls_stream_is_recorded(lib, name):
    h, other = ctypes.c_void_p(11), ctypes.c_void_p(12)
    w, w2 = Tensor(), Tensor()
    B.ra_weights_attach(h, w)
    B.ra_weights_attach(other, w2)
    try:
        CALLS[name](h, 70)
        assert 70 in lib.streams[name]
        assert w.on == [70] and w2.on == []
        CALLS[name](h, 70)                   # once for each stream ..
        CALLS[name](h, 71)
        assert w.on == [70, 71]
        again = Tensor()
        B.ra_weights_attach(h, again)        # .. and tensor
        CALLS[name](h, 70)
        assert again.on == [70] and w.on == [70, 71]
        B.ra_weights_attach(h, None)
        CALLS[name](h, 72)
        assert again.on == [70]
    finally:
        B.ra_cache_destroy(h)
        B.ra_cache_destroy(other)
    CALLS[name](other, 73)
    assert w2.on == []


def test_a_refused_attachment_changes_nothing(lib, monkeypatch):
    h, w, refused = ctypes.c_void_p(13), Tensor(), Tensor()
    B.ra_weights_attach(h, w)
    try:
        monkeypatch.setattr(B, "_lib", lambda: type("Refusing", (), {
            "ra_weights_attach": staticmethod(lambda *a: B.RA_ERR_STATE),
            "ra_status_string": staticmethod(lambda st: b"refused")}))
        for t in (refused, None):
            with pytest.raises(B.RandAttnError):
                B.ra_weights_attach(h, t)
        monkeypatch.setattr(B, "_lib", lambda: lib)
        B.ra_end_step(h, 5)
        assert w.on == [5] and refused.on == []
    finally:
        B.ra_cache_destroy(h)
