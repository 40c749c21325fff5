"""The 8-bit cache's and the sparse steps' sizes and refusals, on the CPU."""

import ctypes

from paper_2609_03430_amd import binding as B


def _cfg(**kw):
    return B.make_config(2, 8, 2, 64, max_seqs=2, **kw)


def test_config_and_sizes():
    c = _cfg(dtype=B.RA_E4M3)
    assert B.ra_config_check(c) == B.RA_OK
    assert B.ra_pool_bytes(c, 96) == 96 * 129
    assert B.ra_pool_bytes(_cfg(), 96) == 96 * 256
    assert B.ra_pool_bytes(_cfg(dtype=B.RA_F32), 96) == 96 * 512
    assert B.ra_pool_bytes(c, -1) == 0
    paged = _cfg(dtype=B.RA_E4M3, layout=B.RA_LAYOUT_PAGED, max_prompt_len=9)
    assert B.ra_config_check(paged) == B.RA_OK
    hole = _cfg(dtype=B.RA_E4M3, layout=B.RA_LAYOUT_HOLE_FILL)
    assert B.ra_config_check(hole) == B.RA_ERR_UNSUPPORTED
    assert B.ra_pool_bytes(hole, 96) == 0
    assert B.ra_config_check(_cfg(dtype=3)) == B.RA_ERR_INVALID_ARG
    # no drop lists: an 8-bit cache's events move their rows
    assert B.ra_meta_bytes(c) == B.ra_meta_bytes(_cfg(dtype=B.RA_F32))


def test_sparse_sizes():
    for dtype in (B.RA_BF16, B.RA_E4M3):
        c = _cfg(dtype=dtype)
        assert B.ra_sparse_bytes(c, 3200) == -(-100 * 257 // 256) * 256
        assert B.ra_sparse_bytes(c, 0) == B.ra_sparse_bytes(c, 33) == 0
        lists = -(-2 * 2 * 7 * 4 // 256) * 256
        assert B.ra_sparse_workspace_bytes(c, 7) == B.ra_workspace_bytes(c) + lists
        assert B.ra_sparse_workspace_bytes(c, 0) == B.ra_workspace_bytes(c)
        assert B.ra_sparse_workspace_bytes(c, -1) == 0
        # more blocks than any head chooses from take no more room
        assert B.ra_sparse_workspace_bytes(c, 2 ** 31 - 1) == B.ra_sparse_workspace_bytes(c, 16384)
    for kw in (dict(dtype=B.RA_F32), dict(layout=B.RA_LAYOUT_HOLE_FILL)):
        assert B.ra_sparse_bytes(_cfg(**kw), 3200) == 0
        assert B.ra_sparse_workspace_bytes(_cfg(**kw), 7) == 0


def test_null_handles_are_refused():
    lib = B._lib()
    assert lib.ra_export_rows(None, 0, None, None, 0, None) == B.RA_ERR_INVALID_ARG
    assert lib.ra_sparse_attach(None, None, 0, None) == B.RA_ERR_INVALID_ARG
    assert lib.ra_sparse_attention(None, 0, 1, 1, None, None, None, None, None, 0, None) \
        == B.RA_ERR_INVALID_ARG
    c, out = _cfg(dtype=B.RA_E4M3), ctypes.c_void_p()
    st = lib.ra_cache_create(ctypes.byref(c), None, None, None, 1024, None, 0, None,
                             ctypes.byref(out))
    assert st == B.RA_ERR_INVALID_ARG
