"""Helpers of the 8-bit cache's and the block-sparse steps' tests (not collected)."""

import numpy as np
import torch

from gpu_harness import DEV, OracleSeq, Run, _f64, attn_err
from oracle import blocks, quant
from oracle.attention import softmax_attention
from paper_2609_03430_amd import binding as B
from paper_2609_03430_amd.synth import Workload


class Run8(Run):
    """A Run over an 8-bit cache: bf16 rows in and out."""

    def __init__(self, *args, begin=True, wl_seed=1000, ring=None, scaled=True, stale=True, **kw):
        super().__init__(*args, begin=False, dtype=B.RA_E4M3, wl_seed=wl_seed, ring=ring,
                         scaled=scaled, **kw)
        self.tdtype = torch.bfloat16
        self.wl = Workload(wl_seed, self.L, self.Hq, self.Hkv, 128, self.tdtype, scaled, ring=ring,
                           device=DEV)
        if stale:
            fill_stale(self.cache)
        if begin:
            for slot in range(self.n):
                self.begin(slot)


def fill_stale(cache):
    """Every row of the pools NaN: rows that nothing wrote must not be read."""
    if cache.cfg.dtype == B.RA_E4M3:
        cache.k_pool.fill_(0x7F)
        cache.v_pool.fill_(0x7F)
    else:
        cache.k_pool.fill_(float("nan"))
        cache.v_pool.fill_(float("nan"))


def held(x):
    """bf16 rows as the cache holds them, as bf16 (every such value is a bf16 number)."""
    return torch.from_numpy(quant.held_rows(x.double().cpu().numpy())).to(torch.bfloat16)


class OracleSeq8(OracleSeq):
    """The oracle's view of a sequence whose rows are held in 8 bits."""

    def rows(self, layer, g, P):
        k, v = super().rows(layer, g, P)
        return held(k), held(v)


def oracle_of(run, slot):
    return (OracleSeq8 if run.cfg.dtype == B.RA_E4M3 else OracleSeq)(run, slot)


def sparse_step(run, n_blocks, recent, layers=None):
    """One decode step, the given layers (all by default) through the sparse call."""
    outs = torch.empty(run.L, run.max_seqs, run.Hq, 128, dtype=run.tdtype, device=DEV)
    for layer in range(run.L):
        q, k, v = run.step_inputs(layer)
        if layers is None or layer in layers:
            run.cache.decode_sparse(layer, n_blocks, recent, q, k, v, outs[layer])
        else:
            run.cache.decode(layer, q, k, v, outs[layer])
    evicted = B.ra_end_step(run.h)
    run.steps = [s + 1 for s in run.steps]
    return outs, evicted


def sparse_want(o, layer, step0, n_blocks, recent):
    """[Hq, d] of the oracle, whose replay holds the cache after the step's append."""
    run = o.run
    q = o.wl.q_rows(o.rid, layer, torch.arange(run.Hq), step0).double().numpy()
    out = np.empty_like(q)
    for g in range(run.Hkv):
        k, v = (_f64(x) for x in o.rows(layer, g, o.rep.P[(layer, g)]))
        mine = q[g * run.G:(g + 1) * run.G]
        rows = blocks.attended(mine, k, len(k) - 1, n_blocks, recent)
        for i in range(run.G):
            out[g * run.G + i] = softmax_attention(mine[i], k[rows], v[rows])
    return out


def check_step(run, oracles, outs, ctx=(), sparse=None):
    """A step's outputs against the oracles (which it advances by the step): dense, or
    with sparse = (n_blocks, recent, layers)."""
    for o in oracles:
        o.rep.append()
        for layer in range(run.L):
            if sparse and (sparse[2] is None or layer in sparse[2]):
                want = sparse_want(o, layer, run.steps[o.slot] - 1, sparse[0], sparse[1])
            else:
                want = o.attend(layer, run.steps[o.slot] - 1)
            attn_err(outs[layer, o.slot], want, B.RA_BF16, (o.slot, layer) + tuple(ctx))
        o.rep.end_step()


def status(fn, *args, **kw):
    try:
        fn(*args, **kw)
    except B.RandAttnError as e:
        return e.status
    return B.RA_OK
