"""A cache under score rules beside its model in float64 (not collected).

``Sim`` makes steps, events and transfers on a cache and follows them on plain arrays: per
(slot, layer, KV head) the positions P, the rows K and V as the cache holds them, the
accumulated weights W and a bound E on what the kernel's may differ from them by.
"""

import numpy as np
import torch

from blocks_harness import fill_stale
from gpu_harness import DEV, _f64, note
from oracle import quant
from oracle.rule import rule_attention
from paper_2609_03430_amd import binding as B

EPS = 2.0 ** -24            # half a step of fp32


def held(x, dtype):
    x = x.double().cpu().numpy()
    return quant.held_rows(x) if dtype == B.RA_E4M3 else x


class Sim:
    def __init__(self, L, Hq, Hkv, K, lps, r=16, every=16, dtype=B.RA_BF16,
                 layout=B.RA_LAYOUT_CHRONOLOGICAL, weights=True, max_seqs=None, page_rows=32,
                 seed=1, policy=B.RA_POLICY_RANDOM, extra_rows=0, attn_split=0):
        self.L, self.Hq, self.Hkv, self.G = L, Hq, Hkv, Hq // Hkv
        self.K, self.r, self.every, self.dtype = K, r, every, dtype
        self.n = max_seqs or len(lps)
        self.tdtype = torch.float32 if dtype == B.RA_F32 else torch.bfloat16
        self.gen = torch.Generator().manual_seed(seed)
        self.cfg = B.make_config(L, Hq, Hkv, K, r, every, dtype=dtype, max_seqs=self.n,
                                 layout=layout, page_rows=page_rows, policy=policy, attn_split=attn_split,
                                 max_prompt_len=max(lps, default=0))
        rows = sum(B.ra_seq_rows(self.cfg, lp) for lp in lps) + extra_rows
        self.cache = B.Cache(self.cfg, rows)
        self.h = self.cache.handle
        fill_stale(self.cache)
        self.weighed = weights
        if weights:
            self.cache.attach_weights(max(lps, default=0))
            self.cache.weights.fill_(float("nan"))
        self.seq = {}
        for s, lp in enumerate(lps):
            self.begin(s, lp)

    def rand(self, *shape):
        return torch.randn(*shape, generator=self.gen).to(self.tdtype)

    def begin(self, s, lp):
        k, v = (self.rand(self.L, self.Hkv, lp, 128) for _ in range(2))
        B.ra_seq_begin(self.h, s, lp, 5 + s, s, k.to(DEV), v.to(DEV))
        heads = {}
        for l in range(self.L):
            for g in range(self.Hkv):
                heads[l, g] = dict(P=np.arange(lp), K=held(k[l, g], self.dtype),
                                   V=held(v[l, g], self.dtype), W=np.zeros(lp), E=np.zeros(lp))
        self.seq[s] = dict(lp=lp, step=0, heads=heads)

    def inputs(self):
        return [self.rand(self.n, h, 128) for h in (self.Hq, self.Hkv, self.Hkv)]

    def step(self, rule, kw, ctx=(), stream=None):
        """One step, `kw` the rule's plain values (slopes: a list)."""
        outs, ins = [], []
        for l in range(self.L):
            q, k, v = self.inputs()
            ins.append((q, k, v))
            out = torch.full((self.n, self.Hq, 128), 7.0, dtype=self.tdtype, device=DEV)
            self.cache.decode_biased(l, rule, q.to(DEV), k.to(DEV), v.to(DEV), out, stream)
            outs.append(out)
        evicted = B.ra_end_step(self.h, stream)
        torch.cuda.synchronize()
        for l in range(self.L):
            for s in range(self.n):
                if s not in self.seq:
                    assert (outs[l][s] == 7.0).all()
                    continue
                self.follow(s, l, *ins[l], outs[l], kw, ctx)
        due = 0
        for s, q in self.seq.items():
            q["step"] += 1
            any_head = q["heads"][0, 0]
            m = len(any_head["P"]) - q["lp"] - self.r - self.K
            if q["step"] % self.every == 0 and m > 0:
                self.event(s, m)
                due += 1
        assert evicted == due
        return outs

    def follow(self, s, l, q, k, v, out, kw, ctx):
        plain = {x: y for x, y in kw.items() if x != "slopes"}
        now = self.seq[s]["lp"] + self.seq[s]["step"]
        got = _f64(out[s])
        for g in range(self.Hkv):
            h = self.seq[s]["heads"][l, g]
            h["P"] = np.append(h["P"], now)
            h["K"] = np.vstack([h["K"], held(k[s, g:g + 1], self.dtype)])
            h["V"] = np.vstack([h["V"], held(v[s, g:g + 1], self.dtype)])
            h["W"], h["E"] = np.append(h["W"], 0.0), np.append(h["E"], 0.0)
            n = len(h["P"])
            for i in range(g * self.G, (g + 1) * self.G):
                slope = kw["slopes"][i] if kw.get("slopes") else 0.0
                qi = q[s, i].double().numpy()
                want, p = rule_attention(qi, h["K"], h["V"], h["P"], now, slope=slope, **plain)
                # A score sums 128 products in fp32 (a rounding each, and one per product of
                # fp32 rows), is scaled (two), capped (four steps of the cap) and lowered
                # (three steps of slope * distance); its weight's relative error is that, the
                # weighted mean of it over the rows (the sum l) and a rounding per row summed.
                scale = kw.get("scale") or 128 ** -0.5
                dot = scale * (np.abs(h["K"]) @ np.abs(qi))
                d = EPS * (131 * dot + 8 * kw.get("cap", 0.0) + 4 * slope * (now - h["P"]) + 8)
                d = np.where(p > 0, d, 0.0)
                rel = 1.01 * (d + p @ d + (2 * n + 16) * EPS)
                err = p * rel + 2.0 ** -120
                # the weights in two bf16 parts: 2^-16 of each; an output's own rounding
                seen = p > 0
                V = np.abs(h["V"][seen])
                parts = 0.0 if self.dtype == B.RA_F32 else 2.0 ** -16
                bound = (err[seen] + parts * p[seen]) @ V + 2 * n * EPS * (p[seen] @ V)
                half = EPS if self.dtype == B.RA_F32 else 2.0 ** -8
                bound = bound + half * (np.abs(want) + bound) + 1e-30
                worst = np.max(np.abs(got[i] - want) / bound)
                note("out_ratio", worst)
                assert worst <= 1.0, (worst, s, l, i, n, now) + tuple(ctx)
                if self.weighed:
                    h["W"] += p
                    h["E"] += err + EPS * (h["W"] + 2)

    def event(self, s, m):
        """The event's kept rows, read back: none dropped that weighs more than a kept one."""
        lp = self.seq[s]["lp"]
        n = len(self.seq[s]["heads"][0, 0]["P"]) - m
        assert B.ra_get_seq_info(self.h, s).len == n
        pos = torch.empty(self.L, self.Hkv, n, dtype=torch.int32, device=DEV)
        B.ra_export_positions(self.h, s, pos)
        pos = pos.cpu().numpy()
        for (l, g), h in self.seq[s]["heads"].items():
            keep = np.isin(h["P"], pos[l, g])
            assert keep.sum() == n and np.array_equal(h["P"][keep], pos[l, g])
            assert keep[:lp].all() and (self.r == 0 or keep[-self.r:].all())
            if self.weighed and keep[lp:len(keep) - self.r].any():
                cand = np.arange(lp, len(keep) - self.r)
                gone, kept = cand[~keep[cand]], cand[keep[cand]]
                assert (h["W"][gone] - h["E"][gone]).max() <= (h["W"][kept] + h["E"][kept]).min()
            for x in ("P", "K", "V", "W", "E"):
                h[x] = h[x][keep]

    def export(self, s):
        n = B.ra_get_seq_info(self.h, s).len
        shape = (self.L, self.Hkv, n)
        pos = torch.empty(shape, dtype=torch.int32, device=DEV)
        k, v = (torch.empty(*shape, 128, dtype=self.tdtype, device=DEV) for _ in range(2))
        B.ra_export_positions(self.h, s, pos)
        B.ra_export_rows(self.h, s, k, v)
        w = None
        if self.weighed:
            w = torch.empty(shape, device=DEV)
            B.ra_export_weights(self.h, s, w)
        torch.cuda.synchronize()
        return pos, k, v, w

    def check(self, ctx=()):
        """Every slot's positions and rows are the model's, its weights within their bound."""
        for s in self.seq:
            pos, k, v, w = self.export(s)
            for (l, g), h in self.seq[s]["heads"].items():
                assert np.array_equal(pos[l, g].cpu().numpy(), h["P"]), (s, l, g) + tuple(ctx)
                assert np.array_equal(_f64(k[l, g]), h["K"]), (s, l, g) + tuple(ctx)
                assert np.array_equal(_f64(v[l, g]), h["V"]), (s, l, g) + tuple(ctx)
                if w is not None and len(h["W"]):
                    ratio = np.max(np.abs(_f64(w[l, g]) - h["W"]) / (h["E"] + 1e-30))
                    note("weight_ratio", ratio)
                    assert ratio <= 1.0, (ratio, s, l, g) + tuple(ctx)

    def rule(self, kw):
        kw = dict(kw)
        if kw.get("slopes"):
            kw["slopes"] = torch.tensor(kw["slopes"], dtype=torch.float32, device=DEV)
        return B.make_score_rule(**kw)

    def close(self):
        self.cache.close()


def slopes(Hq):
    """Slopes that fp32 holds exactly."""
    return [2.0 ** -(1 + i % 8) for i in range(Hq)]
