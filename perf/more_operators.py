"""Cases of rotary positions, biased decode attention and eviction by accumulated
attention weight, and their plain forms.

Four operators, over heads of 128 channels:

rotate   Rotary positions.  Of each row the first `dims` channels are rotated by the
         row's position p: pair i of dims / 2, the channels (i, i + dims / 2) or (2i,
         2i + 1), turns by p * f_i, f_i = base^(-2i / dims); the others stay.
             a' = m (a cos - b sin),  b' = m (b cos + a sin)
         Long contexts change f_i: "linear" divides it by `factor`; "rotations" takes
         f_i (t + (1 - t) / factor), t = (n_i - low) / (high - low) within [0, 1], of the
         n_i = original_len f_i / 2 pi turns a pair makes in the original context;
         "channels" takes t = 1 - (i - i_hi) / (i_lo - i_hi) within [0, 1], i_hi =
         floor(i(high)) and i_lo = ceil(i(low)) within [0, dims - 1], i(n) = dims
         ln(original_len / (2 pi n)) / (2 ln base).  A step's queries and keys take the
         next position of their request, rows those of their head or first, first + 1, ..
biased   Decode steps whose scores are changed before the softmax: s = scale q.k, then
         cap tanh(s / cap), then - slope_h (p_new - p_j) with p the cached positions; a row
         with p_new - p_j >= window is not attended, unless p_j < prefix.
weighed  The same steps, which also add up what each cached row is attended with:
         w_j += the sum of its softmax weights over the KV head's query heads (a new row
         starts at 0).  A pass starts from weights of 0.
event    A request restored (its rows and accumulated weights), evicted by weight, and
         saved: of the rows between the prompt and the `recent` last ones, in each KV
         head of each layer, the `keep` of largest w stay (the earliest go first among
         equal ones); rows, positions and weights are compacted in order.
"""

import math

import torch

own = False

D = 128


# ---- the cases --------------------------------------------------------------------

def _rotary(base=10000.0, dims=128, pairs="halves", scaling="none", factor=1.0, low=1.0,
            high=4.0, original_len=8192, magnitude=1.0):
    return dict(base=base, dims=dims, pairs=pairs, scaling=scaling, factor=factor, low=low,
                high=high, original_len=original_len, magnitude=magnitude)


def _case(kind, **kw):
    """layers, q_heads / kv_heads, batch requests; biased and weighed: prompts of
    prompt_lo to prompt_hi rows and `steps` decode steps to a pass."""
    base = dict(kind=kind, cache="bf16", layers=1, q_heads=32, kv_heads=8, batch=1)
    if kind == "rotate":
        # what = "step": a step's queries and keys, steps in [far / 2, far] made before;
        # "rows": `rows` rows of every head of every layer, from position `far` on, or
        # with spread > 1 of positions of their own, about `spread` apart
        base.update(_rotary(), what="step", rows=0, far=1000, spread=1)
    elif kind == "event":
        base.update(prompt_lo=512, prompt_hi=512, keep=1024, recent=64, extra=48,
                    layout="chronological", page_rows=64)
    else:
        base.update(prompt_lo=512, prompt_hi=512, steps=1, cap=0.0, slopes=False, window=0,
                    prefix=0, layout="chronological", page_rows=64, graph=False)
    base.update(kw)
    return base


def listed():
    return [
        # A step's queries and keys of a batch far into its generations, 40/8 heads; pairs
        # slowed by their turns in the original context.
        _case("rotate", name="rotate-step", q_heads=40, batch=32, far=100000, base=500000.0,
              scaling="rotations", factor=8.0),
        # The keys of a prompt of 4,096 rows, 8 heads of 36 layers, before it is cached.
        _case("rotate", name="rotate-prompt", what="rows", layers=36, rows=4096, far=0,
              base=1000000.0),
        # The kept fp32 keys of an evicted cache, each head's at positions of its own: part of
        # the channels, adjacent pairs, an odd number of rows.
        _case("rotate", name="rotate-kept", what="rows", cache="f32", layers=5, kv_heads=10,
              rows=2113, far=0, spread=9, dims=96, pairs="adjacent", scaling="channels",
              factor=16.0, low=1.0, high=32.0, original_len=4096, magnitude=1.2772588722239782),
        # The smallest steps: one layer of 4/2 fp32 heads over 200 rows, capped.
        _case("biased", name="biased-tiny", cache="f32", q_heads=4, kv_heads=2, prompt_lo=200,
              prompt_hi=200, steps=8, cap=30.0),
        # A batch of 32 requests, 40/8 heads, 9,216 rows each, capped (two of its layers).
        _case("biased", name="biased-batch", layers=2, q_heads=40, batch=32, prompt_lo=9216,
              prompt_hi=9216, steps=2, cap=50.0),
        # Layers with a sliding window over one long 8-bit request whose first rows stay in
        # sight, in captured steps.
        _case("biased", name="biased-window", cache="e4m3", layers=8, prompt_lo=131072,
              prompt_hi=131072, steps=2, window=4096, prefix=64, graph=True),
        # Paged requests of mixed lengths whose scores fall with the distance, 40/10 heads.
        _case("biased", name="biased-paged", layers=2, q_heads=40, kv_heads=10, batch=48,
              prompt_lo=300, prompt_hi=4100, steps=2, slopes=True, layout="paged"),
        # One request of 2,176 rows, eight layers.
        _case("weighed", name="weighed-one", layers=8, prompt_lo=2176, prompt_hi=2176, steps=2),
        # A batch of 32 requests, 40/8 heads, 9,216 rows each.
        _case("weighed", name="weighed-batch", layers=2, q_heads=40, batch=32, prompt_lo=9216,
              prompt_hi=9216, steps=2),
        # Paged 8-bit requests of mixed lengths, 64/8 heads, capped.
        _case("weighed", name="weighed-paged", cache="e4m3", layers=2, q_heads=64, batch=24,
              prompt_lo=400, prompt_hi=12000, steps=2, cap=50.0, layout="paged"),
        # The event of a small model's request.
        _case("event", name="event-small", layers=2, q_heads=4, kv_heads=2, prompt_lo=33,
              prompt_hi=33, keep=448),
        # The event of a request of a 36-layer model, 4,096 rows kept in each of 288 heads.
        _case("event", name="event-request", layers=36, keep=4032, prompt_lo=512,
              prompt_hi=512),
    ]


def draw(rng):
    """One more case: sizes log-uniform over the listed ones' range."""
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rotate", "biased", "biased", "weighed", "weighed", "event"])
    q_heads, kv_heads = rng.choice([(32, 8), (40, 8), (64, 8), (40, 10), (4, 2), (8, 8), (16, 1),
                                    (12, 4), (6, 2)])
    c = _case(kind, q_heads=q_heads, kv_heads=kv_heads)
    c["batch"] = size(1, 64)
    c["layers"] = rng.choice([1, 1, 2, 3, 4, 8, 36])
    if kind == "rotate":
        c["cache"] = rng.choice(["bf16", "bf16", "f32"])
        c["what"] = rng.choice(["step", "rows"])
        c["base"] = float(rng.choice([10000, 500000, 1000000]))
        c["dims"] = rng.choice([128, 128, 64, 96, 32, 80, 2, 126])
        c["pairs"] = rng.choice(["halves", "adjacent"])
        c["scaling"] = rng.choice(["none", "linear", "rotations", "channels"])
        c["factor"] = float(rng.choice([1, 4, 8, 32]))
        if c["scaling"] == "channels":
            c["high"] = 32.0
            c["magnitude"] = 0.1 * math.log(c["factor"]) + 1.0
        c["original_len"] = rng.choice([2048, 4096, 8192, 32768])
        if c["what"] == "step":
            c["layers"] = 1
            c["far"] = size(1, 200000)
            return c
        c["batch"] = 1
        c["rows"] = size(1, 9000)
        c["far"] = rng.choice([0, 0, size(1, 100000)])
        c["spread"] = rng.choice([1, 1, 2, 9])
        while c["layers"] * kv_heads * c["rows"] > 1.2e6:
            c["layers"] = (c["layers"] + 1) // 2
        return c
    c["layout"] = rng.choice(["chronological", "chronological", "paged"])
    c["page_rows"] = rng.choice([32, 64, 128, 256])
    c["cache"] = rng.choice(["bf16", "bf16", "e4m3", "f32"])
    if kind == "event":
        c["batch"] = rng.choice([1, 1, 2, 3])
        c["prompt_lo"] = c["prompt_hi"] = size(1, 2000)
        c["recent"] = rng.choice([0, 1, 33, 64, 100])
        # the event is the request's first: no trigger before it
        c["keep"] = max(0, -(-(size(1, 6000) + c["recent"]) // 64) * 64 - c["recent"])
        c["extra"] = rng.randint(1, 63)
        while c["batch"] * _rows(c) > 1.4e6:
            c["layers"], c["batch"] = (c["layers"] + 1) // 2, 1
        return c
    c["prompt_lo"] = size(1, 20000)
    c["prompt_hi"] = rng.choice([c["prompt_lo"], max(c["prompt_lo"], size(64, 20000))])
    c["steps"] = rng.choice([1, 1, 2, 3])
    c["cap"] = rng.choice([0.0, 30.0, 50.0])
    c["slopes"] = rng.random() < 0.3
    if rng.random() < 0.3:
        c["window"] = size(1, 8192)
        c["prefix"] = rng.choice([0, 0, 4, 64, 100])
    if kind == "biased":
        c["graph"] = c["layout"] != "paged" and rng.random() < 0.25
    # no larger than the listed cases
    def large():
        return work(c)["bytes"] > 4.5e9

    while large() and c["steps"] > 1:
        c["steps"] -= 1
    while large() and c["batch"] > 1:
        c["batch"] = (c["batch"] + 1) // 2
    while large() and c["layers"] > 1:
        c["layers"] = (c["layers"] + 1) // 2
    # a plain pass is some hundred launches per layer and length
    while c["layers"] * len(set(_lengths(c))) * c["steps"] > 150 and c["layers"] > 1:
        c["layers"] = (c["layers"] + 1) // 2
    return c


def _lengths(c):
    """Prompt length of every request: spread over the case's range, in mixed order."""
    n = c["prompt_hi"] - c["prompt_lo"]
    return [c["prompt_lo"] + int(n * ((i * 0.6180339887498949 + 0.37) % 1.0))
            for i in range(c["batch"])]


def _rows(c):
    """Cached rows of an event's request, over its heads."""
    return c["layers"] * c["kv_heads"] * (c["prompt_lo"] + c["keep"] + c["recent"] + c["extra"])


def _elem(c):
    return 4 if c["cache"] == "f32" else 2


def _row_bytes(c):
    """One cached row, key and value."""
    return 2 * (D + 1) if c["cache"] == "e4m3" else 2 * _elem(c) * D


def _seen(c, length):
    """Rows attended at a step over `length` cached rows, which are positions 0 .."""
    if not c["window"]:
        return length + 1
    first = max(0, length - c["window"] + 1)
    return length + 1 - first + min(first, c["prefix"])


def work(case):
    c = case
    if c["kind"] == "rotate":
        if c["what"] == "step":
            rows = c["batch"] * (c["q_heads"] + c["kv_heads"])
        else:
            rows = c["layers"] * c["kv_heads"] * c["rows"]
        nbytes = rows * 2 * D * _elem(c)
        if c["spread"] > 1:
            nbytes += 4 * rows
        return {"bytes": nbytes, "flops": rows * c["dims"] * 3}
    if c["kind"] == "event":
        rows = c["batch"] * _rows(c)
        kept = rows - c["batch"] * c["layers"] * c["kv_heads"] * c["extra"]
        # rows and weights in, the kept ones and their positions out; a comparison each
        return {"bytes": rows * (2 * _elem(c) * D + 4) + kept * (2 * _elem(c) * D + 8),
                "flops": rows}
    steps, group = c["steps"], c["q_heads"] // c["kv_heads"]
    heads = c["layers"] * c["kv_heads"]
    nbytes = float(_elem(c) * D * c["layers"] * c["batch"] * steps *
                   (2 * c["q_heads"] + 2 * c["kv_heads"]))
    flops = 0.0
    for n in _lengths(c):
        for t in range(steps):
            rows = heads * _seen(c, n + t)
            nbytes += rows * _row_bytes(c)
            flops += rows * group * 4 * D
            if c["slopes"] or c["window"]:
                nbytes += 4 * rows                       # positions
            if c["kind"] == "weighed":
                nbytes += 8 * rows                       # weights, read and written
    return {"bytes": nbytes, "flops": flops}


# ---- inputs ------------------------------------------------------------------------

def _device():
    return torch.device("cuda")


def _gen(seed, what):
    g = torch.Generator(device=_device())
    return g.manual_seed((int(seed) * 1000003 + what) % (1 << 62))


def _dtype(c):
    return torch.float32 if c["cache"] == "f32" else torch.bfloat16


def _keys(c, seed, i, n, which):
    """Key (which = 0) or value (1) rows of request i: [layers][kv_heads][n][D].
    Channels of different scale, a few of them large; keys share a direction with
    their neighbours (runs of 48 rows), as the keys of one passage do."""
    g = _gen(seed, 100 + 2 * i + which)
    dev = _device()
    shape = (c["layers"], c["kv_heads"])
    u = torch.rand(*shape, 1, D, generator=_gen(seed, 1 + which), device=dev)
    scale = 0.5 + 1.5 * u + 6.0 * (u > 0.98)
    x = torch.randn(*shape, n, D, generator=g, device=dev)
    if which == 0:
        runs = torch.randn(*shape, (n + 47) // 48, D, generator=g, device=dev)
        x = x.mul_(0.8).add_(runs.repeat_interleave(48, 2)[:, :, :n], alpha=0.6)
    return x.mul_(scale).to(_dtype(c))


def _step_inputs(c, seed):
    """Queries, keys and values: [steps][layers][batch][heads][D]."""
    g = _gen(seed, 3)
    shape = (c["steps"], c["layers"], c["batch"])
    return [torch.randn(*shape, h, D, generator=g, device=_device()).to(_dtype(c))
            for h in (c["q_heads"], c["kv_heads"], c["kv_heads"])]


def _slopes(c):
    """A slope per query head, 2^(-8 (h + 1) / q_heads), as models with such biases have."""
    h = torch.arange(1, c["q_heads"] + 1, dtype=torch.float64)
    return torch.exp2(-8.0 * h / c["q_heads"]).float().to(_device())


def _steps_made(c, seed):
    """Decode steps behind every request of a rotated step."""
    g = torch.Generator().manual_seed(int(seed) * 7 + 5)
    return torch.randint(c["far"] // 2, c["far"] + 1, (c["batch"],), generator=g).tolist()


def _row_positions(c, seed):
    """Positions of the rows of every head, [layers * kv_heads][rows] int32 (spread > 1)."""
    gaps = torch.randint(1, 2 * c["spread"], (c["layers"] * c["kv_heads"], c["rows"]),
                         generator=_gen(seed, 4), device=_device())
    return (gaps.cumsum(1) + (c["far"] - 1)).to(torch.int32)


def _event_inputs(c, seed, i):
    """Keys, values and accumulated weights of the rows of request i.  The weights spread
    over several orders of magnitude and many are alike: small ones are held coarsely."""
    n = c["prompt_lo"] + c["keep"] + c["recent"] + c["extra"]
    k, v = (_keys(c, seed, i, n, w) for w in (0, 1))
    w = torch.randn(c["layers"], c["kv_heads"], n, generator=_gen(seed, 50 + i), device=_device())
    return k, v, torch.exp(1.5 * w).mul_(64).floor_().div_(64)


class State:
    """What a program holds between calls."""


def prepare(case, seed):
    c = case
    s = State()
    s.case = c
    if c["kind"] == "rotate":
        g = _gen(seed, 3)
        if c["what"] == "step":
            s.x = [torch.randn(c["batch"], h, D, generator=g, device=_device()).to(_dtype(c))
                   for h in (c["q_heads"], c["kv_heads"])]
            s.made = _steps_made(c, seed)
            s.positions = torch.tensor([n + 1 for n in s.made], device=_device())   # (one prompt row)
        else:
            s.x = [_keys(c, seed, 0, c["rows"], 0).view(-1, c["rows"], D)]
            s.positions = _row_positions(c, seed) if c["spread"] > 1 else None
        if own:
            _own_rotate_state(s)
        return s
    s.lens = _lengths(c)
    if c["kind"] == "event":
        s.inputs = [_event_inputs(c, seed, i) for i in range(c["batch"])]
        if own:
            _own_event_state(s, seed)
        return s
    s.q, s.k, s.v = _step_inputs(c, seed)
    s.slopes = _slopes(c) if c["slopes"] else None
    if own:
        _own_steps_state(s, seed)
        return s
    s.groups = []          # requests of one length: (indices, K, V), as they are held
    for n in sorted(set(s.lens)):
        at = [i for i, m in enumerate(s.lens) if m == n]
        k, v = (torch.stack([_keys(c, seed, i, n, w) for i in at]) for w in (0, 1))
        s.groups.append((at, _held(c, k), _held(c, v)))
    return s


# ---- the plain forms ----------------------------------------------------------------

def _frequencies(c):
    """Turns per position of every pair, [dims / 2] in 64 bits."""
    half = c["dims"] // 2
    i = torch.arange(half, dtype=torch.float64, device=_device())
    f = c["base"] ** (-2.0 * i / c["dims"])
    if c["scaling"] == "linear":
        f = f / c["factor"]
    elif c["scaling"] == "rotations":
        turns = c["original_len"] * f / (2 * math.pi)
        t = ((turns - c["low"]) / (c["high"] - c["low"])).clamp(0, 1)
        f = f * (t + (1 - t) / c["factor"])
    elif c["scaling"] == "channels":
        def at(turns):
            return (c["dims"] * math.log(c["original_len"] / (2 * math.pi * turns)) /
                    (2 * math.log(c["base"])))
        first = max(math.floor(at(c["high"])), 0)
        last = min(math.ceil(at(c["low"])), c["dims"] - 1)
        t = 1 - ((i - first) / max(last - first, 0.001)).clamp(0, 1)
        f = f * (t + (1 - t) / c["factor"])
    return f / (2 * math.pi)


def _rotated(c, x, positions):
    """Rows x [..., D] at `positions` (broadcast over the rows)."""
    half = c["dims"] // 2
    turns = positions.double()[..., None] * _frequencies(c)
    angle = (turns - turns.floor()) * (2 * math.pi)
    cos, sin = ((f(angle) * c["magnitude"]).float() for f in (torch.cos, torch.sin))
    y = x.float().clone()
    if c["pairs"] == "halves":
        a, b = y[..., :half], y[..., half:2 * half]
    else:
        a, b = y[..., 0:2 * half:2], y[..., 1:2 * half:2]
    ra, rb = a * cos - b * sin, b * cos + a * sin
    a.copy_(ra)
    b.copy_(rb)
    return y.to(x.dtype)


def _quantise(x):
    """(codes, exponents) of rows [..., D]: E4M3 codes and int32 exponents."""
    x = x.float()
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True))      # amax = 2m * 2^(e - 1)
    s = torch.where(2 * m <= 1.75, e - 9, e - 8).clamp(min=-126)
    return torch.ldexp(x, -s).to(torch.float8_e4m3fn), s


def _held(c, x):
    return _quantise(x) if c["cache"] == "e4m3" else (x, None)


def _rows_of(held):
    x, s = held
    return x if s is None else torch.ldexp(x.float(), s).to(torch.bfloat16)


def _weights(c, q, k, first, slopes):
    """Softmax weights of q [n, kv, G, D] over rows k [n, kv, rows, D]: of positions
    0 .., the last being the step's own."""
    s = (q @ k.float().transpose(2, 3)) * (D ** -0.5)
    if c["cap"]:
        s = c["cap"] * torch.tanh(s / c["cap"])
    dist = first - torch.arange(k.shape[2], device=k.device)
    if slopes is not None:
        s = s - slopes.view(1, k.shape[1], -1, 1) * dist
    if c["window"]:
        hidden = (dist >= c["window"]) & (first - dist >= c["prefix"])
        s = s.masked_fill(hidden, -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    return p / p.sum(-1, keepdim=True)


def _plain_steps(s):
    c = s.case
    out = torch.empty_like(s.q)
    kv, group = c["kv_heads"], c["q_heads"] // c["kv_heads"]
    totals = [None] * c["batch"]
    for at, K, V in s.groups:
        n, rows = len(at), s.lens[at[0]]
        total = torch.zeros(n, c["layers"], kv, rows, device=out.device)
        for l in range(c["layers"]):
            k = _rows_of(tuple(None if x is None else x[:, l] for x in K))
            v = _rows_of(tuple(None if x is None else x[:, l] for x in V))
            for t in range(c["steps"]):
                new = [_rows_of(_held(c, x[t, l, at])).view(n, kv, 1, D) for x in (s.k, s.v)]
                k, v = torch.cat([k, new[0]], 2), torch.cat([v, new[1]], 2)
                q = s.q[t, l, at].float().view(n, kv, group, D)
                p = _weights(c, q, k, rows + t, s.slopes)
                out[t, l, at] = (p @ v.float()).reshape(n, -1, D).to(out.dtype)
                if c["kind"] == "weighed":
                    total[:, l] += p.sum(2)[..., :rows]
        for j, i in enumerate(at):
            totals[i] = total[j]
    return [out, totals] if c["kind"] == "weighed" else out


def _plain_event(s):
    c = s.case
    lp, m = c["prompt_lo"], c["extra"]
    outs = []
    for k, v, w in s.inputs:
        n = w.shape[2]
        score = w[:, :, lp:n - c["recent"]]
        gone = torch.sort(score, dim=2, stable=True).indices[:, :, :m] + lp
        keep = torch.ones(w.shape, dtype=torch.bool, device=w.device).scatter_(2, gone, False)
        at = keep.nonzero()[:, 2].view(c["layers"], c["kv_heads"], n - m)
        head = torch.arange(c["layers"] * c["kv_heads"], device=w.device)[:, None] * n
        flat = (at.view(-1, n - m) + head).flatten()
        outs.append([at.to(torch.int32), k.view(-1, D)[flat].view(*at.shape, D),
                     v.view(-1, D)[flat].view(*at.shape, D), w.flatten()[flat].view(at.shape)])
    return outs


# ---- the framework's calls ------------------------------------------------------------

def _cache_dtype(ra, c):
    return {"f32": ra.RA_F32, "bf16": ra.RA_BF16, "e4m3": ra.RA_E4M3}[c["cache"]]


def _own_rotate_state(s):
    from paper_2609_03430_amd import binding as ra
    c = s.case
    s.ra = ra
    s.rotary = ra.make_rotary(
        c["base"], dims=c["dims"],
        pairs=ra.RA_PAIRS_HALVES if c["pairs"] == "halves" else ra.RA_PAIRS_ADJACENT,
        scaling={"none": ra.RA_ROTARY_PLAIN, "linear": ra.RA_ROTARY_LINEAR,
                 "rotations": ra.RA_ROTARY_ROTATIONS,
                 "channels": ra.RA_ROTARY_CHANNELS}[c["scaling"]],
        factor=c["factor"], low=c["low"], high=c["high"], original_len=c["original_len"],
        magnitude=c["magnitude"])
    s.out = [torch.empty_like(x) for x in s.x]
    if c["what"] == "step":
        # the generated rows are evicted down to a few: a long generation's cache
        cfg = ra.make_config(1, c["q_heads"], c["kv_heads"], 64, recent_r=0, evict_every=1024,
                             dtype=_cache_dtype(ra, c), max_seqs=c["batch"])
        s.cache = ra.Cache(cfg, ra.ra_required_slots(cfg, [1] * c["batch"]))
        for i, n in enumerate(s.made):
            ra.ra_seq_begin(s.cache.handle, i, 1, 1, i)
            ra.ra_seq_fast_forward(s.cache.handle, i, n)


def _open_cache(s, keep, recent, every):
    from paper_2609_03430_amd import binding as ra
    c = s.case
    s.ra = ra
    cfg = ra.make_config(
        c["layers"], c["q_heads"], c["kv_heads"], keep, recent_r=recent, evict_every=every,
        dtype=_cache_dtype(ra, c), max_seqs=c["batch"],
        layout=ra.RA_LAYOUT_PAGED if c["layout"] == "paged" else ra.RA_LAYOUT_CHRONOLOGICAL,
        page_rows=c["page_rows"], max_prompt_len=max(s.lens))
    s.cache = ra.Cache(cfg, ra.ra_required_slots(cfg, s.lens))
    if c["kind"] != "biased":
        s.cache.attach_weights(max(s.lens))


def _own_steps_state(s, seed):
    c = s.case
    # nothing generated is kept past the pass: the event of its last step drops it
    _open_cache(s, 0, 0, c["steps"])
    ra = s.ra
    s.rule = ra.make_score_rule(cap=c["cap"], slopes=s.slopes, window=c["window"],
                                prefix=c["prefix"])
    s.out = torch.zeros_like(s.q)
    s.calls = [[(l, s.q[t, l], s.k[t, l], s.v[t, l], s.out[t, l]) for l in range(c["layers"])]
               for t in range(c["steps"])]
    for i, n in enumerate(s.lens):
        k, v = (_keys(c, seed, i, n, w) for w in (0, 1))
        ra.ra_seq_begin(s.cache.handle, i, n, int(seed) & 0xFFFFFFFF, i, k, v)
    if c["kind"] == "weighed":
        s.totals = [torch.empty(c["layers"], c["kv_heads"], n, device=_device()) for n in s.lens]
    # a pass makes the same steps again: where the rule reads positions, its first one is
    # given the slots' records (of steps made) as they are now
    s.records = s.cache.meta.clone() if c["slopes"] or c["window"] else None
    s.graph = None
    if c["graph"]:
        ra.ra_graph_mode(s.cache.handle, True)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        s.graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            _own_steps(s)
            with torch.cuda.graph(s.graph, stream=side):
                _own_steps(s)
        torch.cuda.current_stream().wait_stream(side)


def _own_steps(s):
    for step in s.calls:
        for l, q, k, v, out in step:
            s.cache.decode_biased(l, s.rule, q, k, v, out)
        s.ra.ra_end_step(s.cache.handle)


def _own_event_state(s, seed):
    c = s.case
    _open_cache(s, c["keep"], c["recent"], 64)
    kept = c["prompt_lo"] + c["keep"] + c["recent"]
    shape = (c["layers"], c["kv_heads"], kept)
    s.back = [[torch.empty(shape, dtype=torch.int32, device=_device()),
               torch.empty(*shape, D, dtype=_dtype(c), device=_device()),
               torch.empty(*shape, D, dtype=_dtype(c), device=_device()),
               torch.empty(shape, device=_device())] for _ in s.inputs]


def _own_event(s):
    ra, c, h = s.ra, s.case, s.cache.handle
    made = c["keep"] + c["recent"] + c["extra"]
    for i, ((k, v, w), (pos, k_out, v_out, w_out)) in enumerate(zip(s.inputs, s.back)):
        ra.ra_seq_begin(h, i, c["prompt_lo"], 1, i)
        ra.ra_seq_fast_forward(h, i, made)
        ra.ra_write_rows(h, i, k, v)
        ra.ra_write_weights(h, i, w)
        ra.ra_evict_now(h, i)
        ra.ra_export_positions(h, i, pos)
        ra.ra_export_rows(h, i, k_out, v_out)
        ra.ra_export_weights(h, i, w_out)
        ra.ra_seq_end(h, i)
    return s.back


def _own_run(s):
    c, ra = s.case, s.ra
    if c["kind"] == "rotate":
        if c["what"] == "step":
            ra.ra_rotate_step(s.cache.handle, s.rotary, s.x[0], s.x[1], s.out[0], s.out[1])
        else:
            ra.ra_rotate_rows(s.rotary, s.x[0], s.out[0], first=c["far"], positions=s.positions)
        return s.out
    if c["kind"] == "event":
        return _own_event(s)
    if s.records is not None:
        s.cache.meta.copy_(s.records)
    if s.graph is not None:
        s.graph.replay()
        return s.out
    if c["kind"] == "weighed":
        s.cache.weights.zero_()
    _own_steps(s)
    if c["kind"] == "biased":
        return s.out
    for i, w in enumerate(s.totals):
        ra.ra_export_weights(s.cache.handle, i, w)
    return [s.out, s.totals]


def run(state):
    s = state
    c = s.case
    if own:
        return _own_run(s)
    if c["kind"] == "rotate":
        if c["what"] == "step":
            return [_rotated(c, x, s.positions[:, None]) for x in s.x]
        at = s.positions
        if at is None:
            at = torch.arange(c["far"], c["far"] + c["rows"], device=s.x[0].device)
        return [_rotated(c, s.x[0], at)]
    if c["kind"] == "event":
        return [[pos, *([_rows_of(_held(c, x)) for x in rows]), w]
                for pos, *rows, w in _plain_event(s)]
    return _plain_steps(s)


# ---- the definition in 64 bits ----------------------------------------------------------

def _exact_rows(x):
    """Rows [..., D] as an 8-bit cache holds them, in 64 bits: the nearest of the E4M3
    grid, whose step at |y| is 2^(floor(log2 |y|) - 3) and 2^-9 at the least."""
    x = x.double()
    amax = x.abs().amax(-1, keepdim=True)
    s = torch.ceil(torch.log2(torch.clamp(amax, min=2.0 ** -200) / 448.0))
    s = torch.where(torch.exp2(s) * 448.0 < amax, s + 1, s)          # log2 rounded down
    s = torch.where(torch.exp2(s - 1) * 448.0 >= amax, s - 1, s)     # or up
    s = s.clamp(min=-126.0)
    y = x * torch.exp2(-s)
    step = torch.exp2(torch.floor(torch.log2(torch.clamp(y.abs(), min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * torch.exp2(s)


def _exact_angles(c, positions):
    """Angles [.., dims / 2] of whole positions, one pair at a time."""
    angles = []
    for i in range(c["dims"] // 2):
        f = math.exp(-2.0 * i / c["dims"] * math.log(c["base"]))
        blend = 1.0
        if c["scaling"] == "linear":
            blend = 0.0
        elif c["scaling"] == "rotations":
            turns = c["original_len"] * f / math.tau
            blend = min(1.0, max(0.0, (turns - c["low"]) / (c["high"] - c["low"])))
        elif c["scaling"] == "channels":
            edge = [c["dims"] / 2 * (math.log(c["original_len"] / math.tau / n) /
                                     math.log(c["base"])) for n in (c["high"], c["low"])]
            a, b = max(0, math.floor(edge[0])), min(c["dims"] - 1, math.ceil(edge[1]))
            blend = 1.0 - min(1.0, max(0.0, (i - a) / max(b - a, 1e-3)))
        f = blend * f + (1.0 - blend) * f / c["factor"]
        angles.append(torch.remainder(positions.double() * f, math.tau))
    return torch.stack(angles, -1)


def _exact_rotated(c, x, positions):
    x = x.double()
    z = torch.polar(torch.tensor(c["magnitude"], dtype=torch.float64, device=x.device),
                    _exact_angles(c, positions))
    half = c["dims"] // 2
    head, rest = x[..., :c["dims"]], x[..., c["dims"]:]
    if c["pairs"] == "halves":
        turned = torch.complex(head[..., :half].contiguous(), head[..., half:].contiguous()) * z
        head = torch.cat([turned.real, turned.imag], -1)
    else:
        turned = torch.view_as_complex(head.contiguous().view(*head.shape[:-1], half, 2)) * z
        head = torch.view_as_real(turned).flatten(-2)
    return torch.cat([head, rest], -1)


def _exact_steps(c, seed):
    lens = _lengths(c)
    if c["layers"] * c["kv_heads"] * c["steps"] * c["batch"] > 6000:
        return None                      # a dozen launches for each head: too long
    stored = _exact_rows if c["cache"] == "e4m3" else torch.Tensor.double
    group = c["q_heads"] // c["kv_heads"]
    q, k_new, v_new = _step_inputs(c, seed)
    slopes = _slopes(c).double() if c["slopes"] else None
    out = torch.empty(q.shape, dtype=torch.float64, device=_device())
    totals = []
    for i, n in enumerate(lens):
        K, V = _keys(c, seed, i, n, 0), _keys(c, seed, i, n, 1)
        total = torch.zeros(c["layers"], c["kv_heads"], n, dtype=torch.float64, device=_device())
        for l in range(c["layers"]):
            for g in range(c["kv_heads"]):
                k = torch.cat([stored(K[l, g]), stored(k_new[:, l, i, g])])
                v = torch.cat([stored(V[l, g]), stored(v_new[:, l, i, g])])
                mine = slice(g * group, (g + 1) * group)
                for t in range(c["steps"]):
                    at = n + t                                    # the step's position
                    rows = torch.arange(at + 1, device=k.device)
                    if c["window"]:
                        rows = rows[(rows > at - c["window"]) | (rows < c["prefix"])]
                    z = q[t, l, i, mine].double() @ k[rows].T / math.sqrt(D)
                    if c["cap"]:
                        z = torch.tanh(z / c["cap"]) * c["cap"]
                    if slopes is not None:
                        z = z + slopes[mine, None] * (rows - at)
                    p = torch.softmax(z, -1)
                    out[t, l, i, mine] = p @ v[rows]
                    old = rows < n
                    total[l, g, rows[old]] += p[:, old].sum(0)
        totals.append(total)
    return [out, totals] if c["kind"] == "weighed" else out


def exact(case, seed):
    c = case
    if c["kind"] in ("biased", "weighed"):
        return _exact_steps(c, seed)
    if c["kind"] == "event":
        stored = _exact_rows if c["cache"] == "e4m3" else torch.Tensor.double
        outs = []
        for i in range(c["batch"]):
            k, v, w = _event_inputs(c, seed, i)
            lp, n = c["prompt_lo"], w.shape[2]
            kept = []
            for row in w.flatten(0, 1).cpu().tolist():
                among = sorted(range(lp, n - c["recent"]), key=lambda j: (row[j], j))
                gone = set(among[:c["extra"]])
                kept.append([j for j in range(n) if j not in gone])
            at = torch.tensor(kept, device=w.device).view(c["layers"], c["kv_heads"], -1)
            rows = [torch.take_along_dim(x, at[..., None], 2) for x in (k, v)]
            outs.append([at.to(torch.int32), *(stored(x) for x in rows),
                         torch.take_along_dim(w, at, 2).double()])
        return outs
    if c["what"] == "step":
        g = _gen(seed, 3)
        at = torch.tensor([n + 1 for n in _steps_made(c, seed)], device=_device())[:, None]
        return [_exact_rotated(c, torch.randn(c["batch"], h, D, generator=g, device=_device())
                               .to(_dtype(c)), at) for h in (c["q_heads"], c["kv_heads"])]
    x = _keys(c, seed, 0, c["rows"], 0).view(-1, c["rows"], D)
    at = (_row_positions(c, seed) if c["spread"] > 1
          else torch.arange(c["far"], c["far"] + c["rows"], device=x.device))
    return [_exact_rotated(c, x, at)]
