"""Steps that mix dense and block-sparse layers on the GPU while sequences of very
different lengths come and go: every active sequence has its output and its appended
row at every layer."""

import numpy as np
import pytest

from blocks_harness import Run8, check_step, oracle_of, sparse_step
from gpu_harness import Run, check_heads, log
from paper_2609_03430_amd import binding as B

pytestmark = pytest.mark.gpu
CHRON, PAGED = B.RA_LAYOUT_CHRONOLOGICAL, B.RA_LAYOUT_PAGED
BF16, E4M3 = B.RA_BF16, B.RA_E4M3


def _run(dtype, **kw):
    run = Run8(begin=False, **kw) if dtype == E4M3 else Run(dtype=dtype, begin=False, **kw)
    run.active = set()
    run.cache.attach_sparse(8)
    run.cache.bounds.fill_(0x55)
    return run


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("layout", [CHRON, PAGED])
@pytest.mark.parametrize("first,then", [
    ([0, 1], [2, 3]),        # admitted into slots past those of the step before
    ([1, 3], [0, 2]),        # .. and before and between them
])
def test_admitted_between_a_sparse_first_and_a_dense_first_step(first, then, layout, dtype):
    run = _run(dtype, L=3, Hq=6, Hkv=2, K=64, lps=[300, 40, 700, 0], r=16, every=64, layout=layout,
               page_rows=32, max_seqs=4)
    oracles = {}

    def admit(slots):
        for s in slots:
            run.begin(s)
            oracles[s] = oracle_of(run, s)

    def step(layers):
        outs, _ = sparse_step(run, 2, 16, layers)
        check_step(run, list(oracles.values()), outs, (sorted(oracles), layers), (2, 16, layers))
    admit(first)
    step({0, 1, 2})                       # the order of the two slots is made here
    admit(then)
    step({1})                             # dense, sparse, dense
    step({1, 2})
    run.end(first[0])                     # one slot given to another sequence
    oracles.pop(first[0])
    run.lps[first[0]], run.rids[first[0]] = 13, 40
    admit([first[0]])
    step({2})
    step({0, 2})
    check_heads(run, list(oracles.values()))
    run.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("layout", [CHRON, PAGED])
def test_slots_change_under_mixed_steps(layout, dtype):
    """Any mix of layers from step to step, events among them, sequences of 0 to 500
    prompt rows ended and admitted."""
    run = _run(dtype, L=3, Hq=4, Hkv=1, K=60, lps=[0] * 5, r=8, every=12, layout=layout,
               page_rows=64, max_seqs=5, max_prompt_len=500, pool_rows=64 * 3 * 60)
    rng = np.random.default_rng(23)
    rep, rid, events, admitted = {}, 100, 0, 0
    for t in range(120):
        free = [s for s in range(5) if s not in rep]
        if free and (len(rep) < 2 or rng.random() < 0.3):
            s = int(rng.choice(free))
            run.lps[s], run.rids[s] = int(rng.choice([0, 1, 33, 200, 500])), rid
            rid += 1
            run.begin(s)
            rep[s] = oracle_of(run, s)
            admitted += 1
        elif len(rep) > 2 and rng.random() < 0.2:
            s = int(rng.choice(sorted(rep)))
            run.end(s)
            rep.pop(s)
        layers = {l for l in range(3) if rng.random() < 0.5}
        log("mixed step %d: slots %s, sparse layers %s" % (t, sorted(rep), sorted(layers)))
        outs, evicted = sparse_step(run, 3, 8, layers)
        check_step(run, list(rep.values()), outs, (t, sorted(layers)), (3, 8, layers))
        events += evicted
    check_heads(run, list(rep.values()))
    assert events >= 5 and admitted >= 10
    run.close()
