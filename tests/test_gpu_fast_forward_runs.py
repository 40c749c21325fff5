"""A fast forward over many triggers, whose launches run from event to event, against the same
steps in fast forwards of a few: slots of different lengths and phases, in the layouts and
sizes whose events are launched one by one."""

import numpy as np
import pytest

from paper_2609_03430_amd import binding as B

pytestmark = pytest.mark.gpu
CHRON, HOLE, PAGED = B.RA_LAYOUT_CHRONOLOGICAL, B.RA_LAYOUT_HOLE_FILL, B.RA_LAYOUT_PAGED


def _state(c, slots):
    out = []
    for s in slots:
        i = B.ra_get_seq_info(c.handle, s)
        out.append((i.len, i.step, i.event))
        for l in range(2):
            for g in range(2):
                out.append(B.ra_read_positions(c.handle, s, l, g, i.len).tolist())
    return out


@pytest.mark.parametrize("layout,K,policy", [
    (HOLE, 200, B.RA_POLICY_RANDOM), (HOLE, 700, B.RA_POLICY_SHARED),
    (PAGED, 300, B.RA_POLICY_RANDOM), (CHRON, 9300, B.RA_POLICY_RANDOM),
    (CHRON, 500, B.RA_POLICY_EXTERNAL)])
def test_one_call_or_many(layout, K, policy):
    lps, r, every = [40, 0, 129], 16, 32
    steps = 450 if policy == B.RA_POLICY_EXTERNAL else K + r + 7 * every + 5
    got = []
    for part in (steps, 23):
        cfg = B.make_config(2, 4, 2, K, r, every, layout=layout, policy=policy, max_seqs=3,
                            max_prompt_len=max(lps))
        c = B.Cache(cfg, B.ra_required_slots(cfg, lps))
        for s, lp in enumerate(lps):
            B.ra_seq_begin(c.handle, s, lp, 3, s)
        B.ra_seq_fast_forward(c.handle, 1, 50)              # phases of their own
        B.ra_seq_fast_forward(c.handle, 2, 9)
        for at in range(0, steps, part):
            B.ra_fast_forward(c.handle, min(part, steps - at))
        got.append(_state(c, range(3)))
        c.close()
    assert got[0] == got[1]
    events = [x[2] for x in got[0] if isinstance(x, tuple)]
    assert (events == [0, 0, 0]) == (policy == B.RA_POLICY_EXTERNAL), events
    if policy != B.RA_POLICY_EXTERNAL:
        assert min(events) >= 6
    for x in got[0]:
        assert isinstance(x, tuple) or len(set(x)) == len(x) and np.min(x or [0]) >= 0
