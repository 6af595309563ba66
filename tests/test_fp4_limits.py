"""The largest plans over 4-bit pages, 64 nodes and 800 pages: they run, and larger ones are refused."""
import pytest

import paper_2609_22283_amd as sc
from paper_2609_22283_amd.binding import sc_attention_form

# prefix states (a page each), nodes
FULL = [(799, 1), (736, 64)]


@pytest.mark.parametrize("prefix,nodes", FULL + [(800, 1), (737, 64), (3, 65)])
@pytest.mark.parametrize("nq", [1, 2048])
def test_what_is_planned(prefix, nodes, nq):
    """CPU only: nothing is launched."""
    cache = sc.sc_cache_create(1 << 20, 1, 1, 128, 64, 1, prefix + nodes, sc.SC_DTYPE_FP4)
    for first in range(0, prefix + nodes, 50):  # reserves the states' slots
        pack = [(c, 1) for c in range(first, min(first + 50, prefix + nodes))]
        sc.sc_plan_build(sc.sc_selection_build("clean", 1, 0, pack), cache)
    own = [(prefix + i, 1) for i in range(nodes)]
    plan = sc.sc_plan_share(sc.sc_plan_condition(cache, own, nq), [(c, 1) for c in range(prefix)])
    if (prefix, nodes) in FULL:
        assert sc_attention_form(plan, cache)[0] in (0, 16, 32) and sc.sc_attention_workspace_bytes(plan, cache) >= 0
        return
    with pytest.raises(sc.ScError) as e:
        sc_attention_form(plan, cache)
    assert e.value.code == sc.SC_EUNSUPPORTED and sc.sc_attention_workspace_bytes(plan, cache) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("prefix,nodes", FULL)
@pytest.mark.parametrize("nq", [1, 40])
def test_the_largest_plans(prefix, nodes, nq):
    from fp4_cases import Held, attend, check, condition_plan, oracle
    pre, own = [(c, 0) for c in range(prefix)], [(prefix + i, 0) for i in range(nodes)]
    h = Held(1, 32, 1, pre + own, seed=81)
    plan = condition_plan(h, pre, own, nq)
    qd, q = h.queries(nodes * nq, 2.0)
    want, tol = oracle(h, [pre + [st] for st in own], q, nq)
    check(attend(h, plan, qd), want, tol)
