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


def test_pages_whose_bytes_32_bits_count():
    """CPU only: a page of 2^25 tokens has more than 4 GiB a head, which the attention would read in the wrong places."""
    def pool(tokens, dtype=sc.SC_DTYPE_FP4):
        return sc.sc_cache_pool_bytes(1, 1, 128, tokens, 1, 1, dtype)
    assert pool(1 << 24) == (1 << 24) // 32 * 4352 and pool(1 << 25, sc.SC_DTYPE_BF16) == 512 << 25
    for tokens in ((1 << 24) + 8, 1 << 25, (1 << 31) - 8):
        assert pool(tokens) == 0
        with pytest.raises(sc.ScError) as e:
            sc.sc_cache_create(1 << 20, 1, 1, 128, tokens, 1, 1, sc.SC_DTYPE_FP4)
        assert e.value.code == sc.SC_EUNSUPPORTED


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
