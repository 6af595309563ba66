"""What a plan whose pages have gone may still be asked (CPU only): a cache moves to a pool of fewer slots,
and plans over the old slots live on."""
import pytest

import paper_2609_22283_amd as sc
from paper_2609_22283_amd.binding import sc_attention_form

PAGES = 700


def _plan(dtype, tpp=64, shared=0, nq=4096):
    """A plan over 700 pages, of nodes so long that 4-bit pages would be taken out as bf16 first"""
    cache = sc.sc_cache_create(1 << 20, 1, 2, 128, tpp, 50, PAGES, dtype)
    states = [(c, 1) for c in range(PAGES // 50)]
    # reserves the states' slots: nothing is launched
    sc.sc_plan_build(sc.sc_selection_build("clean", 1, 0, states), cache)
    plan = sc.sc_plan_condition(cache, states[shared:], nq)
    return cache, sc.sc_plan_share(plan, states[:shared]) if shared else plan, states


def _queries(plan, cache):
    return sc.sc_attention_workspace_bytes(plan, cache), sc.sc_attention_weigh_workspace_bytes(plan, cache)


@pytest.mark.parametrize("shared", [0, 3])
@pytest.mark.parametrize("n_slots", [1, 10, PAGES, 5000])
@pytest.mark.parametrize("asked_before", [False, True])
def test_a_plan_from_before_a_move(shared, n_slots, asked_before):
    cache, plan, states = _plan(sc.SC_DTYPE_FP4, shared=shared)
    if asked_before:
        assert sc.sc_attention_workspace_bytes(plan, cache) > 0 and sc_attention_form(plan, cache)[0] == 0
    for st in states:
        cache.release(st)
    cache.move(1 << 50, n_slots)
    for _ in range(2):
        assert _queries(plan, cache) == (0, 0)
        for ask in (lambda: sc_attention_form(plan, cache), lambda: sc.sc_attention(plan, cache, 0, 64, 64, 1.0),
                    lambda: sc.sc_attention_noalloc(plan, cache, 0, 64, 64, 1.0)):
            with pytest.raises(sc.ScError) as e:
                ask()
            assert e.value.code == sc.SC_ESTALE


@pytest.mark.parametrize("gone", [0, 7])
def test_a_plan_over_a_released_state(gone):
    cache, plan, states = _plan(sc.SC_DTYPE_FP4, shared=3)
    cache.release(states[gone])
    assert _queries(plan, cache) == (0, 0)
    with pytest.raises(sc.ScError) as e:
        sc_attention_form(plan, cache)
    assert e.value.code == sc.SC_ESTALE


@pytest.mark.parametrize("dtype", [sc.SC_DTYPE_BF16, sc.SC_DTYPE_F32])
@pytest.mark.parametrize("shared", [0, 3])
def test_other_caches_answer_as_before(dtype, shared):
    """The size of what a plan over bf16 or fp32 pages needs does not depend on them."""
    cache, plan, states = _plan(dtype, shared=shared)
    want, form = _queries(plan, cache), sc_attention_form(plan, cache)
    fresh = _plan(dtype, shared=shared)
    for st in states:
        fresh[0].release(st)
    fresh[0].move(1 << 50, 1)
    assert _queries(fresh[1], fresh[0]) == want and sc_attention_form(fresh[1], fresh[0]) == form
    with pytest.raises(sc.ScError) as e:
        sc.sc_attention(fresh[1], fresh[0], 0, 64, 64, 1.0, 64, 1 << 40)
    assert e.value.code == sc.SC_ESTALE
