"""Host side of the bounded, shared history on the CPU: the plans of sc_plan_share,
sizes, and everything the entry points refuse before they launch (no kernel runs: a
refused call launches nothing; device pointers here are never read)."""
import pytest

import paper_2609_22283_amd as sc

A, B, C, D = (0, 0), (1, 0), (2, 0), (3, 0)
PTR = 1 << 20  # stands for device memory, 16-byte aligned


def _cache(n_slots=16, ppc=2, tpp=64, layers=2, dtype=sc.SC_DTYPE_BF16, hd=128, heads=2):
    return sc.sc_cache_create(PTR, layers, heads, hd, tpp, ppc, n_slots, dtype)


def _reserve(cache, states):
    """Gives states slots (unwritten), in order."""
    return sc.sc_plan_build(sc.sc_selection_build("clean", 4, 0, states), cache)


def _code(fn, *args, **kw):
    with pytest.raises(sc.ScError) as e:
        fn(*args, **kw)
    return e.value.code


def test_share_lists():
    cache = _cache()
    _reserve(cache, [A, B, C, D])
    base = sc.sc_plan_condition(cache, [C, D, C], 5)
    plan = sc.sc_plan_share(base, [B, A])
    off, slots, tokens, frames = plan.tables()
    pre = cache.slots(B) + cache.slots(A)
    assert off == [0, 6, 12, 18]
    assert slots == (pre + cache.slots(C)) + (pre + cache.slots(D)) + (pre + cache.slots(C))
    assert tokens == [64] * 18
    assert frames[:4] == [2, 3, 0, 1]
    assert base.tables()[0] == [0, 2, 4, 6]
    del base
    assert plan.tables()[0] == [0, 6, 12, 18]


def test_share_of_an_empty_pack():
    cache = _cache()
    _reserve(cache, [A])
    empty = sc.sc_plan_build(sc.sc_selection_build("clean", 4, 0, []), cache)
    assert sc.sc_plan_share(empty, [A]).tables() == ([0], [], [], [])


def test_share_refusals():
    cache = _cache()
    _reserve(cache, [A, B, C])
    plan = sc.sc_plan_condition(cache, [C], 3)
    assert _code(sc.sc_plan_share, plan, []) == sc.SC_EINVAL
    assert _code(sc.sc_plan_share, plan, [D]) == sc.SC_ENOTFOUND
    assert _code(sc.sc_plan_share, plan, [A, A]) == sc.SC_EINVAL
    assert _code(sc.sc_plan_share, plan, [A, C]) == sc.SC_EINVAL
    twice = sc.sc_plan_share(plan, [A])
    assert _code(sc.sc_plan_share, twice, [A]) == sc.SC_EINVAL
    assert sc.sc_plan_share(twice, [B]).tables()[1] == cache.slots(B) + cache.slots(A) + cache.slots(C)
    assert sc.lib.sc_plan_share(None, None, 1, None) == sc.SC_EINVAL
    cache.release(A)
    assert _code(sc.sc_attention, twice, cache, 0, PTR, PTR, 0.1, PTR, 1 << 30) == sc.SC_ESTALE


def test_share_limits():
    """800 pages with the prefix counted once, 64 nodes, and rows by partials beyond the lists."""
    cache = _cache(n_slots=900, ppc=1, tpp=32, layers=1)
    states = [(c, 0) for c in range(900)]
    _reserve(cache, states)

    def form(prefix, nodes, nq):
        own = states[prefix:prefix + nodes]
        return sc.sc_attention_form(sc.sc_plan_share(sc.sc_plan_condition(cache, own, nq), states[:prefix]), cache)

    assert form(736, 64, 1)[2] < 0
    assert _code(form, 737, 64, 1) == sc.SC_EUNSUPPORTED
    assert _code(form, 10, 65, 1) == sc.SC_EUNSUPPORTED
    # 32-token pages: more than 64 queries a node need the shared form's partials
    assert form(10, 4, 2000)[2] < 0
    assert _code(form, 10, 4, 20000) == sc.SC_EUNSUPPORTED
    small = _cache(tpp=24, ppc=1)
    _reserve(small, [A, B])
    plan = sc.sc_plan_share(sc.sc_plan_condition(small, [B], 1), [A])
    assert _code(sc.sc_attention_form, plan, small) == sc.SC_EUNSUPPORTED


def test_share_workspace():
    cache = _cache(n_slots=300, ppc=1, layers=1)
    states = [(c, 0) for c in range(300)]
    _reserve(cache, states)
    plan = sc.sc_plan_share(sc.sc_plan_condition(cache, states[290:], 1), states[:290])
    pieces = -sc.sc_attention_form(plan, cache)[2]
    nb = sc.sc_attention_workspace_bytes(plan, cache)
    # partials of at least the prefix's pieces and one of the own pages, per row and head
    assert nb >= (pieces + 1) * 10 * 2 * 130 * 4 and nb % 16 == 0
    f32 = _cache(n_slots=300, ppc=1, layers=1, dtype=sc.SC_DTYPE_F32)
    _reserve(f32, states)
    plan = sc.sc_plan_share(sc.sc_plan_condition(f32, states[290:], 1), states[:290])
    assert sc.sc_attention_workspace_bytes(plan, f32) > 0


def test_weigh_sizes_and_refusals():
    cache = _cache()
    assert sc.sc_cache_weights_bytes(cache) == 2 * 16 * 2 * 64 * 4
    _reserve(cache, [A, B])
    plan = sc.sc_plan_condition(cache, [A, B], 7)
    nb = sc.sc_attention_weigh_workspace_bytes(plan, cache)
    assert nb >= sc.sc_attention_workspace_bytes(plan, cache) + 2 * 7 * 2 * 4
    call = lambda **k: sc.sc_attention_weigh(  # noqa: E731
        plan, k.get("cache", cache), k.get("layer", 0), k.get("q", PTR), PTR, k.get("scale", 0.1),
        k.get("weights", PTR), k.get("ws", PTR), k.get("nb", nb))
    for bad in (dict(q=0), dict(q=PTR + 8), dict(weights=0), dict(scale=float("nan")), dict(scale=float("inf")), dict(layer=2),
                dict(layer=-1), dict(cache=_cache())):
        assert _code(call, **bad) == sc.SC_EINVAL, bad
    assert _code(call) == sc.SC_EUNAVAILABLE  # slots reserved, nothing written
    assert sc.sc_attention_weigh_workspace_bytes(plan, _cache()) == 0
    assert _code(cache.weights_clear, D, PTR) == sc.SC_ENOTFOUND
    assert _code(cache.weights_clear, A, 0) == sc.SC_EINVAL


def test_condense_refusals():
    cache = _cache(n_slots=6)
    _reserve(cache, [A, B])
    call = lambda src, into=C, layer=0, n=1, w=PTR, kept=PTR: cache.condense(layer, n, src, into, w, kept)  # noqa: E731
    assert _code(call, []) == sc.SC_EINVAL
    assert _code(call, [A, A]) == sc.SC_EINVAL
    assert _code(call, [A, C]) == sc.SC_EINVAL
    assert _code(call, [A], (-1, 0)) == sc.SC_EINVAL
    assert _code(call, [A], layer=2) == sc.SC_EINVAL
    assert _code(call, [A], layer=-1) == sc.SC_EINVAL
    assert _code(call, [A], layer=1, n=2) == sc.SC_EINVAL
    assert _code(call, [A], n=0) == sc.SC_EINVAL
    assert _code(call, [A], w=0) == sc.SC_EINVAL
    assert _code(call, [A], kept=0) == sc.SC_EINVAL
    assert _code(call, [D]) == sc.SC_ENOTFOUND
    assert _code(call, [A, B]) == sc.SC_EUNAVAILABLE
    assert cache.free_slot_count() == 2 and not cache.contains(C)
    wide = _cache(n_slots=802, ppc=1, layers=1)
    states = [(c, 0) for c in range(801)]
    _reserve(wide, states)
    assert _code(wide.condense, 0, 1, states[:800], states[800], PTR, PTR) == sc.SC_EUNSUPPORTED


def test_share_own_lists_longer_than_the_prefix():
    """Rows for which two partials each have room and three do not, lists of more than 800
    pages, and own lists twice the prefix's length: one piece of each."""
    cache = _cache(n_slots=400, ppc=40, layers=1, heads=10)
    pack = [(c, 0) for c in range(3, 7)]
    _reserve(cache, [(c, 0) for c in range(9)])
    plan = sc.sc_plan_build(sc.sc_selection_build("clean", 4, 3, pack), cache)
    plan = sc.sc_plan_share(plan, [(7, 0), (8, 0)])
    queries, _, pieces = sc.sc_attention_form(plan, cache)
    assert queries > 0 and pieces == -1
    assert sc.sc_attention_workspace_bytes(plan, cache) == 2 * 4 * 2560 * 10 * 130 * 4
