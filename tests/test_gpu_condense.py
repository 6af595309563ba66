"""Cache.condense against a sort: the numbers each head keeps, and the pages and
weights gathered by them, bit for bit.  Ties, zeros, infinities and NaN among the
weights, one source and many, sources in any order, layers of their own, the
ways a head's weights are held, and rolling one memory state forward."""
import pytest
import torch

import paper_2609_22283_amd as sc

from memory_cases import MemCache

pytestmark = pytest.mark.gpu


def _want(case, w, sources, layer):
    """[heads, n] numbers kept, ascending: by weight descending, then by number."""
    flat = torch.stack([w[layer, slot] for s in sources for slot in case.cache.slots(s)], 1).flatten(1).double()
    flat = torch.where(torch.isnan(flat), torch.full_like(flat, -float("inf")), flat)
    nan = torch.stack([w[layer, slot] for s in sources for slot in case.cache.slots(s)], 1).flatten(1).isnan()
    order = torch.sort(flat, dim=-1, descending=True, stable=True).indices
    # NaN after -inf
    rank = torch.gather(nan.to(torch.int64), -1, order)
    order = torch.gather(order, -1, torch.sort(rank, dim=-1, stable=True).indices)
    return order[:, :case.n].sort(-1).values


def _check(case, w, sources, into, layer=0, n_layers=1):
    before, pool = w.clone(), case.pool.clone()
    kept = torch.full((n_layers, case.heads, case.n), -1, dtype=torch.int32, device="cuda")
    case.cache.condense(layer, n_layers, sources, into, w, kept)
    torch.cuda.synchronize()
    dst = case.cache.slots(into)
    for l in range(layer, layer + n_layers):
        want = _want(case, before, sources, l)
        assert torch.equal(kept[l - layer].long(), want)
        k = torch.cat([case.kv[s][l][0] for s in sources]).transpose(0, 1)  # [heads, N, d]
        v = torch.cat([case.kv[s][l][1] for s in sources]).transpose(0, 1)
        pick = want[..., None].expand(-1, -1, case.hd)
        gk, gv = case.pages(into, l)
        bits = torch.int16 if case.dtype == "bf16" else torch.int32
        assert torch.equal(gk.view(bits), torch.gather(k, 1, pick).transpose(0, 1).contiguous().view(bits))
        assert torch.equal(gv.view(bits), torch.gather(v, 1, pick).transpose(0, 1).contiguous().view(bits))
        flat = torch.stack([before[l, slot] for s in sources for slot in case.cache.slots(s)], 1).flatten(1)
        ww = torch.gather(flat, -1, want).view(case.heads, case.ppc, case.tpp).transpose(0, 1)
        assert torch.equal(w[l, dst].view(torch.int32), ww.contiguous().view(torch.int32))
        assert case.cache.contains(into, l)
    # nothing else is written
    rest = torch.ones(w.shape[:2], dtype=torch.bool, device="cuda")
    rest[layer:layer + n_layers, dst] = False
    assert torch.equal(w[rest].view(torch.int32), before[rest].view(torch.int32))
    per = case.pool.view(case.layers, case.n_slots, -1)
    assert torch.equal(per[rest], pool.view(case.layers, case.n_slots, -1)[rest])
    return kept


CASES = [  # dtype, heads, head dim, tokens per page, pages per state, sources, layers
    ("bf16", 2, 128, 8, 1, 2, 1),
    ("bf16", 3, 128, 72, 2, 1, 2),        # one source: a copy
    ("bf16", 12, 128, 64, 1, 21, 3),
    ("bf16", 12, 128, 64, 1, 3, 30),      # few tokens, more work-groups than run at once
    ("bf16", 2, 64, 104, 3, 5, 1),
    ("f32", 2, 64, 104, 3, 2, 1),
    ("f32", 1, 128, 40, 1, 7, 2),
    ("bf16", 2, 128, 1560, 3, 1, 1),      # 4680 tokens: 8 of a thread's of 1024
    ("bf16", 2, 128, 1560, 3, 3, 1),      # 14040 tokens: 16
    ("bf16", 1, 128, 1560, 3, 8, 1),      # 37440 tokens: 40
    ("bf16", 1, 128, 1560, 3, 9, 1),      # 42120 tokens: read again in each pass
]


@pytest.mark.parametrize("kind", ["tail", "ties"])
@pytest.mark.parametrize("dtype,heads,hd,tpp,ppc,sources,layers", CASES)
def test_condense(dtype, heads, hd, tpp, ppc, sources, layers, kind):
    states = [(c, 1) for c in range(sources)]
    case = MemCache(dtype, heads, hd, tpp, ppc, states, layers=layers, seed=101)
    w = torch.exp(2.0 * case.normal((layers, case.n_slots, heads, tpp)))
    if kind == "ties":  # few distinct values, zeros of both signs among them
        w = torch.round(w.clamp_max(3.0)) * torch.where(case.normal(w.shape) > 0, 1.0, -1.0)
    _check(case, w, states[::-1], (9, 0), 0, layers)


def test_condense_odd_weights():
    """All equal; infinities and NaN; the smallest and largest numbers."""
    states = [(c, 0) for c in range(4)]
    special = torch.tensor([float("nan"), float("inf"), -float("inf"), 0.0, -0.0, 1e-45, -1e-45, 3e38, -3e38, 1.0],
                           device="cuda")
    for which in range(3):
        case = MemCache("bf16", 2, 128, 40, 2, states, seed=102)
        shape = (1, case.n_slots, 2, 40)
        w = torch.zeros(shape, device="cuda") if which == 0 else \
            special[torch.randint(0, 10, shape, generator=case.gen, device="cuda")]
        if which == 2:
            w = torch.where(case.normal(shape) > -1.0, torch.full_like(w, float("nan")), w)
        _check(case, w, states, (7, 7))


def test_condense_some_layers_then_the_rest():
    states = [(0, 0), (1, 0), (2, 0)]
    case = MemCache("bf16", 2, 128, 64, 1, states, layers=4, seed=103)
    w = case.weights()
    _check(case, w, states, (5, 0), 1, 2)
    assert not case.cache.contains((5, 0), 0) and not case.cache.contains((5, 0), 3)
    with pytest.raises(sc.ScError) as e:
        case.cache.condense(2, 2, states, (5, 0), w, torch.empty((2, 2, 64), dtype=torch.int32, device="cuda"))
    assert e.value.code == sc.SC_EEXIST
    _check(case, w, states, (5, 0), 0, 1)
    _check(case, w, states, (5, 0), 3, 1)


def test_condense_captured():
    """Captured and replayed: each replay folds by the weights that it finds."""
    states = [(c, 0) for c in range(3)]
    case = MemCache("bf16", 2, 128, 72, 2, states, layers=2, seed=105)
    w = case.weights()
    kept = torch.empty((2, 2, case.n), dtype=torch.int32, device="cuda")
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        case.cache.condense(0, 2, states, (3, 0), w, kept)
    for _ in range(3):
        w.copy_(torch.exp(case.normal(w.shape)))
        before = w.clone()
        g.replay()
        torch.cuda.synchronize()
        for l in range(2):
            want = _want(case, before, states, l)
            assert torch.equal(kept[l].long(), want)
            k, v = (torch.cat([case.kv[s][l][i] for s in states]).transpose(0, 1) for i in (0, 1))
            pick = want[..., None].expand(-1, -1, 128)
            gk, gv = case.pages((3, 0), l)
            assert torch.equal(gk, torch.gather(k, 1, pick).transpose(0, 1))
            assert torch.equal(gv, torch.gather(v, 1, pick).transpose(0, 1))


def test_rolling_memory():
    """The operators together: a window weighed, its oldest states folded into the memory,
    the memory read by the next pack as a shared prefix, and weighed in turn; slots
    freed by the fold are used again."""
    H, tpp, W = 3, 64, 2
    case = MemCache("bf16", H, 128, tpp, 1, [(c, 0) for c in range(W + 1)], spare=2, seed=104)
    w = torch.zeros((1, case.n_slots, H, tpp), device="cuda")
    memory = None
    for c in range(W, 7):
        if c > W:
            k, v = (case.normal((tpp, H, 128)).to(torch.bfloat16) for _ in range(2))
            case.cache.append(0, (c, 0), k, v)
            case.cache.weights_clear((c, 0), w)
            case.kv[(c, 0)] = [(k, v)]
        plan = sc.sc_plan_build(sc.sc_selection_build("clean", 4, W, [(c, 0)]), case.cache)
        reads = [(c - r, 0) for r in range(W, -1, -1)]
        if memory is not None:
            plan = sc.sc_plan_share(plan, [memory])
            reads = [memory] + reads
        q = case.queries(tpp)
        nb = sc.sc_attention_weigh_workspace_bytes(plan, case.cache)
        ws, o = torch.empty(nb, dtype=torch.uint8, device="cuda"), torch.empty_like(q)
        before = w.clone()
        sc.sc_attention_weigh(plan, case.cache, 0, q, o, 128 ** -0.5, w, ws, nb)
        torch.cuda.synchronize()
        want, sums = case.attend(q, [reads], 128 ** -0.5)
        exp = case.weights_after(before, sums)
        assert float((o.double() - want).norm() / want.norm()) < 1e-2
        assert float((w.double() - exp).abs().max()) < 1e-4
        old = (c - W, 0)
        sources = [old] if memory is None else [memory, old]
        into = (c - W, 1)
        kept = _check(case, w, sources, into)
        k, v = case.pages(into)
        case.kv[into] = [(k.clone(), v.clone())]
        assert kept.shape == (1, H, tpp)
        for s in sources:
            case.cache.release(s)
        memory = into
    assert case.cache.free_slot_count() == case.n_slots - W - 1
