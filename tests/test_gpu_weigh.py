"""sc_attention_weigh against the formula in 64 bits: outputs and the weight that
every cached key received, added to what the array held.

Packs whose nodes read overlapping windows (pages with one reader and with
several), pages that end inside key tiles, the forms of the attention under it (keys
over waves, 64, 128 and 256 queries, whole and in pieces), single queries, negative
scales and a prefix shared by the pack.  Tolerances: the weights' from the
arithmetic (memory_cases.weight_bound), the outputs' those of the attention."""
import pytest
import torch

import paper_2609_22283_amd as sc

from memory_cases import MemCache, close, weight_bound

pytestmark = pytest.mark.gpu


def _run(case, plan, q, scale, w, layer=0):
    nb = sc.sc_attention_weigh_workspace_bytes(plan, case.cache)
    ws = torch.full((nb,), 0xFF, dtype=torch.uint8, device="cuda")
    o = torch.full_like(q, float("nan"))
    sc.sc_attention_weigh(plan, case.cache, layer, q, o, scale, w, ws, nb)
    torch.cuda.synchronize()
    return o


def _check(case, plan, reads, nq, scale=None, layer=0):
    scale = case.hd ** -0.5 if scale is None else scale
    q = case.queries(len(reads) * nq)
    w = case.weights()
    before = w.clone()
    o = _run(case, plan, q, scale, w, layer)
    want, sums = case.attend(q, reads, scale, layer)
    close(case.dtype, o, want, "o")
    exp = case.weights_after(before, sums, layer)
    keys = max(len(r) for r in reads) * case.n
    tol = weight_bound(case, q, scale, keys) * (exp - before.double()) + exp * 2.0 ** -23
    assert ((w.double() - exp).abs() <= tol).all(), float(((w.double() - exp).abs() / tol.clamp_min(1e-30)).max())
    untouched = exp == before.double()
    assert torch.equal(w[untouched], before[untouched])
    # again, from the same weights: the same bits
    w2 = before.clone()
    o2 = _run(case, plan, q, scale, w2, layer)
    assert torch.equal(w2, w) and torch.equal(o2, o)


def _pack(policy, K, W, nodes, case):
    """Plan of a pack and the states each node reads (all appended)."""
    sel = sc.sc_selection_build(policy, K, W, nodes)
    off, ch, lv, _ = sel.tables()
    reads = [list(zip(ch[off[i]:off[i + 1]], lv[off[i]:off[i + 1]])) for i in range(len(nodes))]
    return sc.sc_plan_build(sel, case.cache), reads


# dtype, heads, head dim, tokens per page, pages per chunk, window, nodes
PACKS = [
    ("bf16", 2, 128, 40, 1, 6, 3),     # keys over waves, pages ending inside tiles
    ("bf16", 12, 128, 64, 1, 20, 1),
    ("bf16", 12, 128, 40, 1, 3, 32),   # 64-query units, many nodes
    ("bf16", 12, 128, 64, 1, 40, 3),   # 64-query units in pieces
    ("bf16", 12, 128, 264, 1, 6, 3),   # 128-query units
    ("bf16", 2, 128, 104, 3, 6, 4),    # 128-query units in pieces
    ("bf16", 7, 128, 600, 2, 3, 5),    # 256-query units
    ("bf16", 3, 128, 600, 2, 1, 3),    # 256-query units in pieces
    ("bf16", 1, 128, 64, 1, 0, 1),     # a node alone with itself
    ("f32", 2, 128, 104, 3, 3, 4),
    ("f32", 3, 64, 8, 1, 5, 2),
    ("f32", 1, 64, 16, 1, 0, 1),
]


@pytest.mark.parametrize("dtype,heads,hd,tpp,ppc,W,nodes", PACKS)
def test_weigh_pack(dtype, heads, hd, tpp, ppc, W, nodes):
    pack = [(W + i, 2) for i in range(nodes)]
    case = MemCache(dtype, heads, hd, tpp, ppc, [(c, 2) for c in range(W + nodes)], seed=71)
    plan, reads = _pack("same", 4, W, pack, case)
    _check(case, plan, reads, case.n)


@pytest.mark.parametrize("nq", [1, 5, 33, 200])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weigh_condition(dtype, nq):
    """Nodes of any number of rows that name one state or several; the second of two layers."""
    case = MemCache(dtype, 3, 128, 72, 2, [(0, 0), (1, 0), (2, 0)], layers=2, seed=72)
    names = [(0, 0), (2, 0), (0, 0), (1, 0)]
    plan = sc.sc_plan_condition(case.cache, names, nq)
    _check(case, plan, [[s] for s in names], nq, layer=1)


@pytest.mark.parametrize("scale", [-0.06, 0.0, 0.2])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weigh_scales(dtype, scale):
    case = MemCache(dtype, 2, 128, 64, 1, [(c, 0) for c in range(5)], seed=73)
    plan, reads = _pack("clean", 4, 4, [(4, 0)], case)
    _check(case, plan, reads, case.n, scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weigh_shared_prefix(dtype):
    """Over a prefix shared by the pack: its pages are weighed by every node."""
    states = [(c, 0) for c in range(12)]
    case = MemCache(dtype, 4, 128, 64, 1, states, seed=74)
    own = states[8:]
    plan = sc.sc_plan_share(sc.sc_plan_condition(case.cache, own, 3), states[:8])
    _check(case, plan, [states[:8] + [s] for s in own], 3)


def test_weigh_many_reader_sets():
    """More than 64 sets of readers and more than 512 pages: several launches."""
    W, nodes = 9, 60
    case = MemCache("bf16", 1, 128, 64, 1, [(c, 1) for c in range(W + nodes)], seed=75)
    pack = [(W + i, 1) for i in range(nodes)]
    plan, reads = _pack("same", 4, W, pack, case)
    assert sum(map(len, reads)) == 600 and len({tuple(i for i, r in enumerate(reads) if s in r) for s in case.kv}) > 64
    _check(case, plan, reads, case.n)
    states = [(c, 0) for c in range(600)]
    case = MemCache("bf16", 1, 128, 64, 1, states, seed=76)
    plan = sc.sc_plan_share(sc.sc_plan_condition(case.cache, states[598:], 2), states[:598])
    _check(case, plan, [states[:598] + [s] for s in states[598:]], 2)


@pytest.mark.parametrize("rising", [False, True])
def test_weigh_far_logits(rising):
    """Logits that rise some 150 log2 units after the first page (the unit forms redo
    their items), or fall: the early or the late keys get no weight."""
    def key_fn(st, k):
        k = k.clone()
        k[:, :, 0] = 1200.0 if (st[0] > 0) == rising else 0.0
        return k

    for heads, tpp, W in ((2, 64, 4), (12, 264, 6)):
        case = MemCache("bf16", heads, 128, tpp, 1, [(c, 0) for c in range(W + 1)], seed=77, key_fn=key_fn)
        plan, reads = _pack("clean", 4, W, [(W, 0)], case)
        scale = 128 ** -0.5
        q = case.queries(case.n)
        q[:, :, 0] = 1.0
        w = torch.zeros_like(case.weights())
        o = _run(case, plan, q, scale, w)
        want, sums = case.attend(q, reads, scale)
        close("bf16", o, want, "o")
        exp = case.weights_after(torch.zeros_like(w), sums)
        assert ((w.double() - exp).abs() <= weight_bound(case, q, scale, (W + 1) * case.n) * exp + 1e-30).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weigh_keys_without_a_finite_logit(dtype):
    """Keys of -inf logits (a channel of -inf against queries of 1) get no weight and change
    nothing, also where they fill whole pages of the prefix and pieces of them."""
    dead = {(c, 0) for c in (0, 1, 2, 5)}

    def key_fn(st, k):
        k = k.clone()
        k[:, :, 3] = -float("inf") if st in dead else 0.0
        return k

    states = [(c, 0) for c in range(10)]
    for nodes, nq in ((1, 64), (4, 2)):
        case = MemCache(dtype, 2, 128, 64, 1, states, seed=78, key_fn=key_fn)
        own = states[10 - nodes:]
        pre = states[:10 - nodes]
        plan = sc.sc_plan_share(sc.sc_plan_condition(case.cache, own, nq), pre)
        q = case.queries(nodes * nq)
        q[:, :, 3] = 1.0
        w = torch.zeros_like(case.weights())
        o = _run(case, plan, q, 0.1, w)
        want, sums = case.attend(q, [pre + [s] for s in own], 0.1)
        close(dtype, o, want, "o")
        for st in dead:
            assert (w[0, case.cache.slots(st)] == 0).all()
        assert abs(float(w.sum()) - 2 * nodes * nq) < 1e-3 * nodes * nq


def test_weigh_captured():
    """Captured and replayed: every replay adds once more, in the same bits as eager calls."""
    case = MemCache("bf16", 3, 128, 72, 2, [(c, 2) for c in range(5)], seed=79)
    plan, _ = _pack("same", 4, 3, [(3, 2), (4, 2)], case)
    q, scale = case.queries(2 * case.n), 128 ** -0.5
    nb = sc.sc_attention_weigh_workspace_bytes(plan, case.cache)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    o, w = torch.empty_like(q), case.weights()
    eager_w = w.clone()
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        sc.sc_attention_weigh(plan, case.cache, 0, q, o, scale, w, ws, nb)
    for _ in range(3):
        want = _run(case, plan, q, scale, eager_w)
        o.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(w, eager_w) and torch.equal(o, want)


def test_weights_clear():
    case = MemCache("bf16", 3, 128, 40, 2, [(0, 0), (1, 0), (2, 0)], layers=3, seed=80)
    w = case.weights()
    want = w.clone()
    want[:, case.cache.slots((1, 0))] = 0
    case.cache.weights_clear((1, 0), w)
    torch.cuda.synchronize()
    assert torch.equal(w, want)


def test_weigh_rejects_a_stale_plan():
    case = MemCache("bf16", 2, 128, 64, 1, [(c, 0) for c in range(3)], seed=81)
    plan, _ = _pack("clean", 4, 2, [(2, 0)], case)
    case.cache.release((0, 0))
    q = case.queries(case.n)
    with pytest.raises(sc.ScError) as e:
        _run(case, plan, q, 0.1, case.weights())
    assert e.value.code == sc.SC_ESTALE


def test_weigh_workspace_is_checked():
    case = MemCache("bf16", 2, 128, 64, 1, [(c, 0) for c in range(3)], seed=82)
    plan, _ = _pack("clean", 4, 2, [(2, 0)], case)
    nb = sc.sc_attention_weigh_workspace_bytes(plan, case.cache)
    q, w = case.queries(case.n), case.weights()
    ws = torch.full((nb + 16,), 0x5A, dtype=torch.uint8, device="cuda")
    o = torch.empty_like(q)
    for bad in ((ws, nb - 1), (None, nb), (ws[8:], nb)):
        with pytest.raises(sc.ScError) as e:
            sc.sc_attention_weigh(plan, case.cache, 0, q, o, 0.1, w, *bad)
        assert e.value.code == sc.SC_EINVAL
    sc.sc_attention_weigh(plan, case.cache, 0, q, o, 0.1, w, ws, nb)
    torch.cuda.synchronize()
    assert (ws[nb:] == 0x5A).all()


@pytest.mark.parametrize("heads,tpp,prefix,nodes,nq", [
    (12, 64, 20, 1, 64), (12, 128, 10, 1, 128), (12, 40, 6, 1, 40), (12, 64, 8, 8, 1), (12, 64, 24, 4, 16),
    (24, 64, 16, 2, 33), (12, 72, 5, 64, 1), (7, 264, 3, 3, 20),
])
def test_weigh_few_rows(heads, tpp, prefix, nodes, nq):
    """Few rows over a prefix and pages of their own, where the weighing merges the
    attention's partials itself, or the attention does."""
    states = [(c, 0) for c in range(prefix + nodes)]
    case = MemCache("bf16", heads, 128, tpp, 1, states, seed=83)
    own = states[prefix:]
    plan = sc.sc_plan_share(sc.sc_plan_condition(case.cache, own, nq), states[:prefix])
    _check(case, plan, [states[:prefix] + [s] for s in own], nq)


def test_weigh_merges_few_partials():
    """One frame of 64 tokens over its window leaves few partials: no launch merges them."""
    case = MemCache("bf16", 12, 128, 64, 1, [(c, 0) for c in range(21)], seed=84)
    plan, reads = _pack("clean", 4, 20, [(20, 0)], case)
    sc.sc_timer_enable(True)
    try:
        _check(case, plan, reads, 64)
        assert sc.sc_timer_read("attention_weigh")[0] == 2 and sc.sc_timer_read("attention_combine")[0] == 0
    finally:
        sc.sc_timer_enable(False)
