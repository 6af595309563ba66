"""Attention over plans whose nodes share a prefix (sc_plan_share) against the formula
in 64 bits: one to 64 nodes of one to several hundred rows, prefixes from one page
to hundreds, own lists of different lengths, pages that end inside key tiles, both
ways such a plan can run (asserted), the entry points that take it, and a block."""
import pytest
import torch

import paper_2609_22283_amd as sc

from memory_cases import MemCache, close

pytestmark = pytest.mark.gpu


def _run(case, plan, q, scale, layer=0):
    nb = sc.sc_attention_workspace_bytes(plan, case.cache)
    ws = torch.full((max(16, nb),), 0xFF, dtype=torch.uint8, device="cuda")
    o = torch.full_like(q, float("nan"))
    sc.sc_attention(plan, case.cache, layer, q, o, scale, ws, nb)
    torch.cuda.synchronize()
    return o


# dtype, heads, head dim, tokens per page, pages per state, prefix states, nodes, rows per node
CASES = [
    ("bf16", 12, 128, 64, 1, 8, 4, 1),
    ("bf16", 12, 128, 64, 1, 256, 32, 1),
    ("bf16", 2, 128, 32, 1, 1, 64, 1),      # the smallest pages, the most nodes
    ("bf16", 7, 128, 40, 2, 30, 11, 3),
    ("bf16", 3, 128, 72, 1, 60, 5, 31),
    ("bf16", 12, 128, 128, 1, 128, 16, 128),
    ("bf16", 2, 128, 104, 3, 9, 3, 312),
    ("bf16", 1, 128, 64, 1, 700, 2, 1),
    ("bf16", 2, 128, 264, 2, 5, 7, 200),
    ("bf16", 12, 128, 1560, 1, 2, 1, 1),
    ("f32", 2, 128, 104, 3, 9, 3, 50),
    ("f32", 3, 64, 8, 1, 1, 64, 1),
    ("f32", 12, 64, 16, 2, 100, 6, 1),
    ("f32", 2, 128, 40, 1, 200, 2, 70),
]


@pytest.mark.parametrize("dtype,heads,hd,tpp,ppc,prefix,nodes,nq", CASES)
def test_share(dtype, heads, hd, tpp, ppc, prefix, nodes, nq):
    states = [(c, 0) for c in range(prefix + nodes)]
    case = MemCache(dtype, heads, hd, tpp, ppc, states, seed=91)
    own = states[prefix:]
    plan = sc.sc_plan_share(sc.sc_plan_condition(case.cache, own, nq), states[:prefix])
    q, scale = case.queries(nodes * nq), hd ** -0.5
    o = _run(case, plan, q, scale)
    want, _ = case.attend(q, [states[:prefix] + [s] for s in own], scale)
    close(dtype, o, want, "o")
    assert torch.equal(_run(case, plan, q, scale), o)
    o2 = torch.full_like(q, float("nan"))
    sc.sc_attention_noalloc(plan, case.cache, 0, q, o2, scale)
    torch.cuda.synchronize()
    close(dtype, o2, want, "noalloc")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_share_own_lists_of_different_lengths(dtype):
    """Early chunks' windows are shorter: own lists of one to four states; a memory of two
    states before them, in two steps; a negative scale."""
    states = [(c, 0) for c in range(4)] + [(50, 0), (60, 0)]
    case = MemCache(dtype, 3, 128, 72, 2, states, seed=92)
    pack = [(c, 0) for c in range(4)]
    plan = sc.sc_plan_build(sc.sc_selection_build("clean", 4, 3, pack), case.cache)
    plan = sc.sc_plan_share(sc.sc_plan_share(plan, [(60, 0)]), [(50, 0)])
    off, slots, _, _ = plan.tables()
    assert [b - a for a, b in zip(off, off[1:])] == [6, 8, 10, 12]
    assert slots[off[2]:off[2] + 4] == case.cache.slots((50, 0)) + case.cache.slots((60, 0))
    q = case.queries(4 * case.n)
    reads = [[(50, 0), (60, 0)] + [(r, 0) for r in range(c + 1)] for c in range(4)]
    for scale in (128 ** -0.5, -0.05):
        close(dtype, _run(case, plan, q, scale), case.attend(q, reads, scale)[0], "o")


def test_share_forms():
    """Few rows run over the shared prefix once, a pack of long chunks over its lists."""
    states = [(c, 0) for c in range(70)]
    case = MemCache("bf16", 12, 128, 64, 1, states, seed=93)
    few = sc.sc_plan_share(sc.sc_plan_condition(case.cache, states[60:], 1), states[:60])
    assert sc.sc_attention_form(few, case.cache)[2] < 0
    big = MemCache("bf16", 12, 128, 1560, 1, [(c, 0) for c in range(4)], seed=94)
    plan = sc.sc_plan_share(sc.sc_plan_condition(big.cache, [(2, 0), (3, 0)], 4680), [(0, 0), (1, 0)])
    assert sc.sc_attention_form(plan, big.cache)[2] > 0
    q = big.queries(2 * 4680)
    o = _run(big, plan, q, 128 ** -0.5)
    want, _ = big.attend(q, [[(0, 0), (1, 0), (2, 0)], [(0, 0), (1, 0), (3, 0)]], 128 ** -0.5)
    close("bf16", o, want, "o")


def test_share_far_logits():
    """Prefix and own keys whose logits lie some 150 log2 units apart, either way."""
    for far in ("prefix", "own"):
        def key_fn(st, k):
            k = k.clone()
            k[:, :, 0] = 1200.0 if (st[0] < 20) == (far == "prefix") else 0.0
            return k
        for nodes, nq in ((6, 1), (4, 100), (3, 300)):
            states = [(c, 0) for c in range(20 + nodes)]
            case = MemCache("bf16", 4, 128, 64, 1, states, seed=95, key_fn=key_fn)
            plan = sc.sc_plan_share(sc.sc_plan_condition(case.cache, states[20:], nq), states[:20])
            q = case.queries(nodes * nq)
            q[:, :, 0] = 1.0
            want, _ = case.attend(q, [states[:20] + [s] for s in states[20:]], 128 ** -0.5)
            close("bf16", _run(case, plan, q, 128 ** -0.5), want, f"{far} {nodes} x {nq}")


def test_share_infinite_values():
    """A channel of +inf in every value row stays +inf (no 0 x inf past a page list's end)."""
    states = [(c, 0) for c in range(9)]

    def value_fn(st, v):
        v = v.clone()
        v[:, :, 5] = float("inf")
        return v

    case = MemCache("bf16", 2, 128, 40, 1, states, seed=96, value_fn=value_fn)
    plan = sc.sc_plan_share(sc.sc_plan_condition(case.cache, states[6:], 2), states[:6])
    q = case.queries(6)
    o = _run(case, plan, q, 128 ** -0.5)
    assert (o[:, :, 5] == float("inf")).all()
    want, _ = case.attend(q, [states[:6] + [s] for s in states[6:]], 128 ** -0.5)
    rest = [i for i in range(128) if i != 5]
    close("bf16", o[:, :, rest], want[:, :, rest], "o")


def test_share_rows_behind_the_last_node_stay():
    states = [(c, 0) for c in range(6)]
    case = MemCache("bf16", 3, 128, 64, 1, states, seed=97)
    plan = sc.sc_plan_share(sc.sc_plan_condition(case.cache, states[4:], 5), states[:4])
    q = case.queries(10)
    buf = torch.full((16, 3, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    nb = sc.sc_attention_workspace_bytes(plan, case.cache)
    ws = torch.full((nb + 64,), 0x5A, dtype=torch.uint8, device="cuda")
    sc.sc_attention(plan, case.cache, 0, q, buf, 0.1, ws, nb)
    torch.cuda.synchronize()
    assert (buf[10:] == 7.0).all() and (ws[nb:] == 0x5A).all()
    with pytest.raises(sc.ScError) as e:
        sc.sc_attention(plan, case.cache, 0, q, buf, 0.1, ws, nb - 1)
    assert e.value.code == sc.SC_EINVAL


def test_share_captured():
    states = [(c, 0) for c in range(40)]
    case = MemCache("bf16", 12, 128, 64, 1, states, seed=98)
    plan = sc.sc_plan_share(sc.sc_plan_condition(case.cache, states[32:], 2), states[:32])
    q = case.queries(16)
    nb = sc.sc_attention_workspace_bytes(plan, case.cache)
    ws, o = torch.empty(nb, dtype=torch.uint8, device="cuda"), torch.empty_like(q)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        sc.sc_attention(plan, case.cache, 0, q, o, 0.1, ws, nb)
    for _ in range(3):
        q.copy_(case.queries(16))
        want = _run(case, plan, q, 0.1)
        o.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want)


@pytest.mark.parametrize("hd", [64, 128])
def test_share_pool_off_16_byte_boundaries(hd):
    """An fp32 pool that is only element-aligned: the same sums through other loads."""
    states = [(c, 0) for c in range(9)]
    case = MemCache("f32", 2, hd, 40, 1, states, seed=99)
    own = states[6:]
    plan = sc.sc_plan_share(sc.sc_plan_condition(case.cache, own, 20), states[:6])
    q = case.queries(60)
    aligned = _run(case, plan, q, 0.1)
    want, _ = case.attend(q, [states[:6] + [s] for s in own], 0.1)
    raw = torch.zeros(case.pool.numel() + 16, dtype=torch.uint8, device="cuda")
    pool = raw[4:4 + case.pool.numel()]
    cache = sc.sc_cache_create(pool, 1, 2, hd, 40, 1, case.n_slots, sc.SC_DTYPE_F32)
    for st in states:
        cache.append(0, st, *case.kv[st][0])
    case.cache = cache
    plan = sc.sc_plan_share(sc.sc_plan_condition(cache, own, 20), states[:6])
    shifted = _run(case, plan, q, 0.1)
    close("f32", shifted, want, "o")
    assert torch.equal(shifted, aligned)
