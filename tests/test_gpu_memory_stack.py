"""Blocks, stacks and the pipeline with a bounded memory of the history.

A shared prefix as a block's plan against the same states in the window (one
block, the gate of two GPU results of one function); a stack that weighs its keys
against single blocks and sc_attention_weigh on their queries; the pipeline with a
memory: as long as the memory holds one chunk whole, a window of W and the memory
are a window of W + 1, and later it is a fold.
"""
import pytest

import paper_2609_22283_amd as sc
from paper_2609_22283_amd.pipeline import StackPipeline
from synth import TAG_K, TAG_V, TAG_W_DOWN, TAG_W_O, TAG_W_QKV, TAG_W_UP, TAG_X, normal
from synth.configs import SMALL

from gpu_cases import from_device, to_device, torch_mod
from test_gpu_pipeline import T_SCHED, _setup, _stack_gate

pytestmark = pytest.mark.gpu

HEADS, D, MLP, GH, GW, DIMS = 2, 256, 512, 8, 13, (44, 42, 42)
TPP = GH * GW


def _layers(n):
    gen = lambda shape, tag: to_device(normal(shape, (31, tag), 0.05), sc.SC_DTYPE_BF16)[0]  # noqa: E731
    return [sc.BlockWeights(D, HEADS, 128, MLP, gen((3 * D, D), TAG_W_QKV + 100 * l), gen((D, D), TAG_W_O + 100 * l),
                            gen((MLP, D), TAG_W_UP + 100 * l), gen((D, MLP), TAG_W_DOWN + 100 * l)) for l in range(n)]


def _rope():
    torch = torch_mod()
    table = torch.empty(sc.sc_rope_table_bytes(GH, GW, DIMS, 64), dtype=torch.uint8, device="cuda")
    return sc.sc_rope_table_build(table, GH, GW, DIMS, 64)


def _cache(n_layers, states, n_slots):
    """A cache with `states` appended at every layer."""
    torch = torch_mod()
    args = (n_layers, HEADS, 128, TPP, 1, n_slots, sc.SC_DTYPE_BF16)
    pool = torch.full((sc.sc_cache_pool_bytes(*args),), 0xFF, dtype=torch.uint8, device="cuda")
    cache = sc.sc_cache_create(pool, *args)
    for l in range(n_layers):
        for st in states:
            k, v = (to_device(normal((TPP, HEADS, 128), (32, tag, l) + st), sc.SC_DTYPE_BF16)[0]
                    for tag in (TAG_K, TAG_V))
            cache.append(l, st, k, v, rope=_rp)
    return cache


@pytest.fixture(autouse=True)
def _rope_table():
    global _rp
    _rp = _rope()


def test_block_over_a_shared_prefix():
    """Two nodes that read chunk 1 as a shared prefix beside a window of two, and by a sparse
    window of four (clean history: the same keys)."""
    torch = torch_mod()
    w = _layers(1)[0]
    nodes = [(4, 1), (5, 2)]
    T = 2 * TPP
    x0 = to_device(normal((T, D), (33, TAG_X)), sc.SC_DTYPE_BF16)[0]
    nb = sc.sc_block_workspace_bytes(w, T)
    got = []
    for shared in (True, False):
        cache = _cache(1, [(c, 0) for c in range(5)], 8)
        if shared:
            plan = sc.sc_plan_build(sc.sc_selection_build("clean", 4, 2, nodes), cache)
            plan = sc.sc_plan_share(plan, [(1, 0)])
        else:
            mask = [[1, 1, 0, 0]] * 5
            mask[1] = [1, 1, 1, 0]       # (4, 1): offsets 1, 2 and chunk 1
            mask[2] = [1, 1, 0, 1]       # (5, 2): offsets 1, 2 and chunk 1
            plan = sc.sc_plan_build(sc.sc_selection_build("clean", 4, 4, nodes, r_mask=mask), cache)
        x, ws = x0.clone(), torch.full((nb,), 0xFF, dtype=torch.uint8, device="cuda")
        sc.sc_block_forward(w, cache, 0, plan, x, _rp, ws, nb)
        torch.cuda.synchronize()
        got.append(x.double())
    assert torch.isfinite(got[0]).all()
    # each is within 0.0034 of the exact block in the 2-norm
    assert float((got[0] - got[1]).norm() / got[1].norm()) <= 2 * 0.0034


@pytest.mark.parametrize("shared", [False, True])
def test_stack_weighs_its_keys(shared):
    torch = torch_mod()
    L, nodes = 3, [(3, 1), (4, 2)]
    hist = [(c, 0) for c in range(4)]
    T, layers, scale = 2 * TPP, _layers(3), 128 ** -0.5
    x0 = to_device(normal((T, D), (34, TAG_X)), sc.SC_DTYPE_BF16)[0]
    nb = sc.sc_block_workspace_bytes(layers[0], T)

    def start():
        cache = _cache(L, hist, 8)
        plan = sc.sc_plan_build(sc.sc_selection_build("clean", 4, 2, nodes), cache)
        if shared:
            plan = sc.sc_plan_share(plan, [(0, 0)])
        ws = torch.full((nb,), 0xFF, dtype=torch.uint8, device="cuda")
        wnb = sc.sc_attention_weigh_workspace_bytes(plan, cache)
        w = torch.zeros((L, 8, HEADS, TPP), dtype=torch.float32, device="cuda")
        return cache, plan, ws, x0.clone(), w, torch.empty(wnb, dtype=torch.uint8, device="cuda"), wnb

    cache, plan, ws, x, w, wws, wnb = start()
    with pytest.raises(sc.ScError) as e:
        sc.sc_stack_forward_weigh(layers, cache, plan, x, _rp, ws, nb, w, wws, wnb - 1)
    assert e.value.code == sc.SC_EINVAL and torch.equal(x, x0)
    sc.sc_stack_forward_weigh(layers, cache, plan, x, _rp, ws, nb, w, wws, wnb)
    cache2, plan2, ws2, x2, w2, wws2, _ = start()
    q_off, _ = sc.sc_block_workspace_views(layers[0], T)
    o = torch.empty((T, HEADS, 128), dtype=torch.bfloat16, device="cuda")
    for l, layer in enumerate(layers):
        sc.sc_block_forward(layer, cache2, l, plan2, x2, _rp, ws2, nb)
        q = ws2[q_off:q_off + T * D * 2].view(torch.bfloat16)
        sc.sc_attention_weigh(plan2, cache2, l, q, o, scale, w2, wws2, wnb)
    torch.cuda.synchronize()
    assert float((x.double() - x2.double()).norm() / x2.double().norm()) <= 2 * 0.0034 * L
    assert torch.equal(w[0], w2[0])  # the same q and k in the first layer
    for l in range(1, L):  # q and k of two stacks within the gate: 0.0068 per layer of logits below 2^3
        assert float((w[l] - w2[l]).norm() / w2[l].norm()) <= 0.0068 * l * 8
    # every row hands out a weight of one per head
    assert torch.allclose(w.sum((1, 3)), torch.full((L, HEADS), float(T), device="cuda"), rtol=1e-4)
    read = {s for st in hist[(0 if shared else 1):] + nodes for s in cache.slots(st)}
    for slot in range(8):
        assert bool((w[:, slot] > 0).all()) == (slot in read)


def _pipe(make, **kw):
    p = make()
    return StackPipeline(layers=p.layers, cache=p.cache, rope=p.rope, xs=p.xs, noise=p.noise, policy=p.policy, K=p.K,
                         W=kw.pop("W", p.W), B=p.B, t_sched=T_SCHED, refresh=True, **kw)


def test_pipeline_memory_of_one_chunk_is_a_wider_window():
    """Serial clean history over four chunks: once chunk 0 has left a window of two, it is the
    memory, whole, and chunk 3 reads what a window of three reads."""
    torch = torch_mod()
    make, _, _, keep = _setup(SMALL, 2, 4, 2, "clean", seed=25, n_slots=60)
    runs = []
    for kw in (dict(memory=True), dict(W=3)):
        p = _pipe(make, **kw)
        p.run("serial")
        torch.cuda.synchronize()
        assert p.cache.free_slot_count() == 60 and p.memory is None
        runs.append(from_device(p.xs))
    for c in range(4):
        _stack_gate(runs[0][c], runs[1][c], 2, ("memory", c), runs=2)


@pytest.mark.parametrize("mode,policy", [("packed", "prog"), ("sequential", "same"), ("serial", "prog")])
def test_pipeline_folds_what_leaves_the_window(mode, policy):
    """Eight chunks over a window of two: the memory is folded again and again, read by every
    later node, and two runs give the same bits."""
    torch = torch_mod()
    make, _, _, keep = _setup(SMALL, 2, 8, 2, policy, seed=26, n_slots=120)
    seen, runs = [], []
    for memory in (True, True, False):
        p = _pipe(make, memory=memory)
        if memory:
            fold = p.cache.condense

            def spy(layer, n, sources, into, *a, **k):
                seen.append((list(sources), into))
                fold(layer, n, sources, into, *a, **k)

            p.cache.condense = spy
        p.run(mode)
        torch.cuda.synchronize()
        assert p.cache.free_slot_count() == 120
        runs.append(p.xs.clone())
        if memory:
            assert torch.isfinite(p.weights).all()
    assert torch.equal(runs[0], runs[1])
    half = len(seen) // 2
    assert half >= 3 and seen[:half] == seen[half:]
    folded = [st for sources, _ in seen[:half] for st in sources if st[1] == 0]
    assert folded == sorted(set(folded)) and folded[0] == (0, 0)  # every clean chunk once, in order
    for (_, into), (sources, _) in zip(seen[:half], seen[1:half]):
        assert sources[0] == into                               # each fold starts from the last
    assert torch.isfinite(runs[0].float()).all()
    assert not torch.equal(runs[0][-1], runs[2][-1])            # the last chunk has read the memory


def test_pipeline_memory_refuses_layer_hooks():
    make, _, _, keep = _setup(SMALL, 2, 3, 2, "clean", seed=27, n_slots=60)
    p = _pipe(make, memory=True)
    with pytest.raises(ValueError):
        p.run("serial", layer_hooks={0: lambda *a: None})


def test_pipeline_memory_times_its_launches():
    make, _, _, keep = _setup(SMALL, 2, 6, 2, "prog", seed=28, n_slots=100)
    p = _pipe(make, memory=True)
    p.run("packed", kernel_timer_rounds=(0, len(p.rounds()) - 1))
    layers = len(p.layers)
    assert p.kernel_times["attention_weigh"][0] >= layers * len(p.rounds())
    assert p.kernel_times["condense"][0] >= 1
