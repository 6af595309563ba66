"""A scale of zero: every key that a node reads weighs the same, 1 / n of n keys, also where
the keys end inside a tile.  The forms that scale the logits (weighing, a shared
prefix) over waves, 64, 128 and 256 queries, whole and in pieces, a merge by the
weighing itself; scales too small for a normal fp32 number; the entry point without a
workspace.  Tolerances as for any scale."""
import pytest
import torch

import paper_2609_22283_amd as sc

from memory_cases import MemCache, close
from test_gpu_share import _run as run_share
from test_gpu_weigh import _check, _pack

pytestmark = pytest.mark.gpu

SCALES = [0.0, -0.0, 1e-42]

# heads, tokens per page, pages per chunk, window, nodes: no node's keys fill whole tiles
PACKS = [
    (2, 40, 1, 6, 3),      # keys over waves
    (12, 72, 1, 20, 1),    # few rows: the weighing merges the attention's partials
    (12, 40, 1, 2, 32),    # 64-query units
    (12, 72, 1, 40, 3),    # in pieces
    (12, 264, 1, 6, 3),    # 128-query units
    (2, 104, 3, 6, 4),     # in pieces
    (7, 600, 2, 2, 5),     # 256-query units
    (3, 600, 1, 2, 3),     # in pieces
]


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("heads,tpp,ppc,W,nodes", PACKS)
def test_weigh_at_scale_zero(heads, tpp, ppc, W, nodes, scale):
    assert (W + 1) * ppc * tpp % 32
    pack = [(W + i, 2) for i in range(nodes)]
    case = MemCache("bf16", heads, 128, tpp, ppc, [(c, 2) for c in range(W + nodes)], seed=111)
    plan, reads = _pack("same", 4, W, pack, case)
    _check(case, plan, reads, case.n, scale)


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("dtype,heads,tpp,prefix,nodes,nq", [
    ("bf16", 12, 40, 8, 4, 1), ("bf16", 3, 72, 61, 5, 31), ("bf16", 12, 72, 30, 4, 100), ("bf16", 2, 72, 9, 3, 300),
    ("bf16", 12, 1560, 3, 2, 600), ("bf16", 2, 40, 1, 64, 1), ("f32", 2, 40, 9, 3, 50),
])
def test_share_at_scale_zero(dtype, heads, tpp, prefix, nodes, nq, scale):
    states = [(c, 0) for c in range(prefix + nodes)]
    case = MemCache(dtype, heads, 128, tpp, 1, states, seed=112)
    own = states[prefix:]
    plan = sc.sc_plan_share(sc.sc_plan_condition(case.cache, own, nq), states[:prefix])
    q = case.queries(nodes * nq)
    want, _ = case.attend(q, [states[:prefix] + [s] for s in own], scale)
    close(dtype, run_share(case, plan, q, scale), want, "o")
    o = torch.full_like(q, float("nan"))
    sc.sc_attention_noalloc(plan, case.cache, 0, q, o, scale)
    torch.cuda.synchronize()
    close(dtype, o, want, "noalloc")
    _check(case, plan, [states[:prefix] + [s] for s in own], nq, scale)


def test_zero_scale_keeps_what_lies_behind():
    """Accumulated weights of slots that the plan does not read stay, at a scale of zero too."""
    case = MemCache("bf16", 2, 128, 40, 1, [(c, 0) for c in range(4)], seed=113)
    plan, _ = _pack("clean", 4, 1, [(3, 0)], case)
    q, w = case.queries(case.n), case.weights()
    before = w.clone()
    nb = sc.sc_attention_weigh_workspace_bytes(plan, case.cache)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    sc.sc_attention_weigh(plan, case.cache, 0, q, torch.empty_like(q), 0.0, w, ws, nb)
    torch.cuda.synchronize()
    read = case.cache.slots((2, 0)) + case.cache.slots((3, 0))
    rest = [s for s in range(case.n_slots) if s not in read]
    assert torch.equal(w[:, rest], before[:, rest])
    got = (w - before)[:, read].double()
    # 40 rows, 80 keys: half a row's worth a key, added to less than 0.25 (fp32)
    assert float((got - 0.5).abs().max()) <= 0.5 * (80 / 32 + 128) * 2.0 ** -24 + 2.0 ** -18
