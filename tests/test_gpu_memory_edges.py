"""What the bounded, shared history says of itself and no other test shows: infinite
values over fp32 pages that end inside key tiles (with and without a shared prefix,
weighed and not), and a shared plan as that of a block's cross-attention."""
import numpy as np
import pytest
import torch

import paper_2609_22283_amd as sc
from synth.configs import SMALL

from gpu_cases import ConditionCase
from memory_cases import MemCache, close
from test_gpu_block import BlockCase
from test_gpu_share import _run as run_share
from test_gpu_weigh import _pack, _run as run_weigh

pytestmark = pytest.mark.gpu


def _infinite(st, v):
    """Channel 5 of every token +inf; of channel 9, that of the state's last token."""
    v = v.clone()
    v[:, :, 5] = float("inf")
    v[-1, :, 9] = -float("inf")
    return v


def _expect(dtype, o, want):
    assert (o[:, :, 5] == float("inf")).all() and (o[:, :, 9] == -float("inf")).all()
    rest = [i for i in range(o.shape[2]) if i not in (5, 9)]
    close(dtype, o[:, :, rest], want[:, :, rest], "o")


@pytest.mark.parametrize("dtype,hd", [("f32", 64), ("f32", 128), ("bf16", 128)])
@pytest.mark.parametrize("tpp", [40, 104])
@pytest.mark.parametrize("nodes,nq", [(3, 2), (2, 40)])
def test_infinite_values_over_a_shared_prefix(dtype, hd, tpp, nodes, nq):
    states = [(c, 0) for c in range(6 + nodes)]
    case = MemCache(dtype, 2, hd, tpp, 1, states, seed=131, value_fn=_infinite)
    own, scale = states[6:], hd ** -0.5
    plan = sc.sc_plan_share(sc.sc_plan_condition(case.cache, own, nq), states[:6])
    q = case.queries(nodes * nq)
    want, _ = case.attend(q, [states[:6] + [s] for s in own], scale)
    _expect(dtype, run_share(case, plan, q, scale), want)
    w = torch.zeros_like(case.weights())
    _expect(dtype, run_weigh(case, plan, q, scale, w), want)
    assert torch.isfinite(w).all()  # values have no part in the weights


@pytest.mark.parametrize("dtype,hd", [("f32", 64), ("f32", 128), ("bf16", 128)])
@pytest.mark.parametrize("tpp,ppc,W,nodes", [(40, 1, 3, 1), (104, 3, 2, 3), (264, 1, 6, 2)])
def test_infinite_values_weighed(dtype, hd, tpp, ppc, W, nodes):
    case = MemCache(dtype, 2, hd, tpp, ppc, [(c, 2) for c in range(W + nodes)], seed=132, value_fn=_infinite)
    plan, reads = _pack("same", 4, W, [(W + i, 2) for i in range(nodes)], case)
    q = case.queries(nodes * case.n)
    want, _ = case.attend(q, reads, hd ** -0.5)
    w = torch.zeros_like(case.weights())
    _expect(dtype, run_weigh(case, plan, q, hd ** -0.5, w), want)
    assert torch.isfinite(w).all()


def test_cross_attention_over_a_shared_condition():
    """Every node of a block reads condition 0 first and one of its own: as over a condition
    cache in which each state holds both, page after page."""
    L, pack = 72, [(6, 0), (7, 1), (8, 2)]
    cc = ConditionCase(SMALL, L, seed=51, n_cond=3, q_norm=True, k_norm=True)
    own = [1, 2, 1]
    H, d = SMALL.heads, SMALL.head_dim
    args = (1, H, d, L, 2, 4, sc.SC_DTYPE_BF16)
    pool = torch.full((sc.sc_cache_pool_bytes(*args),), 0xFF, dtype=torch.uint8, device="cuda")
    both = sc.sc_cache_create(pool, *args)
    pages = cc.pool.view(torch.bfloat16).view(3, 2, -1)
    kv = [[pages[cc.cache.slots((i, 0))[0], half] for half in (0, 1)] for i in range(3)]
    k = [x.view(H, L, d).transpose(0, 1) for x, _ in kv]
    v = [x.view(H, d, L).permute(2, 0, 1) for _, x in kv]
    for i in (1, 2):
        both.append(0, (i, 0), torch.cat([k[0], k[i]]).contiguous(), torch.cat([v[0], v[i]]).contiguous())
    outs = []
    for which in ("shared", "both", "own"):
        case = BlockCase(SMALL, "prog", pack, [(c, 0) for c in range(6)], seed=52, cross=cc)
        cache = both if which == "both" else cc.cache
        plan = sc.sc_plan_condition(cache, [(i, 0) for i in own], SMALL.tokens_per_chunk)
        if which == "shared":
            plan = sc.sc_plan_share(plan, [(0, 0)])
        case.bw = case.bw.with_cross(sc.CrossAttn(cc.w_dev["w_q"], cc.w_dev["w_o"], cache, plan, q_norm=cc.g_q_dev))
        outs.append(torch.from_numpy(np.concatenate(case.run())))
    got, want, less = outs
    assert torch.isfinite(got).all()
    # each is within 0.0034 of the exact block in the 2-norm
    assert float((got - want).norm() / want.norm()) <= 2 * 0.0034
    assert float((less - want).norm() / want.norm()) > 4 * 0.0034  # condition 0 is seen in the output
