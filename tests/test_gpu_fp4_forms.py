"""Every way of running the attention over 4-bit pages, each where it is chosen: tiles of 16 rows
with four waves and with eight, and of 32 rows, keys in pieces, a prefix read once or by each node, and bf16 pages taken out first; without
a workspace; and as a block's cross-attention."""
import numpy as np
import pytest
import torch

import paper_2609_22283_amd as sc
from paper_2609_22283_amd.binding import sc_attention_form

from fp4_cases import D, Held, attend, bf16_pages, check, condition_plan, oracle
from gpu_cases import ConditionCase
from test_gpu_block import SMALL, BlockCase, block_gate
from test_gpu_condition import PACK, RESIDENT, ROUNDINGS

pytestmark = pytest.mark.gpu

# heads, tokens per page, frames, prefix states, nodes, rows a node; tile rows (0: bf16 pages), the
# waves of a work-group, and pieces: 1, "pieces", or "prefix" where that is read once for all rows
FORMS = [
    ((1, 64, 1, 0, 1, 1), 16, 4, 1),
    ((2, 40, 2, 9, 5, 17), 16, 8, 1),
    ((1, 1560, 3, 0, 1, 65), 16, 4, "pieces"),
    ((1, 8, 1, 700, 1, 1), 16, 8, "pieces"),
    ((1, 64, 1, 40, 64, 1), 16, 4, "prefix"),
    ((1, 512, 1, 60, 32, 1), 16, 8, "prefix"),
    ((12, 64, 1, 100, 16, 4), 16, 8, "prefix"),
    ((2, 64, 1, 0, 4, 2000), 32, 4, 1),
    ((3, 520, 1, 30, 3, 256), 32, 4, "pieces"),
    ((3, 64, 1, 120, 3, 500), 32, 4, "prefix"),
    ((12, 64, 1, 0, 2, 2000), 0, 1, 1),
    ((3, 104, 1, 120, 3, 1024), 0, 1, 1),
    ((2, 520, 3, 6, 2, 4680), 0, 1, 1),
]


def _case(heads, tpp, frames, prefix, nodes, nq):
    pre, own = [(c, 0) for c in range(prefix)], [(prefix + i, 0) for i in range(nodes)]
    h = Held(heads, tpp, frames, pre + own, seed=nq + 1)
    plan = condition_plan(h, pre, own, nq)
    return h, plan, [pre + [st] for st in own]


def _sampled(h, reads, q, nq):
    """Rows of every node (the first, the last and some between) and the oracle's outputs for them"""
    at = sorted(set(np.linspace(0, nq - 1, 24).astype(int)))
    rows = np.array([i * nq + r for i in range(len(reads)) for r in at])
    return rows, oracle(h, reads, q[rows], len(at))


def _form(plan, cache):
    tile, waves, pieces = sc_attention_form(plan, cache)
    return tile, waves, "prefix" if pieces < 0 else "pieces" if pieces > 1 else pieces


@pytest.mark.parametrize("shape,tile,waves,pieces", FORMS)
def test_every_form(shape, tile, waves, pieces):
    h, plan, reads = _case(*shape)
    nodes, nq = shape[-2:]
    assert _form(plan, h.cache) == (tile, waves, pieces)
    qd, q = h.queries(nodes * nq, 2.0)
    rows, (want, tol) = _sampled(h, reads, q, nq)
    got = attend(h, plan, qd)
    assert np.isfinite(got).all()
    check(got[rows], want, tol)
    np.testing.assert_array_equal(got, attend(h, plan, qd))  # equal calls, equal bits


@pytest.mark.parametrize("shape", [s for s, *_ in FORMS] + [(4, 104, 3, 60, 4, 2048)])
def test_without_a_workspace(shape):
    """The call that has an array of its own, which the last shape's fastest way does not fit into."""
    h, plan, reads = _case(*shape)
    nodes, nq = shape[-2:]
    qd, q = h.queries(nodes * nq, 2.0)
    rows, (want, tol) = _sampled(h, reads, q, nq)
    room, most = sc.sc_attention_noalloc_scratch_bytes(), sc.sc_attention_workspace_bytes(plan, h.cache)
    assert (most > room) == (shape == (4, 104, 3, 60, 4, 2048))
    o = torch.full((nodes * nq + 1, h.heads, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    sc.sc_attention_noalloc(plan, h.cache, 0, qd, o, D ** -0.5)
    torch.cuda.synchronize()
    got = o.float().cpu().double().numpy()
    check(got[rows], want, tol)
    assert np.isfinite(got[:-1]).all() and np.isnan(got[-1]).all()


@pytest.mark.parametrize("shape", [(1, 64, 1, 0, 1, 1), (3, 104, 1, 120, 3, 1024)])
def test_refusals(shape):
    h, plan, _ = _case(*shape)
    rows = shape[-2] * shape[-1]
    q = torch.zeros(rows * h.heads * D + 8, dtype=torch.bfloat16, device="cuda")
    o = torch.full_like(q, 7.0)
    nb = sc.sc_attention_workspace_bytes(plan, h.cache)
    ws = torch.zeros(nb + 32, dtype=torch.uint8, device="cuda")
    for scale, x, w in ((float("nan"), q, ws), (float("inf"), q, ws), (1.0, q[4:], ws), (1.0, q, ws[8:])):
        with pytest.raises(sc.ScError) as e:
            sc.sc_attention(plan, h.cache, 0, x, o, scale, w, nb)
        assert e.value.code == sc.SC_EINVAL
    if nb:
        with pytest.raises(sc.ScError) as e:
            sc.sc_attention(plan, h.cache, 0, q, o, 1.0, ws, nb - 1)
        assert e.value.code == sc.SC_EINVAL
        with pytest.raises(sc.ScError) as e:
            sc.sc_attention(plan, h.cache, 0, q, o, 1.0, None, nb)
        assert e.value.code == sc.SC_EINVAL
    with pytest.raises(sc.ScError) as e:
        sc.sc_attention_noalloc(plan, h.cache, 0, q, o, float("nan"))
    assert e.value.code == sc.SC_EINVAL
    torch.cuda.synchronize()
    assert bool((o == 7.0).all())


@pytest.mark.parametrize("tokens,norms", [(64, False), (136, True)])
def test_a_condition_in_4_bits(tokens, norms):
    """A block whose cross-attention reads a condition held in 4 bits: against the oracle over the held
    values, with the roundings of the block over a bf16 condition (one of which it does not make)."""
    cross = ConditionCase(SMALL, tokens, seed=41, q_norm=norms, k_norm=norms)
    args = (1, SMALL.heads, D, tokens, 1, 1)
    pools = [torch.full((sc.sc_cache_pool_bytes(*args, dt),), 0xff, dtype=torch.uint8, device="cuda")
             for dt in (sc.SC_DTYPE_FP4, sc.SC_DTYPE_BF16)]
    held, back = (sc.sc_cache_create(p, *args, dt) for p, dt in zip(pools, (sc.SC_DTYPE_FP4, sc.SC_DTYPE_BF16)))
    st = [(0, 0)]
    cross.cache.copy(st, held, st, 0, 1)
    held.copy(st, back, st, 0, 1)
    torch.cuda.synchronize()
    k, v = bf16_pages(pools[1], SMALL.heads, tokens, 1)
    far = max(np.abs(k[0, 0].transpose(1, 0, 2) - cross.kv[0][0]).max(), np.abs(v[0, 0].transpose(2, 0, 1) - cross.kv[0][1]).max())
    assert far > 0.1  # the oracle sees other values than those of the bf16 condition
    cross.kv[0] = (k[0, 0].transpose(1, 0, 2), v[0, 0].transpose(2, 0, 1))
    cross.cache = held
    case = BlockCase(SMALL, "prog", PACK, RESIDENT, seed=42, cross=cross)
    got = case.run()
    want, _ = case.oracle()
    for i in range(len(PACK)):
        block_gate(got[i], want[i], f"node {PACK[i]}", ROUNDINGS["cross_norm" if norms else "cross"])


def test_pages_behind_four_gigabytes():
    """States in the last slots of a pool whose offsets do not fit 32 bits: appended, attended over, copied
    out and back, and moved to the front of another pool."""
    heads, tpp, frames, nq = 12, 1560, 3, 3
    slot = sc.sc_cache_pool_bytes(1, heads, D, tpp, frames, 1, sc.SC_DTYPE_FP4)
    fill = (1 << 32) // slot // frames // 2 + 3  # states in front, in two layers of them
    h = Held(heads, tpp, frames, [], extra_slots=(fill + 4) * frames, layers=2, layer=1, seed=51)
    assert (fill + 4) * frames * slot + fill * frames * slot > 1 << 32
    keep = [sc.sc_plan_build(sc.sc_selection_build("clean", 1, 0, [(c, 1) for c in range(i, min(i + 64, fill))]), h.cache)
            for i in range(0, fill, 64)]  # reserves their slots
    far = [(5000, 0), (5001, 0)]
    tail = Held(heads, tpp, frames, far, layers=2, layer=1, seed=51)
    tail.cache.copy(far, h.cache, far, 1, 1)
    h.k, h.v = tail.k, tail.v
    assert min(min(h.cache.slots(st)) for st in far) == fill * frames
    kd = torch.zeros((tpp * frames, heads, D), dtype=torch.bfloat16, device="cuda")
    h.cache.append(1, (5002, 0), kd, kd)
    h.k[(5002, 0)] = h.v[(5002, 0)] = np.zeros(kd.shape)
    reads = [far + [(5002, 0)]]
    plan = condition_plan(h, far, [(5002, 0)], nq)
    qd, q = h.queries(nq, 2.0)
    want, tol = oracle(h, reads, q, nq)
    check(attend(h, plan, qd), want, tol)
    wide = torch.full((sc.sc_cache_pool_bytes(2, heads, D, tpp, frames, 6),), 0xff, dtype=torch.uint8, device="cuda")
    out = sc.sc_cache_create(wide, 2, heads, D, tpp, frames, 6)
    h.cache.copy(far, out, far, 1, 1)
    torch.cuda.synchronize()
    k, v = bf16_pages(wide, heads, tpp, 6, 2)
    for st in far:
        s = out.slots(st)
        np.testing.assert_array_equal(k[1][s].transpose(0, 2, 1, 3).reshape(-1, heads, D), h.k[st])
        np.testing.assert_array_equal(v[1][s].transpose(0, 3, 1, 2).reshape(-1, heads, D), h.v[st])
    h.cache.release(far[0])
    out.copy(far[:1], h.cache, far[:1], 1, 1)
    plan = condition_plan(h, far, [(5002, 0)], nq)
    check(attend(h, plan, qd), want, tol, "taken out and held again")
    for c in range(fill):
        h.cache.release((c, 1))
    to = torch.empty(sc.sc_cache_pool_bytes(2, heads, D, tpp, frames, 9, sc.SC_DTYPE_FP4), dtype=torch.uint8, device="cuda")
    h.cache.move(to, 9)
    plan = condition_plan(h, far, [(5002, 0)], nq)
    check(attend(h, plan, qd), want, tol, "moved")
