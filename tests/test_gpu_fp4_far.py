"""Attention over 4-bit pages where the logits lie far from zero: what counts is how they differ.

A key is 4 in channel 0 and a code in channel 1, a query a in channel 0 and b in channel 1, so that the
logits 4 a + b code and their differences are exact in fp32, however large a is."""
import numpy as np
import pytest

import paper_2609_22283_amd as sc
from paper_2609_22283_amd.binding import sc_attention_form

from fp4_cases import D, Held, attend, bf16_dev, check, condition_plan, oracle

pytestmark = pytest.mark.gpu

# 4 a, whose scaled values are 0.1, 1e4, 1e6, 1e7, 5e7 .. 1e9, 1e29 and 1e35
SIZES = [m * s for m in (1.0, 159 / 128, 255 / 128) for s in (1.0, 2.0 ** 17, 2.0 ** 24, 2.0 ** 27, 2.0 ** 29, 2.0 ** 30,
                                                            2.0 ** 33, 2.0 ** 100, 2.0 ** 120)]
SIZES += [-x for x in SIZES]

# heads, tokens per page, frames, prefix states, nodes, rows a node; tile rows (0: bf16 pages) and waves
SHAPES = [
    ((1, 64, 1, 0, 1, 1), 16, 4),
    ((2, 40, 2, 9, 5, 17), 16, 8),
    ((1, 1560, 3, 0, 1, 65), 16, 4),
    ((1, 8, 1, 700, 1, 1), 16, 8),
    ((1, 512, 1, 60, 32, 1), 16, 8),
    ((2, 64, 1, 0, 4, 2000), 32, 4),
    ((3, 520, 1, 30, 3, 256), 32, 4),
    ((3, 104, 1, 120, 3, 1024), 0, 1),
]


def _case(shape, codes, seed=70):
    """codes(state, tokens) -> channel 1 of a state's keys; the other channels are zeros"""
    heads, tpp, frames, prefix, nodes, nq = shape

    def edit(st, k, v):
        k[:] = 0
        k[:, :, 0] = 4.0
        k[:, :, 1] = codes(st, len(k))[:, None]
    pre, own = [(c, 0) for c in range(prefix)], [(prefix + i, 0) for i in range(nodes)]
    h = Held(heads, tpp, frames, pre + own, seed=seed, edit=edit)
    return h, condition_plan(h, pre, own, nq), [pre + [st] for st in own]


def _queries(shape, sizes, small):
    """Row r of every node: sizes[r % len(sizes)] / 4 in channel 0, `small` of its magnitude in channel 1."""
    heads, nodes, nq = shape[0], shape[-2], shape[-1]
    a = np.resize(np.asarray(sizes) / 4, nq)
    q = np.zeros((nodes, nq, heads, D), np.float32)
    q[..., 0] = a[:, None]
    q[..., 1] = np.exp2(np.floor(np.log2(np.abs(a))))[:, None] * small
    qd, qv = bf16_dev(q.reshape(nodes * nq, heads, D))
    np.testing.assert_array_equal(qv, q.reshape(nodes * nq, heads, D))
    return qd, qv


def _kinds(shape, st, n, kinds):
    """Codes 0 and -4, a third of each state's keys 0; every third state of a prefix has none of those."""
    none = st[0] % 3 == 1 and st[0] < shape[3]
    kinds[st] = np.where(np.random.default_rng(st[0]).random(n) < (0.0 if none else 0.3), 0.0, -4.0)
    kinds[st][-1] = -4.0 if none else 0.0
    return kinds[st]


@pytest.mark.parametrize("shape,tile,waves", SHAPES)
def test_keys_far_from_zero(shape, tile, waves):
    """Keys of two kinds, those of code 0 and those of -4, whose logits are an eighth below.  Far from zero
    that leaves the mean of the first kind's values."""
    kinds = {}
    h, plan, reads = _case(shape, lambda st, n: _kinds(shape, st, n, kinds))
    assert sc_attention_form(plan, h.cache)[:2] == (tile, waves)
    nq = shape[-1]
    for turn in range(1 if nq >= len(SIZES) else -(-len(SIZES) // nq)):
        sizes = np.roll(SIZES, -turn * nq)
        qd, q = _queries(shape, sizes, 0.125)
        got = attend(h, plan, qd)
        for i, states in enumerate(reads):
            v = np.concatenate([h.v[s] for s in states])
            top = np.concatenate([kinds[s] for s in states]) == 0
            for r in np.unique(np.linspace(0, nq - 1, 2 * len(SIZES)).astype(int)):
                size, g = np.resize(sizes, nq)[r], got[i * nq + r]
                if abs(size) < 2:  # near zero: both kinds count
                    want, tol = oracle(h, [states], q[i * nq + r:i * nq + r + 1], 1)
                    check(g, want[0], tol[0], f"node {i}, row {r}")
                    continue
                # each exponential is 1 but for its rounding, and the output is rounded (2^-9 each, twice
                # that allowed as in fp4_cases.oracle); what lies below has no weight at all
                want = v[top].mean(0)
                check(g, want, 2.0 ** -8 * (np.abs(want) + np.abs(v[top]).mean(0)), f"node {i}, row {r}, logit {size}")


@pytest.mark.parametrize("nq", [1, 6, 40])
def test_near_one_another_and_far_from_zero(nq):
    """128 keys whose logits are near one another: weighed as they differ.  With a a power of two and
    b = 2^-20 a, half a code is one step of fp32 beside 4 a."""
    grid = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
    shape = (1, 128, 1, 0, 1, nq)
    h, plan, reads = _case(shape, lambda st, n: grid[np.arange(n) * 5 % 8] * np.where(np.arange(n) % 3 == 0, -1, 1))
    sizes = [2.0 ** 26, 2.0 ** 27, 2.0 ** 25, -2.0 ** 26, -2.0 ** 27, -2.0 ** 25]
    for turn in range(1 if nq >= 6 else 6):
        qd, q = _queries(shape, np.roll(sizes, -turn), 2.0 ** -20)
        want, _ = oracle(h, reads, q, nq)
        s = q[:, 0] @ h.k[(0, 0)][:, 0].T * D ** -0.5
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        assert (p.max(-1) < 0.2).all() and (np.sort(p, -1)[:, -20:].min(-1) > 2.0 ** -12).all()
        v = np.abs(h.v[(0, 0)][:, 0])
        # as in fp4_cases.oracle, the logits' differences (34 at most) off by 2^-23 of themselves
        tol = 2.0 ** -8 * np.abs(want[:, 0]) + (2.0 ** -8 + np.expm1(2.0 ** -17)) * (p @ v) + 2.0 ** -22 * p.max(-1, keepdims=True) * v.sum(0)
        check(attend(h, plan, qd)[:, 0], want[:, 0], tol)


@pytest.mark.parametrize("shape,tile,waves", SHAPES)
def test_logits_that_fp32_does_not_hold(shape, tile, waves):
    """Keys whose scaled logits are below all fp32 numbers have no weight beside others."""
    kinds = {}
    h, plan, reads = _case(shape, lambda st, n: _kinds(shape, st, n, kinds))
    nodes, nq = shape[-2:]
    q = np.zeros((nodes * nq, h.heads, D), np.float32)
    q[:, :, 1] = 2.0 ** 125  # times -4 and a scale of 10
    got = attend(h, plan, bf16_dev(q)[0], 10.0)
    for i, states in enumerate(reads):
        v = np.concatenate([h.v[s] for s in states])[np.concatenate([kinds[s] for s in states]) == 0]
        want = v.mean(0)
        for r in (0, nq // 2, nq - 1):
            check(got[i * nq + r], want, 2.0 ** -8 * (np.abs(want) + np.abs(v).mean(0)), f"node {i}, row {r}")


@pytest.mark.parametrize("shape,tile,waves", SHAPES)
def test_rows_of_zeros_at_the_largest_scales(shape, tile, waves):
    h, plan, reads = _case(shape, lambda st, n: np.where(np.arange(n) % 2 == 0, 0.0, -4.0))
    nodes, nq = shape[-2:]
    qd, _ = bf16_dev(np.zeros((nodes * nq, h.heads, D), np.float32))
    for scale in (3e38, -3e38):
        got = attend(h, plan, qd, scale)
        for i, states in enumerate(reads):
            v = np.concatenate([h.v[s] for s in states])
            want = v.mean(0)
            for r in (0, nq // 2, nq - 1):
                check(got[i * nq + r], want, 2.0 ** -8 * (np.abs(want) + np.abs(v).mean(0)), f"node {i}, row {r}, scale {scale}")
