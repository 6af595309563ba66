"""A step over a history in 4 bits captured into a graph: queries rotated, a state appended, recent
states packed and taken out again, the attention; replayed with other inputs beside eager work."""
import numpy as np
import pytest
import torch

import paper_2609_22283_amd as sc
from synth import TAG_K, TAG_Q, TAG_V, normal

from fp4_cases import D, bf16_dev, bf16_pages, make_cache

pytestmark = pytest.mark.gpu

HEADS, GRID, FRAMES, DIMS, NQ = 3, (5, 8), 2, (44, 42, 42), 20
TPP = GRID[0] * GRID[1]


class Step:
    """The buffers and caches of a step; run() is what is captured."""

    def __init__(self):
        table = torch.empty(sc.sc_rope_table_bytes(*GRID, DIMS, 64), dtype=torch.uint8, device="cuda")
        self.rope = sc.sc_rope_table_build(table, *GRID, DIMS, 64)
        self.x, self.k, self.v = (torch.empty(n, HEADS, D, dtype=torch.bfloat16, device="cuda")
                                  for n in (NQ, TPP * FRAMES, TPP * FRAMES))
        self.q, self.o = torch.empty_like(self.x), torch.empty_like(self.x)
        self.pos = torch.empty(NQ, 3, dtype=torch.int32, device="cuda")
        self.wide_pool, self.wide = make_cache(sc.SC_DTYPE_BF16, HEADS, TPP, FRAMES, 4 * FRAMES)
        self.held_pool, self.held = make_cache(sc.SC_DTYPE_FP4, HEADS, TPP, FRAMES, 4 * FRAMES, fill=0xff)
        self.back_pool, self.back = make_cache(sc.SC_DTYPE_BF16, HEADS, TPP, FRAMES, 2 * FRAMES)
        for c in range(3):
            kd, vd = (bf16_dev(normal((TPP * FRAMES, HEADS, D), (61, tag, c)))[0] for tag in (TAG_K, TAG_V))
            self.wide.append(0, (c, 0), kd, vd, rope=self.rope)
        torch.cuda.synchronize()

    def fill(self, i):
        self.x.copy_(bf16_dev(normal((NQ, HEADS, D), (62, TAG_Q, i)))[0])
        self.k.copy_(bf16_dev(normal((TPP * FRAMES, HEADS, D), (62, TAG_K, i)))[0])
        self.v.copy_(bf16_dev(normal((TPP * FRAMES, HEADS, D), (62, TAG_V, i)))[0])
        self.pos.copy_(torch.tensor([[(i + r) % 64, r % GRID[0], r % GRID[1]] for r in range(NQ)], dtype=torch.int32))

    def run(self, stream=None):
        sc.sc_rope_rotate(self.rope, self.x, self.q, self.pos, stream=stream)
        self.held.append(0, (7, 0), self.k, self.v, rope=self.rope, stream=stream)
        past = [(0, 0), (1, 0), (2, 0)]
        self.wide.copy(past, self.held, past, 0, 1, stream=stream)
        self.held.copy([(7, 0), (1, 0)], self.back, [(7, 0), (1, 0)], 0, 1, stream=stream)
        plan = sc.sc_plan_share(sc.sc_plan_condition(self.held, [(7, 0)], NQ), past)
        sc.sc_attention_noalloc(plan, self.held, 0, self.q, self.o, D ** -0.5, stream=stream)

    def results(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (self.q, self.o, self.held_pool, self.back_pool)]


def _eager(i, stream=None):
    s = Step()
    s.fill(i)
    torch.cuda.synchronize()
    s.run(stream)
    return s.results()


def test_a_captured_step():
    want = [_eager(i) for i in range(4)]
    for a, b in zip(want[1], _eager(1, torch.cuda.Stream())):
        assert torch.equal(a, b)
    assert bool(torch.isfinite(want[0][1]).all()) and not torch.equal(want[0][1], want[1][1])
    s = Step()
    s.fill(0)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.run()
    for i in (1, 3, 0, 2):
        s.fill(i)
        g.replay()
        for a, b in zip(want[i], s.results()):
            assert torch.equal(a, b)
        _eager(i)


def test_timers():
    s = Step()
    s.fill(0)
    torch.cuda.synchronize()
    sc.sc_timer_enable(True)
    try:
        s.run()
        torch.cuda.synchronize()
        for kind, n in (("rotate", 1), ("append", 1), ("pages", 2), ("attention", 1)):
            launches, ms = sc.sc_timer_read(kind)
            assert launches == n and ms > 0, kind
    finally:
        sc.sc_timer_enable(False)
    k, _ = bf16_pages(s.back_pool, HEADS, TPP, 2 * FRAMES)
    assert np.isfinite(k).all()
