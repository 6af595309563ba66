"""The pipeline with a memory on the GPU: caches of more layers than the stack, streams,
and a condition beside the memory."""
import pytest

import paper_2609_22283_amd as sc
from paper_2609_22283_amd.pipeline import StackPipeline
from synth.configs import SMALL

from gpu_cases import from_device, torch_mod
from test_gpu_pipeline import T_SCHED, _setup, _stack_gate

pytestmark = pytest.mark.gpu


def _pipe(make, cache=None, **kw):
    p = make()
    return StackPipeline(layers=p.layers, cache=cache or p.cache, rope=p.rope, xs=p.xs, noise=p.noise, policy=p.policy,
                         K=p.K, W=kw.pop("W", p.W), B=p.B, t_sched=T_SCHED, refresh=True, **kw)


def test_cache_of_more_layers_than_the_stack():
    """Six chunks over a window of two, folded again and again: the same bits whether the cache
    holds the stack's two layers or a third, which stays as it was."""
    torch = torch_mod()
    make, _, _, keep = _setup(SMALL, 2, 6, 2, "prog", seed=31, n_slots=90)
    runs = []
    for layers in (2, 3):
        args = (layers, SMALL.heads, SMALL.head_dim, SMALL.tokens_per_page, SMALL.frames_per_chunk, 90)
        pool = torch.full((sc.sc_cache_pool_bytes(*args),), 0xFF, dtype=torch.uint8, device="cuda")
        p = _pipe(make, sc.sc_cache_create(pool, *args), memory=True)
        p.run("packed")
        torch.cuda.synchronize()
        assert p.cache.free_slot_count() == 90 and p.memory is None
        assert bool((pool.view(layers, -1)[2:] == 0xFF).all())
        assert bool((p.weights[2:] == 0).all())
        runs.append((p.xs.clone(), p.weights[:2].clone()))
    assert torch.isfinite(runs[0][0].float()).all()
    assert torch.equal(runs[0][0], runs[1][0]) and torch.equal(runs[0][1], runs[1][1])


def test_made_on_a_busy_stream_run_on_another():
    """A pipeline made behind long work of one stream and run on another: its weights start from
    zeros that have landed, and the run has the bits of one on a single stream."""
    torch = torch_mod()
    make, _, _, keep = _setup(SMALL, 2, 6, 2, "prog", seed=32, n_slots=90)
    base = make()
    p = _pipe(make, memory=True)
    p.run("packed")
    torch.cuda.synchronize()
    want, weights = p.xs.clone(), p.weights.clone()
    side = torch.cuda.Stream()
    a = torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    for _ in range(20):  # some tens of ms
        a = (a @ a) * 1e-2
    q = StackPipeline(layers=base.layers, cache=base.cache, rope=base.rope, xs=base.xs, noise=base.noise,
                      policy=base.policy, K=base.K, W=base.W, B=base.B, t_sched=T_SCHED, refresh=True, memory=True)
    assert torch.cuda.current_stream().query()  # the zeros have landed
    with torch.cuda.stream(side):
        q.run("packed")
    torch.cuda.synchronize()
    assert torch.equal(q.xs, want) and torch.equal(q.weights, weights)


def test_memory_beside_a_condition():
    """The full block form with a memory: serial clean history, a window of two and a memory of
    one chunk against a window of three, as without a condition; and a packed stream
    whose conditions change under it, twice with the same bits."""
    torch = torch_mod()
    switch = lambda c: 0 if c < 3 else 1  # noqa: E731
    make, _, _, keep, _ = _setup(SMALL, 2, 4, 2, "clean", seed=33, n_slots=60, full=True, n_cond=2, cond_of=switch)
    runs = []
    for kw in (dict(memory=True), dict(W=3)):
        p = _pipe(make, condition=make().condition, **kw)
        p.run("serial")
        torch.cuda.synchronize()
        assert p.cache.free_slot_count() == 60 and p.memory is None
        runs.append(from_device(p.xs))
    for c in range(4):
        _stack_gate(runs[0][c], runs[1][c], 2, ("memory beside a condition", c), runs=2)
    make, _, _, keep2, _ = _setup(SMALL, 2, 8, 2, "prog", seed=34, n_slots=120, full=True, n_cond=2, cond_of=switch)
    runs = []
    for memory in (True, True, False):
        p = _pipe(make, condition=make().condition, memory=memory)
        p.run("packed")
        torch.cuda.synchronize()
        runs.append(p.xs.clone())
    assert torch.isfinite(runs[0].float()).all()
    assert torch.equal(runs[0], runs[1]) and not torch.equal(runs[0][-1], runs[2][-1])
