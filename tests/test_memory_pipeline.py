"""The pipeline with a memory on the CPU: what it folds, and what it does when a fold
fails or is refused (no kernel runs: device pointers here are never read)."""
import pytest
import torch

import paper_2609_22283_amd as sc
from paper_2609_22283_amd.pipeline import StackPipeline

PTR = 1 << 20  # stands for device memory, 16-byte aligned
HEADS, TPP, PPC, D, MLP = 2, 40, 1, 256, 512


def _pipe(layers=2, cache_layers=2, B=8, **kw):
    cache = sc.sc_cache_create(PTR, cache_layers, HEADS, 128, TPP, PPC, 40)
    ws = [sc.BlockWeights(D, HEADS, 128, MLP, PTR, PTR, PTR, PTR) for _ in range(layers)]
    xs = torch.zeros((B, TPP * PPC, D), dtype=torch.bfloat16)
    return StackPipeline(layers=ws, cache=cache, rope=None, xs=xs, noise=xs, policy="clean", K=4, W=2, B=B,
                         t_sched=(0.0, 0.25, 0.5, 0.75, 1.0), memory=True, **kw)


def _cached(p, states):
    """States that the pipeline has run, with slots (unwritten)."""
    sc.sc_plan_build(sc.sc_selection_build("clean", 4, 0, states), p.cache)
    p.cached = set(states)


def test_folds_the_stack_layers():
    """A cache may hold more layers than the stack: the fold takes those of the stack."""
    p = _pipe(layers=2, cache_layers=3)
    _cached(p, [(0, 0), (1, 0), (2, 0)])
    seen = []
    p.cache.condense = lambda layer, n_layers, *a: seen.append((layer, n_layers))
    p._fold_unread([(4, 4)])
    assert seen == [(0, 2)]
    assert tuple(p.kept.shape) == (2, HEADS, TPP * PPC)
    assert tuple(p.weights.shape) == (3, 40, HEADS, TPP)


def test_a_failed_fold_keeps_its_states():
    """A fold that fails leaves the memory and the states that were to join it as they are:
    cached, known to the pipeline, and folded by the next attempt."""
    p = _pipe()
    _cached(p, [(0, 0), (1, 0), (1, 3), (2, 0)])
    p.memory = (0, 0)
    p.cached.discard((0, 0))
    for _ in range(2):
        with pytest.raises(sc.ScError) as e:  # nothing is written yet
            p._fold_unread([(4, 4)])
        assert e.value.code == sc.SC_EUNAVAILABLE
        assert p.memory == (0, 0) and p.cached == {(1, 0), (2, 0)}
        assert all(p.cache.contains(st) for st in [(0, 0), (1, 0), (2, 0)]) and not p.cache.contains((1, 3))
    folds = []
    p.cache.condense = lambda layer, n, sources, into, *a: folds.append((sources, into))
    p._fold_unread([(4, 4)])
    assert folds == [([(0, 0), (1, 0)], (1, 5))]
    assert p.memory == (1, 5) and p.cached == {(2, 0)}
    assert not p.cache.contains((0, 0)) and not p.cache.contains((1, 0))


def test_memory_needs_the_refresh_node():
    """Only clean states join the memory, and only the refresh node makes them: without it the
    history would be lost in silence."""
    with pytest.raises(ValueError):
        _pipe(refresh=False)
    assert _pipe(refresh=True).memory is None


@pytest.mark.parametrize("mode", ["packed", "sequential", "serial"])
def test_layer_hooks_are_refused_before_anything_runs(mode):
    """In whichever round the hook is: no state has slots, no weight is cleared."""
    p = _pipe()
    for r in (0, 3, len(p.rounds()) - 1):
        with pytest.raises(ValueError):
            p.run(mode, layer_hooks={r: lambda *a: None})
        assert p.cache.free_slot_count() == 40 and p.cached == set()
    with pytest.raises(ValueError):
        p.forward([(0, 4)], lambda *a: None)
    assert p.cache.free_slot_count() == 40
