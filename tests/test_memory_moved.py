"""A pipeline with a memory whose cache goes to a pool of another size: its weights, one row a slot, have to
go along (CPU only: nothing is cached, nothing is launched)."""
import pytest
import torch

from test_memory_pipeline import HEADS, TPP, _cached, _pipe


@pytest.mark.parametrize("n_slots", [20, 60])
def test_weights_of_the_old_slots_are_refused(n_slots):
    """They end, or lie, elsewhere than the kernels would write."""
    p = _pipe()
    p.cache.move(1 << 50, n_slots)
    for f in (lambda: p.forward([(0, 4)]), p.run, lambda: p.run("serial"), lambda: p._fold_unread([])):
        with pytest.raises(ValueError):
            f()
        assert p.cache.free_slot_count() == n_slots and p.cached == set() and p.memory is None


def test_moved_weights_are_taken():
    p = _pipe()
    p.cache.move(1 << 50, 60)
    p.weights = torch.zeros(2, 60, HEADS, TPP)
    _cached(p, [(0, 0), (1, 0), (2, 0)])
    seen = []
    p.cache.condense = lambda layer, n_layers, sources, into, weights, *a: seen.append(weights)
    p._fold_unread([(4, 4)])
    assert len(seen) == 1 and seen[0] is p.weights
