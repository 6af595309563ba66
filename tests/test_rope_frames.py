"""Chunks beyond a rope table, however far, are refused before anything is launched (CPU only)."""
import pytest

import paper_2609_22283_amd as sc
from paper_2609_22283_amd import binding

FRAMES = 64
# pages of a chunk, chunk: the first beyond the table, and those whose frames pass 31 and 32 bits
FAR = [(1, FRAMES), (4, FRAMES // 4), (4, 1 << 29), (4, (1 << 29) + 3), (4, 1 << 30), (1, (1 << 31) - 1), (2, (1 << 31) - 1),
       (32, (1 << 27) - 1), (32, (1 << 31) - 1)]


def _case(pages, dtype):
    cache = sc.sc_cache_create(1 << 20, 1, 2, 128, 64, pages, 2 * pages, dtype)
    return cache, binding.Rope(binding.sc_rope_desc(8, 8, 44, 42, 42, FRAMES, 10000.0), 1 << 40)


def _refused(f, *args, **kw):
    with pytest.raises(sc.ScError) as e:
        f(*args, **kw)
    assert e.value.code == sc.SC_EINVAL and "rope table" in str(e.value)


@pytest.mark.parametrize("dtype", [sc.SC_DTYPE_BF16, sc.SC_DTYPE_F32, sc.SC_DTYPE_FP4])
@pytest.mark.parametrize("pages,chunk", FAR)
def test_appends(dtype, pages, chunk):
    cache, rope = _case(pages, dtype)
    _refused(cache.append, 0, (chunk, 0), 1 << 41, 1 << 41, rope=rope)
    assert cache.free_slot_count() == 2 * pages


@pytest.mark.parametrize("pages,chunk", FAR)
def test_blocks(pages, chunk):
    cache, rope = _case(pages, sc.SC_DTYPE_BF16)
    plan = sc.sc_plan_build(sc.sc_selection_build("clean", 1, 0, [(chunk, 1)]), cache)
    w = sc.BlockWeights(256, 2, 128, 256, 16, 16, 16, 16)
    _refused(sc.sc_block_forward, w, cache, 0, plan, 16, rope, 16, 1 << 40)
    _refused(sc.sc_stack_forward, [w], cache, plan, 16, rope, 16, 1 << 40)
