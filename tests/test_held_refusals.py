"""What the calls of 4-bit caches, their pages and rotary positions refuse, before anything is
launched (CPU only), and the pages' oracle by hand."""
import ctypes as C
import math

import numpy as np
import pytest

import paper_2609_22283_amd as sc
from oracle.held import held, held_keys, held_values


def _cache(dtype=sc.SC_DTYPE_FP4, layers=2, heads=2, head_dim=128, tpp=40, frames=1, slots=6, pool=1 << 20):
    return sc.sc_cache_create(pool, layers, heads, head_dim, tpp, frames, slots, dtype)


def _refused(code, f, *args, **kw):
    with pytest.raises(sc.ScError) as e:
        f(*args, **kw)
    assert e.value.code == code, e.value


def test_held_values_by_hand():
    x = np.zeros(32)
    x[:13] = [7.9, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.26, -0.74, -5.1, 6.5, 1e-9]
    np.testing.assert_array_equal(held(x)[:13], [6, 0, 1, 1, 2, 2, 4, 4, 0.5, -0.5, -6, 6, 0])
    np.testing.assert_array_equal(held(x * 2.0 ** -20), held(x) * 2.0 ** -20)
    np.testing.assert_array_equal(held(np.zeros(32)), 0)
    tiny = np.full(32, 2.0 ** -133)  # the smallest bf16 number, far below the unit 2^-127
    np.testing.assert_array_equal(held(tiny), 0)
    np.testing.assert_array_equal(held(np.full(8, 2.0 ** -128)), 2.0 ** -128)
    assert np.isnan(held(np.r_[np.inf, np.zeros(31)])).all() and np.isnan(held(np.r_[np.nan, np.ones(31)])).all()
    k = np.random.default_rng(0).normal(size=(5, 2, 128))
    np.testing.assert_array_equal(held_keys(k)[3, 1, 64:96], held(k[3, 1, 64:96]))
    v = np.random.default_rng(1).normal(size=(80, 2, 128))
    hv = held_values(v, 40)
    np.testing.assert_array_equal(hv[32:40, 1, 7], held(v[32:40, 1, 7]))  # a page ends at 40
    np.testing.assert_array_equal(hv[40:72, 0, 9], held(v[40:72, 0, 9]))
    np.testing.assert_array_equal(held_keys(held_keys(k)), held_keys(k))  # held once, held for good


def test_pool_of_a_4_bit_cache():
    per = 4352  # bytes of 32 tokens x 128 channels, keys and values
    assert sc.sc_cache_pool_bytes(2, 3, 128, 32, 1, 5, sc.SC_DTYPE_FP4) == 2 * 5 * 3 * per
    assert sc.sc_cache_pool_bytes(1, 1, 128, 1560, 1, 1, sc.SC_DTYPE_FP4) == 49 * per
    assert sc.sc_cache_pool_bytes(1, 1, 128, 8, 1, 1, sc.SC_DTYPE_FP4) == per
    assert sc.sc_cache_pool_bytes(1, 1, 64, 32, 1, 1, sc.SC_DTYPE_FP4) == 0
    _refused(sc.SC_EUNSUPPORTED, _cache, head_dim=64)
    _refused(sc.SC_EINVAL, _cache, pool=(1 << 20) + 8)
    _refused(sc.SC_EINVAL, _cache, dtype=3)
    _refused(sc.SC_EINVAL, _cache, tpp=36)


def test_what_takes_no_4_bit_cache():
    c = _cache()
    sel = sc.sc_selection_build("clean", 1, 0, [(0, 1)])
    plan = sc.sc_plan_build(sel, c)
    _refused(sc.SC_EUNAVAILABLE, sc.sc_attention, plan, c, 0, 64, 64, 1.0)
    w = sc.BlockWeights(256, 2, 128, 256, 16, 16, 16, 16)
    _refused(sc.SC_EUNSUPPORTED, sc.sc_block_forward, w, c, 0, plan, 16, None, 16, 1 << 40)
    _refused(sc.SC_EUNSUPPORTED, sc.sc_stack_forward, [w], c, plan, 16, None, 16, 1 << 40)
    _refused(sc.SC_EUNSUPPORTED, sc.sc_stack_forward_weigh, [w], c, plan, 16, None, 16, 1 << 40, 16, 16, 1 << 40)
    assert sc.sc_attention_weigh_workspace_bytes(plan, c) == 0
    _refused(sc.SC_EUNSUPPORTED, sc.sc_condition_append, c, 0, (5, 0), 16, 16, 16, None, 16, 1 << 40)
    _refused(sc.SC_EUNSUPPORTED, c.condense, 0, 1, [(0, 1)], (1, 0), 16, 16)


def test_copies_forks_and_moves():
    a, b = _cache(), _cache(pool=1 << 30)
    _refused(sc.SC_EINVAL, a.copy, [(0, 0)], b, [(0, 0), (1, 0)], 0, 1)
    _refused(sc.SC_EINVAL, a.copy, [], b, [], 0, 1)
    _refused(sc.SC_ENOTFOUND, a.copy, [(0, 0)], b, [(0, 0)], 0, 1)
    sc.sc_plan_build(sc.sc_selection_build("clean", 1, 0, [(0, 1)]), a)  # reserves (0, 1)
    _refused(sc.SC_EUNAVAILABLE, a.copy, [(0, 1)], b, [(0, 1)], 0, 1)
    _refused(sc.SC_EUNAVAILABLE, a.fork)
    _refused(sc.SC_EINVAL, a.copy, [(0, 1)], _cache(tpp=48, pool=1 << 30), [(0, 1)], 0, 1)
    _refused(sc.SC_EUNSUPPORTED, a.copy, [(0, 1)], _cache(dtype=sc.SC_DTYPE_F32, pool=1 << 30), [(0, 1)], 0, 1)
    _refused(sc.SC_EINVAL, a.copy, [(0, 1)], _cache(pool=(1 << 20) + 4352), [(0, 1)], 0, 1)  # overlapping pools
    a.compact()  # slot 0 is the lowest: nothing to launch
    _refused(sc.SC_EINVAL, a.move, None, 6)
    _refused(sc.SC_EINVAL, a.move, 1 << 30, 0)
    _refused(sc.SC_EINVAL, a.move, (1 << 30) + 8, 6)
    _refused(sc.SC_EINVAL, a.move, 1 << 20, 6)
    _refused(sc.SC_EINVAL, a.move, 1 << 30, 6, weights=1 << 31)
    _refused(sc.SC_EINVAL, a.move, 1 << 30, 6, weights=1 << 31, moved_weights=(1 << 31) + 4)
    assert a.desc.n_slots == 6 and a.free_slot_count() == 5
    f = b.fork()
    b.move(1 << 29, 9)  # nothing is cached: nothing to launch
    assert f.desc.n_slots == b.desc.n_slots == 9 and f.free_slot_count() == 9 and f.pool == 1 << 29


def _rotate(rope_dims=(4, 2, 2), table=1 << 20, x=1 << 24, y=1 << 25, pos=1 << 26, frames=8, grid=(4, 4), **kw):
    d = dict(n_rows=3, n_heads=2, head_dim=16, dtype=sc.SC_DTYPE_BF16, layout=0, transpose=0, x_row=32, x_head=16,
             y_row=32, y_head=16)
    d.update(kw)
    from paper_2609_22283_amd import binding as b
    rope = b.sc_rope(b.sc_rope_desc(*grid, *rope_dims, frames, 10000.0), table)
    desc = b.sc_rotate_desc(*[d[n] for n, _ in b.sc_rotate_desc._fields_])
    return b.lib.sc_rope_rotate(C.byref(rope), C.byref(desc), x, y, pos, None)


def test_rotations():
    bad = [dict(n_rows=-1), dict(n_heads=0), dict(head_dim=0), dict(layout=2), dict(rope_dims=(18, 0, 0)),
           dict(rope_dims=(0, 0, 0)), dict(rope_dims=(3, 1, 0)), dict(rope_dims=(-2, 4, 4)), dict(grid=(0, 4)), dict(frames=0),
           dict(x=None), dict(y=None), dict(pos=None), dict(table=None), dict(x=(1 << 24) + 1), dict(pos=(1 << 26) + 2),
           dict(dtype=sc.SC_DTYPE_F32, y=(1 << 25) + 2), dict(y=(1 << 24) + 32), dict(y=1 << 24, y_row=64),
           dict(y_row=16), dict(y_head=8), dict(y_row=0), dict(y_head=0), dict(y_row=40, y_head=90),
           dict(y=(1 << 24) - 32), dict(n_heads=1, y_row=8)]
    for kw in bad:
        assert _rotate(**kw) == sc.SC_EINVAL, kw
    assert _rotate(dtype=sc.SC_DTYPE_FP4) == sc.SC_EUNSUPPORTED
    assert _rotate(n_heads=65536, y=1 << 50, x_row=1 << 20, y_row=1 << 20) == sc.SC_EUNSUPPORTED
    assert _rotate(n_rows=0) == 0 and _rotate(n_rows=0, x=None, y=None, pos=None) == 0


def test_rotation_of_torch_tensors():
    import torch
    rope = sc.binding.Rope(sc.binding.sc_rope_desc(1, 1, 8, 0, 0, 16, 10000.0), 1 << 20)
    x = torch.zeros(3, 2, 8)
    p = torch.zeros(3, 3, dtype=torch.int32)
    for bad in [(x[0], x[0], p), (x, x[:2], p), (x, x.double(), p), (x.half(), x.half(), p), (x, x, p[:2]), (x, x, p.long()),
                (x, x, p.t()), (x.transpose(1, 2), x.transpose(1, 2), p)]:
        _refused(sc.SC_EINVAL, sc.sc_rope_rotate, rope, *bad)
    _refused(sc.SC_EINVAL, sc.sc_rope_rotate, rope, x, x, p, layout="other")


def test_scaled_tables():
    ok = dict(kind="yarn", factor=4.0, original=1024.0)
    for change in [dict(kind="other"), dict(more=1), dict(factor=0.5), dict(factor=math.inf), dict(factor=math.nan),
                   dict(original=0), dict(original=math.nan), dict(beta_fast=1.0), dict(beta_slow=math.inf), dict(magnitude=0),
                   dict(magnitude=-1.0), dict(magnitude=math.inf)]:
        _refused(sc.SC_EINVAL, sc.sc_rope_table_build, 1 << 20, 4, 4, (4, 2, 2), 8, scaling={**ok, **change})
    _refused(sc.SC_EINVAL, sc.sc_rope_table_build, None, 4, 4, (4, 2, 2), 8, scaling=ok)
    _refused(sc.SC_EINVAL, sc.sc_rope_table_build, 1 << 20, 4, 4, (3, 2, 2), 8, scaling=ok)
    _refused(sc.SC_EINVAL, sc.sc_rope_table_build, 1 << 20, 4, 0, (4, 2, 2), 8, scaling=ok)
