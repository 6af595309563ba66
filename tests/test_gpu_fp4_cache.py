"""States held in 4 bits: what append and copy leave in the pages, bit for bit."""
import numpy as np
import pytest
import torch

import paper_2609_22283_amd as sc
from oracle.held import held_keys, held_values
from synth import TAG_K, TAG_V, normal

from fp4_cases import D, bf16_dev, bf16_pages, make_cache

pytestmark = pytest.mark.gpu


def _values(k, v, heads, tpp, frames):
    """[frame, head, token, d], [frame, head, d, token] of held k and v [tokens, head, d]"""
    kk = held_keys(k).reshape(frames, tpp, heads, D).transpose(0, 2, 1, 3)
    vv = held_values(v, tpp).reshape(frames, tpp, heads, D).transpose(0, 2, 3, 1)
    return kk, vv


def _out(cache, state, heads, tpp, frames, layer=0, layers=1):
    """What a state's pages stand for, by way of a bf16 cache"""
    pool, out = make_cache(sc.SC_DTYPE_BF16, heads, tpp, frames, frames, layers)
    cache.copy([state], out, [state], layer, 1)
    torch.cuda.synchronize()
    k, v = bf16_pages(pool, heads, tpp, frames, layers)
    return k[layer], v[layer]


@pytest.mark.parametrize("heads,tpp,frames", [(1, 8, 1), (3, 24, 2), (2, 32, 1), (12, 40, 3), (7, 64, 1), (1, 104, 32),
                                              (12, 1560, 3)])
def test_append_holds_the_nearest_codes(heads, tpp, frames):
    n = tpp * frames
    kd, k = bf16_dev(normal((n, heads, D), (1, TAG_K)) * np.exp(normal((1, heads, D), (2, TAG_K))))
    vd, v = bf16_dev(normal((n, heads, D), (1, TAG_V)) * np.exp(normal((1, heads, D), (2, TAG_V))))
    _, cache = make_cache(sc.SC_DTYPE_FP4, heads, tpp, frames, frames)
    cache.append(0, (0, 0), kd, vd)
    got_k, got_v = _out(cache, (0, 0), heads, tpp, frames)
    want_k, want_v = _values(k, v, heads, tpp, frames)
    np.testing.assert_array_equal(got_k, want_k)
    np.testing.assert_array_equal(got_v, want_v)


def test_every_bf16_value_as_the_largest_and_beside_larger_ones():
    """All finite bf16 numbers, each the largest of its group beside its fractions, subnormals among them."""
    bits = np.concatenate([np.arange(0x0000, 0x7f80), np.arange(0x8000, 0xff80)]).astype(np.uint32)
    top = (bits << 16).view(np.float32)
    part = np.array([0, 0.04, 0.06, 1 / 16, 0.09, 0.125, 0.15, 3 / 16, 0.22, 0.25, 0.3, 0.3125, 0.37, 0.4375, 0.5, 0.55,
                     0.625, 0.7, 0.75, 0.8, 0.875, 0.9, 0.93, 0.96, 0.98, 1, -1, -0.5, -0.3125, -0.125, -0.05, -0.01],
                    np.float32)
    x = (top[:, None] * part).reshape(-1, 4, 32)  # rows of 128 channels
    x = np.concatenate([x, np.zeros((-len(x) % 64, 4, 32), np.float32)]).reshape(-1, 1, D)
    tpp, n = 64, x.shape[0]
    frames, done = 16, 0
    while done < n:
        rows = x[done:done + tpp * frames]
        rows = np.concatenate([rows, np.zeros((tpp * frames - len(rows), 1, D), np.float32)])
        kd, k = bf16_dev(rows)
        # the same numbers as groups of tokens: a block's 32 x 128 values, taken the other way
        vd, v = bf16_dev(rows.reshape(-1, D, 32).transpose(0, 2, 1).reshape(-1, 1, D))
        _, cache = make_cache(sc.SC_DTYPE_FP4, 1, tpp, frames, frames)
        cache.append(0, (0, 0), kd, vd)
        got_k, got_v = _out(cache, (0, 0), 1, tpp, frames)
        want_k, want_v = _values(k, v, 1, tpp, frames)
        np.testing.assert_array_equal(got_k, want_k)
        np.testing.assert_array_equal(got_v, want_v)
        done += tpp * frames


@pytest.mark.parametrize("tpp", [24, 32, 72])
def test_groups_with_infinities_and_nan(tpp):
    k, v = normal((tpp, 2, D), (3, TAG_K)), normal((tpp, 2, D), (3, TAG_V))
    k[1, 0, 5], k[2, 1, 64], k[tpp - 1, 0, 127] = np.inf, -np.inf, np.nan
    v[0, 0, 7], v[tpp - 1, 1, 0], v[tpp // 2, 1, 100] = -np.inf, np.nan, np.inf
    kd, kv = bf16_dev(k)
    vd, vv = bf16_dev(v)
    _, cache = make_cache(sc.SC_DTYPE_FP4, 2, tpp, 1, 1)
    cache.append(0, (0, 0), kd, vd)
    got_k, got_v = _out(cache, (0, 0), 2, tpp, 1)
    want_k, want_v = _values(kv, vv, 2, tpp, 1)
    assert np.isnan(want_k).sum() == 96
    np.testing.assert_array_equal(got_k, want_k)
    np.testing.assert_array_equal(got_v, want_v)


@pytest.mark.parametrize("grid_h,grid_w,frames,dims", [(8, 13, 3, (44, 42, 42)), (4, 2, 2, (128, 0, 0)), (5, 8, 1, (2, 62, 64))])
def test_append_rotates_as_the_bf16_cache_does(grid_h, grid_w, frames, dims):
    """Appending with a rotation is the bf16 cache's append and a copy, to the last bit of the pool."""
    heads, tpp = 3, grid_h * grid_w
    kd, _ = bf16_dev(normal((tpp * frames, heads, D), (4, TAG_K)))
    vd, _ = bf16_dev(normal((tpp * frames, heads, D), (4, TAG_V)))
    table = torch.empty(sc.sc_rope_table_bytes(grid_h, grid_w, dims, 40), dtype=torch.uint8, device="cuda")
    rope = sc.sc_rope_table_build(table, grid_h, grid_w, dims, 40)
    wide, src = make_cache(sc.SC_DTYPE_BF16, heads, tpp, frames, frames)
    a, one = make_cache(sc.SC_DTYPE_FP4, heads, tpp, frames, frames)
    b, two = make_cache(sc.SC_DTYPE_FP4, heads, tpp, frames, frames)
    src.append(0, (9, 1), kd, vd, rope=rope)
    src.copy([(9, 1)], one, [(9, 1)], 0, 1)
    two.append(0, (9, 1), kd, vd, rope=rope)
    torch.cuda.synchronize()
    assert torch.equal(a, b)


def test_append_reads_unaligned_rows_and_writes_its_pages_alone():
    heads, tpp, frames, layers, slots = 2, 40, 2, 3, 6
    kd, k = bf16_dev(normal((tpp * frames, heads, D), (5, TAG_K)))
    vd, v = bf16_dev(normal((tpp * frames, heads, D), (5, TAG_V)))
    shifted = []
    for t in (kd, vd):
        buf = torch.zeros(t.numel() + 1, dtype=torch.bfloat16, device="cuda")
        buf[1:] = t.flatten()
        shifted.append(buf[1:])
    pool, cache = make_cache(sc.SC_DTYPE_FP4, heads, tpp, frames, slots, layers, fill=0xa5)
    cache.append(0, (0, 0), kd, vd)
    cache.append(1, (7, 2), shifted[0], shifted[1])
    torch.cuda.synchronize()
    p = pool.view(layers, slots, -1).cpu()
    at = cache.slots((7, 2))
    assert torch.equal(p[1, at], p[0, cache.slots((0, 0))])
    left = torch.ones(layers, slots, dtype=torch.bool)
    left[1, at] = left[0, cache.slots((0, 0))] = False
    assert (p[left] == 0xa5).all()


@pytest.mark.parametrize("heads,tpp,frames", [(2, 8, 1), (3, 56, 2), (12, 64, 1), (1, 1560, 3)])
def test_copies_go_out_and_back(heads, tpp, frames):
    """bf16 -> 4 bits -> bf16 -> 4 bits: the values of the oracle, and the same codes again;
    states of several layers at once, onto free slots in another order, neighbours untouched."""
    layers, states = 3, [(0, 0), (1, 0), (2, 1)]
    wide, src = make_cache(sc.SC_DTYPE_BF16, heads, tpp, frames, 3 * frames, layers)
    held, cache = make_cache(sc.SC_DTYPE_FP4, heads, tpp, frames, 4 * frames, layers, fill=0xa5)
    again, twice = make_cache(sc.SC_DTYPE_FP4, heads, tpp, frames, 3 * frames, layers)
    values = {}
    for l in range(layers):
        for st in states:
            kd, k = bf16_dev(normal((tpp * frames, heads, D), (6, TAG_K, l) + st))
            vd, v = bf16_dev(normal((tpp * frames, heads, D), (6, TAG_V, l) + st))
            src.append(l, st, kd, vd)
            values[l, st] = _values(k, v, heads, tpp, frames)
    src.copy(states[:1], cache, [(9, 0)], 1, 1)
    src.copy(states, cache, states[::-1], 1, 2)
    back, out = make_cache(sc.SC_DTYPE_BF16, heads, tpp, frames, 3 * frames, layers, fill=0xa5)
    cache.copy(states[::-1], out, states, 1, 2)
    out.copy(states, twice, states, 1, 2)
    torch.cuda.synchronize()
    k, v = bf16_pages(back, heads, tpp, 3 * frames, layers)
    for l in (1, 2):
        for st in states:
            np.testing.assert_array_equal(k[l, out.slots(st)], values[l, st][0])
            np.testing.assert_array_equal(v[l, out.slots(st)], values[l, st][1])
    assert (back.view(layers, -1)[0] == 0xa5).all() and (held.view(layers, 4 * frames, -1)[0] == 0xa5).all()
    a, b = held.view(layers, 4 * frames, -1), again.view(layers, 3 * frames, -1)
    for st, to in zip(states, states[::-1]):
        assert torch.equal(a[1:, cache.slots(to)], b[1:, twice.slots(st)])
    assert (a[2, cache.slots((9, 0))] == 0xa5).all()


@pytest.mark.parametrize("dtype,head_dim,tpp", [(sc.SC_DTYPE_BF16, 64, 8), (sc.SC_DTYPE_BF16, 128, 24), (sc.SC_DTYPE_F32, 64, 104),
                                                (sc.SC_DTYPE_F32, 128, 40), (sc.SC_DTYPE_FP4, 128, 40)])
def test_pages_are_copied_as_they_are(dtype, head_dim, tpp):
    """Any bytes, at a pool that is only aligned to its elements, 500 pages in one call."""
    heads, layers, n = 3, 2, 250
    args = (layers, heads, head_dim, tpp, 2, 4 * n, dtype)
    size = sc.sc_cache_pool_bytes(*args)
    off = {sc.SC_DTYPE_BF16: 2, sc.SC_DTYPE_F32: 4, sc.SC_DTYPE_FP4: 16}[dtype]
    buf = torch.randint(0, 256, (size + off,), dtype=torch.uint8, device="cuda")
    pool = buf[off:]
    c = sc.sc_cache_create(pool, *args)
    q = torch.zeros(2 * tpp, heads, head_dim, dtype=torch.float32 if dtype == sc.SC_DTYPE_F32 else torch.bfloat16, device="cuda")
    for i in range(n):
        for l in range(layers):
            c.append(l, (i, 0), q, q)
    pool.copy_(torch.randint(0, 256, (size,), dtype=torch.uint8, device="cuda"))
    before = pool.clone().view(layers, 4 * n, -1)
    c.copy([(i, 0) for i in range(n)], c, [(n - 1 - i, 1) for i in range(n)], 0, layers)
    torch.cuda.synchronize()
    after = pool.view(layers, 4 * n, -1)
    src = [s for i in range(n) for s in c.slots((i, 0))]
    dst = [s for i in range(n) for s in c.slots((n - 1 - i, 1))]
    assert torch.equal(after[:, dst], before[:, src])
    assert torch.equal(after[:, src], before[:, src])


def test_compact_and_move_on_the_gpu():
    """Pages and weights land in the slots that the handles name, forks' too; a smaller pool, then a larger."""
    heads, tpp, frames, layers, slots = 2, 40, 2, 3, 40
    pool, c = make_cache(sc.SC_DTYPE_FP4, heads, tpp, frames, slots, layers)
    kd, _ = bf16_dev(normal((tpp * frames, heads, D), (7, TAG_K)))
    for i in range(20):
        for l in range(layers):
            c.append(l, (i, 0), kd, kd)
    pool.copy_(torch.randint(0, 256, pool.shape, dtype=torch.uint8, device="cuda"))
    w = torch.randn(layers, slots, heads, tpp, device="cuda")
    pages, weights = pool.clone().view(layers, slots, -1), w.clone()
    named = {(i, 0): c.slots((i, 0)) for i in range(20)}
    f = c.fork()
    for i in range(0, 20, 3):
        c.release((i, 0))
        if i % 2:
            f.release((i, 0))
    left = [(i, 0) for i in range(20) if not (i % 3 == 0 and i % 2)]

    def holds(pool, w, n):
        torch.cuda.synchronize()
        for h in (c, f):
            for st in left:
                if h.contains(st):
                    at = h.slots(st)
                    assert max(at) < 2 * len(left)
                    assert torch.equal(pool.view(layers, n, -1)[:, at], pages[:, named[st]])
                    assert torch.equal(w[:, at], weights[:, named[st]])
        assert all(f.contains(st) for st in left)

    c.compact(w)
    holds(pool, w, slots)
    for n in (2 * len(left), 50):
        to = torch.zeros(sc.sc_cache_pool_bytes(layers, heads, D, tpp, frames, n, sc.SC_DTYPE_FP4), dtype=torch.uint8, device="cuda")
        w2 = torch.zeros(layers, n, heads, tpp, device="cuda")
        f.move(to, n, weights=w, moved_weights=w2)
        assert c.desc.n_slots == f.desc.n_slots == n and c.pool is to
        w = w2
        holds(to, w, n)


@pytest.mark.parametrize("given", [True, False])
def test_the_pool_left_behind_is_not_reused_early(given):
    """Moved on a busy stream: the old pool, which nothing else holds, is handed out again only behind
    the move."""
    heads, tpp, n = 2, 64, 40
    args = (1, heads, D, tpp, 1, n, sc.SC_DTYPE_FP4)
    size = sc.sc_cache_pool_bytes(*args)
    torch.cuda.empty_cache()
    c = sc.sc_cache_create(torch.empty(size, dtype=torch.uint8, device="cuda"), *args)
    kd, _ = bf16_dev(normal((tpp, heads, D), (8, TAG_K)))
    for i in range(n):
        c.append(0, (i, 0), kd, kd)
    want, to = c.pool.clone(), torch.zeros(size, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(100_000_000)
        if not given:
            c.move(to, n)
    if given:
        c.move(to, n, stream=s)
    other = torch.zeros(size, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    assert torch.equal(to, want) and not bool(other.any())


def test_copies_of_a_pool_aligned_to_its_elements():
    heads, tpp, frames = 3, 56, 2
    args = (1, heads, D, tpp, frames, frames, sc.SC_DTYPE_BF16)
    size = sc.sc_cache_pool_bytes(*args)
    bufs = [torch.full((size + 16,), 0x5a, dtype=torch.uint8, device="cuda") for _ in range(2)]
    src, out = (sc.sc_cache_create(b[2:size + 2], *args) for b in bufs)
    _, held = make_cache(sc.SC_DTYPE_FP4, heads, tpp, frames, frames)
    kd, k = bf16_dev(normal((tpp * frames, heads, D), (9, TAG_K)))
    vd, v = bf16_dev(normal((tpp * frames, heads, D), (9, TAG_V)))
    src.append(0, (0, 0), kd, vd)
    src.copy([(0, 0)], held, [(0, 0)], 0, 1)
    held.copy([(0, 0)], out, [(0, 0)], 0, 1)
    torch.cuda.synchronize()
    got = bf16_pages(bufs[1][2:size + 2].clone(), heads, tpp, frames)
    want = _values(k, v, heads, tpp, frames)
    np.testing.assert_array_equal(got[0][0], want[0])
    np.testing.assert_array_equal(got[1][0], want[1])
    assert bool((bufs[1][:2] == 0x5a).all()) and bool((bufs[1][size + 2:] == 0x5a).all())
