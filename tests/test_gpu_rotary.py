"""Rotary positions of the rows of a tensor against an fp64 rotation, and the tables whose time
axis is scaled against their formulas."""
import math

import numpy as np
import pytest
import torch

import paper_2609_22283_amd as sc
from synth import normal

pytestmark = pytest.mark.gpu

THETA = 10000.0
SCALINGS = {"none": None, "unscaled": dict(kind="none"), "linear": dict(kind="linear", factor=3.5),
            "ntk": dict(kind="ntk", factor=8.0),
            "yarn": dict(kind="yarn", factor=16.0, original=4096, beta_fast=32, beta_slow=1,
                         magnitude=0.1 * math.log(16.0) + 1.0)}


def _freq(dim, scaling):
    i = np.arange(dim // 2)
    s = scaling or {}
    f = THETA ** (-2.0 * i / dim)
    if s.get("kind") == "linear":
        return f / s["factor"]
    if s.get("kind") == "ntk" and dim > 2:
        return (THETA * s["factor"] ** (dim / (dim - 2))) ** (-2.0 * i / dim)
    if s.get("kind") == "yarn":
        g = np.clip((s["original"] * f / (2 * math.pi) - s["beta_slow"]) / (s["beta_fast"] - s["beta_slow"]), 0, 1)
        return f * (g + (1 - g) / s["factor"])
    return f


def _angles(pos, dims, scaling):
    parts = [pos[:, a:a + 1].astype(np.float64) * _freq(d, scaling if a == 0 else None)
             for a, d in enumerate(dims) if d]
    return np.concatenate(parts, 1)


def _rotated(x, pos, dims, layout, transpose, scaling=None):
    part = sum(dims)
    m = (scaling or {}).get("magnitude", 1.0)
    ang = _angles(pos, dims, scaling)[:, None]
    c, s = m * np.cos(ang), m * np.sin(ang) * (-1 if transpose else 1)
    a, b = (np.arange(0, part, 2), np.arange(1, part, 2)) if layout == "interleaved" else (
        np.arange(part // 2), np.arange(part // 2, part))
    y = x.copy()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y, (np.abs(x[..., a]) + np.abs(x[..., b])) * m, a, b


def _rope(dims, grid=(30, 52), frames=1 << 16, scaling=None):
    table = torch.empty(sc.sc_rope_table_bytes(*grid, dims, frames), dtype=torch.uint8, device="cuda")
    return sc.sc_rope_table_build(table, *grid, dims, frames, theta=THETA, scaling=scaling)


def _positions(rows, frames=1 << 16, grid=(30, 52), seed=0):
    rng = np.random.default_rng(seed)
    pos = np.stack([rng.integers(0, n, rows) for n in (frames, *grid)], 1).astype(np.int32)
    pos[0] = 0
    pos[-1] = (frames - 1, grid[0] - 1, grid[1] - 1)
    return pos, torch.from_numpy(pos).cuda()


def _check(got, x, pos, dims, layout, transpose, scaling, dtype):
    """cos and sin are rounded to fp32 (2^-24 each), the rotation is two fp32 operations (2^-24
    each, of at most the pair's magnitudes), and the result is rounded to its type."""
    want, mag, a, b = _rotated(x, pos, dims, layout, transpose, scaling)
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    tol = half * np.abs(want)
    for ch in (a, b):
        tol[..., ch] += 4 * 2.0 ** -24 * mag
    rest = np.setdiff1d(np.arange(x.shape[-1]), np.concatenate([a, b]))
    np.testing.assert_array_equal(got[..., rest], x[..., rest])
    assert (np.abs(got - want) <= tol).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("rows,heads,head_dim,dims", [
    (1, 1, 2, (2, 0, 0)), (3, 2, 7, (2, 2, 0)), (5, 1, 40, (10, 6, 2)), (17, 3, 64, (64, 0, 0)), (257, 12, 128, (44, 42, 42)),
    (33, 2, 80, (8, 0, 32)), (64, 5, 96, (0, 48, 0)), (19, 2, 256, (86, 84, 84)), (9, 3, 127, (62, 64, 0)), (4, 1, 1000, (500, 2, 2))])
def test_rows_at_their_positions(rows, heads, head_dim, dims, layout, dtype):
    for transpose in (False, True):
        x = torch.from_numpy(normal((rows, heads, head_dim), (1, rows)).astype(np.float32)).to(dtype).cuda()
        pos, pd = _positions(rows)
        y = torch.full_like(x, float("nan"))
        sc.sc_rope_rotate(_rope(dims), x, y, pd, layout=layout, transpose=transpose)
        torch.cuda.synchronize()
        xv = x.cpu().double().numpy()
        _check(y.cpu().double().numpy(), xv, pos, dims, layout, transpose, None, dtype)
        sc.sc_rope_rotate(_rope(dims), x, x, pd, layout=layout, transpose=transpose)  # in place
        torch.cuda.synchronize()
        assert torch.equal(x, y)


@pytest.mark.parametrize("scaling", SCALINGS)
@pytest.mark.parametrize("dims", [(128, 0, 0), (2, 4, 6), (44, 42, 42), (64, 0, 0)])
def test_scaled_tables(scaling, dims):
    s = SCALINGS[scaling]
    x = torch.from_numpy(normal((201, 2, 128), (2, 1)).astype(np.float32)).cuda()
    pos, pd = _positions(201, seed=1)
    y = torch.empty_like(x)
    sc.sc_rope_rotate(_rope(dims, scaling=s), x, y, pd, layout="half")
    torch.cuda.synchronize()
    _check(y.cpu().double().numpy(), x.cpu().double().numpy(), pos, dims, "half", False, s, torch.float32)
    if scaling == "unscaled":
        a, b = (_rope(dims, scaling=v).table for v in (None, s))
        torch.cuda.synchronize()
        assert torch.equal(a, b)


def test_a_scaled_table_rotates_cached_keys():
    """It goes wherever an sc_rope goes: keys appended with it are the rows rotated with it."""
    dims, grid, heads, s = (44, 42, 42), (8, 9), 2, SCALINGS["yarn"]
    rope = _rope(dims, grid=grid, frames=64, scaling=s)
    k = torch.from_numpy(normal((72, heads, 128), (3, 1)).astype(np.float32)).to(torch.bfloat16).cuda()
    pool = torch.empty(sc.sc_cache_pool_bytes(1, heads, 128, 72, 1, 1), dtype=torch.uint8, device="cuda")
    cache = sc.sc_cache_create(pool, 1, heads, 128, 72, 1, 1)
    cache.append(0, (50, 0), k, k, rope=rope)
    pos = torch.tensor([[50, i // 9, i % 9] for i in range(72)], dtype=torch.int32, device="cuda")
    y = torch.empty_like(k)
    sc.sc_rope_rotate(rope, k, y, pos)
    torch.cuda.synchronize()
    held = pool.view(torch.bfloat16).view(2, heads, 72, 128)[0].transpose(0, 1)
    assert torch.equal(held, y)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_strides_padding_and_shared_rows(layout, dtype):
    dims, heads, hd, rows = (20, 10, 10), 3, 48, 37
    wide = torch.from_numpy(normal((rows, 3 * heads * hd + 1), (4, 1)).astype(np.float32)).to(dtype).cuda()
    pos, pd = _positions(rows, seed=2)
    for r, p in ((3, (-1, 0, 0)), (7, (1 << 16, 0, 0)), (8, (5, 30, 0)), (9, (5, 0, 52)), (11, (5, -3, 2))):
        pos[r] = p
    pd.copy_(torch.from_numpy(pos))
    pad = [3, 7, 8, 9, 11]
    live = [r for r in range(rows) if r not in pad]
    rope = _rope(dims)
    x = wide[:, 1:1 + heads * hd].unflatten(1, (heads, hd))  # element-aligned, rows far apart
    y = torch.full((heads, rows, hd), 7.0, dtype=dtype, device="cuda").transpose(0, 1)  # heads outermost
    before = wide.clone()
    sc.sc_rope_rotate(rope, x, y, pd, layout=layout)
    torch.cuda.synchronize()
    assert torch.equal(wide, before)
    got = y.cpu().double().numpy()
    assert (got[pad] == 7.0).all()
    _check(got[live], x.cpu().double().numpy()[live], pos[live], dims, layout, False, None, dtype)
    # one row for all, and one head for all
    z = torch.empty(rows, heads, hd, dtype=dtype, device="cuda")
    for src in (x[:1].expand(rows, heads, hd), x[:, :1].expand(rows, heads, hd)):
        sc.sc_rope_rotate(rope, src, z, pd, layout=layout)
        torch.cuda.synchronize()
        _check(z.cpu().double().numpy()[live], src.cpu().double().numpy()[live], pos[live], dims, layout, False, None, dtype)
    # in place in the wider tensor: nothing beside the slice changes
    sc.sc_rope_rotate(rope, x, x, pd, layout=layout)
    torch.cuda.synchronize()
    assert torch.equal(x[live].contiguous(), y[live].contiguous())
    assert torch.equal(wide[:, 0], before[:, 0]) and torch.equal(wide[:, 1 + heads * hd:], before[:, 1 + heads * hd:])
    assert torch.equal(x[pad].contiguous(), before[pad, 1:1 + heads * hd].unflatten(1, (heads, hd)))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("rows,heads,head_dim,dims", [
    (9001, 5, 40, (14, 14, 12)), (9000, 6, 44, (10, 6, 6)), (9000, 9, 34, (26, 0, 0)), (9000, 4, 80, (28, 26, 26)), (9001, 7, 128, (64, 0, 0))])
def test_rows_by_four_heads(rows, heads, head_dim, dims, layout, dtype):
    """Many rows, whose threads take four heads each: odd numbers of heads, runs that end inside the
    rotated part and inside the rest, reads that stay in the caches and that do not."""
    x = torch.from_numpy(normal((rows, heads, head_dim), (3, heads)).astype(np.float32)).to(dtype).cuda()
    pos, pd = _positions(rows, seed=heads)
    y = torch.full_like(x, float("nan"))
    sc.sc_rope_rotate(_rope(dims), x, y, pd, layout=layout)
    torch.cuda.synchronize()
    _check(y.cpu().double().numpy(), x.cpu().double().numpy(), pos, dims, layout, False, None, dtype)


def test_many_rows_and_far_offsets():
    """More elements than 2^31 in the tensor that the rows are strided through."""
    rows, stride = 70000, 40000  # 2.8e9 elements between the first and the last row
    big = torch.zeros(rows * stride, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((rows, 1, 64), (stride, 64, 1))
    src = torch.from_numpy(normal((rows, 1, 64), (5, 1)).astype(np.float32)).to(torch.bfloat16).cuda()
    x.copy_(src)
    pos, pd = _positions(rows, seed=3)
    sc.sc_rope_rotate(_rope((32, 16, 16)), x, x, pd)
    torch.cuda.synchronize()
    at = np.r_[0:50, rows - 50:rows]
    _check(x[at].cpu().double().numpy(), src[at].cpu().double().numpy(), pos[at], (32, 16, 16), "interleaved", False, None, torch.bfloat16)


@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_the_transpose_is_the_gradient(layout):
    """<g, R x> = <R^T g, x>, and against differences: R is linear, so one step of any length gives
    its derivative up to the roundings of R (x + e) and R x."""
    dims, s = (20, 12, 8), SCALINGS["yarn"]
    rope = _rope(dims, scaling=s)
    x, g, e = (torch.from_numpy(normal((23, 2, 44), (6, i)).astype(np.float32)).cuda() for i in range(3))
    pos, pd = _positions(23, seed=4)

    def rot(v, transpose=False):
        y = torch.empty_like(v)
        sc.sc_rope_rotate(rope, v, y, pd, layout=layout, transpose=transpose)
        torch.cuda.synchronize()
        return y.double()

    dx = rot(g, True)
    want, _, _, _ = _rotated(g.cpu().double().numpy(), pos, dims, layout, True, s)
    assert np.abs(dx.cpu().numpy() - want).max() <= 6 * 2.0 ** -24 * 2 * 1.3 * g.abs().max().item()
    change = ((rot(x + e) - rot(x)) * g.double()).sum().item()
    along = (dx * ((x + e).double() - x.double())).sum().item()
    size = (g.abs().double().sum() * 8 * (x.abs().max() + e.abs().max())).item()
    assert abs(change - along) <= 8 * 2.0 ** -24 * size
    ident = torch.empty_like(x)
    plain = _rope(dims)
    sc.sc_rope_rotate(plain, x, ident, pd, layout=layout)
    sc.sc_rope_rotate(plain, ident, ident, pd, layout=layout, transpose=True)
    torch.cuda.synchronize()
    assert (ident - x).abs().max().item() <= 16 * 2.0 ** -24 * x.abs().max().item()


def test_no_rows_another_stream_and_a_graph():
    rope = _rope((44, 42, 42))
    x = torch.from_numpy(normal((40, 12, 128), (7, 1)).astype(np.float32)).to(torch.bfloat16).cuda()
    pos, pd = _positions(40, seed=5)
    y = torch.empty_like(x)
    sc.sc_rope_rotate(rope, x[:0], y[:0], pd[:0])
    sc.sc_rope_rotate(rope, x, y, pd)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    z = torch.zeros_like(x)
    torch.cuda.synchronize()
    sc.sc_rope_rotate(rope, x, z, pd, stream=s)
    s.synchronize()
    assert torch.equal(y, z)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sc.sc_rope_rotate(rope, x, z, pd)
    for shift in (1, 2, 3):
        x.copy_(x.roll(1, 0))
        pd.copy_(pd.roll(shift, 0))
        g.replay()
        sc.sc_rope_rotate(rope, x, y, pd)
        torch.cuda.synchronize()
        assert torch.equal(y, z)
