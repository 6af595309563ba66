"""The operators of a history held in 4 bits, as measurable cases.

  attend   sc_attention over a cache whose keys and values are held in 4 bits
           (a code of four bits each, a power of two for every 32 of them)
  hold     Cache.append into such a cache, and Cache.copy out of it: what the
           state's pages stand for, as a bf16 cache holds it
  park     Cache.copy of a bf16 cache's states into a 4-bit one and back
  move     Cache.move: a cache's pages gathered into another pool
  rotate   sc_rope_rotate: rotary positions of the rows of a tensor

With ``own`` false every operator runs in its plain form, elementary torch
operations in 32 bits.  Sizes are those of the repository's configurations (12
heads of 128, 30x52 tokens per latent frame, three frames per chunk, the short
streaming frames of 64 and 128 tokens) and of the range between them.
"""
from __future__ import annotations

import math

import torch

own = False

K_LEVELS = 4
Q_SCALE = 2.0  # logits of standard deviation 2: some keys matter, most do not
D = 128        # channels of a head in the caches
GROUP = 32     # values that share a scale
THETA = 10000.0


# ------------------------------------------------------------------- the cases
def _pack(name, heads, grid_h, grid_w, frames, nodes, window, policy="prog"):
    """The packed nodes of a streaming step over their windows, every state in 4 bits."""
    return {"name": name, "kind": "attend", "heads": heads, "tpp": grid_h * grid_w, "frames": frames,
            "nodes": nodes, "nq": grid_h * grid_w * frames, "prefix": 0, "window": window, "policy": policy}


def _tokens(name, heads, tpp, frames, nodes, nq, prefix):
    """``nq`` rows of every node over ``prefix`` states that all nodes read and one of its own."""
    return {"name": name, "kind": "attend", "heads": heads, "tpp": tpp, "frames": frames, "nodes": nodes,
            "nq": nq, "prefix": prefix, "window": -1, "policy": ""}


def _hold(name, heads, grid_h, grid_w, frames, dims):
    return {"name": name, "kind": "hold", "heads": heads, "grid_h": grid_h, "grid_w": grid_w,
            "tpp": grid_h * grid_w, "frames": frames, "dim_t": dims[0], "dim_h": dims[1], "dim_w": dims[2]}


def _park(name, heads, tpp, frames, states, layers):
    return {"name": name, "kind": "park", "heads": heads, "tpp": tpp, "frames": frames, "states": states,
            "layers": layers}


def _move(name, heads, tpp, frames, states, layers):
    """Every second state of a full cache has been released."""
    return {"name": name, "kind": "move", "heads": heads, "tpp": tpp, "frames": frames, "states": states,
            "layers": layers}


def _rotate(name, dtype, rows, heads, head_dim, dims, layout, scaling="none", transpose=False, fused=False):
    """``dims``: rotated channels of the three axes; ``fused``: the rows are the first third of a wider tensor."""
    return {"name": name, "kind": "rotate", "dtype": dtype, "rows": rows, "heads": heads, "head_dim": head_dim,
            "dim_t": dims[0], "dim_h": dims[1], "dim_w": dims[2], "layout": layout, "scaling": scaling,
            "transpose": transpose, "fused": fused}


def listed():
    return [
        # the next token of one stream over a short history: latency alone
        _tokens("attend_one_token", 12, 64, 8, 1, 1, 0),
        # single tokens of 16 streams over long histories of their own: reading these is the work
        _tokens("attend_tokens_long", 12, 512, 32, 16, 1, 0),
        # sixteen candidates of 16 rows each, from one history
        _tokens("attend_candidates", 12, 128, 1, 16, 16, 128),
        # one short frame over its window: a streaming step
        _pack("attend_short_frame", 12, 8, 8, 1, 1, 20, "clean"),
        # three nodes at a reduced resolution, every tile ragged
        _pack("attend_mid_ragged", 12, 11, 24, 3, 3, 6, "same"),
        # the headline pack: four nodes of a progressive diagonal over their windows
        _pack("attend_wan_pack4", 12, 30, 52, 3, 4, 6),
        # a short frame enters the cache
        _hold("hold_frame", 12, 8, 8, 1, (44, 42, 42)),
        # a full-size chunk enters the cache
        _hold("hold_wan_chunk", 12, 30, 52, 3, (44, 42, 42)),
        # the window of a short stream, in every layer of a 30-block model, set aside and recalled
        _park("park_window", 12, 64, 1, 20, 30),
        # a fragmented cache of two full-size chunks in eight layers goes to a smaller pool
        _move("move_wan_stack", 12, 1560, 3, 2, 8),
        # queries of 16 single tokens at far positions, half of every head, from a fused projection
        _rotate("rotate_tokens", "bf16", 16, 12, 128, (64, 0, 0), "half", "yarn", False, True),
        # the queries of the headline pack
        _rotate("rotate_wan_pack4", "bf16", 4 * 4680, 12, 128, (44, 42, 42), "interleaved"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _even_split(rng, total):
    """Three even numbers that add up to the even ``total``, the first at least 2."""
    t = 2 * rng.randint(1, total // 2)
    h = 2 * rng.randint(0, (total - t) // 2)
    return t, h, total - t - h


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "hold", "park", "move", "rotate"])
    heads = rng.choice([1, 2, 7, 12])
    if kind == "attend" and rng.random() < 0.4:
        tpp, frames = 8 * _log_int(rng, 1, 195), rng.choice([1, 2, 3])
        policy = rng.choice(["prog", "prog", "same", "clean"])
        window = rng.randint(0, 6) if tpp * frames > 400 else rng.randint(0, 20)
        case = _pack("", heads, 1, tpp, frames, 1 if policy == "clean" else rng.randint(1, 4), window, policy)
    elif kind == "attend":
        nodes, nq = _log_int(rng, 1, 64), _log_int(rng, 1, 512)
        tpp, frames = 8 * _log_int(rng, 1, 64), rng.choice([1, 1, 2, 8, 32])
        nodes = max(1, min(nodes, 4096 // nq, 700 // frames, (1 << 18) // (tpp * frames)))
        most = min(768 // frames - nodes, (1 << 17) // (tpp * frames), (1 << 26) // (nodes * nq * tpp * frames))
        case = _tokens("", heads, tpp, frames, nodes, nq, rng.choice([0, 1]) * _log_int(rng, 1, max(1, most)))
        if case["prefix"] > most:
            case["prefix"] = 0
    elif kind == "hold":
        grid_h, grid_w = 8 * _log_int(rng, 1, 5), _log_int(rng, 1, 52)
        case = _hold("", heads, grid_h, grid_w, rng.choice([1, 2, 3]), _even_split(rng, D))
    elif kind == "park":
        tpp, frames = 8 * _log_int(rng, 1, 195), rng.choice([1, 2, 3])
        states = rng.randint(1, 4) if tpp * frames > 400 else _log_int(rng, 1, 24)
        case = _park("", heads, tpp, frames, states, rng.choice([1, 2]) if tpp * frames > 400 else _log_int(rng, 1, 30))
    elif kind == "move":
        tpp, frames = 8 * _log_int(rng, 1, 195), rng.choice([1, 2, 3])
        states = rng.randint(1, 4) if tpp * frames > 400 else _log_int(rng, 1, 24)
        case = _move("", heads, tpp, frames, states, rng.choice([1, 2, 4]) if tpp * frames > 400 else _log_int(rng, 1, 30))
    else:
        head_dim = rng.choice([40, 64, 80, 128])
        part = rng.choice([head_dim, head_dim, head_dim // 2])
        case = _rotate("", rng.choice(["bf16", "bf16", "f32"]), _log_int(rng, 1, 16384), heads, head_dim,
                       _even_split(rng, part), rng.choice(["interleaved", "half"]),
                       rng.choice(["none", "linear", "ntk", "yarn"]), rng.random() < 0.3, rng.random() < 0.5)
    case.pop("name")
    return case


# ------------------------------------------------------------------ case geometry
def _window_nodes(case):
    """The pack of an attend case with a window, oldest chunk first, behind a full window of history."""
    first, n = case["window"], case["nodes"]
    if case["policy"] == "clean":
        return [(first, K_LEVELS)]
    return [(first + i, 2 if case["policy"] == "same" else 1 + i) for i in range(n)]


def _segments(case, node):
    """States that node (c, j) reads: its window, oldest first, then itself."""
    c, j = node
    level = {"clean": lambda r: 0, "same": lambda r: j, "prog": lambda r: max(j - r, 0)}[case["policy"]]
    return [(c - r, level(r)) for r in range(min(case["window"], c), 0, -1)] + [node]


def _cached(case):
    """The states in the cache, in slot order."""
    if case["kind"] == "attend" and case["window"] >= 0:
        level = 2 if case["policy"] == "same" else 0
        return [(c, level) for c in range(case["window"])] + _window_nodes(case)
    if case["kind"] == "attend":
        return [(c, 0) for c in range(case["prefix"] + case["nodes"])]
    if case["kind"] == "hold":
        return [(5, 0)]
    return [(c, 0) for c in range(case["states"])]


def _reads(case):
    """For each node, the indices (in _cached) of the states that it reads, in order."""
    if case["window"] >= 0:
        at = {st: i for i, st in enumerate(_cached(case))}
        return [[at[st] for st in _segments(case, nd)] for nd in _window_nodes(case)]
    return [list(range(case["prefix"])) + [case["prefix"] + i] for i in range(case["nodes"])]


SCALED = {"none": None, "linear": dict(kind="linear", factor=4.0), "ntk": dict(kind="ntk", factor=4.0),
          "yarn": dict(kind="yarn", factor=8.0, original=4096.0, beta_fast=32.0, beta_slow=1.0,
                       magnitude=0.1 * math.log(8.0) + 1.0)}
MAX_FRAMES = 32768


def _grid(case):
    """(frames, rows, columns) that the positions of a rotate case come from."""
    return MAX_FRAMES, 30 if case["dim_h"] else 1, 52 if case["dim_w"] else 1


# ----------------------------------------------------------------------- inputs
class _State:
    pass


def _normal(shape, gen, dev):
    return torch.randn(shape, generator=gen, device=dev, dtype=torch.float32)


def _inputs(case, seed):
    """Keys and values as a model's projections leave them: normal entries, some channels larger than
    others; queries of normal entries; positions spread over the table."""
    dev = "cuda" if torch.cuda.is_available() else "cpu"
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    H = case["heads"]
    if case["kind"] == "rotate":
        dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        wide = _normal((case["rows"], (3 if case["fused"] else 1) * H, case["head_dim"]), gen, dev).to(dt)
        pos = torch.stack([torch.randint(0, n, (case["rows"],), generator=gen, device=dev) for n in _grid(case)], 1)
        return {"wide": wide, "x": wide[:, :H], "pos": pos.to(torch.int32).contiguous()}
    n, states, layers = case["tpp"] * case["frames"], len(_cached(case)), case.get("layers", 1)
    size = torch.exp(0.5 * _normal((2, H, D), gen, dev))
    t = {"k": [], "v": []}
    for _ in range(layers):  # one layer at a time: the fp32 draws of a stack do not lie beside each other
        t["k"].append((_normal((states, n, H, D), gen, dev) * size[0]).to(torch.bfloat16))
        t["v"].append((_normal((states, n, H, D), gen, dev) * size[1]).to(torch.bfloat16))
    if case["kind"] == "attend":
        q = _normal((case["nodes"] * case["nq"], H, D), gen, dev) / size[0]
        t["q"] = (q * Q_SCALE).to(torch.bfloat16)
    return t


def _pool(sc, layers, case, slots, dtype):
    args = (layers, case["heads"], D, case["tpp"], case["frames"], slots, dtype)
    pool = torch.zeros(sc.sc_cache_pool_bytes(*args), dtype=torch.uint8, device="cuda")
    return pool, sc.sc_cache_create(pool, *args)


def _pages(pool, layers, case, slots):
    """A bf16 pool's pages: K [layer, slot, head, token, channel], V [layer, slot, head, channel, token]."""
    H, tpp = case["heads"], case["tpp"]
    p = pool.view(torch.bfloat16).view(layers, -1, 2, H, tpp * D)[:, :slots]
    return p[:, :, 0].unflatten(-1, (tpp, D)), p[:, :, 1].unflatten(-1, (D, tpp))


def prepare(case, seed):
    s = _State()
    s.case, s.t = case, _inputs(case, seed)
    t, kind, F = s.t, case["kind"], case.get("frames", 0)
    if kind == "rotate":
        s.y = torch.empty(t["x"].shape, dtype=t["x"].dtype, device=t["x"].device)
    if not own:
        dev = t["x" if kind == "rotate" else "k"][0].device
        if kind == "attend":  # the cache as it is held: codes of four bits and the scales' exponents
            s.k, s.v = _plain_codes(_key_groups(t["k"][0])), _plain_codes(_value_groups(t["v"][0], case))
        if kind == "hold":
            c = _cached(case)[0][0]
            tok = torch.arange(F * case["tpp"], device=dev)
            at = tok % case["tpp"]
            s.cos, s.sin = _plain_table(torch.stack([c * F + tok // case["tpp"], at // case["grid_w"],
                                                     at % case["grid_w"]], 1), case, None)
        if kind == "rotate":  # the table that a program keeps: cosines and sines of every position of an axis
            s.axes = [_plain_axis(torch.arange(n, device=dev), d, SCALED[case["scaling"]] if a == 0 else None)
                      for a, (n, d) in enumerate(zip(_grid(case), (case["dim_t"], case["dim_h"], case["dim_w"])))]
        if kind == "move":
            s.pool = torch.stack([torch.cat([x.flatten(1) for x in _plain_pages(t, l, case)], 1).unflatten(0, (-1, F))
                                  for l in range(case["layers"])])  # [layer, state, frame, ...] of the kept states
            full = torch.zeros((case["layers"], 2 * case["states"]) + s.pool.shape[2:], dtype=s.pool.dtype, device=dev)
            full[:, 1::2] = s.pool
            s.pool, s.used = full, torch.arange(1, 2 * case["states"], 2, device=dev)
        return s

    import paper_2609_22283_amd as sc
    s.sc = sc
    states = [] if kind == "rotate" else _cached(case)
    if kind == "rotate":
        F_, h, w = _grid(case)
        dims = (case["dim_t"], case["dim_h"], case["dim_w"])
        table = torch.empty(sc.sc_rope_table_bytes(h, w, dims, F_), dtype=torch.uint8, device="cuda")
        s.rope = sc.sc_rope_table_build(table, h, w, dims, F_, theta=THETA, scaling=SCALED[case["scaling"]])
        return s
    if kind == "attend":
        _, s.cache = _pool(sc, 1, case, len(states) * F, sc.SC_DTYPE_FP4)
        for i, st in enumerate(states):
            s.cache.append(0, st, t["k"][0][i], t["v"][0][i])
        if case["window"] >= 0:
            s.plan = sc.sc_plan_build(
                sc.sc_selection_build(case["policy"], K_LEVELS, case["window"], _window_nodes(case)), s.cache)
        else:
            s.plan = sc.sc_plan_condition(s.cache, states[case["prefix"]:], case["nq"])
            if case["prefix"]:
                s.plan = sc.sc_plan_share(s.plan, states[:case["prefix"]])
        s.o, s.scale = torch.empty_like(t["q"]), D ** -0.5
        s.ws_bytes = sc.sc_attention_workspace_bytes(s.plan, s.cache)
        s.ws = torch.empty(max(16, s.ws_bytes), dtype=torch.uint8, device="cuda")
    elif kind == "hold":
        dims = (case["dim_t"], case["dim_h"], case["dim_w"])
        frames = (states[0][0] + 1) * F
        table = torch.empty(sc.sc_rope_table_bytes(case["grid_h"], case["grid_w"], dims, frames), dtype=torch.uint8,
                            device="cuda")
        s.rope = sc.sc_rope_table_build(table, case["grid_h"], case["grid_w"], dims, frames, theta=THETA)
        _, s.cache = _pool(sc, 1, case, F, sc.SC_DTYPE_FP4)
        pool, s.out = _pool(sc, 1, case, F, sc.SC_DTYPE_BF16)
        s.pages = _pages(pool, 1, case, F)
    elif kind == "park":
        L, slots = case["layers"], case["states"] * F
        _, s.src = _pool(sc, L, case, slots, sc.SC_DTYPE_BF16)
        for l in range(L):
            for i, st in enumerate(states):
                s.src.append(l, st, t["k"][l][i], t["v"][l][i])
        _, s.cache = _pool(sc, L, case, slots, sc.SC_DTYPE_FP4)
        pool, s.out = _pool(sc, L, case, slots, sc.SC_DTYPE_BF16)
        s.pages = _pages(pool, L, case, slots)
    else:
        L, n = case["layers"], case["states"]
        pool, s.cache = _pool(sc, L, case, 2 * n * F, sc.SC_DTYPE_BF16)
        for l in range(L):
            for i in range(2 * n):
                s.cache.append(l, (i, 0), t["k"][l][i // 2], t["v"][l][i // 2])
        for i in range(n):
            s.cache.release((2 * i, 0))
        bytes_ = sc.sc_cache_pool_bytes(L, case["heads"], D, case["tpp"], F, n * F, sc.SC_DTYPE_BF16)
        s.pools = [torch.zeros(bytes_, dtype=torch.uint8, device="cuda") for _ in range(2)]
    return s


# -------------------------------------------------------------------- one pass
def run(s):
    """attend: the outputs; hold, park and move: the pages' keys and values; rotate: the rotated rows."""
    t, case, kind = s.t, s.case, s.case["kind"]
    if not own:
        return {"attend": _plain_attend, "hold": _plain_hold, "park": _plain_park, "move": _plain_move,
                "rotate": _plain_rotate}[kind](s)
    sc, states = s.sc, [] if kind == "rotate" else _cached(case)
    if kind == "attend":
        sc.sc_attention(s.plan, s.cache, 0, t["q"], s.o, s.scale, s.ws, s.ws_bytes)
        return {"o": s.o}
    if kind == "rotate":
        sc.sc_rope_rotate(s.rope, t["x"], s.y, t["pos"], layout=case["layout"], transpose=case["transpose"])
        return {"y": s.y}
    if kind == "move":
        n = case["states"] * case["frames"]
        s.cache.move(s.pools[0], n)
        s.pools.reverse()
        k, v = _pages(s.pools[1], case["layers"], case, n)
        return {"k": k, "v": v}
    if kind == "hold":
        s.cache.append(0, states[0], t["k"][0][0], t["v"][0][0], rope=s.rope)
        s.cache.copy(states, s.out, states, 0, 1)
    else:
        s.src.copy(states, s.cache, states, 0, case["layers"])
        s.cache.copy(states, s.out, states, 0, case["layers"])
    for st in states:
        s.cache.release(st)
        s.out.release(st)
    return {"k": s.pages[0], "v": s.pages[1]}


# ------------------------------------------------------------------ plain forms
def _key_groups(k):
    """[..., token, head, channel] -> [..., token, head, channel / 32, 32]"""
    return k.unflatten(-1, (-1, GROUP))


def _value_groups(v, case):
    """[state, tokens, head, channel] -> [state * frame, token / 32, head, channel, 32], zeros behind a page's end"""
    v = v.reshape((-1, case["tpp"]) + v.shape[-2:])
    pad = -case["tpp"] % GROUP
    v = torch.cat([v, v.new_zeros((v.shape[0], pad) + v.shape[2:])], 1) if pad else v
    return v.unflatten(1, (-1, GROUP)).movedim(2, -1)


def _plain_codes(x):
    """Codes of four bits of groups [..., 32] and the exponent that each group shares."""
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    e = torch.clamp(torch.frexp(top).exponent - 3, min=-127)
    a = torch.ldexp(x.abs(), -e)
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    return code + 8 * (x < 0), e


def _plain_values(held):
    code, e = held
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=code.device)
    grid = torch.cat([grid, -grid])
    return torch.ldexp(grid[code.long()], e)


def _ungroup_values(g, case):
    """Back from _value_groups: [page, token, head, channel]"""
    return g.movedim(-1, 2).flatten(1, 2)[:, :case["tpp"]]


def _heads_first(x):
    return x.movedim(-2, -3).contiguous()


def _plain_attend(s):
    case, q = s.case, s.t["q"]
    H, nq, n = case["heads"], case["nq"], case["tpp"] * case["frames"]
    k = _plain_values(s.k).flatten(-2)
    v = _ungroup_values(_plain_values(s.v), case).reshape(-1, n, H, D)
    o = torch.empty_like(q)
    for i, row in enumerate(_reads(case)):
        kt = _heads_first(k[row].flatten(0, 1)).transpose(-1, -2).contiguous()
        p = torch.matmul(_heads_first(q[i * nq:(i + 1) * nq].float()), kt).mul_(D ** -0.5)
        p -= p.amax(-1, keepdim=True)
        p.exp_()
        p /= p.sum(-1, keepdim=True)
        o[i * nq:(i + 1) * nq] = torch.matmul(p, _heads_first(v[row].flatten(0, 1))).movedim(0, 1)
    return {"o": o}


def _plain_axis(pos, dim, scaled):
    """Cosines and sines [position, pair] of one axis, the angles in 64 bits."""
    i = torch.arange(dim // 2, dtype=torch.float64, device=pos.device)
    theta, kind = THETA, scaled["kind"] if scaled else ""
    if kind == "ntk" and dim > 2:
        theta *= scaled["factor"] ** (dim / (dim - 2))
    freq = theta ** (-2.0 * i / max(dim, 1))
    if kind == "linear":
        freq = freq / scaled["factor"]
    if kind == "yarn":
        turns = scaled["original"] * freq / (2 * math.pi)
        keep = ((turns - scaled["beta_slow"]) / (scaled["beta_fast"] - scaled["beta_slow"])).clamp(0, 1)
        freq = freq * (keep + (1 - keep) / scaled["factor"])
    ang = pos.double()[:, None] * freq
    return torch.cos(ang), torch.sin(ang)


def _plain_table(pos, case, scaled):
    """Cosines and sines [row, pair] at positions [row, 3], the axes' pairs one after another."""
    parts = [_plain_axis(pos[:, a], case[d], scaled if a == 0 else None) for a, d in enumerate(("dim_t", "dim_h", "dim_w"))]
    m = scaled.get("magnitude", 1.0) if scaled else 1.0
    return tuple((torch.cat([p[j] for p in parts], 1) * m).float()[:, None] for j in (0, 1))


def _plain_pages(t, l, case):
    """A layer's pages as a bf16 cache holds them: [state * frame, head, token, channel], [.., head, channel, token]"""
    shape = (-1, case["tpp"], case["heads"], D)
    return t["k"][l].reshape(shape).permute(0, 2, 1, 3), t["v"][l].reshape(shape).permute(0, 2, 3, 1)


def _plain_hold(s):
    """The keys are rotated and rounded as the bf16 cache rounds them: a product in 32 bits, then a fused multiply-add."""
    case, k = s.case, s.t["k"][0].float()
    x0, x1, c, n = k[..., 0::2], k[..., 1::2], s.cos.double(), s.sin
    k0 = (x0.double() * c - (x1 * n).double()).float()
    k1 = (x0.double() * n.double() + (x1 * s.cos).double()).float()
    k = torch.stack([k0, k1], -1).flatten(-2).to(torch.bfloat16)
    k = _plain_values(_plain_codes(_key_groups(k))).flatten(-2)
    v = _ungroup_values(_plain_values(_plain_codes(_value_groups(s.t["v"][0], case))), case)
    k = k.reshape(v.shape)
    return {"k": k.to(torch.bfloat16).permute(0, 2, 1, 3).contiguous()[None],
            "v": v.to(torch.bfloat16).permute(0, 2, 3, 1).contiguous()[None]}


def _plain_park(s):
    case, ks, vs = s.case, [], []
    for l in range(case["layers"]):
        k = _plain_values(_plain_codes(_key_groups(s.t["k"][l]))).flatten(-2)
        v = _ungroup_values(_plain_values(_plain_codes(_value_groups(s.t["v"][l], case))), case)
        ks.append(k.to(torch.bfloat16).reshape(v.shape).permute(0, 2, 1, 3).contiguous())
        vs.append(v.to(torch.bfloat16).permute(0, 2, 3, 1).contiguous())
    return {"k": torch.stack(ks), "v": torch.stack(vs)}


def _plain_move(s):
    case = s.case
    H, tpp = case["heads"], case["tpp"]
    p = s.pool[:, s.used].flatten(1, 2)  # [layer, page, keys and values]
    k, v = p[:, :, :H * tpp * D], p[:, :, H * tpp * D:]
    return {"k": k.unflatten(-1, (H, tpp, D)), "v": v.unflatten(-1, (H, D, tpp))}


def _plain_rotate(s):
    case, x = s.case, s.t["x"].float()
    part = case["dim_t"] + case["dim_h"] + case["dim_w"]
    m = (SCALED[case["scaling"]] or {}).get("magnitude", 1.0)
    pos = s.t["pos"].long()
    c, n = ((torch.cat([ax[j][pos[:, a]] for a, ax in enumerate(s.axes)], 1) * m).float()[:, None] for j in (0, 1))
    n = -n if case["transpose"] else n
    y = x.clone()
    if case["layout"] == "half":
        a, b = slice(0, part // 2), slice(part // 2, part)
    else:
        a, b = slice(0, part, 2), slice(1, part, 2)
    y[..., a] = x[..., a] * c - x[..., b] * n
    y[..., b] = x[..., a] * n + x[..., b] * c
    return {"y": y.to(s.t["x"].dtype)}


# ------------------------------------------------------------------- its work
def work(case):
    """Every input read once, every output written once; 4-bit pages at 17 bytes for 32 values."""
    H = case["heads"]
    if case["kind"] == "rotate":
        size = 4 if case["dtype"] == "f32" else 2
        n = case["rows"] * H * case["head_dim"]
        return {"bytes": 2.0 * size * n + 12.0 * case["rows"], "flops": 0.0}
    n = case["tpp"] * case["frames"]
    held = 17.0 / 32.0
    if case["kind"] == "attend":
        reads = _reads(case)
        keys = n * len({i for r in reads for i in r})
        pairs = case["nq"] * n * sum(len(r) for r in reads)
        return {"bytes": 4.0 * H * D * case["nodes"] * case["nq"] + 2.0 * held * H * D * keys, "flops": 4.0 * H * D * pairs}
    values = 2.0 * H * D * n * len(_cached(case)) * case.get("layers", 1)
    return {"bytes": values * (4.0 if case["kind"] == "move" else 4.0 + held), "flops": 0.0}


# ------------------------------------------------------------- the exact results
def _exact_held(x):
    """Groups [..., 32] as the values that their codes stand for: multiples of a half, one or two of the
    shared power of two, by size, the nearest (of two the even one), six at most."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(torch.where(top > 0, top, torch.ones_like(top)))) - 2
    unit = torch.exp2(torch.clamp(e, min=-127))
    a = x.abs() / unit
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).double()
    return torch.sign(x) * torch.clamp(torch.round(a / step) * step, max=6.0) * unit


def _exact_pages(k, v, case):
    """Held keys [page, head, token, channel] and values [page, head, channel, token] of bf16 ones
    [states, tokens, head, channel]."""
    H, tpp = case["heads"], case["tpp"]
    shape = (-1, tpp, H, D)
    kk = _exact_held(k.reshape(-1, GROUP)).reshape(shape).permute(0, 2, 1, 3)
    vt = v.reshape(shape).permute(0, 2, 3, 1).double()  # [page, head, channel, token]
    vv = torch.cat([_exact_held(g) for g in vt.split(GROUP, -1)], -1)
    return kk.contiguous(), vv.contiguous()


def exact(case, seed):
    t, kind = _inputs(case, seed), case["kind"]
    if kind == "attend":
        return _exact_attend(case, t)
    if kind == "rotate":
        return _exact_rotate(case, t)
    if kind == "move":
        pages = [_plain_layout(t["k"][l], t["v"][l], case) for l in range(case["layers"])]
        return {"k": torch.stack([p[0] for p in pages]), "v": torch.stack([p[1] for p in pages])}
    if kind == "park":
        pages = [_exact_pages(t["k"][l], t["v"][l], case) for l in range(case["layers"])]
        return {"k": torch.stack([p[0] for p in pages]), "v": torch.stack([p[1] for p in pages])}
    # hold: the rotation as the bf16 cache does it, whose roundings are part of what the codes are taken from
    F, tpp, w = case["frames"], case["tpp"], case["grid_w"]
    k = t["k"][0].double()
    out = torch.empty_like(k)
    pair = 0
    for axis, dim in enumerate((case["dim_t"], case["dim_h"], case["dim_w"])):
        for i in range(dim // 2):
            tok = torch.arange(F * tpp, device=k.device, dtype=torch.float64)
            at = tok % tpp
            p = [_cached(case)[0][0] * F + torch.floor(tok / tpp), torch.floor(at / w), at % w][axis]
            ang = p * THETA ** (-2.0 * i / dim)
            c, n = (f(ang).float().double()[:, None] for f in (torch.cos, torch.sin))
            x0, x1 = k[..., 2 * pair], k[..., 2 * pair + 1]
            out[..., 2 * pair] = (x0 * c - (x1 * n).float().double()).float().double()
            out[..., 2 * pair + 1] = (x0 * n + (x1 * c).float().double()).float().double()
            pair += 1
    kk, vv = _exact_pages(out.to(torch.bfloat16), t["v"][0], case)
    return {"k": kk[None], "v": vv[None]}


def _plain_layout(k, v, case):
    shape = (-1, case["tpp"], case["heads"], D)
    return (k.double().reshape(shape).permute(0, 2, 1, 3).contiguous(),
            v.double().reshape(shape).permute(0, 2, 3, 1).contiguous())


def _exact_attend(case, t):
    H, nq = case["heads"], case["nq"]
    if work(case)["flops"] > 2e13:
        return None
    F = case["frames"]
    k, v = _exact_pages(t["k"][0], t["v"][0], case)
    o = torch.empty(t["q"].shape, dtype=torch.float64, device=t["q"].device)
    for i, row in enumerate(_reads(case)):
        pages = [j * F + f for j in row for f in range(F)]
        for h in range(H):
            p = t["q"][i * nq:(i + 1) * nq, h].double() @ k[pages, h].reshape(-1, D).T / math.sqrt(D)
            o[i * nq:(i + 1) * nq, h] = torch.softmax(p, -1) @ v[pages, h].transpose(1, 2).reshape(-1, D)
    return {"o": o}


def _exact_rotate(case, t):
    x = t["x"].double()
    y = x.clone()
    half = (case["dim_t"] + case["dim_h"] + case["dim_w"]) // 2
    sc = SCALED[case["scaling"]] or {}
    m, pair = sc.get("magnitude", 1.0), 0
    for axis, dim in enumerate((case["dim_t"], case["dim_h"], case["dim_w"])):
        for i in range(dim // 2):
            f = THETA ** (-2.0 * i / dim)
            if axis == 0 and sc.get("kind") == "linear":
                f /= sc["factor"]
            if axis == 0 and sc.get("kind") == "ntk" and dim > 2:
                f = (THETA * sc["factor"] ** (dim / (dim - 2.0))) ** (-2.0 * i / dim)
            if axis == 0 and sc.get("kind") == "yarn":
                keep = (sc["original"] * f / (2 * math.pi) - sc["beta_slow"]) / (sc["beta_fast"] - sc["beta_slow"])
                keep = min(1.0, max(0.0, keep))
                f = f * keep + f / sc["factor"] * (1.0 - keep)
            z = torch.polar(torch.full_like(t["pos"][:, 0], m, dtype=torch.float64), t["pos"][:, axis].double() * f)[:, None]
            z = z.conj() if case["transpose"] else z
            a, b = (pair, pair + half) if case["layout"] == "half" else (2 * pair, 2 * pair + 1)
            r = torch.complex(x[..., a], x[..., b]) * z
            y[..., a], y[..., b] = r.real, r.imag
            pair += 1
    return {"y": y}
