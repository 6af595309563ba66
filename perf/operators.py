"""The operators of a bounded, shared history, as measurable cases.

  weigh     sc_attention_weigh: the packed attention, with the weight that every
            cached key received added to an array kept beside the cache
  condense  Cache.condense: the heaviest tokens of several states, head by head,
            gathered into the pages of one
  share     sc_attention over sc_plan_share: nodes that read a long prefix, the
            same for all, before the pages of their own

With ``own`` false every operator runs in its plain form, elementary torch
operations in 32 bits.  Sizes are those of the repository's configurations
(12 heads of 128, 30x52 tokens per latent frame, three frames per chunk, the
short streaming frames of 64 and 128 tokens, the small ragged test geometries)
and of the range between them.
"""
from __future__ import annotations

import math

import torch

own = False

K_LEVELS = 4
Q_SCALE = 2.0  # logits of standard deviation 2: some keys matter, most do not


# ------------------------------------------------------------------- the cases
def _weigh(name, dtype, heads, head_dim, grid_h, grid_w, frames, nodes, window, policy="prog"):
    return {"name": name, "kind": "weigh", "dtype": dtype, "heads": heads, "head_dim": head_dim,
            "tpp": grid_h * grid_w, "frames": frames, "nodes": nodes, "window": window, "policy": policy}


def _condense(name, dtype, heads, head_dim, tpp, frames, sources, layers):
    return {"name": name, "kind": "condense", "dtype": dtype, "heads": heads, "head_dim": head_dim,
            "tpp": tpp, "frames": frames, "sources": sources, "layers": layers}


def _share(name, dtype, heads, head_dim, tpp, frames, nodes, nq, prefix):
    """Every node reads ``prefix`` shared states and one state of its own."""
    return {"name": name, "kind": "share", "dtype": dtype, "heads": heads, "head_dim": head_dim,
            "tpp": tpp, "frames": frames, "nodes": nodes, "nq": nq, "prefix": prefix}


def listed():
    return [
        # one short frame weighed against its window: the smallest call of a streaming step
        _weigh("weigh_short_serial", "bf16", 12, 128, 8, 8, 1, 1, 20, "clean"),
        # an fp32 cache, pages that end inside key tiles
        _weigh("weigh_f32_small", "f32", 2, 128, 8, 13, 3, 4, 3),
        # three nodes at a reduced resolution, every tile ragged
        _weigh("weigh_mid_ragged", "bf16", 12, 128, 11, 24, 3, 3, 6, "same"),
        # the headline pack: four nodes of a progressive diagonal over their windows
        _weigh("weigh_wan_pack4", "bf16", 12, 128, 30, 52, 3, 4, 6),
        # single tokens of a few answers over one short prompt: latency alone
        _share("share_few_tokens", "bf16", 12, 128, 64, 1, 4, 1, 8),
        # single tokens of 32 continuations of one long history: reading it once is the work
        _share("share_tokens", "bf16", 12, 128, 64, 1, 32, 1, 256),
        # sixteen candidates for the next 128-token frame, from one history
        _share("share_candidates", "bf16", 12, 128, 128, 1, 16, 128, 128),
        # four full-size chunks that read one memory of two chunks beside themselves
        _share("share_wan_memory", "bf16", 12, 128, 1560, 3, 4, 4680, 2),
        # a small fp32 cache
        _condense("condense_f32_small", "f32", 2, 64, 104, 3, 2, 1),
        # a short stream's whole window folded to one frame, in every layer of a 30-block model
        _condense("condense_short_stack", "bf16", 12, 128, 64, 1, 21, 30),
        # three full-size chunks to one, one layer
        _condense("condense_wan_layer", "bf16", 12, 128, 1560, 3, 3, 1),
        # two full-size chunks to one in eight layers at once
        _condense("condense_wan_stack", "bf16", 12, 128, 1560, 3, 2, 8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["weigh", "condense", "share"])
    f32 = rng.random() < 0.3
    dtype, heads = ("f32", rng.choice([2, 3, 12])) if f32 else ("bf16", rng.choice([2, 7, 12]))
    head_dim = rng.choice([64, 128]) if f32 or kind == "condense" else 128
    tpp, frames = 8 * _log_int(rng, 8, 195), rng.choice([1, 2, 3])
    if f32:
        tpp = 8 * _log_int(rng, 2, 24)
    if kind == "weigh":
        policy = rng.choice(["prog", "prog", "same", "clean"])
        window = rng.randint(0, 6) if tpp * frames > 400 else rng.randint(0, 20)
        nodes = 1 if policy == "clean" else rng.randint(1, 4)
        case = _weigh("", dtype, heads, head_dim, 1, tpp, frames, nodes, window, policy)
    elif kind == "condense":
        layers = rng.choice([1, 1, 2, 4, 8]) if tpp * frames > 400 else _log_int(rng, 1, 30)
        case = _condense("", dtype, heads, head_dim, tpp, frames, rng.randint(2, 4 if tpp > 400 else 16), layers)
    else:
        nodes, nq = _log_int(rng, 1, 64), _log_int(rng, 1, 512)
        tpp, frames = min(tpp, 512), rng.choice([1, 1, 2])
        nodes = max(1, min(nodes, 4096 // nq, 32768 // (tpp * frames)))
        most = min(768 // frames - nodes, 32768 // (tpp * frames), (1 << 25) // (nodes * nq * tpp * frames))
        case = _share("", dtype, heads, head_dim, tpp, frames, nodes, nq, _log_int(rng, 1, max(1, most)))
    case.pop("name")
    return case


# ------------------------------------------------------------------ case geometry
def _window_nodes(case):
    """The pack of a weigh case, oldest chunk first, behind a full window of history."""
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
    if case["kind"] == "weigh":
        level = 2 if case["policy"] == "same" else 0
        return [(c, level) for c in range(case["window"])] + _window_nodes(case)
    if case["kind"] == "condense":
        return [(c, 0) for c in range(case["sources"])]
    return [(c, 0) for c in range(case["prefix"] + case["nodes"])]


def _reads(case):
    """For each node, the indices (in _cached) of the states that it reads, in order."""
    if case["kind"] == "weigh":
        at = {st: i for i, st in enumerate(_cached(case))}
        return [[at[st] for st in _segments(case, nd)] for nd in _window_nodes(case)]
    return [list(range(case["prefix"])) + [case["prefix"] + i] for i in range(case["nodes"])]


def _queries(case):
    return case["nq"] if case["kind"] == "share" else case["tpp"] * case["frames"]


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


# ----------------------------------------------------------------------- inputs
class _State:
    pass


def _inputs(case, seed):
    """Cached K/V [states, tokens, heads, head_dim] (per layer for condense) and
    queries of normal entries; weights as attention leaves them: a heavy tail,
    of about what one pass adds, and some tokens that nothing has read yet."""
    dev = "cuda" if torch.cuda.is_available() else "cpu"
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def normal(shape):
        return torch.randn(shape, generator=gen, device=dev, dtype=torch.float32)

    H, d, tpp, F = case["heads"], case["head_dim"], case["tpp"], case["frames"]
    n, states, layers = tpp * F, len(_cached(case)), case.get("layers", 1)
    t = {"k": [], "v": []}
    for _ in range(layers):  # one layer at a time: the fp32 draws of a stack do not lie beside each other
        t["k"].append(normal((states, n, H, d)).to(_dtype(case)))
        t["v"].append(normal((states, n, H, d)).to(_dtype(case)))
    if case["kind"] != "condense":
        t["k"], t["v"] = t["k"][0], t["v"][0]
        t["q"] = (normal((case["nodes"] * _queries(case), H, d)) * Q_SCALE).to(_dtype(case))
    if case["kind"] != "share":
        slots = (states + 1) * F if case["kind"] == "condense" else states * F
        w = torch.exp(2.0 * normal((layers, slots, H, tpp)))
        if case["kind"] == "weigh":
            w *= 0.1 * case["nodes"] / states  # a pass gives its queries' count, spread over the keys
        unread = torch.rand((layers, slots, H, tpp), generator=gen, device=dev) < 0.1
        t["weights"] = torch.where(unread, torch.zeros_like(w), w)
    return t


def _page_index(case, device):
    """[nodes, pages] slots that each node reads."""
    F = case["frames"]
    return torch.tensor([[s * F + f for s in row for f in range(F)] for row in _reads(case)], device=device)


def prepare(case, seed):
    s = _State()
    s.case, s.t = case, _inputs(case, seed)
    t, kind = s.t, case["kind"]
    H, d, tpp, F = case["heads"], case["head_dim"], case["tpp"], case["frames"]
    states = _cached(case)
    if not own:
        dev = t["k"][0].device
        if kind != "condense":
            s.reads = torch.tensor(_reads(case), device=dev)
            s.pages = _page_index(case, dev)
        return s

    import paper_2609_22283_amd as sc
    s.sc = sc
    dt = sc.SC_DTYPE_F32 if case["dtype"] == "f32" else sc.SC_DTYPE_BF16
    layers = case.get("layers", 1)
    slots = (len(states) + (1 if kind == "condense" else 0)) * F
    args = (layers, H, d, tpp, F, slots, dt)
    pool = torch.empty(sc.sc_cache_pool_bytes(*args), dtype=torch.uint8, device="cuda")
    s.cache = sc.sc_cache_create(pool, *args)
    s.scale = d ** -0.5
    for i, st in enumerate(states):
        for l in range(layers):
            k, v = (t["k"][l], t["v"][l]) if kind == "condense" else (t["k"], t["v"])
            s.cache.append(l, st, k[i], v[i])
    if kind == "condense":
        pages = pool.view(_dtype(case)).view(layers, slots, 2, H, tpp * d)[:, len(states) * F:]
        s.k = pages[:, :, 0].view(layers, F, H, tpp, d)
        s.v = pages[:, :, 1].view(layers, F, H, d, tpp)
        s.kept = torch.empty((layers, H, F * tpp), dtype=torch.int32, device="cuda")
        return s
    s.o = torch.empty_like(t["q"])
    if kind == "weigh":
        sel = sc.sc_selection_build(case["policy"], K_LEVELS, case["window"], _window_nodes(case))
        s.plan = sc.sc_plan_build(sel, s.cache)
        s.ws_bytes = sc.sc_attention_weigh_workspace_bytes(s.plan, s.cache)
    else:
        alone = sc.sc_plan_condition(s.cache, states[case["prefix"]:], case["nq"])
        s.plan = sc.sc_plan_share(alone, states[:case["prefix"]])
        s.ws_bytes = sc.sc_attention_workspace_bytes(s.plan, s.cache)
    s.ws = torch.empty(max(16, s.ws_bytes), dtype=torch.uint8, device="cuda")
    return s


# -------------------------------------------------------------------- one pass
def run(s):
    """weigh: the outputs and the accumulated weights [slots, heads, tokens];
    share: the outputs; condense: the new state's pages, its weights and the
    indices of the tokens that each head kept."""
    t, kind = s.t, s.case["kind"]
    if own:
        sc = s.sc
        if kind == "weigh":
            sc.sc_attention_weigh(s.plan, s.cache, 0, t["q"], s.o, s.scale, t["weights"], s.ws, s.ws_bytes)
            return {"o": s.o, "weights": t["weights"]}
        if kind == "share":
            sc.sc_attention(s.plan, s.cache, 0, t["q"], s.o, s.scale, s.ws, s.ws_bytes)
            return {"o": s.o}
        n = s.case["sources"]
        s.cache.condense(0, s.case["layers"], [(c, 0) for c in range(n)], (n, 0), t["weights"], s.kept)
        s.cache.release((n, 0))
        return {"k": s.k, "v": s.v, "weights": t["weights"][:, n * s.case["frames"]:], "kept": s.kept}
    if kind == "condense":
        return _plain_condense(s)
    return _plain_attention(s)


def _heads_first(x):
    return x.float().movedim(-2, -3).contiguous()


def _softmax_(x):
    x -= x.amax(-1, keepdim=True)
    x.exp_()
    x /= x.sum(-1, keepdim=True)
    return x


def _plain_attention(s):
    case, t = s.case, s.t
    H, d, nodes, nq = case["heads"], case["head_dim"], case["nodes"], _queries(case)
    if case["kind"] == "weigh":
        q = _heads_first(t["q"].view(nodes, nq, H, d))
        k = _heads_first(t["k"][s.reads].flatten(1, 2))
        v = _heads_first(t["v"][s.reads].flatten(1, 2))
        p = torch.matmul(q, k.transpose(-1, -2))
        p = _softmax_(p.mul_(d ** -0.5))
        o = torch.matmul(p, v).movedim(1, 2).reshape(-1, H, d).to(_dtype(case))
        got = p.sum(-2).view(nodes, H, s.pages.shape[1], case["tpp"]).transpose(1, 2)
        t["weights"][0].index_add_(0, s.pages.reshape(-1), got.flatten(0, 1))
        return {"o": o, "weights": t["weights"]}
    # the prefix's products once for all rows, the own ones node by node (batched)
    P = case["prefix"]
    kp, vp = (_heads_first(x[:P].flatten(0, 1)) for x in (t["k"], t["v"]))
    ko, vo = (_heads_first(x[P:]) for x in (t["k"], t["v"]))
    q = _heads_first(t["q"])
    a = torch.matmul(q, kp.transpose(-1, -2)).view(H, nodes, nq, -1)
    qn = q.view(H, nodes, nq, d).transpose(0, 1).contiguous()
    b = torch.matmul(qn, ko.transpose(-1, -2)).transpose(0, 1)
    p = _softmax_(torch.cat([a, b], -1).mul_(d ** -0.5))
    m = kp.shape[1]
    o = torch.matmul(p[..., :m].reshape(H, nodes * nq, m), vp).view(H, nodes, nq, d)
    o = o + torch.matmul(p[..., m:].transpose(0, 1).contiguous(), vo).transpose(0, 1)
    return {"o": o.movedim(0, 2).reshape(-1, H, d).to(_dtype(case))}


def _plain_condense(s):
    case, t = s.case, s.t
    H, d, tpp, F, n = case["heads"], case["head_dim"], case["tpp"], case["frames"], case["sources"]
    L = case["layers"]
    w = t["weights"]
    flat = w[:, :n * F].transpose(1, 2).reshape(L, H, n * F * tpp)
    order = torch.sort(flat, dim=-1, descending=True, stable=True).indices[..., :F * tpp]
    kept = torch.sort(order, dim=-1).values
    w[:, n * F:] = torch.gather(flat, -1, kept).view(L, H, F, tpp).transpose(1, 2)
    pick = kept[..., None].expand(-1, -1, -1, d)

    def gathered(x):
        x = torch.stack(x).flatten(1, 2).transpose(1, 2)  # [layer, head, token, channel]
        return torch.gather(x, 2, pick).view(L, H, F, tpp, d).transpose(1, 2)

    k, v = gathered(t["k"]), gathered(t["v"]).transpose(-1, -2)
    return {"k": k.contiguous(), "v": v.contiguous(), "weights": w[:, n * F:], "kept": kept.to(torch.int32)}


# ------------------------------------------------------------------- its work
def _pairs(case):
    """(query, key) pairs and distinct keys of an attention case."""
    n, reads = case["tpp"] * case["frames"], _reads(case)
    return _queries(case) * n * sum(len(r) for r in reads), n * len({i for r in reads for i in r})


def work(case):
    size, D = 4 if case["dtype"] == "f32" else 2, case["heads"] * case["head_dim"]
    if case["kind"] == "condense":
        n, N = case["tpp"] * case["frames"], case["sources"] * case["tpp"] * case["frames"]
        return {"bytes": case["layers"] * (4.0 * size * n * D + case["heads"] * (4.0 * N + 8.0 * n)), "flops": 0.0}
    pairs, keys = _pairs(case)
    nbytes = 2.0 * size * D * (case["nodes"] * _queries(case) + keys)
    if case["kind"] == "weigh":
        nbytes += 8.0 * case["heads"] * keys
    return {"bytes": nbytes, "flops": 4.0 * D * pairs}


# ------------------------------------------------------------- the exact results
def exact(case, seed):
    t = _inputs(case, seed)
    H, d, tpp, F = case["heads"], case["head_dim"], case["tpp"], case["frames"]
    if case["kind"] == "condense":
        return _exact_condense(case, t)
    if 4.0 * H * d * _pairs(case)[0] > 2e13:
        return None
    nq = _queries(case)
    o = torch.empty(t["q"].shape, dtype=torch.float64, device=t["q"].device)
    w = t["weights"].double() if case["kind"] == "weigh" else None
    for i, row in enumerate(_reads(case)):
        for h in range(H):
            k = torch.cat([t["k"][j, :, h] for j in row]).double()
            v = torch.cat([t["v"][j, :, h] for j in row]).double()
            p = torch.softmax(t["q"][i * nq:(i + 1) * nq, h].double() @ k.T / math.sqrt(d), -1)
            o[i * nq:(i + 1) * nq, h] = p @ v
            if w is not None:
                each = p.sum(0).split(tpp)
                for j, state in enumerate(row):
                    for f in range(F):
                        w[0, state * F + f, h] += each[j * F + f]
    return {"o": o} if w is None else {"o": o, "weights": w}


def _exact_condense(case, t):
    """The n heaviest of every head by rank: a token's rank is the number of
    heavier tokens, and of equal ones before it."""
    H, d, tpp, F, n, L = (case[k] for k in ("heads", "head_dim", "tpp", "frames", "sources", "layers"))
    dev, N, m = t["k"][0].device, n * F * tpp, F * tpp
    k = torch.empty((L, F, H, tpp, d), dtype=torch.float64, device=dev)
    v = torch.empty((L, F, H, d, tpp), dtype=torch.float64, device=dev)
    w = torch.empty((L, F, H, tpp), dtype=torch.float64, device=dev)
    kept = torch.empty((L, H, m), dtype=torch.int32, device=dev)
    for l in range(L):
        for h in range(H):
            x = t["weights"][l, :n * F, h].reshape(-1).double()
            low = x.sort().values[N - m]  # the lightest weight that is kept
            equal = x == low
            take = (x > low) | (equal & (equal.cumsum(0) <= m - int((x > low).sum())))
            idx = torch.nonzero(take).view(-1)
            kept[l, h] = idx.to(torch.int32)
            w[l, :, h] = x[idx].view(F, tpp)
            k[l, :, h] = t["k"][l][:, :, h].reshape(N, d)[idx].double().view(F, tpp, d)
            v[l, :, h] = t["v"][l][:, :, h].reshape(N, d)[idx].double().view(F, tpp, d).transpose(1, 2)
    return {"k": k, "v": v, "weights": w, "kept": kept}
