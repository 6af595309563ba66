"""Helpers of the tests of the bounded, shared history: a poisoned cache with known
K/V in it, and the operators' formulas in 64 bits."""
from __future__ import annotations

import torch

import paper_2609_22283_amd as sc

DTYPES = {"bf16": (torch.bfloat16, sc.SC_DTYPE_BF16), "f32": (torch.float32, sc.SC_DTYPE_F32)}


class MemCache:
    """A cache of `states` (appended in order), every byte of its pool NaN before, with
    `spare` free states' slots.  kv[state][layer]: (k, v) [tokens, heads, d] on the GPU."""

    def __init__(self, dtype, heads, hd, tpp, ppc, states, layers=1, spare=2, seed=0, key_fn=None, value_fn=None):
        self.dtype, self.heads, self.hd, self.tpp, self.ppc = dtype, heads, hd, tpp, ppc
        self.layers, self.n = layers, tpp * ppc
        self.tdt, code = DTYPES[dtype]
        self.n_slots = (len(states) + spare) * ppc
        args = (layers, heads, hd, tpp, ppc, self.n_slots, code)
        self.pool = torch.full((sc.sc_cache_pool_bytes(*args),), 0xFF, dtype=torch.uint8, device="cuda")
        self.cache = sc.sc_cache_create(self.pool, *args)
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        self.kv = {}
        for st in states:
            per = []
            for layer in range(layers):
                k, v = self.normal((self.n, heads, hd)), self.normal((self.n, heads, hd))
                k = (k if key_fn is None else key_fn(st, k)).to(self.tdt)
                v = (v if value_fn is None else value_fn(st, v)).to(self.tdt)
                self.cache.append(layer, st, k, v)
                per.append((k, v))
            self.kv[st] = per

    def normal(self, shape, scale=1.0):
        return torch.randn(shape, generator=self.gen, device="cuda") * scale

    def queries(self, rows, scale=2.0):
        return self.normal((rows, self.heads, self.hd), scale).to(self.tdt)

    def weights(self):
        """A weights array of the cache: small positive values, which an operator adds to."""
        w = torch.rand((self.layers, self.n_slots, self.heads, self.tpp), generator=self.gen, device="cuda") * 0.25
        assert w.numel() * 4 == sc.sc_cache_weights_bytes(self.cache)
        return w

    def pages(self, state, layer=0):
        """(k [tokens, heads, d], v likewise) as they lie in the state's pages."""
        size = 2 if self.dtype == "bf16" else 4
        flat = self.pool.view(torch.int16 if size == 2 else torch.int32).view(self.layers, self.n_slots, 2, -1)
        got = flat[layer, self.cache.slots(state)].view(self.tdt)
        k = got[:, 0].reshape(self.ppc, self.heads, self.tpp, self.hd).transpose(1, 2).reshape(self.n, self.heads, self.hd)
        v = got[:, 1].reshape(self.ppc, self.heads, self.hd, self.tpp).permute(0, 3, 1, 2).reshape(self.n, self.heads, self.hd)
        return k, v

    def attend(self, q, reads, scale, layer=0):
        """(o [rows, heads, d], probability column sums per state {state: [heads, tokens]})
        in 64 bits; reads: per node the states that it reads, q its rows after the other's."""
        nq = q.shape[0] // len(reads)
        o = torch.empty(q.shape, dtype=torch.float64, device="cuda")
        sums = {}
        for i, states in enumerate(reads):
            for h in range(self.heads):
                k = torch.cat([self.kv[s][layer][0][:, h] for s in states]).double()
                v = torch.cat([self.kv[s][layer][1][:, h] for s in states]).double()
                p = torch.softmax(q[i * nq:(i + 1) * nq, h].double() @ k.T * scale, -1)
                o[i * nq:(i + 1) * nq, h] = p @ v
                for s, part in zip(states, p.sum(0).split(self.n)):
                    sums.setdefault(s, torch.zeros((self.heads, self.n), dtype=torch.float64, device="cuda"))[h] += part
        return o, sums

    def weights_after(self, before, sums, layer=0):
        w = before.double()
        for s, part in sums.items():
            for f, slot in enumerate(self.cache.slots(s)):
                w[layer, slot] += part[:, f * self.tpp:(f + 1) * self.tpp]
        return w


def weight_bound(case, q, scale, keys):
    """Largest relative error of a probability computed in fp32 from the stored
    values: a d-term dot product is off by (d + 2) 2^-24 sum |q k| at most, which
    moves the exponent of the numerator and those of the row's sum; the sum itself
    and its logarithm (below 2^6 in size), the exponential and the sums over
    rows add a few units of 2^-24 for each of keys / 32 + 128 additions."""
    qa = q.float().abs().amax(0)
    big = max(float((qa * k.float().abs().amax(0)).sum(-1).max()) for per in case.kv.values() for k, _ in per)
    return 2 * abs(scale) * big * (case.hd + 2) * 2.0 ** -24 + (keys / 32 + 128) * 2.0 ** -24 + 2.0 ** -18


def bf16_close(got, want, what):
    """The attention's gates (bf16): largest and mean error, and per head relative."""
    d = (got.double() - want).abs()
    assert torch.isfinite(got).all(), what
    top = max(1.0, float(want.abs().max()))
    assert float(d.max()) <= 2e-2 * top, f"{what}: max {float(d.max()):.3g}"
    assert float(d.mean()) <= 2e-3 * top, f"{what}: mean {float(d.mean()):.3g}"
    for h in range(want.shape[1]):
        rel = float((got[:, h].double() - want[:, h]).norm() / want[:, h].norm())
        assert rel <= 1e-2, f"{what}: head {h} relative {rel:.3g}"


def close(dtype, got, want, what):
    if dtype == "bf16":
        bf16_close(got, want, what)
    else:
        assert float((got.double() - want).abs().max()) <= 1e-4, what
