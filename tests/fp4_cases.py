"""Caches in 4 bits for the GPU tests: seeded states, their held values, an attention oracle
and what the roundings of the path may add up to."""
import math

import numpy as np
import torch

import paper_2609_22283_amd as sc
from oracle.held import held_keys, held_values
from synth import TAG_K, TAG_Q, TAG_V, bf16_bits, bf16_value, normal

D = 128


def bf16_dev(x):
    """fp32 numpy -> bf16 device tensor (rounded to nearest even), and its values in fp64"""
    bits = bf16_bits(np.ascontiguousarray(x, dtype=np.float32))
    t = torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16)
    return t, bf16_value(bits).astype(np.float64)


def make_cache(dtype, heads, tpp, frames, slots, layers=1, fill=0x5a):
    args = (layers, heads, D, tpp, frames, slots, dtype)
    pool = torch.full((sc.sc_cache_pool_bytes(*args),), fill, dtype=torch.uint8, device="cuda")
    return pool, sc.sc_cache_create(pool, *args)


def bf16_pages(pool, heads, tpp, slots, layers=1):
    """A bf16 pool: K [layer, slot, head, token, d], V [layer, slot, head, d, token], fp64 numpy"""
    p = pool.view(torch.bfloat16).view(layers, slots, 2, heads, tpp * D).float().cpu().double().numpy()
    return p[:, :, 0].reshape(layers, slots, heads, tpp, D), p[:, :, 1].reshape(layers, slots, heads, D, tpp)


class Held:
    """A 4-bit cache with states appended in layer ``layer``; k and v hold their values."""

    def __init__(self, heads, tpp, frames, states, extra_slots=0, layers=1, layer=0, seed=0, spread=1.0, edit=None):
        self.heads, self.tpp, self.frames, self.layer, self.seed = heads, tpp, frames, layer, seed
        self.pool, self.cache = make_cache(sc.SC_DTYPE_FP4, heads, tpp, frames,
                                           len(states) * frames + extra_slots, layers, fill=0xff)
        n = tpp * frames
        self.k, self.v = {}, {}
        for st in states:
            k, v = (normal((n, heads, D), (seed, tag) + st) * spread for tag in (TAG_K, TAG_V))
            if edit is not None:
                edit(st, k, v)
            kd, kv = bf16_dev(k)
            vd, vv = bf16_dev(v)
            self.cache.append(layer, st, kd, vd)
            self.k[st], self.v[st] = held_keys(kv), held_values(vv, tpp)
        torch.cuda.synchronize()

    def queries(self, rows, scale=1.0):
        return bf16_dev(normal((rows, self.heads, D), (self.seed, TAG_Q, rows)) * scale)


def attend(h: Held, plan, q, scale=D ** -0.5, stream=None):
    o = torch.full_like(q, float("nan"))
    nb = sc.sc_attention_workspace_bytes(plan, h.cache)
    ws = torch.full((max(16, nb),), 0xff, dtype=torch.uint8, device="cuda")
    sc.sc_attention(plan, h.cache, h.layer, q, o, scale, ws, nb, stream=stream)
    torch.cuda.synchronize()
    return o.float().cpu().double().numpy()


def oracle(h: Held, reads, q, nq, scale=D ** -0.5):
    """(outputs, what they may be off by): reads[i] are the states of node i.

    With p the exact probabilities, a kernel's are off by a factor from the logits' error
    d and by the rounding of the exponentials to 8 bits, 2^-8 each at most; the output is
    rounded to bf16, 2^-8 of it.  d: 128 products summed in fp32, 2^-24 of the sum of their
    magnitudes at each step, and queries split into two numbers of four bits leave 2^-20
    of the row's largest value in each.  What is small beside the largest exponential near it is
    not held to 8 bits of itself: scaled so that the largest is 2^8, the second of two e4m3
    numbers that hold one together (the first one's rest times 2^4) ends at steps of 2^-9,
    2^-13 in the first one's scale, so that half a step is 2^-22 of the largest; in the
    same way what is below the smallest fp32 number becomes 0."""
    out, tol = np.empty(q.shape), np.empty(q.shape)
    for i, states in enumerate(reads):
        r = slice(i * nq, (i + 1) * nq)
        for x in range(h.heads):
            k = np.concatenate([h.k[s][:, x] for s in states])
            v = np.concatenate([h.v[s][:, x] for s in states])
            qq = q[r, x]
            s = qq @ k.T * scale
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            out[r, x] = p @ v
            mag = abs(scale) * (np.abs(qq) @ np.abs(k).T).max(-1)
            rest = abs(scale) * np.abs(qq).max(-1) * np.abs(k).sum(-1).max()
            d = 128 * 2.0 ** -24 * mag + 2.0 ** -20 * rest
            tol[r, x] = 2.0 ** -8 * np.abs(out[r, x]) + (2.0 ** -8 + np.expm1(2 * d)[:, None]) * (p @ np.abs(v))
            tol[r, x] += 2.0 ** -22 * p.max(-1, keepdims=True) * np.abs(v).sum(0)
    return out, tol


def check(got, want, tol, what=""):
    bad = ~(np.abs(got - want) <= tol)
    worst = np.nanmax(np.abs(got - want) / tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} off, worst {worst:.2f} of its bound"


def condition_plan(h: Held, prefix, own, nq):
    plan = sc.sc_plan_condition(h.cache, own, nq)
    return sc.sc_plan_share(plan, prefix) if prefix else plan
