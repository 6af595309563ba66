"""Round driver of the streaming schedule (Sec. 3.3), on top of the C ABI.

Each chunk's current latent state lives in ``xs[c]`` ([tokens, hidden]
bf16), initialised with the chunk's starting noise x^K.  A forward gathers the
states of its nodes into a staging buffer (node order), runs the block stack
(``sc_stack_forward``), and the sampler writes x^{j-1} back into ``xs[c]``
(``sc_sampler_step``); the refresh node (c, 0) only leaves its K/V in the cache.
After every round the states no later node reads are released
(``sc_cache_release_unread``).  Modes:

  packed      Eq. 7 rounds (plus the refresh node), one forward per round
  sequential  the same rounds, one forward per node, oldest chunk first
  serial      Eq. 2 order, one forward per node, chunk by chunk

With ``condition`` set, every block also cross-attends to a cached
condition sequence (the condition c of Eq. 1): per forward, a condition plan
maps each pack node to the condition its chunk reads (``condition_of``), and
each layer's weights are bound to that plan.

With ``memory`` set, what leaves the history window is not lost: the clean
states that no later node selects are folded into one memory state that every
node reads beside its window.  The stack weighs the keys that it reads
(``sc_stack_forward_weigh``), each head keeps the heaviest tokens of the memory
and the states that join it (``Cache.condense``), and the packs' plans get the
memory as a shared prefix (``sc_plan_share``).  Weights accumulate and do not age:
a token of the memory has gained weight in every forward since it was cached, so
on long streams early tokens hold their places.

Every computation runs in the library; this module sequences calls and moves
device buffers.
"""
from __future__ import annotations

from typing import Dict, List, Sequence, Tuple

from . import binding as sc


class StackPipeline:
    def __init__(self, *, layers: Sequence["sc.BlockWeights"], cache: "sc.Cache", rope: "sc.Rope",
                 xs, noise, policy: str, K: int, W: int, B: int, t_sched: Sequence[float],
                 refresh: bool = True, stream=None, condition=None, memory: bool = False):
        """``memory``: keep one memory state of what leaves the window, of as
        many tokens as a chunk.  The cache needs room for two states more; the
        modes are the same, ``refresh`` is needed (the clean states that it
        leaves are what the memory is made of), layer hooks are refused, and
        states cached before the run are left where they are.  ``condition``: optional dict with
        ``cache`` (an sc.Cache holding the condition K/V of every layer),
        ``cross`` (per layer: (w_q, w_o, q_norm or None)) and ``condition_of``
        (chunk -> cached condition state; default (0, 0))."""
        import torch
        self.torch = torch
        self.layers, self.cache, self.rope = list(layers), cache, rope
        self.xs, self.noise = xs, noise            # [B, n, hidden], [B, K + 2, n, hidden]
        self.policy, self.K, self.W, self.B = policy, K, W, B
        self.t_sched, self.refresh, self.stream = tuple(t_sched), refresh, stream
        self.condition = condition
        self.n_tok, self.hidden = xs.shape[1], xs.shape[2]
        max_pack = K + 1
        self.stage = torch.empty((max_pack * self.n_tok, self.hidden), dtype=xs.dtype, device=xs.device)
        self.ws_bytes = sc.sc_block_workspace_bytes(self.layers[0], max_pack * self.n_tok)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=xs.device)
        self.memory = None   # the cached state that holds it, once something has left the window
        self.weights = None  # accumulated attention weight of every cached key
        if memory:
            if not refresh:
                raise ValueError("a memory holds clean states, which only the refresh nodes leave: it needs refresh=True")
            d = cache.desc
            self.weights = torch.zeros((d.n_layers, d.n_slots, d.n_heads, d.tokens_per_page),
                                       dtype=torch.float32, device=xs.device)
            self.kept = torch.empty((len(self.layers), d.n_heads, self.n_tok), dtype=torch.int32, device=xs.device)
            self.weigh_ws = [torch.empty(0, dtype=torch.uint8, device=xs.device)]
            if xs.is_cuda:  # a run on another stream must not find the zeros still to come
                torch.cuda.current_stream(xs.device).synchronize()
            self.cached = set()  # states of the nodes run so far that are still cached

    # ----------------------------------------------------------- schedules
    def rounds(self) -> List[List[Tuple[int, int]]]:
        n = sc.sc_pipeline_rounds(self.K, self.B, self.refresh)
        return [sc.sc_pipeline_round_nodes(self.K, self.B, self.refresh, r) for r in range(n)]

    def serial_nodes(self) -> List[Tuple[int, int]]:
        n = sc.sc_serial_steps(self.K, self.B, self.refresh)
        return [sc.sc_serial_step_node(self.K, self.B, self.refresh, i) for i in range(n)]

    # ------------------------------------------------------------ forwards
    def forward(self, nodes: Sequence[Tuple[int, int]], layer_hook=None) -> None:
        """One packed forward of ``nodes`` through every layer, then the sampler.

        ``layer_hook(layer, phase, x, plan, layers)``, when given, observes the
        forward layer by layer: it is called with phase "in" before and "out"
        after each layer's block is enqueued (x: the pack's activations,
        layers: the block weights in use).  The layers then run one
        sc_block_forward call each instead of one sc_stack_forward call:
        the same function of the inputs, equal up to the order of fp32 sums
        (a stack takes its layers' first RMSNorm factors from sums that the
        layer before stored)."""
        self._refuse_hooks(layer_hook)
        self._refuse_other_weights()
        n = self.n_tok
        sel = sc.sc_selection_build(self.policy, self.K, self.W, nodes)
        plan = sc.sc_plan_build(sel, self.cache)
        if self.weights is not None:
            for node in nodes:
                self.cache.weights_clear(node, self.weights, self.stream)
            if self.memory is not None:
                plan = sc.sc_plan_share(plan, [self.memory])
        for i, (c, _) in enumerate(nodes):
            self.stage[i * n:(i + 1) * n].copy_(self.xs[c])
        x = self.stage[:len(nodes) * n]
        layers = self.layers
        if self.condition is not None:
            cond = self.condition
            of = cond.get("condition_of") or (lambda c: (0, 0))
            plan_c = sc.sc_plan_condition(cond["cache"], [of(c) for c, _ in nodes], n)
            layers = [w.with_cross(sc.CrossAttn(wq, wo, cond["cache"], plan_c, q_norm=qn))
                      for w, (wq, wo, qn) in zip(self.layers, cond["cross"])]
        if self.weights is not None:
            nb = sc.sc_attention_weigh_workspace_bytes(plan, self.cache)
            if self.weigh_ws[-1].numel() < nb:  # the smaller ones may still be in use
                self.weigh_ws.append(self.torch.empty(nb, dtype=self.torch.uint8, device=x.device))
            sc.sc_stack_forward_weigh(layers, self.cache, plan, x, self.rope, self.ws, self.ws_bytes,
                                      self.weights, self.weigh_ws[-1], nb, self.stream)
            self.cached.update(tuple(node) for node in nodes)
        elif layer_hook is None:
            sc.sc_stack_forward(layers, self.cache, plan, x, self.rope, self.ws, self.ws_bytes,
                                self.stream)
        else:
            for l, w in enumerate(layers):
                layer_hook(l, "in", x, plan, layers)
                sc.sc_block_forward(w, self.cache, l, plan, x, self.rope, self.ws, self.ws_bytes,
                                    self.stream)
                layer_hook(l, "out", x, plan, layers)
        for i, (c, j) in enumerate(nodes):
            if j >= 1:
                sc.sc_sampler_step([(c, j)], self.t_sched, self.K, self.xs[c],
                                   self.stage[i * n:(i + 1) * n], self.noise[c, j],
                                   n * self.hidden, self.stream)

    def _refuse_hooks(self, *hooks) -> None:
        if self.weights is not None and any(h is not None for h in hooks):
            raise ValueError("layer hooks observe single blocks; a stack with a memory runs in one call")

    def _refuse_other_weights(self) -> None:
        if self.weights is not None and self.weights.shape[1] != self.cache.desc.n_slots:
            raise ValueError(f"the weights are those of {self.weights.shape[1]} slots, the cache has {self.cache.desc.n_slots}: "
                             "after Cache.move(..., weights, moved_weights) the pipeline's weights are the moved ones")

    def _fold_unread(self, future: Sequence[Tuple[int, int]]) -> None:
        """Release what no node of ``future`` selects, the clean states among it
        into the memory; the memory too once nothing is left to read it."""
        self._refuse_other_weights()
        off, chunk, level, _ = sc.sc_selection_build(self.policy, self.K, self.W, future).tables()
        needed = {(chunk[s], level[s]) for i in range(len(future)) for s in range(off[i], off[i + 1] - 1)}
        unread = sorted(self.cached - needed)
        leaving = [st for st in unread if st[1] == 0] if future else []
        self._release([st for st in unread if st not in leaving])
        old = [] if self.memory is None else [self.memory]
        if not future:
            self._release(old)
            self.memory = None
        elif len(old + leaving) == 1:
            self.memory = (old + leaving)[0]  # it fits whole
            self.cached -= set(leaving)
        elif leaving:
            into = (leaving[-1][0], self.K + 1)  # a level that no node has
            # the stack's layers: a cache may hold more, which nothing writes
            self.cache.condense(0, len(self.layers), old + leaving, into, self.weights, self.kept,
                                self.stream)
            self._release(old + leaving)  # only now: a fold that fails can be tried again
            self.memory = into

    def _release(self, states: Sequence[Tuple[int, int]]) -> None:
        for st in states:
            self.cache.release(st)
            self.cached.discard(st)

    def run(self, mode: str = "packed", time_rounds: bool = False,
            kernel_timer_rounds: Tuple[int, int] = None, layer_hooks=None,
            stop_after: int = None) -> List[float]:
        """Run the whole schedule; returns per-round (or per-node for serial)
        milliseconds when ``time_rounds``.  With ``kernel_timer_rounds =
        (first, last)`` the library's kernel timer records the launches of
        those rounds; ``self.kernel_times`` then maps kernel kinds to
        (launches, total ms).  ``layer_hooks`` maps a round (a forward in
        serial mode) to a layer hook of its forwards (see ``forward``);
        ``stop_after`` ends the run after that round."""
        torch = self.torch
        self._refuse_hooks(*(layer_hooks or {}).values())
        times = []
        self.kernel_times = {}
        if mode == "serial":
            units = [[node] for node in self.serial_nodes()]
            groups = [[u] for u in units]
        else:
            units = self.rounds()
            groups = [[u] if mode == "packed" else [[node] for node in u] for u in units]
        flat = [node for u in units for node in u]
        done = 0
        for g, group in enumerate(groups):
            if kernel_timer_rounds and g == kernel_timer_rounds[0]:
                sc.sc_timer_enable(True)
            if time_rounds:
                e0 = torch.cuda.Event(enable_timing=True)
                e1 = torch.cuda.Event(enable_timing=True)
                e0.record()
            for nodes in group:
                self.forward(nodes, (layer_hooks or {}).get(g))
                done += len(nodes)
            if self.weights is None:
                sc.sc_cache_release_unread(self.cache, self.policy, self.K, self.W, flat[done:])
            else:
                self._fold_unread(flat[done:])
            if time_rounds:
                e1.record()
                times.append((e0, e1))
            if kernel_timer_rounds and g == kernel_timer_rounds[1]:
                folds = () if self.weights is None else ("attention_weigh", "condense")
                for kind in ("attention", "attention_combine", "gemm_qkv", "gemm_out", "gemm_up",
                             "gemm_down", "qk_norm", "cross_attention", "gemm_cross_q", "gemm_cross_out") + folds:
                    self.kernel_times[kind] = sc.sc_timer_read(kind)
                sc.sc_timer_enable(False)
            if stop_after is not None and g == stop_after:
                break
        if time_rounds:
            torch.cuda.synchronize()
            return [a.elapsed_time(b) for a, b in times]
        return []
