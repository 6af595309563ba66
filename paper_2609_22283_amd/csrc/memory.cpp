// A bounded, shared history: attention that weighs the cached keys, states folded
// into one by these weights, and plans whose nodes share a prefix.
#include <algorithm>
#include <climits>
#include <cmath>
#include <memory>
#include <new>
#include <set>

#include "internal.h"

using namespace sc;

// The entry points' bodies allocate host memory; no exception leaves them.
template <class F>
static int guarded(F body) {
  try {
    return body();
  } catch (const std::bad_alloc&) {
    return fail(SC_EINVAL, "out of host memory");
  }
}

static size_t align256(size_t n) { return (n + 255) & ~size_t(255); }

extern "C" int sc_plan_share(const sc_plan* plan, const sc_node* states, int32_t n, sc_plan** out) {
  return guarded([&]() -> int {
    if (!plan || !states || !out) return fail(SC_EINVAL, "null argument");
    *out = nullptr;
    if (n < 1) return fail(SC_EINVAL, "a shared prefix needs at least one state (got %d)", n);
    const sc_cache* c = plan->cache;
    const std::set<StateKey> read(plan->page_state.begin(), plan->page_state.end());
    std::set<StateKey> seen;
    for (int32_t i = 0; i < n; ++i) {
      const StateKey key(states[i].chunk, states[i].level);
      if (!c->states.count(key)) return fail(SC_ENOTFOUND, "prefix state (%d,%d) not in the cache", key.first, key.second);
      if (read.count(key) || !seen.insert(key).second)
        return fail(SC_EINVAL, "prefix state (%d,%d) would be read twice", key.first, key.second);
    }
    const int32_t ppc = c->d.pages_per_chunk, nodes = (int32_t)plan->nodes.size();
    const int64_t prefix = (int64_t)n * ppc;
    if (prefix * std::max(nodes, 1) + (int64_t)plan->page_slot.size() > INT32_MAX)
      return fail(SC_EUNSUPPORTED, "a prefix of %lld pages for %d nodes", (long long)prefix, nodes);
    std::unique_ptr<sc_plan> p(new sc_plan);
    p->nodes = plan->nodes;
    p->cache = c;
    p->nq = plan->nq;
    if (nodes) p->shared = plan->shared + (int32_t)prefix;
    p->page_off.push_back(0);
    for (int32_t i = 0; i < nodes; ++i) {
      for (int32_t s = 0; s < n; ++s) {
        const StateKey key(states[s].chunk, states[s].level);
        const StateEntry& e = c->states.at(key);
        for (int32_t f = 0; f < ppc; ++f) {
          p->page_slot.push_back(e.slots[f]);
          p->page_tokens.push_back(c->d.tokens_per_page);
          p->page_frame.push_back(key.first * ppc + f);
          p->page_gen.push_back(c->gen[e.slots[f]]);
          p->page_state.push_back(key);
        }
      }
      for (int32_t k = plan->page_off[i]; k < plan->page_off[i + 1]; ++k) {
        p->page_slot.push_back(plan->page_slot[k]);
        p->page_tokens.push_back(plan->page_tokens[k]);
        p->page_frame.push_back(plan->page_frame[k]);
        p->page_gen.push_back(plan->page_gen[k]);
        p->page_state.push_back(plan->page_state[k]);
      }
      p->page_off.push_back((int32_t)p->page_slot.size());
    }
    *out = p.release();
    return SC_OK;
  });
}

// ------------------------------------------------------------------- weights

extern "C" size_t sc_cache_weights_bytes(const sc_cache* c) {
  if (!c) return 0;
  return (size_t)c->d.n_layers * c->d.n_slots * c->d.n_heads * c->d.tokens_per_page * sizeof(float);
}

extern "C" int sc_cache_weights_clear(const sc_cache* c, sc_node st, float* weights, sc_stream stream) {
  if (!c || !weights) return fail(SC_EINVAL, "null argument");
  auto it = c->states.find(StateKey(st.chunk, st.level));
  if (it == c->states.end()) return fail(SC_ENOTFOUND, "state (%d,%d) not cached", st.chunk, st.level);
  return launch_weights_clear(c, it->second.slots.data(), (int32_t)it->second.slots.size(), weights,
                              static_cast<hipStream_t>(stream));
}

extern "C" size_t sc_attention_weigh_workspace_bytes(const sc_plan* p, const sc_cache* c) {
  size_t need = 0;
  guarded([&]() -> int {
    if (!p || !c || p->cache != c || p->nodes.empty() || attention_check(p, c) != SC_OK) return SC_EINVAL;
    need = weigh_attention_bytes(p, c);
    return SC_OK;
  });
  return need;
}

// What the weighing of a plan needs besides the attention itself.
static int weigh_check(const sc_plan* p, const sc_cache* c, const float* weights, const void* ws, size_t ws_bytes) {
  if (!weights) return fail(SC_EINVAL, "null argument");
  if (p->nodes.empty()) return SC_OK;
  const int rc = attention_check(p, c);
  if (rc != SC_OK) return rc;
  const size_t need = weigh_attention_bytes(p, c);
  if (!ws || ws_bytes < need) return fail(SC_EINVAL, "workspace of %zu bytes, need %zu", ws ? ws_bytes : 0, need);
  if (reinterpret_cast<uintptr_t>(ws) & 15) return fail(SC_EINVAL, "workspace must be 16-byte aligned");
  return SC_OK;
}

extern "C" int sc_attention_weigh(const sc_plan* p, const sc_cache* c, int32_t layer, const void* q, void* o,
                                  float scale, float* weights, void* ws, size_t ws_bytes, sc_stream stream) {
  return guarded([&]() -> int {
    if (!p || !c || !q || !o || !weights) return fail(SC_EINVAL, "null argument");
    if (!std::isfinite(scale)) return fail(SC_EINVAL, "scale must be finite");
    if (reinterpret_cast<uintptr_t>(q) & 15) return fail(SC_EINVAL, "q must be 16-byte aligned");
    int rc = plan_check(p, c, layer);
    if (rc != SC_OK || (rc = weigh_check(p, c, weights, ws, ws_bytes)) != SC_OK) return rc;
    if (p->nodes.empty()) return SC_OK;
    // the keys are weighed by q after (or while) o is written
    const uint64_t n = (uint64_t)p->nodes.size() * p->nq * c->d.n_heads * c->d.head_dim * dtype_size(c->d.dtype);
    const uint64_t qa = reinterpret_cast<uintptr_t>(q), oa = reinterpret_cast<uintptr_t>(o);
    if (qa < oa + n && oa < qa + n) return fail(SC_EINVAL, "o overlaps q, which is read after o is written");
    return launch_attention_weigh(p, c, layer, q, o, scale, weights, ws, static_cast<hipStream_t>(stream));
  });
}

extern "C" int sc_stack_forward_weigh(const sc_block_weights* layers, int32_t n_layers, sc_cache* c, const sc_plan* p,
                                      void* x, const sc_rope* rope, void* ws, size_t ws_bytes, float* weights,
                                      void* weigh_ws, size_t weigh_ws_bytes, sc_stream stream) {
  return guarded([&]() -> int {
    if (!c || !p) return fail(SC_EINVAL, "null argument");
    if (p->cache != c) return fail(SC_EINVAL, "plan was built for another cache");
    const int rc = weigh_check(p, c, weights, weigh_ws, weigh_ws_bytes);
    if (rc != SC_OK) return rc;
    const Weighing scope(p, weights, weigh_ws);
    return sc_stack_forward(layers, n_layers, c, p, x, rope, ws, ws_bytes, stream);
  });
}

// ------------------------------------------------------------------ condense

extern "C" int sc_cache_condense(sc_cache* c, int32_t layer, int32_t n_layers, const sc_node* sources, int32_t n,
                                 sc_node into, float* weights, int32_t* kept, sc_stream stream) {
  return guarded([&]() -> int {
    if (!c || !sources || !weights || !kept) return fail(SC_EINVAL, "null argument");
    if (n < 1) return fail(SC_EINVAL, "need at least one source (got %d)", n);
    if (layer < 0 || n_layers < 1 || n_layers > c->d.n_layers - layer)
      return fail(SC_EINVAL, "layers %d .. %d outside [0, %d)", layer, layer + n_layers - 1, c->d.n_layers);
    if (into.chunk < 0 || into.level < 0) return fail(SC_EINVAL, "bad state (%d,%d)", into.chunk, into.level);
    int rc = condense_check(c, n);
    if (rc != SC_OK) return rc;
    const StateKey to(into.chunk, into.level);
    std::set<StateKey> seen;
    for (int32_t i = 0; i < n; ++i) {
      const StateKey key(sources[i].chunk, sources[i].level);
      if (key == to || !seen.insert(key).second)
        return fail(SC_EINVAL, "state (%d,%d) named twice", key.first, key.second);
    }
    std::vector<int32_t> slots;
    for (int32_t i = 0; i < n; ++i) {
      const StateKey key(sources[i].chunk, sources[i].level);
      auto it = c->states.find(key);
      if (it == c->states.end()) return fail(SC_ENOTFOUND, "state (%d,%d) not cached", key.first, key.second);
      for (int32_t l = layer; l < layer + n_layers; ++l)
        if (!it->second.written[l])
          return fail(SC_EUNAVAILABLE, "state (%d,%d) has no K/V at layer %d", key.first, key.second, l);
      slots.insert(slots.end(), it->second.slots.begin(), it->second.slots.end());
    }
    auto it = c->states.find(to);
    if (it != c->states.end())
      for (int32_t l = layer; l < layer + n_layers; ++l)
        if (it->second.written[l]) return fail(SC_EEXIST, "state (%d,%d) layer %d already written", to.first, to.second, l);
    StateEntry* e = nullptr;
    bool fresh = false;
    if ((rc = state_for_append(c, layer, to, &e, &fresh)) != SC_OK) return rc;
    const int32_t n_src = (int32_t)slots.size();
    slots.insert(slots.end(), e->slots.begin(), e->slots.end());
    rc = launch_condense(c, layer, n_layers, slots.data(), n_src, weights, kept, static_cast<hipStream_t>(stream));
    if (rc != SC_OK) {
      if (fresh) sc_cache_release(c, into);
      return rc;
    }
    for (int32_t l = layer; l < layer + n_layers; ++l) set_written(c, *e, l, 1);
    return SC_OK;
  });
}
