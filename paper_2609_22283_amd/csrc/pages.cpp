// Pages of a cache: copied between states, caches and types, shared by a fork,
// gathered at the front of their pool, or moved to another one.
#include <algorithm>
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

static PoolView pool_view(const sc_cache* c, int32_t layer) {
  const uint64_t bytes = (uint64_t)c->d.n_slots * c->slot_bytes;
  return PoolView{c->pool + (uint64_t)layer * bytes, bytes};
}

static bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb) {
  const uint64_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

extern "C" int sc_cache_copy(const sc_cache* from, const sc_node* states, int32_t n, sc_cache* to, const sc_node* into,
                             int32_t layer, int32_t n_layers, sc_stream stream) {
  return guarded([&]() -> int {
    if (!from || !states || !to || !into) return fail(SC_EINVAL, "null argument");
    if (n < 1) return fail(SC_EINVAL, "need at least one state (got %d)", n);
    const sc_cache_desc &a = from->d, &b = to->d;
    if (a.n_heads != b.n_heads || a.head_dim != b.head_dim || a.tokens_per_page != b.tokens_per_page ||
        a.pages_per_chunk != b.pages_per_chunk)
      return fail(SC_EINVAL, "states of %d pages of %d tokens x %d heads x %d do not fit a cache of %d x %d x %d x %d",
                  a.pages_per_chunk, a.tokens_per_page, a.n_heads, a.head_dim, b.pages_per_chunk, b.tokens_per_page,
                  b.n_heads, b.head_dim);
    const bool pack = a.dtype == SC_DTYPE_BF16 && b.dtype == SC_DTYPE_FP4;
    const bool unpack = a.dtype == SC_DTYPE_FP4 && b.dtype == SC_DTYPE_BF16;
    if (a.dtype != b.dtype && !pack && !unpack)
      return fail(SC_EUNSUPPORTED, "states go between caches of one dtype, or of bf16 and 4 bits (got %d and %d)", a.dtype, b.dtype);
    const int32_t most = std::min(a.n_layers, b.n_layers);
    if (layer < 0 || n_layers < 1 || n_layers > most - layer)
      return fail(SC_EINVAL, "layers %d .. %lld outside [0, %d)", layer, (long long)layer + n_layers - 1, most);
    if (from->table != to->table &&
        overlap(from->pool, (uint64_t)a.n_layers * pool_view(from, 0).layer_bytes, to->pool,
                (uint64_t)b.n_layers * pool_view(to, 0).layer_bytes))
      return fail(SC_EINVAL, "the caches' pools overlap");
    std::vector<int32_t> src, dst;
    std::set<StateKey> seen;
    int64_t fresh_states = 0;
    for (int32_t i = 0; i < n; ++i) {
      const StateKey key(states[i].chunk, states[i].level), key_to(into[i].chunk, into[i].level);
      auto it = from->states.find(key);
      if (it == from->states.end()) return fail(SC_ENOTFOUND, "state (%d,%d) not cached", key.first, key.second);
      for (int32_t l = layer; l < layer + n_layers; ++l)
        if (!it->second.written[l])
          return fail(SC_EUNAVAILABLE, "state (%d,%d) has no K/V at layer %d", key.first, key.second, l);
      if (key_to.first < 0 || key_to.second < 0) return fail(SC_EINVAL, "bad state (%d,%d)", key_to.first, key_to.second);
      if (!seen.insert(key_to).second)
        return fail(SC_EINVAL, "state (%d,%d) would be written twice", key_to.first, key_to.second);
      auto at = to->states.find(key_to);
      if (at == to->states.end())
        ++fresh_states;
      else
        for (int32_t l = layer; l < layer + n_layers; ++l)
          if (at->second.written[l])
            return fail(SC_EEXIST, "state (%d,%d) layer %d already written", key_to.first, key_to.second, l);
      src.insert(src.end(), it->second.slots.begin(), it->second.slots.end());
    }
    if (fresh_states * b.pages_per_chunk > free_slots(to))
      return fail(SC_ECAPACITY, "%lld new states need %lld slots, %d free", (long long)fresh_states,
                  (long long)fresh_states * b.pages_per_chunk, free_slots(to));
    std::vector<sc_node> made;
    made.reserve((size_t)n);
    dst.reserve(src.size());
    const auto undo = [&] {
      for (const sc_node& nd : made) sc_cache_release(to, nd);
    };
    try {
      for (int32_t i = 0; i < n; ++i) {
        StateEntry* e = nullptr;
        bool fresh = false;
        const int rc = state_for_append(to, layer, StateKey(into[i].chunk, into[i].level), &e, &fresh);
        if (rc != SC_OK) {
          undo();
          return rc;
        }
        if (fresh) made.push_back(into[i]);
        dst.insert(dst.end(), e->slots.begin(), e->slots.end());
      }
    } catch (const std::bad_alloc&) {
      undo();
      throw;
    }
    const PagePairs pairs{src.data(), dst.data(), (int32_t)src.size()};
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int rc = pack || unpack
                       ? launch_page_convert(pack, pool_view(from, layer), pool_view(to, layer), a, pairs, n_layers, s)
                       : launch_page_moves(pool_view(from, layer), pool_view(to, layer), from->slot_bytes, pairs, n_layers, s);
    if (rc != SC_OK) {
      undo();
      return rc;
    }
    for (int32_t i = 0; i < n; ++i)
      for (int32_t l = layer; l < layer + n_layers; ++l)
        set_written(to, to->states.at(StateKey(into[i].chunk, into[i].level)), l, 1);
    return SC_OK;
  });
}

extern "C" int sc_cache_fork(sc_cache* c, sc_cache** out) {
  return guarded([&]() -> int {
    if (!c || !out) return fail(SC_EINVAL, "null argument");
    *out = nullptr;
    for (const auto& kv : c->states)
      for (int32_t l = 0; l < c->d.n_layers; ++l)
        if (!kv.second.written[l])
          return fail(SC_EUNAVAILABLE, "state (%d,%d) is not written at layer %d: its pages cannot be shared yet",
                      kv.first.first, kv.first.second, l);
    std::unique_ptr<sc_cache> f(new sc_cache(*c));
    c->table->handles.push_back(f.get());
    for (const auto& kv : f->states)
      for (int32_t s : kv.second.slots) ++f->table->refs[s];
    *out = f.release();
    return SC_OK;
  });
}

// Slots of a table change their numbers: to[s], or -1 for a slot that keeps nothing.
static void renumber(SlotTable& t, const std::vector<int32_t>& to) {
  for (sc_cache* h : t.handles)
    for (auto& kv : h->states)
      for (int32_t& s : kv.second.slots) s = to[s];
}

extern "C" int sc_cache_compact(sc_cache* c, float* weights, sc_stream stream) {
  return guarded([&]() -> int {
    if (!c) return fail(SC_EINVAL, "null argument");
    SlotTable& t = *c->table;
    const int32_t n = c->d.n_slots, used = n - free_slots(c);
    std::vector<int32_t> to(n), src, dst;
    int32_t hole = 0;
    for (int32_t s = 0; s < n; ++s) {
      to[s] = t.refs[s] ? s : -1;
      if (s < used || !t.refs[s]) continue;
      while (t.refs[hole]) ++hole;  // one below `used` for every page above it
      src.push_back(s);
      dst.push_back(hole);
      to[s] = hole++;
    }
    if (src.empty()) return SC_OK;
    const PagePairs pairs{src.data(), dst.data(), (int32_t)src.size()};
    hipStream_t st = static_cast<hipStream_t>(stream);
    int rc = launch_page_moves(pool_view(c, 0), pool_view(c, 0), c->slot_bytes, pairs, c->d.n_layers, st);
    if (rc == SC_OK && weights) {
      const uint64_t page = (uint64_t)c->d.n_heads * c->d.tokens_per_page * sizeof(float);
      const PoolView w{reinterpret_cast<char*>(weights), (uint64_t)n * page};
      rc = launch_page_moves(w, w, page, pairs, c->d.n_layers, st);
    }
    if (rc != SC_OK) return rc;  // the pages are where they were, their copies in slots that hold nothing
    for (size_t i = 0; i < src.size(); ++i) {
      t.refs[dst[i]] = t.refs[src[i]];
      t.refs[src[i]] = 0;
      for (sc_cache* h : t.handles) {
        ++h->gen[src[i]];
        ++h->gen[dst[i]];
      }
      for (int32_t l = 0; l < c->d.n_layers; ++l) {
        uint8_t* w = t.written.data() + (size_t)l * n;
        w[dst[i]] = w[src[i]];
        w[src[i]] = 0;
      }
    }
    renumber(t, to);
    return SC_OK;
  });
}

extern "C" int sc_cache_move(sc_cache* c, void* pool, int32_t n_slots, const float* weights, float* moved_weights,
                             sc_stream stream) {
  return guarded([&]() -> int {
    if (!c || !pool) return fail(SC_EINVAL, "null argument");
    if (n_slots < 1) return fail(SC_EINVAL, "need at least one slot (got %d)", n_slots);
    if (!weights != !moved_weights) return fail(SC_EINVAL, "weights move from one array to another: both or neither");
    if (c->d.dtype == SC_DTYPE_FP4 && reinterpret_cast<uintptr_t>(pool) & 15)
      return fail(SC_EINVAL, "the pool of a 4-bit cache must be 16-byte aligned");
    SlotTable& t = *c->table;
    const int32_t n = c->d.n_slots, used = n - free_slots(c);
    if (used > n_slots) return fail(SC_ECAPACITY, "%d slots in use do not fit %d", used, n_slots);
    const uint64_t L = c->d.n_layers, page = (uint64_t)c->d.n_heads * c->d.tokens_per_page * sizeof(float);
    if (overlap(c->pool, L * n * c->slot_bytes, pool, L * n_slots * c->slot_bytes))
      return fail(SC_EINVAL, "the new pool overlaps the old one");
    if (weights && overlap(weights, L * n * page, moved_weights, L * n_slots * page))
      return fail(SC_EINVAL, "the new weights overlap the old ones");
    std::vector<int32_t> to(n, -1), src, dst, refs(n_slots, 0);
    std::vector<uint8_t> written((size_t)L * n_slots, 0);
    for (int32_t s = 0; s < n; ++s)
      if (t.refs[s]) {
        to[s] = (int32_t)dst.size();
        refs[to[s]] = t.refs[s];
        for (uint64_t l = 0; l < L; ++l) written[l * n_slots + to[s]] = t.written[l * n + s];
        src.push_back(s);
        dst.push_back(to[s]);
      }
    // no plan over the old slots fits the new ones, of whatever number
    uint32_t newest = 0;
    for (const sc_cache* h : t.handles)
      for (uint32_t g : h->gen) newest = std::max(newest, g);
    std::vector<std::vector<uint32_t>> gens(t.handles.size(), std::vector<uint32_t>(n_slots, newest + 1));
    if (!src.empty()) {
      const PagePairs pairs{src.data(), dst.data(), (int32_t)src.size()};
      hipStream_t st = static_cast<hipStream_t>(stream);
      const PoolView view{static_cast<char*>(pool), (uint64_t)n_slots * c->slot_bytes};
      int rc = launch_page_moves(pool_view(c, 0), view, c->slot_bytes, pairs, c->d.n_layers, st);
      if (rc == SC_OK && weights)
        rc = launch_page_moves(PoolView{reinterpret_cast<char*>(const_cast<float*>(weights)), (uint64_t)n * page},
                               PoolView{reinterpret_cast<char*>(moved_weights), (uint64_t)n_slots * page}, page, pairs,
                               c->d.n_layers, st);
      if (rc != SC_OK) return rc;
    }
    renumber(t, to);
    t.refs.swap(refs);
    t.written.swap(written);
    for (size_t i = 0; i < t.handles.size(); ++i) {
      sc_cache* h = t.handles[i];
      h->pool = static_cast<char*>(pool);
      h->d.n_slots = n_slots;
      h->gen.swap(gens[i]);
    }
    return SC_OK;
  });
}
