// Pages of caches on the CPU: copies, forks, compaction and moves to other pools, with
// the launchers' stand-ins moving real bytes (page_stubs.cpp).  Every state's pages carry a
// number of their own in each layer, and the pages are looked at after every step.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <random>
#include <vector>

#include "../../paper_2609_22283_amd/csrc/internal.h"

extern int g_launches, g_fail_at;
extern bool g_page_fail;

#define CHECK(x)                                                            \
  do {                                                                      \
    if (!(x)) {                                                             \
      std::fprintf(stderr, "%s:%d: %s (%s)\n", __FILE__, __LINE__, #x, sc_last_error()); \
      std::exit(1);                                                         \
    }                                                                       \
  } while (0)

namespace {

constexpr int kLayers = 3, kPages = 2;

sc_cache_desc desc(int slots, int dtype = SC_DTYPE_BF16) { return sc_cache_desc{kLayers, 1, 128, 8, kPages, slots, dtype}; }

struct Pool {
  std::vector<char> bytes;
  char* p;
  explicit Pool(const sc_cache_desc& d) : bytes(sc_cache_pool_bytes(&d) + 64, 0x5a) {
    p = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(bytes.data()) + 15) & ~uintptr_t(15));
  }
};

int32_t* word(const sc_cache* c, int layer, int slot) {
  return reinterpret_cast<int32_t*>(c->pool + ((size_t)layer * c->d.n_slots + slot) * c->slot_bytes);
}

// Appends a state in every layer and signs its pages.
int append(sc_cache* c, sc_node s, int32_t sign) {
  for (int l = 0; l < kLayers; ++l) {
    const int rc = sc_cache_append(c, l, s, c, c, nullptr, nullptr);
    if (rc != SC_OK) return rc;
    int32_t slots[kPages];
    CHECK(sc_cache_slots(c, s, slots) == SC_OK);
    for (int f = 0; f < kPages; ++f) *word(c, l, slots[f]) = sign * 100 + l * 10 + f;
  }
  return SC_OK;
}

bool signed_by(const sc_cache* c, sc_node s, int32_t sign) {
  int32_t slots[kPages];
  if (sc_cache_slots(c, s, slots) != SC_OK) return false;
  for (int l = 0; l < kLayers; ++l)
    for (int f = 0; f < kPages; ++f)
      if (sc_cache_contains(c, s, l) != 1 || *word(c, l, slots[f]) != sign * 100 + l * 10 + f) return false;
  return true;
}

sc_plan* plan_of(sc_cache* c, sc_node s) {
  sc_plan* p = nullptr;
  CHECK(sc_plan_condition(c, &s, 1, 4, &p) == SC_OK);
  return p;
}

int use(const sc_plan* p, const sc_cache* c) {
  float q = 0, o = 0;
  return sc_attention(p, c, 0, &q, &o, 1.f, nullptr, 0, nullptr);
}

void forks() {
  const sc_cache_desc d = desc(8);
  Pool pool(d);
  sc_cache *a = nullptr, *b = nullptr;
  CHECK(sc_cache_create(&d, pool.p, &a) == SC_OK);
  CHECK(append(a, {0, 0}, 1) == SC_OK && append(a, {1, 0}, 2) == SC_OK);
  CHECK(sc_cache_append(a, 0, sc_node{2, 0}, a, a, nullptr, nullptr) == SC_OK);
  CHECK(sc_cache_fork(a, &b) == SC_EUNAVAILABLE && !b);  // (2, 0) has one layer
  CHECK(sc_cache_release(a, {2, 0}) == SC_OK);
  CHECK(sc_cache_fork(nullptr, &b) == SC_EINVAL && sc_cache_fork(a, nullptr) == SC_EINVAL);
  CHECK(sc_cache_fork(a, &b) == SC_OK);
  CHECK(sc_cache_free_slot_count(a) == 4 && sc_cache_free_slot_count(b) == 4);
  CHECK(signed_by(b, {0, 0}, 1) && signed_by(b, {1, 0}, 2));
  sc_plan *pa = plan_of(a, {0, 0}), *pb = plan_of(b, {0, 0});
  CHECK(use(pa, a) == SC_OK && use(pb, b) == SC_OK);
  CHECK(use(pa, b) == SC_EINVAL);  // another handle's plan
  CHECK(sc_cache_append(b, 0, sc_node{0, 0}, b, b, nullptr, nullptr) == SC_EEXIST);
  // a release is the handle's own: its plans are stale, the fork's are not, no slot is free
  CHECK(sc_cache_release(a, {0, 0}) == SC_OK);
  CHECK(use(pa, a) == SC_ESTALE && use(pb, b) == SC_OK);
  CHECK(sc_cache_free_slot_count(a) == 4 && signed_by(b, {0, 0}, 1));
  // the same name again, in slots of its own
  CHECK(append(a, {0, 0}, 7) == SC_OK);
  CHECK(signed_by(a, {0, 0}, 7) && signed_by(b, {0, 0}, 1));
  CHECK(use(pa, a) == SC_ESTALE && use(pb, b) == SC_OK);
  CHECK(append(b, {3, 0}, 8) == SC_OK && sc_cache_contains(a, {3, 0}, -1) == 0);
  CHECK(sc_cache_free_slot_count(a) == 0 && append(a, {4, 0}, 9) == SC_ECAPACITY);
  CHECK(sc_cache_release(b, {0, 0}) == SC_OK && sc_cache_free_slot_count(a) == 2);
  CHECK(use(pb, b) == SC_ESTALE);
  // a fork of a fork, and the first handle gone before the others
  sc_cache* e = nullptr;
  CHECK(sc_cache_fork(b, &e) == SC_OK);
  sc_plan_free(pa);
  sc_cache_free(a);
  CHECK(sc_cache_free_slot_count(e) == 4);  // (0, 0) of a is gone; (1, 0) and (3, 0) stay
  CHECK(signed_by(e, {1, 0}, 2) && signed_by(b, {1, 0}, 2) && signed_by(e, {3, 0}, 8));
  sc_cache_free(b);
  CHECK(signed_by(e, {1, 0}, 2) && sc_cache_free_slot_count(e) == 4);
  sc_plan_free(pb);
  sc_cache_free(e);
  sc_cache_free(nullptr);
}

void copies() {
  const sc_cache_desc d = desc(8), q = desc(6, SC_DTYPE_FP4);
  Pool pool(d), held(q);
  sc_cache *a = nullptr, *b = nullptr;
  CHECK(sc_cache_create(&d, pool.p, &a) == SC_OK && sc_cache_create(&q, held.p, &b) == SC_OK);
  CHECK(append(a, {0, 0}, 1) == SC_OK && append(a, {1, 0}, 2) == SC_OK);
  const sc_node from[2] = {{0, 0}, {1, 0}}, into[2] = {{5, 1}, {6, 1}};
  const auto copy = [&](const sc_node* f, int n, sc_cache* to, const sc_node* t, int l = 0, int m = kLayers) {
    return sc_cache_copy(a, f, n, to, t, l, m, nullptr);
  };
  CHECK(sc_cache_copy(nullptr, from, 2, b, into, 0, 1, nullptr) == SC_EINVAL);
  CHECK(copy(nullptr, 2, b, into) == SC_EINVAL && copy(from, 2, b, nullptr) == SC_EINVAL && copy(from, 0, b, into) == SC_EINVAL);
  CHECK(copy(from, 2, b, into, 0, 0) == SC_EINVAL && copy(from, 2, b, into, -1, 1) == SC_EINVAL);
  CHECK(copy(from, 2, b, into, 1, kLayers) == SC_EINVAL && copy(from, 2, b, into, 2147483647, 2147483647) == SC_EINVAL);
  const sc_node none[1] = {{9, 9}}, bad[1] = {{-1, 0}}, same[2] = {{5, 1}, {5, 1}};
  CHECK(copy(none, 1, b, into) == SC_ENOTFOUND && copy(from, 1, b, bad) == SC_EINVAL && copy(from, 2, b, same) == SC_EINVAL);
  CHECK(copy(from, 1, a, from) == SC_EEXIST);
  CHECK(sc_cache_free_slot_count(b) == 6);
  g_page_fail = true;  // nothing of a failed copy stays
  CHECK(copy(from, 2, b, into) == SC_EDEVICE && sc_cache_free_slot_count(b) == 6 && !sc_cache_contains(b, into[0], -1));
  g_page_fail = false;
  CHECK(copy(from, 2, b, into) == SC_OK && signed_by(b, into[0], 1) && signed_by(b, into[1], 2));
  CHECK(copy(from, 2, b, into) == SC_EEXIST);
  const sc_node more[2] = {{7, 0}, {8, 0}};
  CHECK(copy(from, 2, b, more) == SC_ECAPACITY && sc_cache_free_slot_count(b) == 2 && !sc_cache_contains(b, more[0], -1));
  // back, one source twice, and layer by layer
  const sc_node twice[2] = {{5, 1}, {5, 1}};
  CHECK(sc_cache_copy(b, twice, 2, a, more, 1, 2, nullptr) == SC_OK);
  CHECK(sc_cache_contains(a, more[0], 0) == 0 && sc_cache_contains(a, more[0], 1) == 1);
  CHECK(copy(more, 1, b, none) == SC_EUNAVAILABLE);
  CHECK(sc_cache_copy(b, twice, 2, a, more, 0, 1, nullptr) == SC_OK && signed_by(a, more[0], 1) && signed_by(a, more[1], 1));
  // caches that do not match
  sc_cache_desc other = desc(4);
  other.tokens_per_page = 16;
  Pool op(other);
  sc_cache* o = nullptr;
  CHECK(sc_cache_create(&other, op.p, &o) == SC_OK && copy(from, 1, o, into) == SC_EINVAL);
  sc_cache_free(o);
  other = desc(4, SC_DTYPE_F32);
  Pool fp(other);
  CHECK(sc_cache_create(&other, fp.p, &o) == SC_OK && copy(from, 1, o, into) == SC_EUNSUPPORTED);
  sc_cache_free(o);
  CHECK(sc_cache_create(&d, pool.p + a->slot_bytes, &o) == SC_OK && copy(from, 1, o, into) == SC_EINVAL);  // pools overlap
  sc_cache_free(o);
  CHECK(sc_cache_create(&q, held.p + 8, &o) == SC_EINVAL);
  sc_cache_desc narrow = desc(4, SC_DTYPE_FP4);
  narrow.head_dim = 64;
  CHECK(sc_cache_create(&narrow, held.p, &o) == SC_EUNSUPPORTED && sc_cache_pool_bytes(&narrow) == 0);
  sc_cache_free(a);
  sc_cache_free(b);
}

void moves() {
  const sc_cache_desc d = desc(10);
  Pool pool(d);
  sc_cache* a = nullptr;
  CHECK(sc_cache_create(&d, pool.p, &a) == SC_OK);
  CHECK(sc_cache_compact(nullptr, nullptr, nullptr) == SC_EINVAL && sc_cache_compact(a, nullptr, nullptr) == SC_OK);
  for (int i = 0; i < 5; ++i) CHECK(append(a, {i, 0}, i + 1) == SC_OK);
  std::vector<float> w(kLayers * 10 * 8);
  for (size_t i = 0; i < w.size(); ++i) w[i] = (float)i;
  sc_plan *low = plan_of(a, {1, 0}), *high = plan_of(a, {4, 0});
  CHECK(sc_cache_release(a, {0, 0}) == SC_OK && sc_cache_release(a, {2, 0}) == SC_OK);
  int32_t was[kPages], is[kPages];
  CHECK(sc_cache_slots(a, {4, 0}, was) == SC_OK);
  g_page_fail = true;
  CHECK(sc_cache_compact(a, w.data(), nullptr) == SC_EDEVICE && signed_by(a, {4, 0}, 5) && use(high, a) == SC_OK);
  g_page_fail = false;
  CHECK(sc_cache_compact(a, w.data(), nullptr) == SC_OK);
  CHECK(sc_cache_slots(a, {4, 0}, is) == SC_OK);
  for (int f = 0; f < kPages; ++f) {
    CHECK(is[f] < 6 && was[f] >= 6);
    for (int l = 0; l < kLayers; ++l)
      for (int t = 0; t < 8; ++t) CHECK(w[(l * 10 + is[f]) * 8 + t] == (float)((l * 10 + was[f]) * 8 + t));
  }
  CHECK(signed_by(a, {1, 0}, 2) && signed_by(a, {3, 0}, 4) && signed_by(a, {4, 0}, 5));
  CHECK(use(low, a) == SC_OK && use(high, a) == SC_ESTALE);  // only the moved pages' plans
  CHECK(append(a, {7, 0}, 8) == SC_OK && signed_by(a, {4, 0}, 5) && sc_cache_release(a, {7, 0}) == SC_OK);
  // to a smaller pool
  const sc_cache_desc small = desc(6), tiny = desc(5);
  Pool sp(small), tp(tiny);
  std::vector<float> w2(kLayers * 6 * 8, -1.f);
  CHECK(sc_cache_move(a, nullptr, 6, nullptr, nullptr, nullptr) == SC_EINVAL);
  CHECK(sc_cache_move(a, sp.p, 0, nullptr, nullptr, nullptr) == SC_EINVAL);
  CHECK(sc_cache_move(a, sp.p, 6, w.data(), nullptr, nullptr) == SC_EINVAL);
  CHECK(sc_cache_move(a, sp.p, 6, w.data(), w.data() + 3, nullptr) == SC_EINVAL);
  CHECK(sc_cache_move(a, tp.p, 5, nullptr, nullptr, nullptr) == SC_ECAPACITY);
  CHECK(sc_cache_move(a, a->pool, 10, nullptr, nullptr, nullptr) == SC_EINVAL);
  sc_cache* b = nullptr;
  CHECK(sc_cache_fork(a, &b) == SC_OK);
  sc_plan* pb = plan_of(b, {4, 0});
  g_page_fail = true;
  CHECK(sc_cache_move(a, sp.p, 6, w.data(), w2.data(), nullptr) == SC_EDEVICE && a->pool == pool.p && use(low, a) == SC_OK);
  g_page_fail = false;
  CHECK(sc_cache_slots(a, {4, 0}, was) == SC_OK);
  CHECK(sc_cache_move(a, sp.p, 6, w.data(), w2.data(), nullptr) == SC_OK);
  CHECK(sc_cache_slots(a, {4, 0}, is) == SC_OK);
  for (int f = 0; f < kPages; ++f)
    for (int l = 0; l < kLayers; ++l) CHECK(w2[(l * 6 + is[f]) * 8 + 3] == w[(l * 10 + was[f]) * 8 + 3]);
  CHECK(a->pool == sp.p && b->pool == sp.p && b->d.n_slots == 6 && sc_cache_free_slot_count(b) == 0);
  CHECK(signed_by(a, {1, 0}, 2) && signed_by(b, {3, 0}, 4) && signed_by(b, {4, 0}, 5));
  // plans of more slots than there are now, and of slots that hold the same numbers
  CHECK(use(low, a) == SC_ESTALE && use(high, a) == SC_ESTALE && use(pb, b) == SC_ESTALE);
  sc_plan* again = plan_of(a, {4, 0});
  CHECK(use(again, a) == SC_OK);
  // and back to a larger one: stale once more, whatever the numbers
  CHECK(sc_cache_move(b, pool.p, 10, nullptr, nullptr, nullptr) == SC_OK);
  CHECK(use(again, a) == SC_ESTALE && use(high, a) == SC_ESTALE && signed_by(a, {4, 0}, 5) && append(a, {8, 0}, 9) == SC_OK);
  sc_plan_free(again);
  sc_plan_free(pb);
  sc_plan_free(low);
  sc_plan_free(high);
  sc_cache_free(b);
  sc_cache_free(a);
}

// Random steps on a family of handles against what each should hold.
void random_steps() {
  std::mt19937 rnd(7);
  for (int trial = 0; trial < 40; ++trial) {
    const int big = 24;
    const sc_cache_desc d = desc(big);
    Pool p0(d), p1(d);
    char* free_pool = p1.p;
    sc_cache* first = nullptr;
    CHECK(sc_cache_create(&d, p0.p, &first) == SC_OK);
    std::vector<sc_cache*> h{first};
    std::vector<std::map<sc::StateKey, int32_t>> holds(1);
    int32_t sign = 1;
    for (int step = 0; step < 120; ++step) {
      const size_t i = rnd() % h.size();
      const sc_node nd{(int32_t)(rnd() % 6), (int32_t)(rnd() % 2)};
      const sc::StateKey key(nd.chunk, nd.level);
      switch (rnd() % 8) {
        case 0:
        case 1:
        case 2:
          if (!holds[i].count(key)) {
            const int rc = append(h[i], nd, sign);
            CHECK(rc == SC_OK || rc == SC_ECAPACITY);
            if (rc == SC_OK) holds[i][key] = sign++;
          }
          break;
        case 3:
          CHECK((sc_cache_release(h[i], nd) == SC_OK) == (holds[i].erase(key) == 1));
          break;
        case 4:
          if (h.size() < 4) {
            sc_cache* f = nullptr;
            CHECK(sc_cache_fork(h[i], &f) == SC_OK);
            h.push_back(f);
            const auto same = holds[i];
            holds.push_back(same);
          } else {
            sc_cache_free(h[i]);
            h.erase(h.begin() + i);
            holds.erase(holds.begin() + i);
          }
          break;
        case 5:
          CHECK(sc_cache_compact(h[i], nullptr, nullptr) == SC_OK);
          break;
        case 6: {
          const int used = h[i]->d.n_slots - sc_cache_free_slot_count(h[i]);
          char* old = h[i]->pool;
          CHECK(sc_cache_move(h[i], free_pool, used < 1 ? 1 : used + (int)(rnd() % (big + 1 - used)), nullptr, nullptr, nullptr) == SC_OK);
          free_pool = old;
          break;
        }
        default: {
          const size_t j = rnd() % h.size();
          const sc_node to{(int32_t)(rnd() % 6), (int32_t)(rnd() % 2)};
          const sc::StateKey tk(to.chunk, to.level);
          const int rc = sc_cache_copy(h[i], &nd, 1, h[j], &to, 0, kLayers, nullptr);
          if (!holds[i].count(key)) CHECK(rc == SC_ENOTFOUND);
          else if (holds[j].count(tk)) CHECK(rc == SC_EEXIST);
          else CHECK(rc == SC_OK || rc == SC_ECAPACITY);
          if (rc == SC_OK) holds[j][tk] = holds[i][key];
        }
      }
      for (size_t j = 0; j < h.size(); ++j) {
        CHECK(h[j]->states.size() == holds[j].size());
        for (const auto& kv : holds[j]) CHECK(signed_by(h[j], sc_node{kv.first.first, kv.first.second}, kv.second));
      }
    }
    for (sc_cache* c : h) sc_cache_free(c);
  }
}

// A block of a handle whose plan names pages of a state that a fork still holds.
void blocks() {
  sc_cache_desc d{1, 2, 128, 8, 1, 8, SC_DTYPE_BF16};
  Pool pool(d);
  sc_cache *a = nullptr, *b = nullptr;
  CHECK(sc_cache_create(&d, pool.p, &a) == SC_OK);
  CHECK(sc_cache_append(a, 0, sc_node{0, 0}, a, a, nullptr, nullptr) == SC_OK && sc_cache_fork(a, &b) == SC_OK);
  sc_policy pol{SC_POLICY_CLEAN, 1, 1, nullptr, nullptr, 0};
  const sc_node nd{1, 1};
  sc_selection* sel = nullptr;
  sc_plan* p = nullptr;
  CHECK(sc_selection_build(&pol, &nd, 1, &sel) == SC_OK && sc_plan_build(sel, a, &p) == SC_OK);
  char x = 0;
  alignas(16) static char wbuf[16];
  sc_block_weights w{};
  w.hidden = 256, w.n_heads = 2, w.head_dim = 128, w.mlp = 256;
  w.w_qkv = w.w_o = w.w_up = w.w_down = wbuf;
  std::vector<char> ws(sc_block_workspace_bytes(&w, 8) + 16);
  void* wsp = reinterpret_cast<void*>((reinterpret_cast<uintptr_t>(ws.data()) + 15) & ~uintptr_t(15));
  CHECK(sc_cache_release(a, {0, 0}) == SC_OK);
  CHECK(sc_block_forward(&w, a, 0, p, &x, nullptr, wsp, ws.size() - 16, nullptr) == SC_ESTALE);
  sc_plan_free(p);
  sc_selection_free(sel);
  sc_cache_free(b);
  sc_cache_free(a);
}

}  // namespace

int main() {
  forks();
  copies();
  moves();
  random_steps();
  blocks();
  std::printf("page checks passed\n");
  return 0;
}
