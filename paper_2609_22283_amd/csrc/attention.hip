// Packed paged block-causal attention (Eq. 6 over the plan's page lists).
//
// For every pack node i and head h: O = softmax(Q K^T * scale) V over the
// keys of node i's pages only.  The visibility mask is never formed: the page
// list is the mask.  Keys are concatenated page after page; every page holds
// a multiple of 8 tokens, so any 8 consecutive keys of the concatenation that
// start at a multiple of 8 lie in one page.
//
// bf16 kernel (head_dim 128), per work-group: 256 queries of one (node, head),
// eight waves of two 16-query blocks.  Key tiles of 64 are copied into LDS
// (double buffered, XOR-swizzled against bank conflicts); each wave computes
// S^T = K Q^T and O^T += V^T P^T with 16x16x32 bf16 MFMAs and keeps an online
// softmax in fp32.  The K rows feeding the S^T MFMA are permuted so that each
// lane's probabilities are exactly the B operand of the PV MFMA, and V is
// stored transposed in the cache so its A operand is one 16-byte LDS read.
// Two narrower forms of it and one that splits a node's keys over the waves of
// a work-group (attn_waves_kernel) serve shorter nodes and contexts;
// attn_schedule chooses.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>
#include <map>
#include <mutex>
#include <new>

#include "attention_core.h"

namespace sc {

// A form of the unit kernel: queries per work-group, 32-key halves per key tile
// and ring depth; attn_shape gives the widest form that a plan's nodes fill (64,
// 128 or 256 queries).  Nodes of at most 64 queries take the streaming form
// (ring 4 when the units fit the 512 work-groups resident with it, else ring 3
// with 768); larger ones a long-context form.  (The streaming form with 128
// queries per work-group measured 2-8 % slower than the long-context one on the
// short-context sweep: its 32-key steps cost more than the deeper ring gains.)
static int32_t shape_queries(int32_t nq) { return nq <= BQ_TINY ? BQ_TINY : nq <= BQ_SMALL ? BQ_SMALL : BQ_MAX; }
// Work-groups resident per CU: at most 8 waves (256 VGPRs each, 2 per SIMD)
// and 160 KB of LDS, 2 x ring x 8 KB per streaming work-group.
static int32_t per_cu(const AttnShape& s) {
  const int32_t by_vgpr = 8 / (s.bq / 32);
  return s.kh == 2 ? by_vgpr : std::min(by_vgpr, (160 * 1024) / (s.ring * 16 * 1024 + 4));
}
static AttnShape attn_shape(const sc_plan* p, const sc_cache* c) {
  AttnShape s;
  s.bq = shape_queries(p->nq);
  s.kh = s.bq == BQ_TINY ? 1 : 2;
  s.ring = 2;
  if (s.kh == 1) {
    const int32_t units = (int32_t)p->nodes.size() * c->d.n_heads * ((p->nq + s.bq - 1) / s.bq);
    s.ring = 4;
    if (units > kCUs * per_cu(s)) s.ring = 3;
  }
  return s;
}

// The workspace of a plan is the room for the partials of this schedule, on the
// widest form: units = heads x nodes x query tiles; the last (units mod resident
// work-groups) are cut into S pieces, S chosen to minimise the tail's rounds (in
// units of one whole unit) plus a per-piece cost of about two key tiles, with
// at most kAttnMaxPieces pieces and no more pieces than the shortest node has
// key tiles.  attn_schedule picks what runs within that room.
static AttnSchedule workspace_schedule(const sc_plan* p, const sc_cache* c) {
  const int32_t n = (int32_t)p->nodes.size();
  AttnSchedule ts;
  ts.sh = attn_shape(p, c);
  const int32_t bq = ts.sh.bq, bk = 32 * ts.sh.kh;
  const int32_t n_qtiles = (p->nq + bq - 1) / bq;
  const int32_t units = n * c->d.n_heads * n_qtiles;
  int64_t tiles = 0;
  int32_t min_tiles = INT32_MAX;
  for (int32_t i = 0; i < n; ++i) {
    const int32_t nt = (int32_t)(((int64_t)(p->page_off[i + 1] - p->page_off[i]) * c->d.tokens_per_page +
                                  bk - 1) / bk);
    tiles += nt;
    min_tiles = std::min(min_tiles, nt);
  }
  const double mean_tiles = (double)tiles / std::max(n, 1);
  const int32_t slots = kCUs * per_cu(ts.sh);  // work-groups resident at once
  ts.tail = units % slots;
  ts.whole = units - ts.tail;
  ts.split = 1;
  // Short units are not cut: the combine launch and the partial traffic are
  // fixed costs that a few-tile unit cannot repay (measured on the short
  // K/V streaming sweep).  The threshold is in 64-key tiles.
  if (ts.tail == 0 || mean_tiles * bk < kAttnMinSplitTiles * 64) return ts;
  double best = 1e30;
  const int32_t smax = std::max(1, std::min({16, kAttnMaxPieces / ts.tail, min_tiles}));
  for (int32_t sp = 1; sp <= smax; ++sp) {
    const double rounds = (double)((ts.tail * sp + slots - 1) / slots);
    const double cost = rounds * (1.0 / sp + 2.0 / mean_tiles);
    if (cost < best - 1e-9) {
      best = cost;
      ts.split = sp;
    }
  }
  return ts;
}

static size_t share_workspace_bytes(const sc_plan* p, const sc_cache* c, bool lse);
size_t attention_workspace_bytes(const sc_plan* p, const sc_cache* c) {
  if (p->nodes.empty()) return 0;
  if (p->shared) return share_workspace_bytes(p, c, false);
  return c->d.dtype == SC_DTYPE_BF16 ? workspace_schedule(p, c).partial_bytes() : 0;
}

// The cheapest schedule whose partials fit `room` bytes, by estimated time in
// us.  n is the units' mean length in 64-key tiles.  Measured (units of 12
// heads, 64 .. 4680 queries, 256 .. 32760 keys, each form and split forced): a
// unit takes
//   256 queries, one work-group per CU   1.5 n + 6
//   128 queries, two per CU              1.6 n + 8 together, 1.05 n + 6 alone
//   64 queries                           2.0 n + 2.5
// a round of pieces 7 us more (the partials' stores), the combine launch 4 us
// and 0.2 us per MB of partials; keys over waves, 32 queries per work-group, 6.5
// + 0.44 n per round and 1 in all.  So few units over short contexts go
// to the waves form (one 64-query node over 1344 keys 17 us, 43 on the 64-query
// form; 128 queries over 512 keys 10.6 us, 14.7), 256-query units that
// leave half the CUs idle to 128-query ones (four nodes of 520 queries over 3640
// keys 66 us, 104 in fifths), and long contexts stay where they were.
static AttnSchedule attn_schedule(const sc_plan* p, const sc_cache* c, size_t room) {
  const int32_t n = (int32_t)p->nodes.size();
  int64_t keys = 0;
  int32_t min_pages = INT32_MAX;
  for (int32_t i = 0; i < n; ++i) {
    const int32_t np = p->page_off[i + 1] - p->page_off[i];
    keys += (int64_t)np * c->d.tokens_per_page;
    min_pages = std::min(min_pages, np);
  }
  const double mean = (double)keys / n / 64.0;
  const auto units_of = [&](int32_t bq) { return n * c->d.n_heads * ((p->nq + bq - 1) / bq); };
  AttnSchedule best;
  best.sh = AttnShape{WV_BQ, 1, 1};
  best.whole = units_of(WV_BQ);
  best.tail = 0;
  best.split = 1;
  double best_cost = (double)((best.whole + kCUs - 1) / kCUs) * (0.44 * mean + 6.5) + 1.0;
  const AttnShape widest = attn_shape(p, c);
  for (int32_t bq = widest.bq; bq >= std::min(widest.bq, BQ_SMALL); bq /= 2) {
    AttnSchedule s;
    s.sh = bq == widest.bq ? widest : AttnShape{bq, 2, 2};
    const int32_t slots = kCUs * per_cu(s.sh), units = units_of(bq);
    s.tail = units % slots;
    s.whole = units - s.tail;
    const double a = bq == BQ_MAX ? 1.5 : bq == BQ_SMALL ? 1.6 : 2.0, f = bq == BQ_MAX ? 6.0 : bq == BQ_SMALL ? 8.0 : 2.5;
    const auto round = [&](int64_t items, double len) {  // the last, partly filled round
      return bq == BQ_SMALL && items <= kCUs ? 1.05 * len + 6.0 : a * len + f;
    };
    const int32_t min_tiles = (int32_t)((int64_t)min_pages * c->d.tokens_per_page / (32 * s.sh.kh));
    for (s.split = 1; s.split <= 16; ++s.split) {
      if (s.split > 1 && (s.tail == 0 || s.split > min_tiles || s.partial_bytes() > room)) break;
      const int64_t items = (int64_t)s.tail * s.split, full = items / slots, rest = items % slots;
      const double len = mean / s.split;
      double cost = (double)(s.whole / slots) * (a * mean + f) + (double)full * (a * len + f);
      if (rest) cost += round(rest, len);
      if (s.split > 1) cost += 7.0 * (double)items / slots + 4.0 + 0.2e-6 * (double)s.partial_bytes();
      if (cost < best_cost - 1e-9) {
        best_cost = cost;
        best = s;
      }
    }
  }
  best.us = best_cost;
  return best;
}

// What a keys-over-waves launch of `units` work-groups reads ahead, on a
// work-group per CU that it leaves idle: as many bytes as these fetch in the
// time the attention takes anyway.
static AttnAhead take_ahead(int32_t units, double us) {
  AttnAhead a;
  std::memset(&a, 0, sizeof a);
  a.units = units;
  ReadAhead* const ra = ReadAhead::current;
  if (!ra || units >= kCUs) return a;
  double room = kAheadBytesPerUs * std::min(1.0, (kCUs - units) / 128.0) * (us - kAheadLostUs);
  while (ra->next < ra->n && room >= 65536.0) {
    ReadAhead::Range& r = ra->range[ra->next];
    const size_t take = std::min(r.bytes, (size_t)room / 16 * 16);
    a.p[a.n] = r.p;
    a.vecs[a.n++] = (uint32_t)(take / 16);
    r.p += take;
    r.bytes -= take;
    room -= (double)take;
    if (r.bytes < 16) ++ra->next;
  }
  return a;
}

size_t attention_workspace_bound() { return (size_t)kAttnMaxPieces * BQ_MAX * (HDB + 2) * sizeof(float); }

static int share_check(const sc_plan* p, const sc_cache* c);
int attention_check(const sc_plan* p, const sc_cache* c) {
  const sc_cache_desc& d = c->d;
  const int32_t n = (int32_t)p->nodes.size();
  if (n > kMaxNodes) return fail(SC_EUNSUPPORTED, "pack of %d nodes exceeds %d", n, kMaxNodes);
  const size_t pages = p->page_slot.size() - (size_t)std::max(n - 1, 0) * p->shared;  // shared ones once
  if (pages > (size_t)kMaxPages) return fail(SC_EUNSUPPORTED, "plan of %zu pages exceeds %d", pages, kMaxPages);
  if (p->shared) {
    const int rc = share_check(p, c);
    if (rc != SC_OK) return rc;
  }
  if (d.dtype == SC_DTYPE_F32) return SC_OK;
  if (d.head_dim != HDB) return fail(SC_EUNSUPPORTED, "bf16 attention needs head_dim 128");
  const int32_t bk = p->shared ? 32 : 32 * attn_shape(p, c).kh;  // a key tile spans at most two pages
  if (d.tokens_per_page < bk)
    return fail(SC_EUNSUPPORTED, "bf16 attention of %d-query nodes needs pages of >= %d tokens (got %d)",
                p->nq, bk, d.tokens_per_page);
  if ((uint64_t)d.n_slots * c->slot_bytes > 0xffffffffull)
    return fail(SC_EUNSUPPORTED, "bf16 attention needs one layer of the pool within 4 GB");
  return SC_OK;
}

// Page lists in a traversal order shared by the pack's nodes.  The softmax
// sum does not depend on the order of a node's keys, so each node's list (its
// states' pages, oldest state first) is rotated to start at the anchor: the
// state read by the most nodes, the oldest of those.  Nodes of a progressive
// or same-level pack read overlapping windows of consecutive chunks; rotated
// this way, their work-groups read the shared states at the same time
// instead of one chunk apart.
// The order is a property of the plan alone: computed on its first launch
// and kept in it (a plan is immutable once built).
static void shared_order(const sc_plan* p, AttnPlan& plan) {
  const int32_t n = (int32_t)p->nodes.size();
  if (p->attn_slot.size() != p->page_slot.size()) {
    std::map<StateKey, int32_t> readers;
    for (int32_t i = 0; i < n; ++i)
      for (int32_t q = p->page_off[i]; q < p->page_off[i + 1]; ++q)
        if (q == p->page_off[i] || p->page_state[q] != p->page_state[q - 1]) ++readers[p->page_state[q]];
    StateKey anchor(INT32_MIN, INT32_MIN);
    int32_t most = 0;
    for (const auto& kv : readers)  // ascending (chunk, level): the oldest wins ties
      if (kv.second > most) {
        most = kv.second;
        anchor = kv.first;
      }
    std::vector<int32_t> order(p->page_slot.size());
    for (int32_t i = 0; i < n; ++i) {
      const int32_t a = p->page_off[i], b = p->page_off[i + 1];
      int32_t r = a;
      while (r < b && p->page_state[r] < anchor) ++r;
      if (r == b) r = a;
      int32_t o = a;
      for (int32_t q = r; q < b; ++q) order[o++] = p->page_slot[q];
      for (int32_t q = a; q < r; ++q) order[o++] = p->page_slot[q];
    }
    p->attn_slot.swap(order);
  }
  for (int32_t i = 0; i <= n; ++i) plan.page_off[i] = p->page_off[i];
  std::copy(p->attn_slot.begin(), p->attn_slot.end(), plan.page_slot);
}

// The fields of a launch that follow from the plan and the cache alone.
static LseGeom attn_geom(const sc_plan* p, const sc_cache* c, int32_t layer, float scale) {
  const sc_cache_desc& d = c->d;
  LseGeom g;
  std::memset(static_cast<void*>(&g), 0, sizeof g);
  g.layer_base = c->pool + (size_t)layer * d.n_slots * c->slot_bytes;
  g.slot_bytes = c->slot_bytes;
  g.kv_half = c->kv_half;
  g.n_nodes = (int32_t)p->nodes.size();
  g.n_heads = d.n_heads;
  g.tpp = d.tokens_per_page;
  g.nq = p->nq;
  g.tpp_div = magic_div((uint32_t)d.tokens_per_page);
  g.scale = scale;
  g.scale_log2 = scale * 1.4426950408889634f;
  g.unit = d.dtype == SC_DTYPE_F32 ? 1.f : logit_unit(scale);
  g.q_flip = std::signbit(scale) ? 0x80008000u : 0u;
  g.rows = g.n_nodes * p->nq;
  g.nq_div = magic_div((uint32_t)p->nq);
  return g;
}

template <>
void launch_form<PlainAttn>(const AttnShape& sh, uint32_t items, const AttnGeom& g, const AttnPlan& plan,
                            const void* q, void* o, int32_t dtype, int32_t head_dim, hipStream_t stream) {
  if (dtype == SC_DTYPE_F32) {
    timer_begin(TK_ATTENTION, stream);
    if (head_dim == 64)
      hipLaunchKernelGGL((attn_f32_kernel<64>), dim3(items), dim3(64 * F32_NW), 0, stream,
                         static_cast<const float*>(q), static_cast<float*>(o), g, plan);
    else
      hipLaunchKernelGGL((attn_f32_kernel<128>), dim3(items), dim3(64 * F32_NW), 0, stream,
                         static_cast<const float*>(q), static_cast<float*>(o), g, plan);
    timer_end(TK_ATTENTION, stream);
    return;
  }
  const uint16_t* qb = static_cast<const uint16_t*>(q);
  uint16_t* ob = static_cast<uint16_t*>(o);
  timer_begin(TK_ATTENTION, stream);
  if (sh.bq == BQ_TINY && sh.ring == 4)
    hipLaunchKernelGGL((attn_bf16_kernel<2, 1, 4>), dim3(items), dim3(128), 0, stream, qb, ob, g, plan);
  else if (sh.bq == BQ_TINY)
    hipLaunchKernelGGL((attn_bf16_kernel<2, 1, 3>), dim3(items), dim3(128), 0, stream, qb, ob, g, plan);
  else if (sh.bq == BQ_SMALL)
    hipLaunchKernelGGL((attn_bf16_kernel<4, 2, 2>), dim3(items), dim3(256), 0, stream, qb, ob, g, plan);
  else
    hipLaunchKernelGGL((attn_bf16_kernel<8, 2, 2>), dim3(items), dim3(512), 0, stream, qb, ob, g, plan);
  timer_end(TK_ATTENTION, stream);
  if (g.tail_units) {
    timer_begin(TK_ATTN_COMBINE, stream);
    const dim3 grid((uint32_t)g.tail_units, (uint32_t)sh.bq / 8);
    if (sh.bq == BQ_TINY)
      hipLaunchKernelGGL((attn_combine_kernel<BQ_TINY, 1>), grid, dim3(256), 0, stream, ob, g, plan);
    else if (sh.bq == BQ_SMALL)
      hipLaunchKernelGGL((attn_combine_kernel<BQ_SMALL, 2>), grid, dim3(256), 0, stream, ob, g, plan);
    else
      hipLaunchKernelGGL((attn_combine_kernel<BQ_MAX, 2>), grid, dim3(256), 0, stream, ob, g, plan);
    timer_end(TK_ATTN_COMBINE, stream);
  }
}

// Launches a plan by a schedule (unused for fp32 caches); exact: on the LseAttn forms,
// with lse where the rows' logarithmic sums go, or NULL.
static int launch_scheduled(const sc_plan* p, const sc_cache* c, int32_t layer, const void* q, void* o, bool exact,
                            float* lse, float scale, void* ws, const AttnSchedule& ts, hipStream_t stream) {
  const sc_cache_desc& d = c->d;
  AttnPlan plan;
  shared_order(p, plan);
  LseGeom g = attn_geom(p, c, layer, scale);
  g.lse = lse;
  uint32_t items;
  if (d.dtype == SC_DTYPE_F32) {
    g.n_qtiles = (p->nq + F32_BQ - 1) / F32_BQ;
    items = (uint32_t)g.n_nodes * d.n_heads * g.n_qtiles;
  } else {
    if (reinterpret_cast<uintptr_t>(ws) & 15) return fail(SC_EINVAL, "workspace must be 16-byte aligned");
    const int32_t bq = ts.sh.bq;
    g.n_qtiles = (p->nq + bq - 1) / bq;
    g.whole_units = ts.whole;
    g.tail_units = ts.tail;
    g.tail_split = ts.split;
    if (ts.split == 1) {  // no pieces: the tail units run whole
      g.whole_units += ts.tail;
      g.tail_units = 0;
    }
    g.part_o = static_cast<float*>(ws);
    g.part_ml = g.part_o + (size_t)g.tail_units * g.tail_split * bq * HDB;
    items = (uint32_t)(g.whole_units + g.tail_units * g.tail_split);
  }
  if (exact) {
    launch_form<LseAttn>(ts.sh, items, g, plan, q, o, d.dtype, d.head_dim, stream);
  } else if (d.dtype == SC_DTYPE_BF16 && ts.sh.bq == WV_BQ) {
    const uint16_t* qb = static_cast<const uint16_t*>(q);
    uint16_t* ob = static_cast<uint16_t*>(o);
    const AttnAhead ahead = take_ahead((int32_t)items, ts.us);
    timer_begin(TK_ATTENTION, stream);
    if (ahead.n)
      hipLaunchKernelGGL((attn_waves_kernel<AttnAhead>), dim3(kCUs), dim3(64 * WV_NW), 0, stream, qb, ob,
                         static_cast<const AttnGeom&>(g), plan, ahead);
    else
      hipLaunchKernelGGL((attn_waves_kernel<NoAhead>), dim3(items), dim3(64 * WV_NW), 0, stream, qb, ob,
                         static_cast<const AttnGeom&>(g), plan, NoAhead{});
    timer_end(TK_ATTENTION, stream);
  } else {
    launch_form<PlainAttn>(ts.sh, items, g, plan, q, o, d.dtype, d.head_dim, stream);
  }
  SC_HIP(hipGetLastError());
  return SC_OK;
}

// ------------------------------------------------------- a prefix shared by the pack
// A plan of sc_plan_share, and any plan whose rows' logarithmic sums are asked for,
// runs in one of two ways, whichever is estimated cheaper:
// its nodes' whole page lists as any plan's (the nodes of long chunks fill their
// query tiles by themselves, and nothing is left to merge), or as a SharePlan,
// which reads the prefix once for all rows: a node of few queries leaves most of
// a query tile empty, and n nodes would read the prefix n times.
// Measured, lists against once (12 heads of 128, bf16 unless said): 8 nodes of 1 query
// over 64 x 64 keys 33.1 us against 13.4, of 16 queries 34.8 against 18.7; 4 of 64
// queries 30.8 against 24.6; 4 of 256 over 32 x 256 keys 65.7 against 76.4; 4 of 4680
// over 9 x 1560 do not fit the partials; fp32, 8 of 16 queries over 64 x 96 keys 149
// against 68.  No prefix, own lists in pieces: 64 queries over 21 x 64 keys 21.2 us
// whole, 17.2 in sevenths; 3 of 792 queries over 21 x 264 keys 94 us whole, 90 in halves.
struct ShareSchedule {
  size_t room = 0;          // it was found for
  bool lse = false;
  bool whole_lists = false;  // the nodes' whole page lists, by `lists`
  AttnSchedule lists{};
  AttnShape sh{};
  int32_t p_tiles = 1, o_tiles = 1;  // key tiles per piece of the prefix and of the own pages
  int32_t p_pieces = 0, o_pieces = 1;
  bool own_waves = false;
  size_t bytes = 0;  // its partials
  double us = 1e30;
};

static int32_t own_pages(const sc_plan* p, int32_t i) { return p->page_off[i + 1] - p->page_off[i] - p->shared; }

// Key tiles of a form over np pages (the fp32 kernel's lie in one page each).
static int64_t share_tiles(const sc_cache* c, const AttnShape& s, int64_t np) {
  const int32_t tpp = c->d.tokens_per_page;
  if (c->d.dtype == SC_DTYPE_F32) return np * ((tpp + F32_BK - 1) / F32_BK);
  return (np * tpp + 32 * s.kh - 1) / (32 * s.kh);
}

static bool lists_fit(const sc_plan* p, const sc_cache* c) {
  return p->page_slot.size() <= (size_t)kMaxPages &&
         (c->d.dtype == SC_DTYPE_F32 || c->d.tokens_per_page >= 32 * attn_shape(p, c).kh);
}

// Own pages of at most so many 32-key tiles are a wave's work (attn_waves_kernel): 32
// nodes of 1 query, 12 heads, over 64 pages of the tokens said and one of their
// own: 34.3 us so at 192 tokens (6 tiles), 38.2 on a work-group each; 43.6 against 40.0
// at 256 (8 tiles).
constexpr int32_t kOwnWaveTiles = 6;

// The time at which `slots` work-groups at once have done classes of items, one class
// after the other: class k is count[k] items of us[k] each.
static double makespan(int64_t slots, const double* count, const double* us, int classes) {
  struct Level {
    double free, at;  // so many slots are free from this time on
  } lv[16] = {{(double)slots, 0.0}};
  int n = 1;
  double end = 0.0;
  for (int k = 0; k < classes; ++k)
    for (double left = count[k]; left > 0;) {
      double early = lv[0].at, late = lv[0].at;
      for (int i = 1; i < n; ++i) {
        early = std::min(early, lv[i].at);
        late = std::max(late, lv[i].at);
      }
      if (left >= 2 * slots && late - early <= us[k]) {  // a round moves every slot on alike
        const double rounds = std::floor(left / slots) - 1;
        for (int i = 0; i < n; ++i) lv[i].at += rounds * us[k];
        end = std::max(end, late + rounds * us[k]);
        left -= rounds * slots;
      }
      int first = 0;
      for (int i = 1; i < n; ++i)
        if (lv[i].at < lv[first].at) first = i;
      const double take = std::min(left, lv[first].free);
      const double at = lv[first].at + us[k];
      end = std::max(end, at);
      left -= take;
      lv[first].free -= take;
      int same = -1;
      for (int i = 0; i < n; ++i)
        if (lv[i].free > 0 && std::fabs(lv[i].at - at) < 1e-3) same = i;
      if (same >= 0)
        lv[same].free += take;
      else if (lv[first].free <= 0)
        lv[first] = Level{take, at};
      else if (n < 16)
        lv[n++] = Level{take, at};
      else
        return end + left * us[k] / slots;
      if (lv[first].free <= 0 && n > 1) lv[first] = lv[--n];
    }
  return end;
}

// The cheapest way within `room` bytes of partials, by estimated time in us: the
// items' times as in attn_schedule (fp32: 0.32 us per 16-key tile of 128 channels and
// 6), dealt out in their order; no less than the
// pages take from HBM, at 5 MB per us and 25 KB per us of a CU (what the copies in
// flight of a work-group fetch); the partials written at the same rate and read by
// the merging kernel, 4 us and 0.2 per MB.
static ShareSchedule find_share_schedule(const sc_plan* p, const sc_cache* c, size_t room, bool lse) {
  const sc_cache_desc& d = c->d;
  const bool f32 = d.dtype == SC_DTYPE_F32;
  const int32_t n = (int32_t)p->nodes.size(), H = d.n_heads;
  const int64_t rows = (int64_t)n * p->nq;
  int64_t own = 0, own_max = 0;
  for (int32_t i = 0; i < n; ++i) {
    own += own_pages(p, i);
    own_max = std::max<int64_t>(own_max, own_pages(p, i));
  }
  ShareSchedule best;
  best.room = room;
  best.lse = lse;
  if (lists_fit(p, c)) {
    best.whole_lists = true;
    if (f32) {
      const double tiles = (double)share_tiles(c, {}, (int64_t)p->page_slot.size()) / n;
      best.us = std::ceil((double)n * H * ((p->nq + F32_BQ - 1) / F32_BQ) / kCUs) * (6.0 + 0.32 * d.head_dim / 128 * tiles);
    } else {
      best.lists = attn_schedule(p, c, std::min(room, workspace_schedule(p, c).partial_bytes()));
      best.bytes = best.lists.partial_bytes();
      // every node's list is read once at least, from the memory-side cache where
      // another node read it before
      best.us = std::max(best.lists.us, (double)p->page_slot.size() * c->slot_bytes / 10e6);
    }
  }
  const double page_bytes = (double)(p->shared + own) * c->slot_bytes;
  const AttnShape forms[] = {{WV_BQ, 1, 1}, {BQ_TINY, 1, 4}, {BQ_SMALL, 2, 2}, {BQ_MAX, 2, 2}};
  for (AttnShape sh : forms) {
    if (f32) sh = AttnShape{F32_BQ, 0, 1};
    if (!f32 && d.tokens_per_page < 32 * sh.kh) continue;
    const int32_t bq = sh.bq, per = f32 || bq == WV_BQ ? 1 : per_cu(sh), slots = kCUs * per;
    const double a = f32 ? 0.32 * d.head_dim / 128 : (bq == BQ_MAX ? 1.5 : bq == BQ_SMALL ? 1.6 : bq == BQ_TINY ? 2.0 : 0.44) * sh.kh / 2;
    const double f = f32 ? 6.0 : bq == BQ_MAX ? 6.0 : bq == BQ_SMALL ? 8.0 : bq == BQ_TINY ? 2.5 : 6.5;
    const int64_t pt = p->shared ? share_tiles(c, sh, p->shared) : 0, ot_max = share_tiles(c, sh, own_max);
    const double p_units = p->shared ? (double)H * ((rows + bq - 1) / bq) : 0.0;
    const double o_units = (double)H * n * ((p->nq + bq - 1) / bq);
    const bool waves = p->shared && bq == WV_BQ && ot_max <= kOwnWaveTiles;
    const int64_t cut = pt ? pt : ot_max;
    // lengths of a piece: the whole prefix, then shorter by a sixteenth each; own pages
    // in pieces of the same length, or whole
    for (int64_t len = cut; len >= 1; len -= std::max<int64_t>(1, len / 16))
      for (const int64_t o_len : {std::min(len, ot_max), ot_max}) {
        if (waves && o_len != ot_max) continue;
        const int64_t pp = (pt + len - 1) / len, oo = (ot_max + o_len - 1) / o_len;
        const size_t bytes = (size_t)((pp + oo) * H * rows) * (d.head_dim + 2) * sizeof(float);
        if (bytes > room || pp * p_units + oo * o_units > INT32_MAX / 2) continue;
        const double ot = (double)share_tiles(c, sh, own) / n;
        const double count[] = {(double)(pt / len) * p_units, pt % len ? p_units : 0.0,
                                waves ? std::ceil(o_units / WV_NW) : o_units * std::ceil(ot / o_len)};
        const double us[] = {a * len + f, a * (double)(pt % len) + f,
                             waves ? 6.0 + 0.9 * ot : a * std::min<double>(o_len, ot) + f};
        const double cus = std::min<double>(kCUs, std::ceil((pt ? pp * p_units : count[2]) / per));
        const double t = std::max(makespan(slots, count, us, 3), page_bytes / std::min(5e6, 25e3 * cus) + 3.0) +
                         (double)bytes / 5e6 + 4.0 + 0.2e-6 * (double)bytes;
        if (t < best.us - 1e-9) {
          best.whole_lists = false;
          best.sh = sh;
          best.p_tiles = (int32_t)len;
          best.o_tiles = (int32_t)o_len;
          best.p_pieces = (int32_t)pp;
          best.o_pieces = (int32_t)oo;
          best.own_waves = waves;
          best.bytes = bytes;
          best.us = t;
        }
      }
    if (f32) break;
  }
  return best;
}

// Found once per plan, for the few rooms that its calls ask for.  Where host memory
// runs out, one that fits no call (its bytes exceed any workspace).
static const ShareSchedule& share_schedule(const sc_plan* p, const sc_cache* c, size_t room, bool lse) {
  for (const auto& s : p->share)
    if (s->room == room && s->lse == lse) return *s;
  try {
    p->share.push_back(std::make_shared<ShareSchedule>(find_share_schedule(p, c, room, lse)));
  } catch (const std::bad_alloc&) {
    static const ShareSchedule none = [] {
      ShareSchedule s;
      s.bytes = SIZE_MAX / 2;
      return s;
    }();
    return none;
  }
  return *p->share.back();
}

static size_t share_workspace_bytes(const sc_plan* p, const sc_cache* c, bool lse) {
  return share_schedule(p, c, attention_workspace_bound(), lse).bytes;
}
size_t attention_lse_workspace_bytes(const sc_plan* p, const sc_cache* c) {
  return p->nodes.empty() ? 0 : share_workspace_bytes(p, c, true);
}

// Neither way fits: more pages in the lists than a launch takes, and more rows
// than the partials of a prefix have room for.
static int share_check(const sc_plan* p, const sc_cache* c) {
  const size_t least = 2 * p->nodes.size() * p->nq * c->d.n_heads * (c->d.head_dim + 2) * sizeof(float);
  if (!lists_fit(p, c) && least > attention_workspace_bound())
    return fail(SC_EUNSUPPORTED, "%zu rows sharing a prefix need %zu bytes of partials, at most %zu",
                p->nodes.size() * (size_t)p->nq, least, attention_workspace_bound());
  return SC_OK;
}

// left: where not NULL the pieces' partials are left as they are (and o unwritten).
static int launch_share(const sc_plan* p, const sc_cache* c, int32_t layer, const void* q, void* o, float* lse,
                        float scale, void* ws, const ShareSchedule& s, ShareMerge* left, hipStream_t stream) {
  if (s.whole_lists) return launch_scheduled(p, c, layer, q, o, true, lse, scale, ws, s.lists, stream);
  if (!s.sh.bq) return fail(SC_EUNSUPPORTED, "no way to run %zu rows over a shared prefix", p->nodes.size() * (size_t)p->nq);
  if (reinterpret_cast<uintptr_t>(ws) & 15) return fail(SC_EINVAL, "workspace must be 16-byte aligned");
  const sc_cache_desc& d = c->d;
  LseGeom g = attn_geom(p, c, layer, scale);
  SharePlan plan;
  g.lse = lse;
  g.p_qtiles = (g.rows + s.sh.bq - 1) / s.sh.bq;
  g.n_qtiles = (p->nq + s.sh.bq - 1) / s.sh.bq;
  g.p_pieces = s.p_pieces;
  g.p_tiles = s.p_tiles;
  g.p_full = p->shared ? (int32_t)(share_tiles(c, s.sh, p->shared) / s.p_tiles) : 0;
  g.o_pieces = s.o_pieces;
  g.o_tiles = s.o_tiles;
  g.own_waves = s.own_waves;
  std::copy(p->page_slot.begin(), p->page_slot.begin() + p->shared, plan.page_slot);
  int32_t pages = p->shared;
  plan.page_off[0] = 0;
  for (int32_t i = 0; i < g.n_nodes; ++i) {
    plan.page_off[i + 1] = pages;
    std::copy(p->page_slot.begin() + p->page_off[i] + p->shared, p->page_slot.begin() + p->page_off[i + 1],
              plan.page_slot + pages);
    pages += own_pages(p, i);
  }
  for (int32_t i = g.n_nodes + 1; i <= kMaxNodes + 1; ++i) plan.page_off[i] = pages;
  const int64_t o_units = (int64_t)g.n_nodes * g.n_qtiles * d.n_heads;
  const int64_t items = (int64_t)g.p_pieces * g.p_qtiles * d.n_heads +
                        (s.own_waves ? (o_units + WV_NW - 1) / WV_NW : o_units * g.o_pieces);
  g.part_o = static_cast<float*>(ws);
  g.part_ml = g.part_o + (size_t)(g.p_pieces + g.o_pieces) * d.n_heads * g.rows * d.head_dim;
  if (left) {
    left->g = g;
    for (int32_t i = 0; i < g.n_nodes; ++i)
      left->pieces[i] = (uint8_t)(g.p_pieces + (s.own_waves ? 1 : (share_tiles(c, s.sh, own_pages(p, i)) + g.o_tiles - 1) / g.o_tiles));
    launch_share_pieces(s.sh, (uint32_t)items, g, plan, q, d.dtype, d.head_dim, stream);
  } else {
    launch_form<ShareAttn>(s.sh, (uint32_t)items, g, plan, q, o, d.dtype, d.head_dim, stream);
  }
  SC_HIP(hipGetLastError());
  return SC_OK;
}

bool attention_leaves_partials(const sc_plan* p, const sc_cache* c) {
  const ShareSchedule& s = share_schedule(p, c, attention_workspace_bound(), true);
  return c->d.dtype == SC_DTYPE_BF16 && !s.whole_lists && s.sh.bq && s.p_pieces + s.o_pieces <= kMergePieces;
}

int launch_attention_partials(const sc_plan* p, const sc_cache* c, int32_t layer, const void* q, float scale, void* ws,
                              ShareMerge* left, hipStream_t stream) {
  return launch_share(p, c, layer, q, nullptr, nullptr, scale, ws, share_schedule(p, c, attention_workspace_bound(), true),
                      left, stream);
}

int launch_attention_lse(const sc_plan* p, const sc_cache* c, int32_t layer, const void* q, void* o, float* lse,
                         float scale, void* ws, size_t ws_bytes, hipStream_t stream) {
  const int rc = attention_check(p, c);
  if (rc != SC_OK) return rc;
  const size_t need = lse ? attention_lse_workspace_bytes(p, c) : attention_workspace_bytes(p, c);
  if (ws_bytes < need || (need && !ws))
    return fail(SC_EINVAL, "attention workspace of %zu bytes, need %zu", ws_bytes, need);
  if (p->shared || lse)
    return launch_share(p, c, layer, q, o, lse, scale, ws, share_schedule(p, c, attention_workspace_bound(), lse),
                        nullptr, stream);
  const AttnSchedule ts = c->d.dtype == SC_DTYPE_F32 ? AttnSchedule{} : attn_schedule(p, c, need);
  return launch_scheduled(p, c, layer, q, o, false, nullptr, scale, ws, ts, stream);
}

int launch_attention(const sc_plan* p, const sc_cache* c, int32_t layer, const void* q, void* o,
                     float scale, void* ws, size_t ws_bytes, hipStream_t stream) {
  if (const Weighing* w = Weighing::current; w && w->plan == p)
    return launch_attention_weigh(p, c, layer, q, o, scale, w->weights, w->ws, stream);
  return launch_attention_lse(p, c, layer, q, o, nullptr, scale, ws, ws_bytes, stream);
}

}  // namespace sc

extern "C" int sc_attention_form(const sc_plan* p, const sc_cache* c, int32_t* queries, int32_t* ring,
                                 int32_t* pieces) {
  using namespace sc;
  if (!p || !c || !queries || !ring || !pieces) return fail(SC_EINVAL, "null argument");
  if (p->cache != c) return fail(SC_EINVAL, "plan was built for another cache");
  if (p->nodes.empty()) return fail(SC_EINVAL, "a plan without nodes launches nothing");
  const int rc = attention_check(p, c);
  if (rc != SC_OK) return rc;
  *queries = F32_BQ;
  *ring = *pieces = 1;
  AttnSchedule ts{};
  if (p->shared) {
    const ShareSchedule& s = share_schedule(p, c, attention_workspace_bound(), false);
    if (!s.whole_lists) {
      *queries = s.sh.bq;
      *ring = s.sh.ring;
      *pieces = -s.p_pieces;
      return SC_OK;
    }
    ts = s.lists;
  }
  if (c->d.dtype == SC_DTYPE_F32) return SC_OK;
  if (!p->shared) ts = attn_schedule(p, c, attention_workspace_bytes(p, c));
  *queries = ts.sh.bq;
  *ring = ts.sh.ring;
  *pieces = ts.split;
  return SC_OK;
}

namespace sc {

// ------------------------------------------------ attention without allocation
// The split-key partials of sc_attention_noalloc live in this library-owned
// array; every GPU the library runs on holds its own copy until the process
// ends.  Host code never passes the array's name to a kernel (on the host it
// is a stand-in, not a device address): the device address comes from
// hipGetSymbolAddress, once per device, with that device current.
constexpr size_t kNoAllocScratchBytes = size_t(64) << 20;
static __device__ __align__(256) char scratch[kNoAllocScratchBytes];

static std::mutex g_scratch_mu;
static std::map<int, void*> g_scratch_ptr;  // device ordinal -> address of its scratch

static int scratch_address(void** out) {
  int dev = -1;
  SC_HIP(hipGetDevice(&dev));
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  auto it = g_scratch_ptr.find(dev);
  if (it == g_scratch_ptr.end()) {
    void* ptr = nullptr;
    const hipError_t e = hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch));
    if (e != hipSuccess) return hip_fail(e, "hipGetSymbolAddress(scratch)");
    if (!ptr || (reinterpret_cast<uintptr_t>(ptr) & 255))
      return fail(SC_EDEVICE, "scratch of device %d at unusable address %p", dev, ptr);
    it = g_scratch_ptr.emplace(dev, ptr).first;
  }
  *out = it->second;
  return SC_OK;
}

}  // namespace sc

extern "C" size_t sc_attention_noalloc_scratch_bytes(void) { return sc::kNoAllocScratchBytes; }

extern "C" int sc_attention_noalloc(const sc_plan* p, const sc_cache* c, int32_t layer, const void* q,
                                    void* o, float scale, sc_stream stream) {
  using namespace sc;
  if (!p || !c || !q || !o) return fail(SC_EINVAL, "null argument");
  int rc = plan_check(p, c, layer);
  if (rc != SC_OK) return rc;
  if (p->nodes.empty()) return SC_OK;
  if ((rc = attention_check(p, c)) != SC_OK) return rc;
  void* ptr = nullptr;
  if ((p->shared || c->d.dtype == SC_DTYPE_BF16) && (rc = scratch_address(&ptr)) != SC_OK) return rc;
  if (p->shared) {
    const ShareSchedule& s = share_schedule(p, c, kNoAllocScratchBytes, false);
    if (s.us >= 1e30) return fail(SC_ECAPACITY, "the rows sharing a prefix need more partials than the scratch holds");
    return launch_share(p, c, layer, q, o, nullptr, scale, ptr, s, nullptr, static_cast<hipStream_t>(stream));
  }
  AttnSchedule ts{};
  if (ptr) ts = attn_schedule(p, c, std::min(kNoAllocScratchBytes, attention_workspace_bytes(p, c)));
  return launch_scheduled(p, c, layer, q, o, false, nullptr, scale, ptr, ts, static_cast<hipStream_t>(stream));
}
