// Device code of the packed paged attention: the kernels that attention.hip
// launches, and the pieces of them that other kernels over the same pages use.
#pragma once

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "device.h"
#include "internal.h"

namespace sc {

constexpr int kMaxNodes = 64;
constexpr int kMaxPages = 800;

struct AttnPlan {
  int32_t page_off[kMaxNodes + 1];
  int32_t page_slot[kMaxPages];
};

// A pack whose nodes read a common prefix before pages of their own.  Its key
// segments are numbered like nodes: segment 0 is the prefix, read by the rows of all
// nodes as one matrix, segment 1 + i the own pages of node i.  Each segment's
// key tiles are cut into pieces of equal length (the last one shorter), and every
// piece leaves a partial.
struct SharePlan {
  int32_t page_off[kMaxNodes + 2];
  int32_t page_slot[kMaxPages];
};

struct AttnGeom {
  const char* layer_base;
  uint64_t slot_bytes, kv_half;
  int32_t n_nodes, n_heads, tpp, nq, n_qtiles;
  DivMagic tpp_div;
  float scale_log2;  // scale * log2(e): softmax evaluated with exp2
  float scale;
  // schedule of the bf16 kernel: whole units, then tail units cut in pieces
  int32_t whole_units, tail_units, tail_split;
  float* part_o;          // [tail_units * tail_split][BQ][128] unnormalised partial outputs
  float* part_ml;         // [tail_units * tail_split][2][BQ] partial max (log2 units) and sum
                          // (BQ: queries per work-group of the instantiation launched)
};

// What the forms that give the rows' logarithmic sums (LseAttn, ShareAttn) need beside.
struct LseGeom : AttnGeom {
  float* lse;             // [head][row] log2 of the row's sum, or null
  float unit;             // logit_unit(scale); fp32 caches: 1
  uint32_t q_flip;        // bf16: sign bits of a negative scale
  int32_t rows;           // rows of the pack, n_nodes * nq
  // ShareAttn: query tiles of the prefix; pieces and tiles per piece of the prefix, and
  // the most pieces and tiles per piece of own pages
  int32_t p_qtiles, p_pieces, p_tiles, o_pieces, o_tiles;
  int32_t p_full;              // pieces of the prefix of full length (p_pieces, or one less)
  int32_t own_waves;           // ShareAttn: a wave to itself for each node, head and query tile (attn_waves_kernel)
  DivMagic nq_div;
};

// What a kernel computes beside the output, and over which plan.
//   PlainAttn  nothing; nodes read their page lists
//   LseAttn    the rows' logarithmic sums as well, exact in fp32: the logits are
//              products of the bf16 values as they are (scaled in fp32, not in q)
//              and the sums are of the unrounded exponentials
//   ShareAttn  the same over a SharePlan
struct PlainAttn {
  using Plan = AttnPlan;
  using Geom = AttnGeom;
  static constexpr bool kLse = false, kShare = false;
};
struct LseAttn {
  using Plan = AttnPlan;
  using Geom = LseGeom;
  static constexpr bool kLse = true, kShare = false;
};
struct ShareAttn {
  using Plan = SharePlan;
  using Geom = LseGeom;
  static constexpr bool kLse = true, kShare = true;
};
// |scale| log2(e) as the factor of the bf16 forms' logits.  Not below the smallest normal
// number: a scale of zero would turn the -inf of a key past the end into NaN, and
// products of q and k below 2^100 times 2^-126 have an exponential of 1 in every bit.
inline float logit_unit(float scale) { return std::max(std::fabs(scale) * 1.4426950408889634f, FLT_MIN); }
template <class M>
__device__ __forceinline__ float unit_of(const typename M::Geom& g) {
  if constexpr (M::kLse) return g.unit;
  return 1.f;
}

struct AttnItem {
  int32_t head, node, qt;
  int32_t ta, tb;   // key tiles [ta, tb) of the unit
  int32_t ntiles;   // key tiles of the whole unit
  int32_t slot;     // partial slot, or -1 for a whole unit
  int32_t row0, rows;  // ShareAttn: the segment's first row and its rows
};

// The item's fields in scalar registers: out of divisions they come in vector ones, which
// the long-context forms have none of to spare (eight spilled registers in the loop
// cost them a third: a reload waits for every copy in flight).
__device__ __forceinline__ void in_scalars(AttnItem& it) {
  it.head = __builtin_amdgcn_readfirstlane(it.head);
  it.node = __builtin_amdgcn_readfirstlane(it.node);
  it.qt = __builtin_amdgcn_readfirstlane(it.qt);
  it.ta = __builtin_amdgcn_readfirstlane(it.ta);
  it.tb = __builtin_amdgcn_readfirstlane(it.tb);
  it.ntiles = __builtin_amdgcn_readfirstlane(it.ntiles);
  it.slot = __builtin_amdgcn_readfirstlane(it.slot);
  it.row0 = __builtin_amdgcn_readfirstlane(it.row0);
  it.rows = __builtin_amdgcn_readfirstlane(it.rows);
}

// First row of an item's node or segment, and its rows.
template <class M>
__device__ __forceinline__ size_t item_row0(const AttnItem& it, const AttnGeom& g) {
  return M::kShare ? (size_t)it.row0 : (size_t)it.node * g.nq;
}
template <class M>
__device__ __forceinline__ int32_t item_rows(const AttnItem& it, const AttnGeom& g) {
  return M::kShare ? it.rows : g.nq;
}

// Key tiles of a SharePlan's segment: of 32 KH keys of the concatenated pages, or
// (KH 0, the fp32 kernel) of 16 keys of one page.
template <int KH>
__device__ __forceinline__ int32_t share_tiles(const SharePlan& plan, const AttnGeom& g, int32_t seg) {
  const int32_t npages = plan.page_off[seg + 1] - plan.page_off[seg];
  return KH ? (npages * g.tpp + 32 * KH - 1) / (32 * (KH ? KH : 1)) : npages * ((g.tpp + 15) / 16);
}

// Items of a SharePlan: the prefix's full pieces, its shorter last ones, the own
// pages'; each kind remapped on its own, since a work-group's XCD is fixed by its
// number and every XCD has to get its share of each.  Query tiles fastest, then (own pages) nodes:
// the work-groups that an XCD runs side by side read the same keys.  A piece past
// the end of a short list is empty (ta == tb).
template <int KH>
__device__ __forceinline__ AttnItem decode_item(const SharePlan& plan, const LseGeom& g, uint32_t b) {
  AttnItem it;
  const uint32_t n0 = (uint32_t)(g.p_pieces * g.p_qtiles * g.n_heads);
  int32_t piece, len;
  if (b < n0) {
    const uint32_t full = (uint32_t)(g.p_full * g.p_qtiles * g.n_heads);
    const int32_t i = (int32_t)(b < full ? xcd_remap(b, full) : full + xcd_remap(b - full, n0 - full));
    const int32_t unit = i % (g.p_qtiles * g.n_heads);
    piece = i / (g.p_qtiles * g.n_heads);
    it.qt = unit % g.p_qtiles;
    it.head = unit / g.p_qtiles;
    it.node = 0;
    it.row0 = 0;
    it.rows = g.rows;
    it.slot = piece;
    len = g.p_tiles;
  } else {
    const int32_t i = (int32_t)xcd_remap(b - n0, gridDim.x - n0), per = g.n_qtiles * g.n_nodes;
    const int32_t unit = i % (per * g.n_heads);
    piece = i / (per * g.n_heads);
    it.qt = unit % g.n_qtiles;
    it.node = 1 + unit / g.n_qtiles % g.n_nodes;
    it.head = unit / per;
    it.row0 = (it.node - 1) * g.nq;
    it.rows = g.nq;
    it.slot = g.p_pieces + piece;
    len = g.o_tiles;
  }
  it.ntiles = share_tiles<KH>(plan, g, it.node);
  it.ta = min(piece * len, it.ntiles);
  it.tb = min(it.ta + len, it.ntiles);
  return it;
}

// Direct global -> LDS copy of 16 bytes per lane (gfx950 LDS DMA): lane i
// of the wave writes bytes [16 i, 16 i + 16) after the wave-uniform LDS
// address, so the XOR swizzle is applied by choosing each lane's source
// (base + off).  Written as inline asm: while a copy it knows of is in
// flight, the compiler waits for every LDS read with lgkmcnt(0), so no
// fragment read could overlap another; the copies themselves complete
// under this wave's explicit vmcnt waits (landed, landed_but).  M0, which
// carries the LDS address, is saved and restored.
__device__ __forceinline__ uint32_t lds_addr(const char* p) {
  return (uint32_t)reinterpret_cast<uintptr_t>(p);
}
__device__ __forceinline__ void dma16(const char* base, uint32_t off, char* lds_wave_base) {
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %3\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, %2\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "v"(off), "s"(base), "s"(lds_addr(lds_wave_base))
      : "memory");
}

// All but this wave's N newest copies have landed.
template <int N>
__device__ __forceinline__ void copies_landed() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// This wave's LDS reads are done: what they read may be copied over.
__device__ __forceinline__ void reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// ------------------------------------------------------------- fp32 kernel
// Work-group: 16 queries of one (node, head).  Its eight waves take eight
// contiguous parts of the node's key tiles (16 keys of one page), each with
// its own online softmax, and merge through LDS at the end, in a fixed order
// and without a workspace.  Both products run on 16x16x4 fp32 MFMAs; their
// operands come straight from the cache as 16-byte loads (fp32 data is only
// 4-byte aligned, which is all these loads need):
//   S^T = K Q^T   the contraction index of MFMA (j, e) in lane group g is
//                 channel 16 j + 4 g + e, so a lane reads runs of 4 channels
//                 of its key row, and of its query row
//   O^T += V^T P^T  MFMA e contracts keys 4 g + e of the tile: lane (g, c)'s
//                 result e of S^T is then its B operand as it stands, and
//                 the A operand a run of 4 tokens of one V^T row
// What bounds it: the fp32 matrix rate of the compute units that hold
// work-groups (a 16-key tile is 64 MFMAs of 32 cycles at head_dim 128), and
// at few tiles per wave the loads' latency.  The split over waves fills the
// chip from one node's queries: one thread per query (the form before) had
// 40 waves in flight and a chain of 128 dependent FMAs per key.
// 4 nodes x 312 queries x 2184 keys, 2 heads of 128: 61 us (46 TFLOP/s; 59 before
// the values behind a page's end were cleared) against 15.6 ms.
// STAGED (pages on 16-byte boundaries): each wave copies its tiles into LDS, K(t + 1)
// over K(t) once that has been read and V(t + 1) likewise, and takes the operands from
// there.  The loads above put adjacent lanes on adjacent rows, so each of their 16
// bytes is a cache access of its own.  16 x 100 rows over 12384 keys, 12 heads of 64:
// 582 us (105 TFLOP/s of 154), 834 without.  Of the vector instructions between the
// products (the products of 16 queries leave little room for them) those forms take the
// exponentials to base 2 (one instruction; the plain form calls expf) and the copies'
// addresses from lane offsets that no tile changes: 695 us before.
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
constexpr int F32_NW = 8, F32_BQ = 16, F32_BK = 16;

template <int HD, class M = PlainAttn, bool STAGED = false>
__global__ __launch_bounds__(64 * F32_NW) void attn_f32_kernel(const float* __restrict__ q, float* __restrict__ o,
                                                               typename M::Geom g, typename M::Plan plan) {
  constexpr int NJ = HD / 16;  // 16-channel blocks
  constexpr int ROW = HD * 4, TILE = F32_BK * ROW, CP = TILE / 1024;  // a K or V^T tile, its copies
  constexpr int PART = F32_NW / 2 * NJ * 64 * 16;
  __shared__ __attribute__((aligned(1024))) char smem[STAGED ? F32_NW * 2 * TILE : PART];
  static_assert(!STAGED || PART <= F32_NW * 2 * TILE, "the merge fits the tiles");
  f32x4(*const part)[NJ][64] = reinterpret_cast<f32x4(*)[NJ][64]>(smem);
  __shared__ float ml[2][F32_NW][F32_BQ];
  const int32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t lg = lane >> 4, c = lane & 15;
  AttnItem it;
  if constexpr (M::kShare) {
    it = decode_item<0>(plan, g, blockIdx.x);
    if (it.ta == it.tb) return;
  } else {
    // query tiles fastest: an XCD's work-groups share the K/V of one or two (node, head)s
    const int32_t unit = (int32_t)xcd_remap(blockIdx.x, gridDim.x);
    it.qt = unit % g.n_qtiles;
    const int32_t nh = unit / g.n_qtiles;
    it.node = nh % g.n_nodes;
    it.head = nh / g.n_nodes;
    it.slot = -1;
  }
  const int32_t node = it.node, head = it.head;
  const size_t row0 = item_row0<M>(it, g);
  const int32_t rows = item_rows<M>(it, g), row = it.qt * F32_BQ + c;
  const size_t qoff = ((row0 + min(row, rows - 1)) * g.n_heads + head) * HD + 4 * lg;
  f32x4 qr[NJ], acc[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    qr[j] = *reinterpret_cast<const f32x4u*>(q + qoff + 16 * j) * (M::kLse ? g.scale_log2 : g.scale);
    acc[j] = f32x4{};
  }
  const int32_t p0 = plan.page_off[node], npages = plan.page_off[node + 1] - p0;
  const int32_t tp = (g.tpp + F32_BK - 1) / F32_BK;  // tiles per page
  int32_t nt = npages * tp, tile0 = 0;
  if constexpr (M::kShare) {
    tile0 = it.ta;
    nt = it.tb - it.ta;
  }
  const int32_t t_end = tile0 + (int32_t)((int64_t)(wave + 1) * nt / F32_NW);
  int32_t t = tile0 + (int32_t)((int64_t)wave * nt / F32_NW), page = t / tp, tt = t - page * tp;
  // K rows of keys past the page's end read its last key, V^T runs past it
  // the page's first tokens (valid memory); their probabilities are zero, and
  // so are these V^T values, since an infinity there would make 0 x inf
  auto load_k = [&](f32x4 (&kf)[NJ]) {
    const float* kb = reinterpret_cast<const float*>(g.layer_base + (size_t)plan.page_slot[p0 + page] * g.slot_bytes) +
                      ((size_t)head * g.tpp + min(F32_BK * tt + c, g.tpp - 1)) * HD + 4 * lg;
#pragma unroll
    for (int j = 0; j < NJ; ++j) kf[j] = *reinterpret_cast<const f32x4u*>(kb + 16 * j);
  };
  // STAGED: 16-byte columns are swizzled by the row (K: its number, V^T: a quarter of it)
  char* const kl = smem + wave * 2 * TILE;
  char* const vl = kl + TILE;
  const auto slot_base = [&](int32_t pg) { return g.layer_base + (size_t)plan.page_slot[p0 + pg] * g.slot_bytes; };
  // A lane's part of the addresses is the same in every tile that lies whole in its
  // page.  Copies go out in fours, with one M0 (copy_group): K copy j adds 1024 j to both
  // addresses and its own bits of the swizzle, V^T copy j 16 rows.
  constexpr int LPR = ROW / 16, RPC = 64 / LPR;  // lanes of a K row, K rows of a copy
  const int32_t kr0 = lane / LPR, kcol0 = (lane % LPR) ^ kr0, vkey0 = 4 * ((lane & 3) ^ (lane >> 4));
  const uint32_t klane0 = (uint32_t)kr0 * ROW + 16 * kcol0;
  uint32_t vlane[STAGED ? CP : 1];
  if constexpr (STAGED)
#pragma unroll
    for (int j = 0; j < CP; ++j)
      vlane[j] = ((uint32_t)(16 * j + (lane >> 2)) * g.tpp + vkey0) * 4 + (kCopyBias - 1024 * (j & 3));
  const auto stage_k = [&](int32_t page, int32_t tt) __attribute__((always_inline)) {
    const char* base = slot_base(page) + ((size_t)head * g.tpp + F32_BK * tt) * ROW;
    const int32_t past = g.tpp - F32_BK * tt;  // rows from here on lie past the page's end
#pragma unroll
    for (int h = 0; h < CP / 4; ++h) {
      uint32_t off[4];
      if (past >= F32_BK) {
#pragma unroll
        for (int j = 0; j < 4; ++j) off[j] = klane0 ^ (16 * RPC * (4 * h + j));
        copy_group<4>(base + 4096 * h, off, lds_addr(kl) + 4096 * h);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int32_t r = RPC * (4 * h + j) + kr0;
          off[j] = (uint32_t)min(r, past - 1) * ROW + 16 * (kcol0 ^ (RPC * (4 * h + j))) + (kCopyBias - 1024 * j);
        }
        copy_group<4>(base - kCopyBias, off, lds_addr(kl) + 4096 * h);
      }
    }
  };
  const auto stage_v = [&](int32_t page, int32_t tt) __attribute__((always_inline)) {
    const char* base = slot_base(page) + g.kv_half + (size_t)head * g.tpp * ROW - kCopyBias;
    const int32_t key = F32_BK * tt;
#pragma unroll
    for (int h = 0; h < CP / 4; ++h) {
      if (key + F32_BK <= g.tpp) {
        copy_group<4>(base + 4 * key, vlane + 4 * h, lds_addr(vl) + 4096 * h);
      } else {
        uint32_t off[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) off[j] = vlane[4 * h + j] + (key + vkey0 < g.tpp ? 4 * key : -4 * vkey0);
        copy_group<4>(base, off, lds_addr(vl) + 4096 * h);
      }
    }
  };
  const auto ex = [](float x) { return M::kLse ? __builtin_amdgcn_exp2f(x) : expf(x); };
  float m = -INFINITY, l = 0.f;
  f32x4 kf[NJ];
  if constexpr (STAGED) {
    // fragments are read out of LDS ahead of the products that need them: V^T(t) while the
    // softmax runs, K(t + 1) while V^T(t) is multiplied
    int32_t kpage = page, ktt = tt;  // of the next K tile to copy
    const auto next = [&](int32_t& pg, int32_t& tl) __attribute__((always_inline)) {
      if (++tl == tp) {
        tl = 0;
        ++pg;
      }
    };
    const auto read_k = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) kf[j] = *reinterpret_cast<const f32x4*>(kl + c * ROW + (((4 * j + lg) ^ c) << 4));
    };
    if (t < t_end) {
      stage_k(kpage, ktt);
      stage_v(page, tt);
      copies_landed<CP>();  // K(t); V^T(t) may still be under way
      read_k();
      reads_done();
      next(kpage, ktt);
      if (t + 1 < t_end) stage_k(kpage, ktt);
    }
    for (; t < t_end; ++t) {
      const bool more = t + 1 < t_end;
      f32x4 s0 = {}, s1 = {};
#pragma unroll
      for (int j = 0; j < NJ; j += 2)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[j][e], qr[j][e], s0, 0, 0, 0);
          s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[j + 1][e], qr[j + 1][e], s1, 0, 0, 0);
        }
      if (more)
        copies_landed<CP>();  // V^T(t); K(t + 1) may still be under way
      else
        copies_landed<0>();
      f32x4 vf[NJ];
#pragma unroll
      for (int j = 0; j < NJ; ++j) vf[j] = *reinterpret_cast<const f32x4*>(vl + (16 * j + c) * 64 + ((lg ^ (c >> 2)) << 4));
      const int32_t k0 = F32_BK * tt + 4 * lg;  // this lane's first key of the tile, within the page
      f32x4 s = s0 + s1;
      if (k0 + 4 > g.tpp) s = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};  // pages hold whole runs of 8 keys
      float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float mn = fmaxf(m, mx);
      if (__builtin_amdgcn_ballot_w64(mn > m)) {
        const float alpha = mn == -INFINITY ? 1.f : ex(m - mn);
        l *= alpha;
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[j] *= alpha;
        m = mn;
      }
      const float ms = m == -INFINITY ? 0.f : m;  // every logit so far -inf: no weight yet
      f32x4 p;
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] = ex(s[e] - ms);
      l += (p[0] + p[1]) + (p[2] + p[3]);
      reads_done();
      if (F32_BK * tt + F32_BK > g.tpp) {  // the page ends in this tile
        asm volatile("");  // a branch, not a selection in every tile
        if (k0 >= g.tpp)
#pragma unroll
          for (int j = 0; j < NJ; ++j) vf[j] = f32x4{};
      }
      if (more) {
        next(page, tt);
        stage_v(page, tt);
        copies_landed<CP>();  // K(t + 1)
        read_k();
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[j][e], p[e], acc[j], 0, 0, 0);
      if (more) {
        reads_done();
        next(kpage, ktt);
        if (t + 2 < t_end) stage_k(kpage, ktt);
      }
    }
  } else {
    if (t < t_end) load_k(kf);
    while (t < t_end) {
      const int32_t k0 = F32_BK * tt + 4 * lg;  // this lane's first key of the tile, within the page
      f32x4 vf[NJ];
      const float* vb = reinterpret_cast<const float*>(g.layer_base + (size_t)plan.page_slot[p0 + page] * g.slot_bytes +
                                                       g.kv_half) +
                        ((size_t)head * HD + c) * g.tpp + (k0 < g.tpp ? k0 : 0);
#pragma unroll
      for (int j = 0; j < NJ; ++j) vf[j] = *reinterpret_cast<const f32x4u*>(vb + (size_t)16 * j * g.tpp);
      const bool page_end = F32_BK * tt + F32_BK > g.tpp;
      f32x4 s0 = {}, s1 = {};
#pragma unroll
      for (int j = 0; j < NJ; j += 2)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[j][e], qr[j][e], s0, 0, 0, 0);
          s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[j + 1][e], qr[j + 1][e], s1, 0, 0, 0);
        }
      ++t;
      if (++tt == tp) {
        tt = 0;
        ++page;
      }
      const bool more = t < t_end;
      if (more) load_k(kf);
      f32x4 s = s0 + s1;
      if (k0 + 4 > g.tpp) s = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};  // pages hold whole runs of 8 keys
      float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float mn = fmaxf(m, mx);
      if (__builtin_amdgcn_ballot_w64(mn > m)) {
        const float alpha = mn == -INFINITY ? 1.f : ex(m - mn);
        l *= alpha;
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[j] *= alpha;
        m = mn;
      }
      const float ms = m == -INFINITY ? 0.f : m;  // every logit so far -inf: no weight yet
      f32x4 p;
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] = ex(s[e] - ms);
      l += (p[0] + p[1]) + (p[2] + p[3]);
      if (page_end && k0 >= g.tpp)
#pragma unroll
        for (int j = 0; j < NJ; ++j) vf[j] = f32x4{};
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[j][e], p[e], acc[j], 0, 0, 0);
    }
  }
  // merge: every wave scales its part to the common maximum, then a tree of
  // LDS additions (a wave without tiles adds zeros), over the tiles
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (lg == 0) {
    ml[0][wave][c] = m;
    ml[1][wave][c] = l;
  }
  __syncthreads();
  float mt = ml[0][0][c], lt = 0.f;
#pragma unroll
  for (int w = 1; w < F32_NW; ++w) mt = fmaxf(mt, ml[0][w][c]);
  // a piece without a finite logit adds zeros to its row
  const float base = M::kShare && mt == -INFINITY ? 0.f : mt;
#pragma unroll
  for (int w = 0; w < F32_NW; ++w) lt += ml[1][w][c] * ex(ml[0][w][c] - base);
  const float f = ex(m - base);
#pragma unroll
  for (int j = 0; j < NJ; ++j) acc[j] *= f;
#pragma unroll
  for (int h = F32_NW / 2; h >= 1; h /= 2) {
    if (wave >= h && wave < 2 * h)
#pragma unroll
      for (int j = 0; j < NJ; ++j) part[wave - h][j][lane] = acc[j];
    __syncthreads();
    if (wave < h)
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[j] += part[wave][j][lane];
    __syncthreads();
  }
  if constexpr (M::kShare) {
    if (wave == 0 && row < rows) {
      const size_t at = ((size_t)it.slot * g.n_heads + head) * g.rows + row0 + row;
#pragma unroll
      for (int j = 0; j < NJ; ++j) *reinterpret_cast<f32x4*>(g.part_o + at * HD + 16 * j + 4 * lg) = acc[j];
      if (lg == 0) {
        g.part_ml[2 * at] = mt;
        g.part_ml[2 * at + 1] = lt;
      }
    }
    return;
  }
  if (wave == 0 && row < g.nq) {
    const float inv = 1.f / lt;
    if constexpr (M::kLse)
      if (g.lse && lg == 0) g.lse[(size_t)head * g.rows + row0 + row] = mt + __builtin_amdgcn_logf(lt);
#pragma unroll
    for (int j = 0; j < NJ; ++j) *reinterpret_cast<f32x4u*>(o + qoff + 16 * j) = acc[j] * inv;
  }
}

// ------------------------------------------------------------- bf16 kernel
// Three work-group shapes: 8 waves x 32 queries (256 per work-group, one
// work-group per CU) and 4 waves x 32 queries (128, two per CU, for nodes of
// at most 128 queries), both with two waves per SIMD and 64-key tiles; and
// 2 waves x 32 queries (64, for nodes of at most 64) on 32-key tiles, whose
// deeper K/V rings (3 or 4 tiles of 16 KB) keep two or three tiles in flight
// per work-group, three or two work-groups per CU.  Such nodes are short and
// their attention streams K/V from HBM: in-flight copies, bounded by LDS,
// set its rate.  A wave's 32 queries are two 16-query blocks of the
// 16x16x32 MFMA; key tiles hold KH halves of 32 keys.
constexpr int HDB = 128;  // head dim of the bf16 kernels
template <int KH>
struct Tile {
  static constexpr int BK = 32 * KH;                  // keys per LDS tile
  static constexpr int KT_BYTES = BK * HDB * 2;       // K tile: BK rows of 256 bytes
  static constexpr int VT_BYTES = HDB * BK * 2;       // V^T tile: 128 rows of 2 BK bytes
};
constexpr int BQ_TINY = 64, BQ_SMALL = 128, BQ_MAX = 256;  // queries per work-group of the three shapes
// Softmax bookkeeping.  Q is pre-scaled by scale*log2(e), so S is in log2
// units, and each S tile starts its accumulation at -m: p = exp2(S)
// directly.  m is the exact maximum of the work item's first tile and is
// never raised inside the loop: later probabilities may exceed 1, which fp32
// sums and bf16 products represent with the same relative precision, up to
// a guard of 2^64 on each lane's tile sum.  A work-group in which any wave
// reaches the guard (logits more than 64 log2 units above the first tile's
// maximum) redoes its item exactly in two passes (attn_exact).  Rescaling in
// place would keep the accumulators and the recomputation live in the loop.
// The row sums come from the matrix cores: one more 16-row block of V^T whose
// first row is all ones turns O^T += V^T P^T into l += sum_k p as well, so
// the sum sees the same bf16 p as the numerator.  Since p >= 0 the final sum
// bounds every partial one, and the guard is checked once, on it.
constexpr float P_GUARD = 18446744073709551616.0f;  // 2^64

// Matrix-core shape: v_mfma_f32_16x16x32_bf16.  Lane l (g = l / 16,
// c = l % 16) supplies row c of A and column c of B with 8 consecutive k
// values 8 g .. 8 g + 7, and receives D[4 g + r][c], r = 0..3.  (The 16x16
// shape sustains more FLOP/s than 32x32x16 under the power cap: half the
// accumulator traffic per FLOP.)
__device__ __forceinline__ f32x4 mfma16(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// XOR swizzle of a K tile row: 16-byte column c of row r is stored at
// c ^ kswz(r).  Bit 4 of the row enters so that the 16 rows one 16-lane
// group reads for an S^T MFMA (see attn_lane) fall on distinct banks.
__device__ __forceinline__ uint32_t kswz(int32_t row) { return (uint32_t)((row & 15) ^ ((row >> 2) & 4)); }

struct AttnLane {
  // per-lane LDS read offsets (bytes) inside one buffer
  // K row of block 0, 16-byte column 4 ds + g (second 32 rows add 8192).  Block 1's
  // rows lie 4 below, which flips bit 2 of the swizzle: its column 4 ds + g is
  // stored where block 0's column 4 (ds ^ 1) + g is, 1024 bytes on.
  uint32_t koff[4];
  __device__ __forceinline__ uint32_t k(int b, int ds) const { return koff[ds ^ b] + 1024u * b; }
  uint32_t voff[2];     // V^T row c, 16-byte column 4 h + g (16-row block db adds 32 BK)
};

// XOR swizzle of a V^T tile row d (16-byte columns): 64-key rows (128 bytes)
// take (d / 2) mod 8, 32-key rows (64 bytes) (d / 4) mod 4, so the 16 rows
// of a PV operand read fall on distinct banks.
template <int KH>
__device__ __forceinline__ uint32_t vswz(int32_t d) {
  return KH == 2 ? (uint32_t)((d >> 1) & 7) : (uint32_t)((d >> 2) & 3);
}

// A row i of the S^T MFMA for 16-key block b of a 32-key half holds key
// 8 (i / 4) + 4 b + i % 4: each lane's four results of blocks 0 and 1 are
// then keys 8 g .. 8 g + 7 of the half -- exactly the B operand of the PV
// MFMA, which therefore needs no shuffle.
template <int KH>
__device__ __forceinline__ AttnLane attn_lane(int32_t c, int32_t g) {
  AttnLane L;
  const int32_t row = 8 * (c >> 2) + (c & 3);
#pragma unroll
  for (int ds = 0; ds < 4; ++ds) L.koff[ds] = row * 256 + (((4 * ds + g) ^ kswz(row)) << 4);
#pragma unroll
  for (int h = 0; h < 2; ++h)
    L.voff[h] = c * (64 * KH) + (((4 * h + g) ^ vswz<KH>(c)) << 4);  // h < KH only is used
  return L;
}

// Q^T operand of a 16-query block: lane holds Q[row][32 ds + 8 g .. +7].
// Rows past the node's end repeat its last row.  The loads are issued with
// the first tile copies (their latencies overlap); scale_q then pre-scales
// the values to log2 units once they have landed.
__device__ __forceinline__ void load_q(const uint16_t* q, const AttnGeom& g, size_t row0, int32_t rows, int32_t head,
                                       int32_t qrow, int32_t lg, bf16x8 (&qreg)[4]) {
  const int32_t qrow_c = qrow < rows ? qrow : rows - 1;
  const uint16_t* qp = q + ((row0 + qrow_c) * g.n_heads + head) * HDB + 8 * lg;
#pragma unroll
  for (int ds = 0; ds < 4; ++ds) qreg[ds] = *reinterpret_cast<const bf16x8*>(qp + 32 * ds);
}

// The forms with logarithmic sums keep the values and scale the logits instead, by
// |scale|: only the sign goes into q.
template <class M>
__device__ __forceinline__ void scale_q(const typename M::Geom& g, bf16x8 (&qreg)[4]) {
  if constexpr (M::kLse) {
#pragma unroll
    for (int ds = 0; ds < 4; ++ds) {
      u32x4 u = __builtin_bit_cast(u32x4, qreg[ds]);
#pragma unroll
      for (int e = 0; e < 4; ++e) u[e] ^= g.q_flip;
      qreg[ds] = __builtin_bit_cast(bf16x8, u);
    }
    return;
  }
#pragma unroll
  for (int ds = 0; ds < 4; ++ds)
#pragma unroll
    for (int e = 0; e < 8; ++e) qreg[ds][e] = static_cast<__bf16>(static_cast<float>(qreg[ds][e]) * g.scale_log2);
}

// Logits of one 64-key tile for a wave's two 16-query blocks:
// s[h][b][qb] holds, in lane (g, c) value r, key 32 h + 8 g + 4 b + r of the
// tile for query c of block qb.
template <int KH>
using STile = f32x4[KH][2][2];

// Sum / maximum of one query's values over the four lane groups.
__device__ __forceinline__ float group_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}
__device__ __forceinline__ float group_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

// A operand of the row-sum MFMA: row 0 all ones, rows 1..15 zero (lane c
// supplies row c).  D[0][query] = sum over the 32 keys of p.
__device__ __forceinline__ bf16x8 ones_row(int32_t c) {
  bf16x8 a;
  const __bf16 v = static_cast<__bf16>(c == 0 ? 1.0f : 0.0f);
#pragma unroll
  for (int e = 0; e < 8; ++e) a[e] = v;
  return a;
}

// Column maxima of a tile, per query block.
template <int KH>
__device__ __forceinline__ void tile_max(const STile<KH>& s, float (&mx)[2]) {
#pragma unroll
  for (int qb = 0; qb < 2; ++qb) {
    float m = s[0][0][qb][0];
#pragma unroll
    for (int h = 0; h < KH; ++h)
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) m = fmaxf(m, s[h][b][qb][r]);
    mx[qb] = group_max(m);
  }
}

// Keys at or past the node's end get no weight (t0: the tile's first key).
template <int KH>
__device__ __forceinline__ void mask_tile(STile<KH>& s, int32_t t0, int32_t nk, int32_t lg) {
#pragma unroll
  for (int h = 0; h < KH; ++h)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int qb = 0; qb < 2; ++qb)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (t0 + 32 * h + 8 * lg + 4 * b + r >= nk) s[h][b][qb][r] = -INFINITY;
}

// p = exp2(s) rounded to bf16: pb[h][qb] is the B operand of the PV MFMA for
// the 32-key half h.
template <int KH>
__device__ __forceinline__ void probs(const STile<KH>& s, bf16x8 (&pb)[KH][2]) {
#pragma unroll
  for (int qb = 0; qb < 2; ++qb)
#pragma unroll
    for (int h = 0; h < KH; ++h)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        pb[h][qb][e] = static_cast<__bf16>(__builtin_amdgcn_exp2f(s[h][e >> 2][qb][e & 3]));
}

// p = exp2(unit s): this lane's sums of the unrounded values are added to l.  Rounded
// to bf16 is p only as the operand of PV, which fp32 MFMAs would do at an eighth of the
// rate (154 TFLOP/s against 1234): at most 2^-8 of each p, independent of each other,
// which in the 2-norm adds as much as the output's own rounding (0.0023 from the exact
// output; 0.0017 for fp32 products rounded once), and less where a row's largest p,
// exactly 1, makes most of it.
// (Taking the maximum off here, by an fma, instead of in the products' accumulators
// was 1 % slower.)
template <int KH>
__device__ __forceinline__ void probs_sum(const STile<KH>& s, float unit, bf16x8 (&pb)[KH][2], float (&l)[2]) {
#pragma unroll
  for (int qb = 0; qb < 2; ++qb) {
    float l0 = 0.f, l1 = 0.f;
#pragma unroll
    for (int h = 0; h < KH; ++h)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p = __builtin_amdgcn_exp2f(s[h][e >> 2][qb][e & 3] * unit);
        pb[h][qb][e] = static_cast<__bf16>(p);
        (e & 1 ? l1 : l0) += p;
      }
    l[qb] += l0 + l1;
  }
}

// The same, also returning this lane's sums of the rounded values per block
// (the exact redo path).
template <int KH>
__device__ __forceinline__ void probs_tile(const STile<KH>& s, bf16x8 (&pb)[KH][2], float (&lt)[2]) {
  const bf16x2 ones = {static_cast<__bf16>(1.0f), static_cast<__bf16>(1.0f)};
#pragma unroll
  for (int qb = 0; qb < 2; ++qb) {
    float l0 = 0.f, l1 = 0.f;
#pragma unroll
    for (int h = 0; h < KH; ++h) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        pb[h][qb][e] = static_cast<__bf16>(__builtin_amdgcn_exp2f(s[h][e >> 2][qb][e & 3]));
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        l0 = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pb[h][qb][e], pb[h][qb][e + 1]}, ones, l0, false);
        l1 = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pb[h][qb][e + 2], pb[h][qb][e + 3]}, ones, l1, false);
      }
    }
    lt[qb] = l0 + l1;
  }
}

// Copies of BK-key K and V^T tiles of one (node, head) from the paged cache
// into LDS, split over the NW waves of a work-group.  A tile spans at most
// two pages (pages hold >= BK tokens), so the page of a key is chosen against
// one wave-uniform boundary.
// Offsets are 32-bit, relative to the layer's slots (the host checks that a
// layer fits in 4 GB); the per-page parts are wave-uniform.  A copy
// instruction moves 1 KB: 4 K rows, or RPI = 512 / BK V^T rows of BK / 8
// 16-byte columns.  Each wave issues KCP of the first and VCP of the second
// per tile; lane (row, physical column p) fetches logical column
// p ^ swizzle(row).  K rows of keys past the node's end fetch its last key,
// V^T columns the tile's first key (valid memory; their probabilities are
// zero).
// KEPT: every copy's lane offsets stay in registers, for the plain forms, which have
// room for them (four nodes of 4680 queries over 32760 keys, 12 heads: 2.899 ms so, 2.922
// otherwise).  The exact forms have none to spare and derive them from the first
// copies'.
template <int NW, int KH, bool KEPT>
struct KvTiles {
  static constexpr int BK = Tile<KH>::BK;
  static constexpr int KCP = BK / (4 * NW), VCP = BK / (4 * NW);
  static constexpr int LPR = BK / 8, RPI = 64 / LPR;  // V^T: lanes per row, rows per copy instruction
  static_assert(LPR == 1 << (KH + 1), "V^T lanes per row");
  static_assert(KCP >= 1 && KCP * 4 * NW == BK, "K copy split");
  struct Slots {
    uint32_t lo, hi;  // byte offsets of the slots of the tile's first page and the next one
    int32_t plo;      // index of the tile's first page within the node
  };
  const char* lbase;
  const int32_t* page_slot;  // the node's page slots
  int32_t npages, nk, tpp, wave;
  uint32_t slot_bytes, khead, vhead, kbad;
  DivMagic tpp_div;
  // Lane offsets of the copies.  Both swizzles are XORs of bits of the row, and copy j
  // adds its own bits to rows that have none there: its offset is the first copy's
  // with a constant XORed in, which costs no register.
  uint32_t kl0;      // K: the first row's bytes and the swizzled column
  uint32_t vl[KH];   // V^T: rows of even and odd copies (their swizzles alternate), with the key's bytes
  int32_t vk0;       // key offset in the tile, of even copies
  uint32_t klane[KEPT ? KCP : 1], vlane[KEPT ? VCP : 1];  // KEPT: of every copy
  int32_t vkeys[KEPT ? VCP : 1];

  template <class Plan>
  __device__ __forceinline__ KvTiles(const Plan& plan, const AttnGeom& g, int32_t node, int32_t head,
                                     int32_t wave_, int32_t lane) {
    const int32_t p0 = plan.page_off[node];
    lbase = g.layer_base;
    page_slot = plan.page_slot + p0;
    npages = plan.page_off[node + 1] - p0;
    tpp = g.tpp;
    nk = npages * tpp;
    wave = wave_;
    slot_bytes = (uint32_t)g.slot_bytes;
    tpp_div = g.tpp_div;
    khead = (uint32_t)head * tpp * HDB * 2;
    vhead = (uint32_t)g.kv_half + (uint32_t)head * HDB * tpp * 2;
    kbad = (uint32_t)page_slot[npages - 1] * slot_bytes + khead + (uint32_t)(tpp - 1) * 256;
    const int32_t krow0 = 4 * KCP * wave + (lane >> 4), kp = lane & 15;
    kl0 = (uint32_t)krow0 * 256 + ((kp ^ kswz(krow0)) << 4);  // plus key t0 * 256
    const int32_t vrow0 = RPI * VCP * wave + (lane >> (KH + 1)), vp = lane & (LPR - 1);  // LPR = 2^(KH+1)
    vk0 = 8 * (vp ^ (int32_t)vswz<KH>(vrow0));
#pragma unroll
    for (int j = 0; j < KH; ++j) vl[j] = (uint32_t)vrow0 * tpp * 2 + (uint32_t)vkey(j) * 2;  // plus key t0 * 2
    if constexpr (KEPT) {
#pragma unroll
      for (int j = 0; j < KCP; ++j) {
        const int32_t row = krow0 + 4 * j;
        klane[j] = (uint32_t)row * 256 + ((kp ^ kswz(row)) << 4);
      }
#pragma unroll
      for (int j = 0; j < VCP; ++j) {
        const int32_t d = vrow0 + RPI * j;
        vkeys[j] = 8 * (vp ^ (int32_t)vswz<KH>(d));
        vlane[j] = (uint32_t)d * tpp * 2 + (uint32_t)vkeys[j] * 2;
      }
    }
  }
  __device__ __forceinline__ int32_t vkey(int j) const { return KH == 2 ? vk0 ^ (32 * (j & 1)) : vk0; }
  // Offset of K copy j from that of the first (kl: kl0).
  static __device__ __forceinline__ uint32_t kxor(uint32_t kl, int j) { return kl ^ (kswz(4 * j) << 4); }
  // Page slots of the tile starting at key t0 >= 0 (two scalar loads),
  // fetched ahead of the copy that uses them so their latency overlaps other
  // work (a step, or the barrier wait before the copy).  Clamped to the
  // node's pages: a tile past the end is never read.
  __device__ __forceinline__ Slots slots(int32_t t0) const {
    Slots sl;
    sl.plo = min((int32_t)fast_div((uint32_t)t0, tpp_div), npages - 1);
    const int32_t phi = sl.plo + 1 < npages ? sl.plo + 1 : sl.plo;
    sl.lo = (uint32_t)page_slot[sl.plo] * slot_bytes;
    sl.hi = (uint32_t)page_slot[phi] * slot_bytes;
    return sl;
  }
  // The 4 K rows of one copy instruction are tile rows 4 (KCP wave + j) ..
  // +3; page boundaries and the node's end are multiples of 8 keys, so the
  // page (or the out-of-range fallback) is one wave-uniform choice per
  // instruction.
  __device__ __forceinline__ void copy_k(int32_t t0, char* kl, const Slots& sl) const {
    const int32_t bkey = (sl.plo + 1) * tpp;
    const uint32_t lo = sl.lo + khead + (uint32_t)(t0 - sl.plo * tpp) * 256;
    const uint32_t hi = sl.hi + khead + (uint32_t)(t0 - bkey) * 256;
    const int32_t lim = nk - t0, split = bkey - t0;
    if constexpr (KEPT) {
#pragma unroll
      for (int j = 0; j < KCP; ++j) {
        const int32_t rg = 4 * KCP * wave + 4 * j;  // first tile row of this copy (wave-uniform)
        const uint32_t src = rg >= lim ? kbad + (klane[j] & 255u) : (rg >= split ? hi : lo) + klane[j];
        dma16(lbase, src, kl + rg * 256);
      }
      return;
    }
    uint32_t k = kl0;
    asm volatile("" : "+v"(k));  // the offsets are made here, not kept
#pragma unroll
    for (int j = 0; j < KCP; ++j) {
      const int32_t rg = 4 * KCP * wave + 4 * j;
      const bool past = rg >= lim;
      const uint32_t base = past ? kbad : (rg >= split ? hi : lo) + 1024u * j;
      dma16(lbase, base + (kxor(k, j) & (past ? 255u : ~0u)), kl + rg * 256);
    }
  }
  // A V^T row holds the tile's BK keys; a page boundary or the node's end
  // falls inside the tile for about one tile in a page, so the per-lane
  // choice is taken only then (wave-uniform branch).
  __device__ __forceinline__ void copy_v(int32_t t0, char* vt, const Slots& sl) const {
    const int32_t bkey = (sl.plo + 1) * tpp;
    const uint32_t lo = sl.lo + vhead + (uint32_t)(t0 - sl.plo * tpp) * 2;
    const int32_t lim = nk - t0, split = bkey - t0;
    if (split >= BK && lim >= BK) {
#pragma unroll
      for (int j = 0; j < VCP; ++j) {
        // opaque, so the offset stays one add of the scalar base (the
        // compiler otherwise re-derives it with a per-lane multiply)
        uint32_t off = KEPT ? vlane[KEPT ? j : 0] : vl[j % KH];
        asm volatile("" : "+v"(off));
        dma16(lbase, lo + (KEPT ? 0u : (uint32_t)(RPI * 2 * j) * tpp) + off, vt + (RPI * VCP * wave + RPI * j) * 2 * BK);
      }
      return;
    }
    const uint32_t hi = sl.hi + vhead + (uint32_t)(t0 - bkey) * 2;
#pragma unroll
    for (int j = 0; j < VCP; ++j) {
      const int32_t rk = KEPT ? vkeys[KEPT ? j : 0] : vkey(j);
      const bool in = rk < lim;
      const uint32_t at = KEPT ? vlane[KEPT ? j : 0] : vl[j % KH] + (uint32_t)(RPI * 2 * j) * tpp, off = in ? at : at - (uint32_t)rk * 2;
      const uint32_t base = (in && rk >= split) ? hi : lo;
      dma16(lbase, base + off, vt + (RPI * VCP * wave + RPI * j) * 2 * BK);
    }
  }
};

__device__ __forceinline__ void landed() {  // this wave's copies are in LDS, then everyone's
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

// The same for all but this wave's n most recent vector-memory operations (a
// wave's loads complete in issue order for this counter), n even, at most
// 16 (wave-uniform).  The barrier is issued without __syncthreads' release
// fence, which would wait for every outstanding copy; the memory clobber
// keeps the compiler from moving LDS accesses across it.
__device__ __forceinline__ void landed_but(int32_t n) {
#define SC_LANDED_BUT(k) \
  case k:                \
    asm volatile("s_waitcnt vmcnt(" #k ")\n\ts_barrier" ::: "memory"); \
    break;
  switch (n) {
    SC_LANDED_BUT(2) SC_LANDED_BUT(4) SC_LANDED_BUT(6) SC_LANDED_BUT(8) SC_LANDED_BUT(10)
    SC_LANDED_BUT(12) SC_LANDED_BUT(14) SC_LANDED_BUT(16)
    default: asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory"); break;
  }
#undef SC_LANDED_BUT
}

// Schedule.  A unit is a (head, node, query tile) triple, numbered head-major
// then node then query tile; a unit's key tiles are processed in order by one
// work-group.  The work-groups an XCD runs side by side are then the query
// tiles of one or two nodes of one head, which read the same K/V tiles at
// about the same time and share them in its L2; every node's page list
// starts at the state most nodes of the pack read (see shared_order), so
// two nodes there read their shared states together too.  (With the node
// fastest, four nodes' streams shared an XCD's L2 and it fetched 11 % more.)
// Equal units fill the resident work-groups in whole rounds but the
// last U mod R; those "tail" units are each cut into S pieces of their key
// range, numbered piece-major (piece p of every tail unit before piece p+1),
// so the last round is S times shorter.  Pieces leave unnormalised partials
// that attn_combine_kernel merges in piece order.
template <int KH>
__device__ __forceinline__ int32_t node_tiles(const AttnPlan& plan, const AttnGeom& g, int32_t node) {
  constexpr int BK = Tile<KH>::BK;
  return ((plan.page_off[node + 1] - plan.page_off[node]) * g.tpp + BK - 1) / BK;
}

template <int KH>
__device__ __forceinline__ AttnItem decode_item(const AttnPlan& plan, const AttnGeom& g, uint32_t b) {
  AttnItem it;
  int32_t unit;
  if (b < (uint32_t)g.whole_units) {
    unit = (int32_t)xcd_remap(b, (uint32_t)g.whole_units);
    it.slot = -1;
  } else {
    const int32_t j = (int32_t)xcd_remap(b - (uint32_t)g.whole_units,
                                         (uint32_t)(g.tail_units * g.tail_split));
    unit = g.whole_units + j % g.tail_units;
    it.slot = j;
  }
  it.qt = unit % g.n_qtiles;
  it.node = (unit / g.n_qtiles) % g.n_nodes;
  it.head = unit / (g.n_qtiles * g.n_nodes);
  it.row0 = it.rows = 0;
  it.ntiles = node_tiles<KH>(plan, g, it.node);
  if (it.slot < 0) {
    it.ta = 0;
    it.tb = it.ntiles;
  } else {
    const int32_t piece = it.slot / g.tail_units;
    it.ta = piece * it.ntiles / g.tail_split;
    it.tb = (piece + 1) * it.ntiles / g.tail_split;
  }
  return it;
}

// The result of a work item for one 16-query block: the normalised output
// of a whole unit, or a piece's unnormalised partial with its max and sum.
// oacc[db] holds, in lane (g, c) value r, O[query c][16 db + 4 g + r].
template <int BQ, class M>
__device__ __forceinline__ void store_rows(const AttnItem& it, const typename M::Geom& g, uint16_t* o,
                                           const f32x4 (&oacc)[8], float m_run, float l_run,
                                           int32_t lrow, int32_t lg) {
  const float l_tot = group_sum(l_run);
  if constexpr (M::kShare) {  // every item is a piece: its valid rows' partials
    const int32_t qrow = it.qt * BQ + lrow;
    if (qrow >= it.rows) return;
    const size_t at = ((size_t)it.slot * g.n_heads + it.head) * g.rows + it.row0 + qrow;
    float* po = g.part_o + at * HDB + 4 * lg;
#pragma unroll
    for (int db = 0; db < 8; ++db) *reinterpret_cast<f32x4*>(po + 16 * db) = oacc[db];
    if (lg == 0) {
      g.part_ml[2 * at] = l_tot == 0.f ? -INFINITY : m_run * unit_of<M>(g);
      g.part_ml[2 * at + 1] = l_tot;
    }
    return;
  }
  if (it.slot < 0) {
    const float inv = 1.f / l_tot;
    const int32_t qrow = it.qt * BQ + lrow;
    if (qrow < g.nq) {
      uint16_t* op = o + (((size_t)it.node * g.nq + qrow) * g.n_heads + it.head) * HDB + 4 * lg;
#pragma unroll
      for (int db = 0; db < 8; ++db) {
        u32x2 v;
        v.x = pack_bf16x2(oacc[db][0] * inv, oacc[db][1] * inv);
        v.y = pack_bf16x2(oacc[db][2] * inv, oacc[db][3] * inv);
        *reinterpret_cast<u32x2*>(op + 16 * db) = v;
      }
      if constexpr (M::kLse)
        if (g.lse && lg == 0)
          g.lse[(size_t)it.head * g.rows + (size_t)it.node * g.nq + qrow] = m_run * unit_of<M>(g) + __builtin_amdgcn_logf(l_tot);
    }
  } else {
    float* po = g.part_o + ((size_t)it.slot * BQ + lrow) * HDB + 4 * lg;
#pragma unroll
    for (int db = 0; db < 8; ++db) *reinterpret_cast<f32x4*>(po + 16 * db) = oacc[db];
    if (lg == 0) {
      g.part_ml[((size_t)it.slot * 2 + 0) * BQ + lrow] = !M::kLse ? m_run : l_tot == 0.f ? -INFINITY : m_run * unit_of<M>(g);
      g.part_ml[((size_t)it.slot * 2 + 1) * BQ + lrow] = l_tot;
    }
  }
}

// S^T of one tile, s[h][b][qb] = K_(h,b) Q_qb^T - m_qb: all 4 KH
// accumulators advance together.
template <int KH>
__device__ __forceinline__ void qk_tile(const char* kl, const AttnLane& L, const bf16x8 (&qreg)[2][4],
                                        STile<KH>& s, const float (&m)[2]) {
  f32x4 acc[KH][2][2];
#pragma unroll
  for (int h = 0; h < KH; ++h)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int qb = 0; qb < 2; ++qb)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[h][b][qb][r] = -m[qb];
#pragma unroll
  for (int ds = 0; ds < 4; ++ds)
#pragma unroll
    for (int h = 0; h < KH; ++h)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const bf16x8 a = *reinterpret_cast<const bf16x8*>(kl + L.k(b, ds) + h * 8192);
        acc[h][b][0] = mfma16(a, qreg[0][ds], acc[h][b][0]);
        acc[h][b][1] = mfma16(a, qreg[1][ds], acc[h][b][1]);
      }
#pragma unroll
  for (int h = 0; h < KH; ++h)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int qb = 0; qb < 2; ++qb) s[h][b][qb] = acc[h][b][qb];
}

// O^T += V^T P^T for a tile whose V^T sits at vl.
template <int KH>
__device__ __forceinline__ void pv_tile(const char* vl, const AttnLane& L, const bf16x8 (&pb)[KH][2],
                                        f32x4 (&oacc)[2][8]) {
#pragma unroll
  for (int h = 0; h < KH; ++h)
#pragma unroll
    for (int db = 0; db < 8; ++db) {
      const bf16x8 a = *reinterpret_cast<const bf16x8*>(vl + L.voff[h] + db * (16 * 2 * Tile<KH>::BK));
      oacc[0][db] = mfma16(a, pb[h][0], oacc[0][db]);
      oacc[1][db] = mfma16(a, pb[h][1], oacc[1][db]);
    }
}

// Columns of a V^T tile past the node's end (t0: the tile's first key) hold a real
// token's values, and an infinity there would make 0 x inf: each lane clears
// what it reads.
template <int KH>
__device__ __forceinline__ void clear_past(char* vl, const AttnLane& L, int32_t t0, int32_t nk, int32_t lg) {
#pragma unroll
  for (int h = 0; h < KH; ++h)
    if (t0 + 32 * h + 8 * lg >= nk)
#pragma unroll
      for (int db = 0; db < 8; ++db)
        *reinterpret_cast<u32x4*>(vl + L.voff[h] + db * (16 * 2 * Tile<KH>::BK)) = u32x4{};
}

// One step of the software-pipelined loop, for tile t: probabilities of
// S(t) (held in s), the next tile's S(t+1) = K(t+1) Q^T - m on the matrix
// cores while the exponentials of tile t run on the vector ALUs, then
// O^T += V(t)^T P(t) and the row sums lsum += 1^T P(t).  K runs one tile
// ahead of V: K(t+1) sits in K buffer KN, V(t) in V buffer VC.
// (The forms with logarithmic sums add up the exponentials themselves, in lsum[qb][0].)
template <class M, int KH, int KN, int VC, bool NEXT, bool MASK>
__device__ __forceinline__ void attn_step(char* smem, const AttnLane& L, const bf16x8 (&qreg)[2][4],
                                          f32x4 (&oacc)[2][8], STile<KH>& s, const float (&m)[2],
                                          f32x4 (&lsum)[2], const bf16x8& ones, int32_t t0, int32_t nk,
                                          int32_t lg, float unit) {
  using T = Tile<KH>;
  if constexpr (NEXT && !MASK && KH == 2) {
    // One stream of 32 fragment reads (the 16 K fragments of S(t+1), then
    // the 16 V^T fragments of tile t), each issued PF fragments ahead of the
    // two MFMAs it feeds; the 32 exponentials of P(t) ride two to a K group.
    // The fences keep that order: left to itself the compiler reads each
    // fragment just before its MFMAs, which then wait out the LDS latency.
    constexpr int PF = 4, NKF = 16, NF = 32;
    const char* kl = smem + KN * T::KT_BYTES;
    const char* vl = smem + 2 * T::KT_BYTES + VC * T::VT_BYTES;
    auto frag = [&](int i) -> bf16x8 {
      if (i < NKF) return *reinterpret_cast<const bf16x8*>(kl + L.k(i & 1, i >> 2) + ((i >> 1) & 1) * 8192);
      const int j = i - NKF;
      return *reinterpret_cast<const bf16x8*>(vl + L.voff[j >> 3] + (j & 7) * (16 * 2 * T::BK));
    };
    STile<2> sn;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int qb = 0; qb < 2; ++qb)
#pragma unroll
          for (int r = 0; r < 4; ++r) sn[h][b][qb][r] = -m[qb];
    bf16x8 pb[2][2];
    // the 32 exponentials, those of half 0 first: spread over the K fragments and the
    // V^T fragments before the first that needs half 1
    constexpr int NE = M::kLse ? 24 : 16;
    auto prob = [&](int x) __attribute__((always_inline)) {
      const int ph = x >> 4, pq = (x >> 3) & 1, pe = x & 7;
      if constexpr (M::kLse) {
        const float p = __builtin_amdgcn_exp2f(s[ph][pe >> 2][pq][pe & 3] * unit);
        pb[ph][pq][pe] = static_cast<__bf16>(p);
        lsum[pq][0] += p;
      } else {
        pb[ph][pq][pe] = static_cast<__bf16>(__builtin_amdgcn_exp2f(s[ph][pe >> 2][pq][pe & 3]));
      }
    };
    bf16x8 ring[PF];
#pragma unroll
    for (int i = 0; i < PF; ++i) ring[i] = frag(i);
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      const bf16x8 f = ring[i % PF];
      if (i + PF < NF) ring[i % PF] = frag(i + PF);
      if (i < NKF) {  // K fragment (ds, h, b) = (i / 4, i / 2 mod 2, i mod 2), as in qk_tile
        const int ds = i >> 2, h = (i >> 1) & 1, b = i & 1;
        sn[h][b][0] = mfma16(f, qreg[0][ds], sn[h][b][0]);
        sn[h][b][1] = mfma16(f, qreg[1][ds], sn[h][b][1]);
      } else {  // V^T fragment (h, db) = (j / 8, j mod 8), as in pv_tile
        const int j = i - NKF, h = j >> 3, db = j & 7;
        oacc[0][db] = mfma16(f, pb[h][0], oacc[0][db]);
        oacc[1][db] = mfma16(f, pb[h][1], oacc[1][db]);
      }
      if (i < NE) {
#pragma unroll
        for (int x = i * 32 / NE; x < (i + 1) * 32 / NE; ++x) prob(x);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (!M::kLse)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        lsum[0] = mfma16(ones, pb[h][0], lsum[0]);
        lsum[1] = mfma16(ones, pb[h][1], lsum[1]);
      }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) s[h][b][qb] = sn[h][b][qb];
    return;
  }
  if constexpr (MASK) mask_tile<KH>(s, t0, nk, lg);
  bf16x8 pb[KH][2];
  if constexpr (M::kLse) {
    float l[2] = {lsum[0][0], lsum[1][0]};
    probs_sum<KH>(s, unit, pb, l);
    lsum[0][0] = l[0];
    lsum[1][0] = l[1];
  } else {
    probs<KH>(s, pb);
  }
  STile<KH> sn;
  if constexpr (NEXT) qk_tile<KH>(smem + KN * T::KT_BYTES, L, qreg, sn, m);
  if constexpr (M::kLse && MASK) clear_past<KH>(smem + 2 * T::KT_BYTES + VC * T::VT_BYTES, L, t0, nk, lg);
  pv_tile<KH>(smem + 2 * T::KT_BYTES + VC * T::VT_BYTES, L, pb, oacc);
  if constexpr (!M::kLse)
#pragma unroll
    for (int h = 0; h < KH; ++h) {
      lsum[0] = mfma16(ones, pb[h][0], lsum[0]);
      lsum[1] = mfma16(ones, pb[h][1], lsum[1]);
    }
  if constexpr (NEXT) {
#pragma unroll
    for (int h = 0; h < KH; ++h)
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) s[h][b][qb] = sn[h][b][qb];
  }
}

// Exact two-pass redo of a work item in which a wave reached the 2^64 guard:
// each query's maximum logit over the item's keys, then the softmax from
// that maximum (every p <= 1).  Single-buffered K and V tiles; slow, and
// taken only for logits far above the first tile's maximum.
template <class M, int NW, int KH>
__device__ __forceinline__ void attn_exact(char* smem, const KvTiles<NW, KH, !M::kLse>& kv, const AttnLane& L,
                                           const bf16x8 (&qreg)[2][4], f32x4 (&oacc)[2][8], float (&m)[2],
                                           float (&l)[2], int32_t ta, int32_t ntiles, int32_t lg, float unit) {
  constexpr int BK = Tile<KH>::BK;
  char* const kl = smem;
  char* const vl = smem + 2 * Tile<KH>::KT_BYTES;
  const int32_t nk = kv.nk;
  const float zero[2] = {0.f, 0.f};
  float mx[2] = {-INFINITY, -INFINITY};
  for (int32_t t = ta; t < ntiles; ++t) {
    kv.copy_k(t * BK, kl, kv.slots(t * BK));
    landed();
    STile<KH> s;
    qk_tile<KH>(kl, L, qreg, s, zero);
    mask_tile<KH>(s, t * BK, nk, lg);
    float tm[2];
    tile_max<KH>(s, tm);
    mx[0] = fmaxf(mx[0], tm[0]);
    mx[1] = fmaxf(mx[1], tm[1]);
    __syncthreads();
  }
#pragma unroll
  for (int qb = 0; qb < 2; ++qb) {
    // a piece without a finite logit adds zeros to its row (LseAttn, ShareAttn)
    m[qb] = M::kLse && mx[qb] == -INFINITY ? 0.f : mx[qb];
    l[qb] = 0.f;
#pragma unroll
    for (int db = 0; db < 8; ++db) oacc[qb][db] = f32x4{};
  }
  for (int32_t t = ta; t < ntiles; ++t) {
    const typename KvTiles<NW, KH, !M::kLse>::Slots sl = kv.slots(t * BK);
    kv.copy_k(t * BK, kl, sl);
    kv.copy_v(t * BK, vl, sl);
    landed();
    STile<KH> s;
    qk_tile<KH>(kl, L, qreg, s, m);
    mask_tile<KH>(s, t * BK, nk, lg);
    bf16x8 pb[KH][2];
    if constexpr (M::kLse) {
      probs_sum<KH>(s, unit, pb, l);
      if (nk < (t + 1) * BK) clear_past<KH>(vl, L, t * BK, nk, lg);
    } else {
      float lt[2];
      probs_tile<KH>(s, pb, lt);
      l[0] += lt[0];
      l[1] += lt[1];
    }
    pv_tile<KH>(vl, L, pb, oacc);
    __syncthreads();
  }
}

// NW = 8: 256 queries per work-group, one work-group per CU; NW = 4: 128
// queries, two per CU; NW = 2: 64 queries, three or two per CU.  Each wave
// owns two 16-query blocks.  KH: 32-key halves per key tile; D: tiles of the
// K and of the V^T ring.  The long-context form (KH = 2, D = 2; NW = 8, 4)
// keeps one tile in flight, its buffer parity unrolled, two waves per SIMD.
// The streaming form (KH = 1, D = 3 or 4: runtime ring slots, D - 1 tiles in
// flight; NW = 2) serves nodes of at most 64 queries, whose attention
// streams K/V from HBM: it trades resident waves for copies in flight.
template <int NW, int KH, int D, class M = PlainAttn>
__global__ __launch_bounds__(64 * NW, NW == 8 || D == 4 ? 1 : 2) void attn_bf16_kernel(const uint16_t* __restrict__ q,
                                                                    uint16_t* __restrict__ o, typename M::Geom g,
                                                                    typename M::Plan plan) {
  constexpr int BQ = 32 * NW;
  using T = Tile<KH>;
  constexpr int BK = T::BK, KT_BYTES = T::KT_BYTES, VT_BYTES = T::VT_BYTES;
  static_assert((D == 2 && KH == 2) || (KH == 1 && (D == 3 || D == 4)), "ring depth");
  // K buffers 0 .. D-1 then V^T buffers 0 .. D-1 (KT_BYTES, VT_BYTES each)
  __shared__ __attribute__((aligned(1024))) char smem[D * (KT_BYTES + VT_BYTES)];
  __shared__ int32_t any_bad;
  AttnItem it = decode_item<KH>(plan, g, blockIdx.x);
  if constexpr (M::kLse) in_scalars(it);
  if (it.ta == it.tb) return;  // empty piece of a unit shorter than the split
  const int32_t ta = it.ta, ntiles = it.tb;  // this item's key tiles: [ta, ntiles)
  const int32_t tid = threadIdx.x, lane = tid & 63;
  const int32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6);  // wave-uniform: LDS copy addresses stay scalar
  const int32_t lg = lane >> 4, c = lane & 15;
  if (tid == 0) any_bad = 0;
  const KvTiles<NW, KH, !M::kLse> kv(plan, g, it.node, it.head, wave, lane);
  const int32_t nk = kv.nk;
  const bool ragged = it.tb == it.ntiles && (nk % BK) != 0;
  bf16x8 qreg[2][4];
  const AttnLane L = attn_lane<KH>(c, lg);

  f32x4 oacc[2][8];
#pragma unroll
  for (int qb = 0; qb < 2; ++qb)
#pragma unroll
    for (int db = 0; db < 8; ++db) oacc[qb][db] = f32x4{};
  float m[2] = {0.f, 0.f}, l[2];
  f32x4 lsum[2] = {f32x4{}, f32x4{}};  // value 0 of lanes 0..15: row sums of the two blocks
  const bf16x8 ones = ones_row(c);
  // A wave whose 32 queries all lie past the node's end (in a node's last
  // query tile) still copies its share of every tile and meets every
  // barrier, but skips the matrix and softmax work.
  const size_t row0 = item_row0<M>(it, g);
  const int32_t rows = item_rows<M>(it, g);
  const bool active = it.qt * BQ + wave * 32 < rows;
  STile<KH> s;
  auto run = [&](auto act) __attribute__((always_inline)) {
    constexpr bool ACT = decltype(act)::value;
    // prologue: K(ta), V(ta), K(ta+1) in flight; S(ta) = K(ta) Q^T; m = its exact column maxima
    {
      const typename KvTiles<NW, KH, !M::kLse>::Slots s0 = kv.slots(ta * BK);
      kv.copy_k(ta * BK, smem, s0);
      kv.copy_v(ta * BK, smem + 2 * KT_BYTES, s0);
      if (ta + 1 < ntiles) kv.copy_k((ta + 1) * BK, smem + KT_BYTES, kv.slots((ta + 1) * BK));
    }
#pragma unroll
    for (int qb = 0; qb < 2; ++qb)
      load_q(q, g, row0, rows, it.head, it.qt * BQ + wave * 32 + 16 * qb + c, lg, qreg[qb]);
    landed();
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) scale_q<M>(g, qreg[qb]);
    if constexpr (ACT) {
      qk_tile<KH>(smem, L, qreg, s, m);
      if (ta + 1 == ntiles && ragged) mask_tile<KH>(s, ta * BK, nk, lg);
      tile_max<KH>(s, m);
#pragma unroll
      for (int h = 0; h < KH; ++h)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int qb = 0; qb < 2; ++qb)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[h][b][qb][r] -= m[qb];
    }
    __syncthreads();  // every wave has read K(ta) before K(ta+2) is copied over it

    // iteration t (buffer parity counted from ta): copy K(t+2) over K(t) and
    // V(t+1) over V(t-1), then step t
    int32_t t = ta;
    typename KvTiles<NW, KH, !M::kLse>::Slots sk = kv.slots(min(ta + 2, it.ntiles - 1) * BK);
    typename KvTiles<NW, KH, !M::kLse>::Slots sv = kv.slots(min(ta + 1, it.ntiles - 1) * BK);
    for (; t + 2 < ntiles; t += 2) {
      kv.copy_k((t + 2) * BK, smem, sk);
      kv.copy_v((t + 1) * BK, smem + 2 * KT_BYTES + VT_BYTES, sv);
      if constexpr (ACT) attn_step<M, KH, 1, 0, true, false>(smem, L, qreg, oacc, s, m, lsum, ones, t * BK, nk, lg, unit_of<M>(g));
      // the next copies' page slots: their scalar loads share the LDS wait
      // counter, so they are issued after the step's fragment reads (a wait
      // for one fragment would otherwise wait for them too)
      __builtin_amdgcn_sched_barrier(0);
      sk = kv.slots(min(t + 3, it.ntiles - 1) * BK);
      sv = kv.slots(min(t + 2, it.ntiles - 1) * BK);
      landed();
      if (t + 3 < ntiles) kv.copy_k((t + 3) * BK, smem + KT_BYTES, sk);
      kv.copy_v((t + 2) * BK, smem + 2 * KT_BYTES, sv);
      if constexpr (ACT)
        attn_step<M, KH, 0, 1, true, false>(smem, L, qreg, oacc, s, m, lsum, ones, (t + 1) * BK, nk, lg, unit_of<M>(g));
      __builtin_amdgcn_sched_barrier(0);
      sk = kv.slots(min(t + 4, it.ntiles - 1) * BK);
      sv = kv.slots(min(t + 3, it.ntiles - 1) * BK);
      landed();
    }
    if (t + 1 < ntiles) {  // two tiles left, parity 0
      kv.copy_v((t + 1) * BK, smem + 2 * KT_BYTES + VT_BYTES, sv);
      if constexpr (ACT) attn_step<M, KH, 1, 0, true, false>(smem, L, qreg, oacc, s, m, lsum, ones, t * BK, nk, lg, unit_of<M>(g));
      landed();
      ++t;
      if constexpr (ACT) {
        if (ragged)
          attn_step<M, KH, 0, 1, false, true>(smem, L, qreg, oacc, s, m, lsum, ones, t * BK, nk, lg, unit_of<M>(g));
        else
          attn_step<M, KH, 0, 1, false, false>(smem, L, qreg, oacc, s, m, lsum, ones, t * BK, nk, lg, unit_of<M>(g));
      }
    } else if constexpr (ACT) {  // one tile left, parity 0 (masking twice is harmless)
      if (ragged)
        attn_step<M, KH, 1, 0, false, true>(smem, L, qreg, oacc, s, m, lsum, ones, t * BK, nk, lg, unit_of<M>(g));
      else
        attn_step<M, KH, 1, 0, false, false>(smem, L, qreg, oacc, s, m, lsum, ones, t * BK, nk, lg, unit_of<M>(g));
    }
  };
  auto weights_of = [&](bf16x8 (&pb)[KH][2]) __attribute__((always_inline)) {
    if constexpr (M::kLse) {
      float ls[2] = {lsum[0][0], lsum[1][0]};
      probs_sum<KH>(s, g.unit, pb, ls);
      lsum[0][0] = ls[0];
      lsum[1][0] = ls[1];
    } else {
      probs<KH>(s, pb);
    }
  };
  auto row_sums = [&](const bf16x8 (&pb)[KH][2]) __attribute__((always_inline)) {
    if constexpr (!M::kLse)
#pragma unroll
      for (int h = 0; h < KH; ++h) {
        lsum[0] = mfma16(ones, pb[h][0], lsum[0]);
        lsum[1] = mfma16(ones, pb[h][1], lsum[1]);
      }
  };
  // The ring form: tile r of the item (key tile ta + r) sits in K slot and
  // V^T slot r mod D.  Copies are issued in pairs (V(j), K(j + 1)), j = 1,
  // 2, ...: pairs up to D - 2 in the prologue, pair r + D - 1 at step r into
  // the slots steps r - 1 (V) and r - 1 (K, read by the QK of step r - 1)
  // have finished with.  After step r, tiles K(r + 2) and V(r + 1) (pair
  // r + 1) must have landed: the wait leaves the copies of the later pairs
  // in flight, counted exactly (a pair past the item's end issues nothing).
  auto run_ring = [&](auto act) __attribute__((always_inline)) {
    constexpr bool ACT = decltype(act)::value;
    using KV = KvTiles<NW, KH, !M::kLse>;
    constexpr int32_t KC = KV::KCP, VC = KV::VCP;
    static_assert(KC % 2 == 0 && VC % 2 == 0 && (D - 2) * (KC + VC) <= 16, "wait counts of landed_but");
    const int32_t n = ntiles - ta;
    auto kbuf = [&](int32_t r) { return smem + (r % D) * KT_BYTES; };
    auto vbuf = [&](int32_t r) { return smem + D * KT_BYTES + (r % D) * VT_BYTES; };
    // copies of pair j (relative tiles); returns nothing, issues V(j) if it
    // exists, then K(j + 1) if it exists
    auto issue_pair = [&](int32_t j) __attribute__((always_inline)) {
      if (j < n) kv.copy_v((ta + j) * BK, vbuf(j), kv.slots((ta + j) * BK));
      if (j + 1 < n) kv.copy_k((ta + j + 1) * BK, kbuf(j + 1), kv.slots((ta + j + 1) * BK));
    };
    // copy instructions of pairs a .. b issued by this wave: V(j) for j < n,
    // K(j + 1) for j < n - 1
    auto copies = [&](int32_t a, int32_t b) {
      return VC * max(0, min(b, n - 1) - a + 1) + KC * max(0, min(b, n - 2) - a + 1);
    };
    {
      const typename KV::Slots s0 = kv.slots(ta * BK);
      kv.copy_k(ta * BK, kbuf(0), s0);
      kv.copy_v(ta * BK, vbuf(0), s0);
      if (n > 1) kv.copy_k((ta + 1) * BK, kbuf(1), kv.slots((ta + 1) * BK));
    }
    if constexpr (ACT) {
#pragma unroll
      for (int qb = 0; qb < 2; ++qb)
        load_q(q, g, row0, rows, it.head, it.qt * BQ + wave * 32 + 16 * qb + c, lg, qreg[qb]);
    }
    landed();
    for (int32_t j = 1; j <= D - 2; ++j) issue_pair(j);
    if constexpr (ACT) {
#pragma unroll
      for (int qb = 0; qb < 2; ++qb) scale_q<M>(g, qreg[qb]);
      qk_tile<KH>(kbuf(0), L, qreg, s, m);
      if (n == 1 && ragged) mask_tile<KH>(s, ta * BK, nk, lg);
      tile_max<KH>(s, m);
#pragma unroll
      for (int qb = 0; qb < 2; ++qb)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[0][b][qb][r] -= m[qb];
    } else {
#pragma unroll
      for (int qb = 0; qb < 2; ++qb)
#pragma unroll
        for (int ds = 0; ds < 4; ++ds) qreg[qb][ds] = bf16x8{};  // defined values for the exact redo
    }
    landed_but(copies(1, D - 2));  // K(ta) read by every wave before pair D - 1 overwrites its slot
    for (int32_t r = 0; r + 1 < n; ++r) {
      issue_pair(r + D - 1);
      if constexpr (ACT) {
        // step r with runtime slots: the same arithmetic as attn_step
        bf16x8 pb[KH][2];
        weights_of(pb);
        STile<KH> sn;
        qk_tile<KH>(kbuf(r + 1), L, qreg, sn, m);
        if (r + 2 == n && ragged) mask_tile<KH>(sn, (ta + r + 1) * BK, nk, lg);
        pv_tile<KH>(vbuf(r), L, pb, oacc);
        row_sums(pb);
#pragma unroll
        for (int h = 0; h < KH; ++h)
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int qb = 0; qb < 2; ++qb) s[h][b][qb] = sn[h][b][qb];
      }
      landed_but(copies(r + 2, r + D - 1));
    }
    if constexpr (ACT) {  // the last tile (already masked if ragged)
      bf16x8 pb[KH][2];
      weights_of(pb);
      if constexpr (M::kLse)
        if (ragged) clear_past<KH>(vbuf(n - 1), L, (ntiles - 1) * BK, nk, lg);
      pv_tile<KH>(vbuf(n - 1), L, pb, oacc);
      row_sums(pb);
    }
  };
  if constexpr (D == 2) {
    if (active)
      run(std::true_type{});
    else
      run(std::false_type{});
  } else {
    if (active)
      run_ring(std::true_type{});
    else
      run_ring(std::false_type{});
  }
  // the guard, on the final sums (also NaN / inf)
  const bool bad = __builtin_amdgcn_ballot_w64(!(lsum[0][0] < P_GUARD && lsum[1][0] < P_GUARD)) != 0;
  l[0] = lsum[0][0];  // zero outside lanes 0..15, so the group sum is the row sum
  l[1] = lsum[1][0];
  if (bad && lane == 0) atomicOr(&any_bad, 1);
  __syncthreads();  // every wave is done with the ring; any_bad is final
  if (any_bad) attn_exact<M>(smem, kv, L, qreg, oacc, m, l, ta, ntiles, lg, unit_of<M>(g));
#pragma unroll
  for (int qb = 0; qb < 2; ++qb) store_rows<BQ, M>(it, g, o, oacc[qb], m[qb], l[qb], wave * 32 + 16 * qb + c, lg);
}

// ------------------------------------------------ bf16 kernel, keys over waves
// For launches whose 64 .. 256-query units would leave most CUs idle.  A
// work-group takes 32 queries of one (node, head); its eight waves take eight
// contiguous parts of the node's 32-key tiles, each through an LDS region of its
// own with an online softmax of its own, and merge through LDS at the end, in
// wave order: no barrier in the loop, no partials in memory, no combine launch.
// K(t + 1) is copied over K(t) once S(t) has read it and V(t + 1) over V(t)
// likewise, so about a tile is in flight per wave, 64 - 128 KB per CU.
// What bounds it: the copies (128 KB per CU and step of 256 keys, 1.7 us) and a
// fixed 7 us of launch, first tile and merge.  One node of 64 queries over 1344
// keys, 12 heads: 17 us (43 on one 64-query unit per head); 4 x 128 over 896:
// 15 us (21); 128 over 512: 10.5 us (14.7).  The same with the operands loaded
// to registers took 25 us for the first: adjacent lanes hold adjacent rows, so
// each 16-byte load is a cache access of its own.
constexpr int WV_NW = 8, WV_BQ = 32, WV_BK = 32;
constexpr int WV_RED = 8 * WV_NW * 2 * 64 * 16;  // merge: [16-channel block][wave][query block][lane] f32x4
static_assert(WV_NW * (Tile<1>::KT_BYTES + Tile<1>::VT_BYTES) <= WV_RED, "the waves' tiles fit the merge buffer");

// A tile of one wave's own: the copies of KvTiles<1, 1>, four to an M0 setting.
// (The biased offsets stay below 2^32: a group's first rows lie at least
// kCopyBias bytes before the end of the slot.)
struct WaveTiles : KvTiles<1, 1, false> {
  using Base = KvTiles<1, 1, false>;
  const char* biased;
  template <class Plan>
  __device__ __forceinline__ WaveTiles(const Plan& plan, const AttnGeom& g, int32_t node, int32_t head,
                                       int32_t lane)
      : Base(plan, g, node, head, 0, lane), biased(lbase - kCopyBias) {}
  __device__ __forceinline__ void copy_k(int32_t t0, uint32_t lds, const Slots& sl) const {
    const int32_t bkey = (sl.plo + 1) * tpp;
    const uint32_t lo = sl.lo + khead + (uint32_t)(t0 - sl.plo * tpp) * 256;
    const uint32_t hi = sl.hi + khead + (uint32_t)(t0 - bkey) * 256;
    const int32_t lim = nk - t0, split = bkey - t0;
#pragma unroll
    for (int h = 0; h < KCP / 4; ++h) {
      uint32_t off[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int32_t rg = 16 * h + 4 * j;
        const uint32_t k = kxor(kl0, 4 * h + j);
        off[j] = (rg >= lim ? kbad + (k & 255u) : (rg >= split ? hi : lo) + 1024u * (4 * h + j) + k) +
                 (kCopyBias - 1024 * j);
      }
      copy_group<4>(biased, off, lds + 4096 * h);
    }
  }
  __device__ __forceinline__ void copy_v(int32_t t0, uint32_t lds, const Slots& sl) const {
    const int32_t bkey = (sl.plo + 1) * tpp;
    const uint32_t lo = sl.lo + vhead + (uint32_t)(t0 - sl.plo * tpp) * 2;
    const uint32_t hi = sl.hi + vhead + (uint32_t)(t0 - bkey) * 2;
    const int32_t lim = nk - t0, split = bkey - t0;
#pragma unroll
    for (int h = 0; h < VCP / 4; ++h) {
      uint32_t off[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int32_t rk = vkey(4 * h + j);
        const bool in = rk < lim;
        off[j] = (in && rk >= split ? hi : lo) + vl[0] + (uint32_t)(RPI * 2 * (4 * h + j)) * tpp - (in ? 0u : (uint32_t)rk * 2) +
                 (kCopyBias - 1024 * j);
      }
      copy_group<4>(biased, off, lds + 4096 * h);
    }
  }
};

// Ranges that the work-groups past the attention's own read and drop (ReadAhead).
// A few dozen of these work-groups take 10 - 18 us and leave most CUs without
// one, while the launches after them wait for weights from HBM: blocks whose
// weights were read last 450 MB ago, 128 tokens with a condition 122.7 -> 111.4
// us, 256 tokens 99.6 -> 91.9, a four-layer stream 2.81 -> 2.71 ms.  It costs 1 us
// where the weights lie in the memory-side cache already (one block called over
// and over: 81.0 -> 81.9).  5 MB per us of the attention's time but its first 3
// us: 4 or 6 MB per us measured within 1 us, 2 MB 2 - 4 us slower.
constexpr double kAheadBytesPerUs = 5.0e6, kAheadLostUs = 3.0;
struct AttnAhead {
  const char* p[ReadAhead::kMax];
  uint32_t vecs[ReadAhead::kMax];  // 16-byte vectors
  int32_t n, units;                // work-groups of the attention itself
};

// Two loads of a thread in flight, 16 KB per work-group: enough for the rate
// above.  Eight crowd the attention's own copies out (256 tokens 94.0 us against
// 91.9, and 84.2 against 81.9 with the weights in the cache already).
__device__ __forceinline__ void read_ahead(const AttnAhead& a) {
  const uint32_t threads = (gridDim.x - (uint32_t)a.units) * (64 * WV_NW);
  const uint32_t first = (blockIdx.x - (uint32_t)a.units) * (64 * WV_NW) + threadIdx.x;
  for (int32_t r = 0; r < a.n; ++r) {
    const u32x4u* p = reinterpret_cast<const u32x4u*>(a.p[r]);
    const uint32_t n = a.vecs[r];
    for (uint32_t i = first; i < n; i += 2 * threads) {
      const u32x4 a = p[i], b = p[min(i + threads, n - 1)];
      asm volatile("" ::"v"(a), "v"(b));
    }
  }
}

struct NoAhead {};

// Ahead: AttnAhead, or NoAhead where nothing is to be read.
template <class Ahead, class M = PlainAttn>
__global__ __launch_bounds__(64 * WV_NW, 2) void attn_waves_kernel(const uint16_t* __restrict__ q,
                                                                   uint16_t* __restrict__ o, typename M::Geom g,
                                                                   typename M::Plan plan, Ahead ahead) {
  uint32_t units = gridDim.x;
  if constexpr (std::is_same_v<Ahead, AttnAhead>) {
    units = (uint32_t)ahead.units;
    if (blockIdx.x >= units) {
      read_ahead(ahead);
      return;
    }
  }
  __shared__ __attribute__((aligned(1024))) char smem[WV_RED];
  __shared__ float ml[2][WV_NW][WV_BQ];
  using KV = WaveTiles;
  constexpr int KC = KV::KCP, VC = KV::VCP;  // copies of a K and of a V^T tile
  const int32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t lg = lane >> 4, c = lane & 15;
  AttnItem it;
  bool alone = false;  // this wave has the item to itself
  if constexpr (M::kShare) {
    const uint32_t n0 = (uint32_t)(g.p_pieces * g.p_qtiles * g.n_heads);
    alone = g.own_waves && blockIdx.x >= n0;
    if (alone) {
      // own pages of a few tiles: nodes fastest within a head, so that the rows of q
      // and the partials of a work-group's waves lie side by side
      const int32_t i = (int32_t)(blockIdx.x - n0) * WV_NW + wave, per = g.n_nodes * g.n_qtiles;
      if (i >= per * g.n_heads) return;
      it.head = i / per;
      it.node = 1 + i % per / g.n_qtiles;
      it.qt = i % g.n_qtiles;
      it.row0 = (it.node - 1) * g.nq;
      it.rows = g.nq;
      it.slot = g.p_pieces;
      it.ta = 0;
      it.tb = share_tiles<1>(plan, g, it.node);
    } else {
      it = decode_item<1>(plan, g, blockIdx.x);
      if (it.ta == it.tb) return;
    }
  } else {
    // query tiles fastest: an XCD's work-groups share the K/V of a few (node, head)s
    const int32_t unit = (int32_t)xcd_remap(blockIdx.x, units);
    it.qt = unit % g.n_qtiles;
    const int32_t nh = unit / g.n_qtiles;
    it.node = nh % g.n_nodes;
    it.head = nh / g.n_nodes;
    it.slot = -1;
  }
  const int32_t qt = it.qt, head = it.head;
  const size_t row0 = item_row0<M>(it, g);
  const int32_t rows = item_rows<M>(it, g);
  const KV kv(plan, g, it.node, head, lane);
  int32_t nt = (kv.nk + WV_BK - 1) / WV_BK, tile0 = 0;
  if constexpr (M::kShare) {
    tile0 = it.ta;
    nt = it.tb - it.ta;
  }
  const int32_t t_end = alone ? nt : tile0 + (wave + 1) * nt / WV_NW;
  int32_t t = alone ? 0 : tile0 + wave * nt / WV_NW;
  char* const kl = smem + wave * (Tile<1>::KT_BYTES + Tile<1>::VT_BYTES);
  char* const vl = kl + Tile<1>::KT_BYTES;
  const uint32_t kd = __builtin_amdgcn_readfirstlane(lds_addr(kl)), vd = kd + Tile<1>::KT_BYTES;  // for the copies
  const AttnLane L = attn_lane<1>(c, lg);
  bf16x8 qreg[2][4];
#pragma unroll
  for (int qb = 0; qb < 2; ++qb) load_q(q, g, row0, rows, head, qt * WV_BQ + 16 * qb + c, lg, qreg[qb]);
  if (t < t_end) {
    const KV::Slots sl = kv.slots(t * WV_BK);
    kv.copy_k(t * WV_BK, kd, sl);
    kv.copy_v(t * WV_BK, vd, sl);
  }
#pragma unroll
  for (int qb = 0; qb < 2; ++qb) scale_q<M>(g, qreg[qb]);
  f32x4 oacc[2][8], lsum[2] = {f32x4{}, f32x4{}};
#pragma unroll
  for (int qb = 0; qb < 2; ++qb)
#pragma unroll
    for (int db = 0; db < 8; ++db) oacc[qb][db] = f32x4{};
  // m: the maximum logit so far (log2 units), the base of the exponents; lim:
  // what a tile's maximum above m has to exceed to raise it (-inf before the
  // first finite one)
  float m[2] = {0.f, 0.f}, lim[2] = {-INFINITY, -INFINITY};
  const bf16x8 ones = ones_row(c);
  while (t < t_end) {
    const int32_t t0 = t * WV_BK, tn = t0 + WV_BK;
    const bool more = t + 1 < t_end;
    const KV::Slots sl = kv.slots(min(tn, kv.nk - 1));
    copies_landed<VC>();  // K(t); V(t) may still be under way
    STile<1> s;
    qk_tile<1>(kl, L, qreg, s, m);
    reads_done();
    if (more) kv.copy_k(tn, kd, sl);
    if (kv.nk < tn) mask_tile<1>(s, t0, kv.nk, lg);
    float mx[2];
    tile_max<1>(s, mx);
    if (__builtin_amdgcn_ballot_w64(mx[0] > lim[0] || mx[1] > lim[1])) {
#pragma unroll
      for (int qb = 0; qb < 2; ++qb) {
        const bool up = mx[qb] > lim[qb];
        const float d = up ? mx[qb] : 0.f;
        const float alpha =
            lim[qb] == 0.f ? __builtin_amdgcn_exp2f(-d * unit_of<M>(g)) : 1.f;  // nothing to scale before the first
        m[qb] += d;
        lim[qb] = up ? 0.f : lim[qb];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[0][b][qb][r] -= d;
        lsum[qb] *= alpha;
#pragma unroll
        for (int db = 0; db < 8; ++db) oacc[qb][db] *= alpha;
      }
    }
    bf16x8 pb[1][2];
    if constexpr (M::kLse) {
      float ls[2] = {lsum[0][0], lsum[1][0]};
      probs_sum<1>(s, g.unit, pb, ls);
      lsum[0][0] = ls[0];
      lsum[1][0] = ls[1];
    } else {
      probs<1>(s, pb);
    }
    if (more) {
      copies_landed<KC>();  // V(t); K(t + 1) may still be under way
    } else {
      copies_landed<0>();
      if (kv.nk < tn) clear_past<1>(vl, L, t0, kv.nk, lg);
    }
    pv_tile<1>(vl, L, pb, oacc);
    if constexpr (!M::kLse)
#pragma unroll
      for (int qb = 0; qb < 2; ++qb) lsum[qb] = mfma16(ones, pb[0][qb], lsum[qb]);
    reads_done();
    if (more) kv.copy_v(tn, vd, sl);
    ++t;
  }
  // merge: a wave without a finite logit adds zeros (weight 2^-inf)
  if constexpr (M::kLse)
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
      lsum[qb][0] = group_sum(lsum[qb][0]);
      m[qb] *= g.unit;  // in log2 units from here on
    }
  if constexpr (M::kShare)
    if (alone) {
#pragma unroll
      for (int qb = 0; qb < 2; ++qb) {
        const int32_t row = qt * WV_BQ + 16 * qb + c;
        if (row >= rows) continue;
        const size_t at = ((size_t)it.slot * g.n_heads + head) * g.rows + row0 + row;
#pragma unroll
        for (int db = 0; db < 8; ++db) *reinterpret_cast<f32x4*>(g.part_o + at * HDB + 16 * db + 4 * lg) = oacc[qb][db];
        if (lg == 0) {
          g.part_ml[2 * at] = lim[qb] == 0.f ? m[qb] : -INFINITY;
          g.part_ml[2 * at + 1] = lsum[qb][0];
        }
      }
      return;
    }
  if (lg == 0)
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
      ml[0][wave][16 * qb + c] = lim[qb] == 0.f ? m[qb] : -INFINITY;
      ml[1][wave][16 * qb + c] = lsum[qb][0];
    }
  __syncthreads();  // every wave is done with its tiles
  f32x4* const red = reinterpret_cast<f32x4*>(smem);
  float inv[2], mrow[2], lrow[2];
#pragma unroll
  for (int qb = 0; qb < 2; ++qb) {
    float mt = -INFINITY, lt = 0.f;
#pragma unroll
    for (int w = 0; w < WV_NW; ++w) mt = fmaxf(mt, ml[0][w][16 * qb + c]);
    const float base = M::kShare && mt == -INFINITY ? 0.f : mt;
#pragma unroll
    for (int w = 0; w < WV_NW; ++w) lt += ml[1][w][16 * qb + c] * __builtin_amdgcn_exp2f(ml[0][w][16 * qb + c] - base);
    inv[qb] = 1.f / lt;
    mrow[qb] = mt;
    lrow[qb] = lt;
    const float f = __builtin_amdgcn_exp2f(ml[0][wave][16 * qb + c] - base);
#pragma unroll
    for (int db = 0; db < 8; ++db) red[((db * WV_NW + wave) * 2 + qb) * 64 + lane] = oacc[qb][db] * f;
  }
  __syncthreads();
  // wave w finishes channels 16 w .. 16 w + 15
#pragma unroll
  for (int qb = 0; qb < 2; ++qb) {
    f32x4 a = red[(wave * WV_NW * 2 + qb) * 64 + lane];
#pragma unroll
    for (int w = 1; w < WV_NW; ++w) a += red[((wave * WV_NW + w) * 2 + qb) * 64 + lane];
    const int32_t row = qt * WV_BQ + 16 * qb + c;
    if constexpr (M::kShare) {
      if (row < rows) {
        const size_t at = ((size_t)it.slot * g.n_heads + head) * g.rows + row0 + row;
        *reinterpret_cast<f32x4*>(g.part_o + at * HDB + 16 * wave + 4 * lg) = a;
        if (wave == 0 && lg == 0) {
          g.part_ml[2 * at] = mrow[qb];
          g.part_ml[2 * at + 1] = lrow[qb];
        }
      }
      continue;
    }
    if (row < rows) {
      if constexpr (M::kLse)
        if (g.lse && wave == 0 && lg == 0) g.lse[(size_t)head * g.rows + row0 + row] = mrow[qb] + __builtin_amdgcn_logf(lrow[qb]);
      u32x2 v;
      v.x = pack_bf16x2(a[0] * inv[qb], a[1] * inv[qb]);
      v.y = pack_bf16x2(a[2] * inv[qb], a[3] * inv[qb]);
      *reinterpret_cast<u32x2*>(o + ((row0 + row) * g.n_heads + head) * HDB + 16 * wave + 4 * lg) = v;
    }
  }
}

// Merges the pieces of each tail unit, in piece order.  A work-group takes 8
// query rows of one tail unit; 32 lanes share a row, each holding 4 of its
// 128 outputs, so every partial row is read as one contiguous 512-byte run.
// With m = max m_p:
//   O = sum_p 2^(m_p - m) O_p / sum_p 2^(m_p - m) l_p.
template <int BQ, int KH, class M = PlainAttn>
__global__ __launch_bounds__(256) void attn_combine_kernel(uint16_t* __restrict__ o, typename M::Geom g, AttnPlan plan) {
  const int32_t tu = blockIdx.x;
  const int32_t unit = g.whole_units + tu;
  const int32_t qt = unit % g.n_qtiles;
  const int32_t node = (unit / g.n_qtiles) % g.n_nodes;
  const int32_t head = unit / (g.n_qtiles * g.n_nodes);
  const int32_t lrow = blockIdx.y * 8 + (threadIdx.x >> 5);
  const int32_t dl = threadIdx.x & 31;
  const int32_t qrow = qt * BQ + lrow;
  if (qrow >= g.nq) return;
  const int32_t nt = node_tiles<KH>(plan, g, node);
  auto nonempty = [&](int32_t p) { return p * nt / g.tail_split < (p + 1) * nt / g.tail_split; };
  float m = -INFINITY;
  for (int32_t p = 0; p < g.tail_split; ++p)
    if (nonempty(p)) m = fmaxf(m, g.part_ml[((size_t)(p * g.tail_units + tu) * 2 + 0) * BQ + lrow]);
  f32x4 acc = {};
  float l = 0.f;
  for (int32_t p = 0; p < g.tail_split; ++p) {
    if (!nonempty(p)) continue;
    const size_t slot = (size_t)p * g.tail_units + tu;
    const float a = __builtin_amdgcn_exp2f(g.part_ml[(slot * 2 + 0) * BQ + lrow] - m);
    l += a * g.part_ml[(slot * 2 + 1) * BQ + lrow];
    const f32x4 v = *reinterpret_cast<const f32x4*>(g.part_o + (slot * BQ + lrow) * HDB + 4 * dl);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += a * v[e];
  }
  const float inv = 1.f / l;
  if constexpr (M::kLse)
    if (g.lse && dl == 0) g.lse[(size_t)head * g.rows + (size_t)node * g.nq + qrow] = m + __builtin_amdgcn_logf(l);
  u32x2 r;
  r.x = pack_bf16x2(acc[0] * inv, acc[1] * inv);
  r.y = pack_bf16x2(acc[2] * inv, acc[3] * inv);
  *reinterpret_cast<u32x2*>(o + (((size_t)node * g.nq + qrow) * g.n_heads + head) * HDB + 4 * dl) = r;
}

// Merges the partials of a SharePlan's rows: the prefix's pieces, then those of the
// row's own node, in that order.  GR groups of 32 lanes share a row (and each
// holds 4 of its HD outputs per lane, or 2): one group where the partials are
// few, eight where there are many and the chain of loads would set the time.  Bound
// by launch and latency: 32 rows of 12 heads and 18 partials 4 us, 2048 and 4 (50 MB)
// 11 us.
// pieces(node): the partials of a row of that node.
template <int HD, int GR, bool F32, class Pieces>
__device__ __forceinline__ void share_combine(void* __restrict__ o, const LseGeom& g, int32_t block, int32_t head,
                                              const Pieces& pieces) {
  constexpr int V = HD / 32;
  typedef float fv __attribute__((ext_vector_type(V)));
  __shared__ fv red[8][32];
  const int32_t grp = threadIdx.x >> 5, dl = threadIdx.x & 31;
  const int32_t row = GR == 8 ? block : block * 8 + grp;
  if (row >= g.rows) return;  // the whole work-group where its lanes share a row
  const int32_t n = pieces((int32_t)fast_div((uint32_t)row, g.nq_div));
  const auto at = [&](int32_t p) { return ((size_t)p * g.n_heads + head) * g.rows + row; };
  const auto ex = [](float x) { return __builtin_amdgcn_exp2f(x); };
  // the first partials are on their way while the maximum is found
  constexpr int AHEAD = 4;
  const int32_t p0 = GR == 8 ? grp : 0;
  fv first[AHEAD];
#pragma unroll
  for (int j = 0; j < AHEAD; ++j)
    first[j] = *reinterpret_cast<const fv*>(g.part_o + at(min(p0 + GR * j, n - 1)) * HD + V * dl);
  const float m0 = dl < n ? g.part_ml[2 * at(dl)] : -INFINITY, l0 = dl < n ? g.part_ml[2 * at(dl) + 1] : 0.f;
  float m = m0;
  for (int32_t p = dl + 32; p < n; p += 32) m = fmaxf(m, g.part_ml[2 * at(p)]);
#pragma unroll
  for (int x = 16; x; x >>= 1) m = fmaxf(m, __shfl_xor(m, x));
  const float e0 = dl < n ? ex(m0 - m) : 0.f;
  float l = e0 * l0;
  for (int32_t p = dl + 32; p < n; p += 32) l += ex(g.part_ml[2 * at(p)] - m) * g.part_ml[2 * at(p) + 1];
#pragma unroll
  for (int x = 16; x; x >>= 1) l += __shfl_xor(l, x);
  fv acc = {};
#pragma unroll
  for (int j = 0; j < AHEAD; ++j)
    if (p0 + GR * j < n) acc += __shfl(e0, p0 + GR * j, 32) * first[j];
#pragma unroll 4
  for (int32_t p = p0 + GR * AHEAD; p < n; p += GR)
    acc += ex(g.part_ml[2 * at(p)] - m) * *reinterpret_cast<const fv*>(g.part_o + at(p) * HD + V * dl);
  if constexpr (GR == 8) {
    red[grp][dl] = acc;
    __syncthreads();
    if (grp) return;
#pragma unroll
    for (int w = 1; w < 8; ++w) acc += red[w][dl];
  }
  const float inv = 1.f / l;
  if (g.lse && dl == 0) g.lse[(size_t)head * g.rows + row] = m + __builtin_amdgcn_logf(l);
  const size_t out = ((size_t)row * g.n_heads + head) * HD + V * dl;
  if constexpr (F32) {
    float* op = static_cast<float*>(o) + out;
#pragma unroll
    for (int e = 0; e < V; ++e) op[e] = acc[e] * inv;
  } else {
    u32x2 r;
    r.x = pack_bf16x2(acc[0] * inv, acc[1] * inv);
    r.y = pack_bf16x2(acc[2] * inv, acc[3] * inv);
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(o) + out) = r;
  }
}
template <int HD, int GR, int KH>
__global__ __launch_bounds__(256) void attn_share_combine_kernel(void* __restrict__ o, LseGeom g, SharePlan plan) {
  share_combine<HD, GR, KH == 0>(o, g, (int32_t)blockIdx.x, (int32_t)blockIdx.y, [&](int32_t node) {
    return g.p_pieces + (g.own_waves ? 1 : (share_tiles<KH>(plan, g, 1 + node) + g.o_tiles - 1) / g.o_tiles);
  });
}

// What is left to merge after a SharePlan's pieces: where their partials lie, and how
// many of them a row of each node has.
struct ShareMerge {
  LseGeom g;
  uint8_t pieces[kMaxNodes];
};

// ---------------------------------------------------------------- launches
// A form of the unit kernel (attn_shape in attention.hip).
struct AttnShape {
  int32_t bq, kh, ring;
};
// A schedule: the form, its whole units, and its tail units with their pieces each.
struct AttnSchedule {
  AttnShape sh;
  int32_t whole, tail, split;
  double us;  // estimated time (attn_schedule)
  size_t partial_bytes() const {
    return split == 1 ? 0 : (size_t)tail * split * sh.bq * (HDB + 2) * sizeof(float);
  }
};


// Enqueues the kernel of a form, and where its pieces left partials the kernel that
// merges them.
template <class M>
void launch_form(const AttnShape& sh, uint32_t items, const typename M::Geom& g, const typename M::Plan& plan, const void* q,
                 void* o, int32_t dtype, int32_t head_dim, hipStream_t stream);
// The pieces of a SharePlan alone (attention_lse.hip).
void launch_share_pieces(const AttnShape& sh, uint32_t items, const LseGeom& g, const SharePlan& plan, const void* q,
                         int32_t dtype, int32_t head_dim, hipStream_t stream);
// Whether a row of a plan leaves few partials (bf16, at most kMergePieces), which launch_weigh can
// merge on its way; and the launch that leaves them (attention.hip).
constexpr int32_t kMergePieces = 16;
bool attention_leaves_partials(const sc_plan* p, const sc_cache* c);
int launch_attention_partials(const sc_plan* p, const sc_cache* c, int32_t layer, const void* q, float scale, void* ws,
                              ShareMerge* left, hipStream_t stream);
template <>  // attention_lse.hip
void launch_form<LseAttn>(const AttnShape&, uint32_t, const LseGeom&, const AttnPlan&, const void*, void*, int32_t,
                          int32_t, hipStream_t);
template <>
void launch_form<ShareAttn>(const AttnShape&, uint32_t, const LseGeom&, const SharePlan&, const void*, void*, int32_t,
                            int32_t, hipStream_t);

}  // namespace sc
