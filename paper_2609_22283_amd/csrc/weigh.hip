// The weight that every cached key received: column sums of the attention's
// probability matrices.
//
//   w[slot][head][token] += sum over the nodes i that read the slot, and their
//                           rows q, of exp2(unit q . k - lse[q])
//
// lse: the rows' logarithmic sums, left by the attention itself (log2 units), so a
// second Q K^T is all that is computed; the probabilities are never stored.  A
// work-group owns keys, holds them in registers and streams through the rows of
// every node that reads them.  Keys read by the same nodes are taken together, page
// after page.  Their rows are cut into items of about one length, a work-group each
// (keys that more nodes read are cut into more), whose sums a second launch adds in
// their order: no atomics, so equal calls give equal bits.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>
#include <map>

#include "attention_core.h"

namespace sc {

constexpr int kWeighPages = 512, kWeighGroups = 64, kWeighSplits = 32;

// Pages in groups with the same readers (bit i: node i).
struct WeighPlan {
  uint64_t readers[kWeighGroups];
  int32_t page0[kWeighGroups + 1];  // a group's pages are page_slot[page0[g] .. page0[g + 1])
  int32_t item0[kWeighGroups];      // its first item of a head (INT32_MAX past the last group)
  int32_t page_slot[kWeighPages];
};

struct WeighGeom {
  const char* layer_base;
  uint64_t slot_bytes;
  float* weights;    // this layer's
  float* part;       // [split][head][key of the launch] sums of the splits' rows, where a group has several
  const float* lse;  // [head][row]
  int32_t n_heads, tpp, nq, rows, items, len, keys;  // items of a head, row tiles of one at most, keys of the launch
  DivMagic tpp_div, nq_div;
  float unit;       // bf16: logit_unit(scale)
  float scale;      // fp32: scale log2(e)
  uint32_t q_flip;  // bf16: sign bits of a negative scale
};

// Tiles of QB rows of a group's readers.
template <int QB>
__host__ __device__ __forceinline__ int32_t weigh_tiles(uint64_t readers, int32_t nq) {
  return (__builtin_popcountll(readers) * nq + QB - 1) / QB;
}

// A work-group's work: KB keys of a group, and tiles [t, t_end) of QB rows of those that
// read them (split `split` of `splits`).
struct WeighItem {
  int32_t head, split, splits, key0, n_keys, page0;  // key0: first key within the group's n_keys
  int32_t n_rows, t, t_end;
  uint64_t readers;
};
template <int KB, int QB>
__device__ __forceinline__ WeighItem weigh_item(const WeighPlan& plan, const WeighGeom& g, uint32_t block, uint32_t of) {
  const int32_t i = (int32_t)xcd_remap(block, of);  // an XCD's work-groups share the rows of a few heads
  WeighItem it;
  it.head = i / g.items;
  const int32_t at = i % g.items;
  const int32_t grp = __builtin_popcountll(__builtin_amdgcn_ballot_w64(plan.item0[threadIdx.x & 63] <= at)) - 1;
  it.readers = plan.readers[grp];
  it.page0 = plan.page0[grp];
  it.n_keys = (plan.page0[grp + 1] - it.page0) * g.tpp;
  it.n_rows = __builtin_popcountll(it.readers) * g.nq;
  const int32_t blocks = (it.n_keys + KB - 1) / KB, tiles = weigh_tiles<QB>(it.readers, g.nq);
  it.splits = (tiles + g.len - 1) / g.len;
  it.split = (at - plan.item0[grp]) / blocks;  // the keys of a split side by side: they share its rows
  it.key0 = (at - plan.item0[grp]) % blocks * KB;
  it.t = (int32_t)((int64_t)it.split * tiles / it.splits);
  it.t_end = (int32_t)((int64_t)(it.split + 1) * tiles / it.splits);
  return it;
}

// Slot and token of a key of the group (clamped to its last one).
struct WeighKey {
  int32_t slot, token;
};
__device__ __forceinline__ WeighKey weigh_key(const WeighPlan& plan, const WeighGeom& g, const WeighItem& it, int32_t key) {
  key = min(key, it.n_keys - 1);
  const int32_t p = (int32_t)fast_div((uint32_t)key, g.tpp_div);
  return WeighKey{plan.page_slot[it.page0 + p], key - p * g.tpp};
}

// The reading nodes in order, one per lane.
__device__ __forceinline__ void list_readers(uint64_t readers, int32_t lane, int32_t* nodes) {
  if (readers >> lane & 1) nodes[__builtin_popcountll(readers & ((1ull << lane) - 1))] = lane;
}

// Row of the pack that is the r-th of the reading nodes' rows.
__device__ __forceinline__ int32_t reader_row(const WeighGeom& g, const int32_t* nodes, int32_t r) {
  const int32_t i = (int32_t)fast_div((uint32_t)r, g.nq_div);
  return nodes[i] * g.nq + (r - i * g.nq);
}

// The 16 columns (queries) of a result added up, in every lane.
__device__ __forceinline__ float column_sum(float x) {
  x += __shfl_xor(x, 1);
  x += __shfl_xor(x, 2);
  x += __shfl_xor(x, 4);
  return x + __shfl_xor(x, 8);
}

typedef float f32x4a __attribute__((ext_vector_type(4), aligned(4)));

// Adds the sums of keys key .. key + 3 (a multiple of 4; pages hold whole runs of 8).
__device__ __forceinline__ void add_weights(const WeighPlan& plan, const WeighGeom& g, const WeighItem& it, int32_t key,
                                            const f32x4& w) {
  if (key >= it.n_keys) return;
  if (it.splits > 1) {
    float* p = g.part + ((size_t)it.split * g.n_heads + it.head) * g.keys + it.page0 * g.tpp + key;
    *reinterpret_cast<f32x4a*>(p) = w;
    return;
  }
  const WeighKey k = weigh_key(plan, g, it, key);
  f32x4a* p = reinterpret_cast<f32x4a*>(g.weights + ((size_t)k.slot * g.n_heads + it.head) * g.tpp + k.token);
  *p = *p + w;
}

// 16 bytes per lane from an address of its own into LDS (see dma16).
__device__ __forceinline__ void dma16_at(const char* p, uint32_t lds) {
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %2\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, off\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "v"(p), "s"(lds)
      : "memory");
}

// bf16: four waves of 16 KW keys each, which stay in registers as the A operand of
// S^T = K Q^T; tiles of 64 rows of q go through LDS (two buffers, 16-byte columns
// swizzled by the row), shared by the waves.  The keys are what stays because the sums
// are theirs: they grow in registers over all rows, where a work-group that kept rows
// would have to add its part of every key's sum to memory.  Bound by the MFMAs under
// the power cap, exponentials beside them: four nodes of 4680 rows over windows of 21
// frames of 1560 keys, 12 heads (1.9 TFLOP), 1.69 ms, 1.1 PFLOP/s where a large
// library product reaches 1.23; three of 792 rows over seven states of 792 keys
// 60 us (0.68 PFLOP/s: last round, ragged tiles).
constexpr int WG_NW = 4, WG_QB = 64;
// lse_of(head, row): a row's logarithmic sum.
template <int KW, class Lse>
__device__ __forceinline__ void weigh_bf16(const uint16_t* __restrict__ q, const WeighGeom& g, const WeighPlan& plan,
                                           uint32_t block, uint32_t of, const Lse& lse_of) {
  __shared__ __attribute__((aligned(1024))) char tiles[2][WG_QB * HDB * 2];
  __shared__ int32_t nodes[kMaxNodes];
  const int32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t lg = lane >> 4, c = lane & 15;
  const WeighItem it = weigh_item<16 * KW * WG_NW, WG_QB>(plan, g, block, of);
  if (wave == 0) list_readers(it.readers, lane, nodes);
  const int32_t key0 = it.key0 + 16 * KW * wave;
  bf16x8 kf[KW][4];
#pragma unroll
  for (int b = 0; b < KW; ++b) {
    const WeighKey k = weigh_key(plan, g, it, key0 + 16 * b + c);
    const char* kp = g.layer_base + (size_t)k.slot * g.slot_bytes + ((size_t)it.head * g.tpp + k.token) * (HDB * 2) + 16 * lg;
#pragma unroll
    for (int ds = 0; ds < 4; ++ds) {
      u32x4 u = *reinterpret_cast<const u32x4*>(kp + 64 * ds);
#pragma unroll
      for (int e = 0; e < 4; ++e) u[e] ^= g.q_flip;
      kf[b][ds] = __builtin_bit_cast(bf16x8, u);
    }
  }
  __syncthreads();
  const int32_t n_rows = it.n_rows;
  const char* qh = reinterpret_cast<const char*>(q) + (size_t)it.head * (HDB * 2);
  const size_t row_bytes = (size_t)g.n_heads * (HDB * 2);
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_addr(tiles[0])) + 4096 * wave;
  // copies this wave's 16 rows of a tile and returns lane l's lse of its row l
  // (past the last row: the last row's values at lse +inf, which gives no weight)
  const auto fetch = [&](int32_t t, int32_t buf) __attribute__((always_inline)) {
    const int32_t r = WG_QB * t + lane, row = reader_row(g, nodes, min(r, n_rows - 1));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int32_t tr = 16 * wave + 4 * j + lg;
      const int32_t src = __shfl(row, tr);
      dma16_at(qh + (size_t)src * row_bytes + ((c ^ (tr & 15)) << 4), lds0 + buf * (WG_QB * HDB * 2) + 1024 * j);
    }
    const float l = lse_of(it.head, row);
    return r < n_rows ? l : INFINITY;
  };
  f32x4 w[KW];
#pragma unroll
  for (int b = 0; b < KW; ++b) w[b] = f32x4{};
  int32_t t = it.t;
  const int32_t t_end = it.t_end;
  float lse = 0.f;
  if (t < t_end) lse = fetch(t, t & 1);
  for (; t < t_end; ++t) {
    landed();
    const float l = lse;
    if (t + 1 < t_end) lse = fetch(t + 1, (t + 1) & 1);
    const char* tile = tiles[t & 1];
#pragma unroll
    for (int qb = 0; qb < WG_QB / 16; ++qb) {
      f32x4 s[KW];
#pragma unroll
      for (int b = 0; b < KW; ++b) s[b] = f32x4{};
#pragma unroll
      for (int ds = 0; ds < 4; ++ds) {
        const bf16x8 f = *reinterpret_cast<const bf16x8*>(tile + (16 * qb + c) * 256 + (((4 * ds + lg) ^ c) << 4));
#pragma unroll
        for (int b = 0; b < KW; ++b) s[b] = mfma16(kf[b][ds], f, s[b]);
      }
      const float lq = __shfl(l, 16 * qb + c);
#pragma unroll
      for (int b = 0; b < KW; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) w[b][r] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][r], g.unit, -lq));
    }
  }
#pragma unroll
  for (int b = 0; b < KW; ++b) {
#pragma unroll
    for (int r = 0; r < 4; ++r) w[b][r] = column_sum(w[b][r]);
    if (c == 0) add_weights(plan, g, it, key0 + 16 * b + 4 * lg, w[b]);
  }
}

template <int KW>
__global__ __launch_bounds__(64 * WG_NW, 2) void weigh_bf16_kernel(const uint16_t* __restrict__ q, WeighGeom g,
                                                                   WeighPlan plan) {
  weigh_bf16<KW>(q, g, plan, blockIdx.x, gridDim.x,
                 [&](int32_t head, int32_t row) { return g.lse[(size_t)head * g.rows + row]; });
}

// The same after an attention that left few partials per row and has not merged them: the
// first work-groups do that, the others take the rows' sums from the partials themselves.
// One launch less, where a row tile or two are all that a work-group streams.  12 heads,
// with the attention: 64 rows over 21 x 64 keys 14.5 us, 17.3 apart; 128 over 11 x 128
// 19.6 against 22.1; 64 over 7 x 64 12.9 against 15.2.  (Up to 32 partials, taken eight at
// a time, cost more than the launch: 23.8 for the second.)
template <int KW>
__global__ __launch_bounds__(64 * WG_NW, 2) void weigh_merge_kernel(const uint16_t* __restrict__ q,
                                                                    uint16_t* __restrict__ o, WeighGeom g, WeighPlan plan,
                                                                    ShareMerge left, int32_t merges) {
  if ((int32_t)blockIdx.x < merges) {
    const int32_t per = (left.g.rows + 7) / 8;
    share_combine<HDB, 1, false>(o, left.g, (int32_t)blockIdx.x % per, (int32_t)blockIdx.x / per,
                                 [&](int32_t node) { return (int32_t)left.pieces[node]; });
    return;
  }
  weigh_bf16<KW>(q, g, plan, blockIdx.x - merges, gridDim.x - merges, [&](int32_t head, int32_t row) {
    const float* ml = left.g.part_ml + 2 * ((size_t)head * g.rows + row);
    const size_t stride = 2 * (size_t)g.n_heads * g.rows;
    const int32_t n = left.pieces[fast_div((uint32_t)row, g.nq_div)];
    float m[kMergePieces], l[kMergePieces], top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int p = 0; p < kMergePieces; ++p) {
      m[p] = p < n ? ml[p * stride] : -INFINITY;
      l[p] = p < n ? ml[p * stride + 1] : 0.f;
    }
#pragma unroll
    for (int p = 0; p < kMergePieces; ++p) top = fmaxf(top, m[p]);
#pragma unroll
    for (int p = 0; p < kMergePieces; ++p) sum += __builtin_amdgcn_exp2f(m[p] - top) * l[p];
    return top + __builtin_amdgcn_logf(sum);
  });
}

// fp32: the same with eight waves of 16 keys, 32-row tiles and fp32 MFMAs, whose
// contraction index of product (j, e) in lane group g is channel 16 j + 4 g + e.
// Bound by the fp32 MFMAs: four nodes of 312 rows over windows of four, 12 heads of 128
// (4.8 GFLOP), 61 us, 78 TFLOP/s of 154; 2 heads 14 us in one round of 252 items.
constexpr int WF_NW = 8, WF_KB = 16 * WF_NW, WF_QB = 32;
template <int HD>
__global__ __launch_bounds__(64 * WF_NW) void weigh_f32_kernel(const float* __restrict__ q, WeighGeom g, WeighPlan plan) {
  constexpr int NJ = HD / 16, ROW = HD * 4, CP = WF_QB * ROW / (1024 * WF_NW), RPC = 1024 / ROW;  // copies of a wave, rows of one
  __shared__ __attribute__((aligned(1024))) char tiles[2][WF_QB * ROW];
  __shared__ int32_t nodes[kMaxNodes];
  const int32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t lg = lane >> 4, c = lane & 15;
  const WeighItem it = weigh_item<WF_KB, WF_QB>(plan, g, blockIdx.x, gridDim.x);
  if (wave == 0) list_readers(it.readers, lane, nodes);
  const int32_t key0 = it.key0 + 16 * wave;
  const WeighKey k = weigh_key(plan, g, it, key0 + c);
  const float* kp = reinterpret_cast<const float*>(g.layer_base + (size_t)k.slot * g.slot_bytes) +
                    ((size_t)it.head * g.tpp + k.token) * HD + 4 * lg;
  f32x4 kf[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) kf[j] = *reinterpret_cast<const f32x4u*>(kp + 16 * j) * g.scale;
  __syncthreads();
  const int32_t n_rows = it.n_rows;
  const char* qh = reinterpret_cast<const char*>(q) + (size_t)it.head * ROW;
  const size_t row_bytes = (size_t)g.n_heads * ROW;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_addr(tiles[0])) + 1024 * CP * wave;
  const auto fetch = [&](int32_t t, int32_t buf) __attribute__((always_inline)) {
    const int32_t r = WF_QB * t + (lane & (WF_QB - 1)), row = reader_row(g, nodes, min(r, n_rows - 1));
#pragma unroll
    for (int j = 0; j < CP; ++j) {
      const int32_t tr = RPC * (CP * wave + j) + lane / (ROW / 16), col = lane & (ROW / 16 - 1);
      const int32_t src = __shfl(row, tr);
      dma16_at(qh + (size_t)src * row_bytes + ((col ^ (tr & 15)) << 4), lds0 + buf * (WF_QB * ROW) + 1024 * j);
    }
    const float l = g.lse[(size_t)it.head * g.rows + row];
    return r < n_rows ? l : INFINITY;
  };
  f32x4 w = {};
  int32_t t = it.t;
  const int32_t t_end = it.t_end;
  float lse = 0.f;
  if (t < t_end) lse = fetch(t, t & 1);
  for (; t < t_end; ++t) {
    landed();
    const float l = lse;
    if (t + 1 < t_end) lse = fetch(t + 1, (t + 1) & 1);
    const char* tile = tiles[t & 1];
#pragma unroll
    for (int rb = 0; rb < WF_QB / 16; ++rb) {
      f32x4 s0 = {}, s1 = {};
#pragma unroll
      for (int j = 0; j < NJ; j += 2) {
        const char* at = tile + (16 * rb + c) * ROW;
        const f32x4 q0 = *reinterpret_cast<const f32x4*>(at + (((4 * j + lg) ^ c) << 4));
        const f32x4 q1 = *reinterpret_cast<const f32x4*>(at + (((4 * j + 4 + lg) ^ c) << 4));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[j][e], q0[e], s0, 0, 0, 0);
          s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[j + 1][e], q1[e], s1, 0, 0, 0);
        }
      }
      s0 += s1;
      const float lq = __shfl(l, 16 * rb + c);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] += __builtin_amdgcn_exp2f(s0[e] - lq);
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = column_sum(w[e]);
  if (c == 0) add_weights(plan, g, it, key0 + 4 * lg, w);
}

// Adds the splits' sums, in their order: four keys of a head to a thread.  QB: the
// rows of a tile.
template <int QB>
__global__ __launch_bounds__(256) void weigh_add_kernel(WeighGeom g, WeighPlan plan) {
  const int32_t key = 4 * (int32_t)(blockIdx.x * 256 + threadIdx.x), head = blockIdx.y;
  if (key >= g.keys) return;
  const int32_t p = (int32_t)fast_div((uint32_t)key, g.tpp_div);
  int32_t grp = 0;
#pragma unroll
  for (int step = kWeighGroups / 2; step; step /= 2)
    if (plan.page0[grp + step] <= p) grp += step;
  const int32_t splits = (weigh_tiles<QB>(plan.readers[grp], g.nq) + g.len - 1) / g.len;
  if (splits == 1) return;
  const float* part = g.part + (size_t)head * g.keys + key;
  const size_t stride = (size_t)g.n_heads * g.keys;
  f32x4 w = *reinterpret_cast<const f32x4a*>(part);
#pragma unroll 4
  for (int32_t s = 1; s < splits; ++s) w += *reinterpret_cast<const f32x4a*>(part + s * stride);
  f32x4a* to = reinterpret_cast<f32x4a*>(g.weights + ((size_t)plan.page_slot[p] * g.n_heads + head) * g.tpp + (key - p * g.tpp));
  *to = *to + w;
}

// Zeroes the weights of slots, one slot of one layer per work-group.
struct SlotList {
  int32_t slot[64];
};
__global__ __launch_bounds__(256) void weights_clear_kernel(float* weights, size_t slot_floats, int32_t n_slots, SlotList s) {
  float* p = weights + ((size_t)blockIdx.y * n_slots + s.slot[blockIdx.x]) * slot_floats;
  for (size_t i = threadIdx.x; i < slot_floats; i += 256) p[i] = 0.f;
}

// How a launch runs: 16-key blocks per wave (bf16), row tiles of an item at most,
// items of a head, keys, and the most splits of a group.
struct WeighForm {
  int32_t kw, len, items, keys, splits;
};
// A plan's distinct pages by their readers, most readers first, in launches of
// bounded argument size.  A property of the plan alone: found on its first use and
// kept in it.
struct WeighLaunches {
  std::vector<WeighPlan> plans;
  std::vector<WeighForm> forms;
  size_t part_bytes;  // the most that a launch's splits leave
};

// The cheapest form by estimated time.  A CU's time per 64-row tile of an item is 1.05
// us with 256 keys (1.07 PFLOP/s), 0.6 with 128 and 0.4 with 64, whose rows feed fewer
// products per LDS read, and 2.2, 1.5 and 1.2 to bring the keys; fp32 2.9 us per 32
// rows and 128 keys of 128 channels, and 3.  Items in rounds over the CUs (a work-group by
// itself takes 1.6 times its share), what the longest one is longer than the mean, and 5 us for
// the launch that adds splits.  Measured with the attention before it: three nodes of
// 792 rows over windows of seven, 12 heads: 159 us with 128 keys in whole rows, 154 with
// 256 in items of 8 to 12 tiles, 160 of 3; four of 4680: 5168 whole, 4970 in
// items of 74, 5060 of 16; fp32, four of 312 rows, 2 heads: 67 us in items of 12,
// 52.7 of 4, 57.7 of 3.
static WeighForm weigh_form(WeighPlan& plan, const sc_cache* c, int32_t nq) {
  const bool f32 = c->d.dtype == SC_DTYPE_F32;
  const int32_t tpp = c->d.tokens_per_page, H = c->d.n_heads;
  const auto tiles_of = [&](int32_t i) {
    return f32 ? weigh_tiles<WF_QB>(plan.readers[i], nq) : weigh_tiles<WG_QB>(plan.readers[i], nq);
  };
  int32_t most = 1;
  for (int32_t i = 0; i < kWeighGroups; ++i) most = std::max(most, tiles_of(i));
  WeighForm best{1, most, 0, 0, 1};
  double best_us = 1e30;
  for (int32_t kw = f32 ? 1 : 4; kw >= 1; kw /= 2) {
    const int32_t kb = f32 ? WF_KB : 16 * kw * WG_NW;
    const double t = f32 ? 2.9 * c->d.head_dim / 128 : kw == 4 ? 1.05 : kw == 2 ? 0.6 : 0.4;
    const double f = f32 ? 3.0 : kw == 4 ? 2.2 : kw == 2 ? 1.5 : 1.2;
    for (int32_t s = 1; s <= kWeighSplits && s <= most; ++s) {
      const int32_t len = (most + s - 1) / s;
      double tiles = 0.0;
      int64_t items = 0, keys = 0;
      for (int32_t i = 0; i < kWeighGroups; ++i) {
        const int64_t k = (int64_t)(plan.page0[i + 1] - plan.page0[i]) * tpp, b = (k + kb - 1) / kb;
        keys += k;
        tiles += (double)b * tiles_of(i);
        items += b * ((tiles_of(i) + len - 1) / len);
      }
      const double rounds = std::max(std::ceil((double)items * H / kCUs), f32 ? 1.0 : 1.6);
      const double mean = tiles / (double)items;
      const double us = rounds * (mean * t + f) + (len - mean) * (f32 ? t : 2.0 * t) + (len < most ? 5.0 : 0.0);
      if (us < best_us * 0.99 && items * H < INT32_MAX) {
        best_us = us;
        best = WeighForm{kw, len, (int32_t)items, (int32_t)keys, (most + len - 1) / len};
      }
    }
  }
  int64_t items = 0;
  for (int32_t i = 0; i < kWeighGroups; ++i) {
    const int32_t kb = f32 ? WF_KB : 16 * best.kw * WG_NW;
    const int64_t b = ((int64_t)(plan.page0[i + 1] - plan.page0[i]) * tpp + kb - 1) / kb;
    plan.item0[i] = b ? (int32_t)items : INT32_MAX;
    items += b * ((tiles_of(i) + best.len - 1) / best.len);
  }
  return best;
}

static const WeighLaunches* weigh_launches(const sc_plan* p, const sc_cache* c) {
  if (p->weigh) return p->weigh.get();
  std::map<int32_t, uint64_t> readers;
  const int32_t n = (int32_t)p->nodes.size();
  const uint64_t all = n == 64 ? ~0ull : (1ull << n) - 1;
  for (int32_t i = 0; i < p->shared; ++i) readers[p->page_slot[i]] = all;
  for (int32_t i = 0; i < n; ++i)
    for (int32_t k = p->page_off[i] + p->shared; k < p->page_off[i + 1]; ++k) readers[p->page_slot[k]] |= 1ull << i;
  std::map<uint64_t, std::vector<int32_t>> groups;
  for (const auto& kv : readers) groups[kv.second].push_back(kv.first);
  std::vector<std::pair<uint64_t, std::vector<int32_t>>> order(groups.begin(), groups.end());
  std::stable_sort(order.begin(), order.end(), [](const auto& a, const auto& b) {
    return __builtin_popcountll(a.first) > __builtin_popcountll(b.first);
  });
  auto out = std::make_shared<WeighLaunches>();
  int32_t pages = kWeighPages, count = kWeighGroups;  // of the launch being filled
  for (const auto& grp : order)
    for (size_t at = 0; at < grp.second.size();) {
      if (pages == kWeighPages || count == kWeighGroups) {
        out->plans.emplace_back();
        std::memset(&out->plans.back(), 0, sizeof(WeighPlan));
        pages = count = 0;
      }
      WeighPlan& w = out->plans.back();
      const size_t take = std::min(grp.second.size() - at, (size_t)(kWeighPages - pages));
      w.readers[count] = grp.first;
      w.page0[count] = pages;
      std::copy(grp.second.begin() + at, grp.second.begin() + at + take, w.page_slot + pages);
      pages += (int32_t)take;
      at += take;
      for (int32_t k = ++count; k <= kWeighGroups; ++k) w.page0[k] = pages;
    }
  out->part_bytes = 0;
  for (WeighPlan& w : out->plans) {
    const WeighForm f = weigh_form(w, c, p->nq);
    out->forms.push_back(f);
    if (f.splits > 1)
      out->part_bytes = std::max(out->part_bytes, (size_t)f.splits * c->d.n_heads * f.keys * sizeof(float));
  }
  p->weigh = out;
  return out.get();
}

// Whether the weighing merges the attention's partials on its way (weigh_merge_kernel).
static bool weigh_merges(const sc_plan* p, const sc_cache* c) {
  const WeighLaunches* all = weigh_launches(p, c);
  return all->plans.size() == 1 && all->forms[0].splits == 1 && all->forms[0].len <= 2 && attention_leaves_partials(p, c);
}

// Adds the weights to the whole array `weights`; part: the launches' part_bytes.  left:
// the partials to merge into o, or NULL.
static int launch_weigh(const sc_plan* p, const sc_cache* c, int32_t layer, const void* q, const float* lse, float scale,
                        float* weights, float* part, void* o, const ShareMerge* left, hipStream_t stream) {
  const sc_cache_desc& d = c->d;
  WeighGeom g;
  std::memset(&g, 0, sizeof g);
  g.layer_base = c->pool + (size_t)layer * d.n_slots * c->slot_bytes;
  g.slot_bytes = c->slot_bytes;
  g.weights = weights + (size_t)layer * d.n_slots * d.n_heads * d.tokens_per_page;
  g.part = part;
  g.lse = lse;
  g.n_heads = d.n_heads;
  g.tpp = d.tokens_per_page;
  g.nq = p->nq;
  g.rows = (int32_t)p->nodes.size() * p->nq;
  g.tpp_div = magic_div((uint32_t)g.tpp);
  g.nq_div = magic_div((uint32_t)g.nq);
  g.unit = logit_unit(scale);
  g.scale = scale * 1.4426950408889634f;
  g.q_flip = std::signbit(scale) ? 0x80008000u : 0u;
  const WeighLaunches* all = weigh_launches(p, c);
  for (size_t i = 0; i < all->plans.size(); ++i) {
    const WeighPlan& plan = all->plans[i];
    const WeighForm& f = all->forms[i];
    g.items = f.items;
    g.len = f.len;
    g.keys = f.keys;
    const dim3 grid((uint32_t)(f.items * d.n_heads));
    timer_begin(TK_ATTN_WEIGH, stream);
    if (d.dtype == SC_DTYPE_F32) {
      const float* qf = static_cast<const float*>(q);
      if (d.head_dim == 64)
        hipLaunchKernelGGL((weigh_f32_kernel<64>), grid, dim3(64 * WF_NW), 0, stream, qf, g, plan);
      else
        hipLaunchKernelGGL((weigh_f32_kernel<128>), grid, dim3(64 * WF_NW), 0, stream, qf, g, plan);
    } else {
      const uint16_t* qb = static_cast<const uint16_t*>(q);
      uint16_t* ob = static_cast<uint16_t*>(o);
      const int32_t merges = left ? (g.rows + 7) / 8 * d.n_heads : 0;
      const dim3 both(grid.x + (uint32_t)merges);
      if (left && f.kw == 4)
        hipLaunchKernelGGL((weigh_merge_kernel<4>), both, dim3(64 * WG_NW), 0, stream, qb, ob, g, plan, *left, merges);
      else if (left && f.kw == 2)
        hipLaunchKernelGGL((weigh_merge_kernel<2>), both, dim3(64 * WG_NW), 0, stream, qb, ob, g, plan, *left, merges);
      else if (left)
        hipLaunchKernelGGL((weigh_merge_kernel<1>), both, dim3(64 * WG_NW), 0, stream, qb, ob, g, plan, *left, merges);
      else if (f.kw == 4)
        hipLaunchKernelGGL((weigh_bf16_kernel<4>), grid, dim3(64 * WG_NW), 0, stream, qb, g, plan);
      else if (f.kw == 2)
        hipLaunchKernelGGL((weigh_bf16_kernel<2>), grid, dim3(64 * WG_NW), 0, stream, qb, g, plan);
      else
        hipLaunchKernelGGL((weigh_bf16_kernel<1>), grid, dim3(64 * WG_NW), 0, stream, qb, g, plan);
    }
    if (f.splits > 1) {
      const dim3 adds((uint32_t)((f.keys / 4 + 255) / 256), (uint32_t)d.n_heads);
      if (d.dtype == SC_DTYPE_F32)
        hipLaunchKernelGGL(weigh_add_kernel<WF_QB>, adds, dim3(256), 0, stream, g, plan);
      else
        hipLaunchKernelGGL(weigh_add_kernel<WG_QB>, adds, dim3(256), 0, stream, g, plan);
    }
    timer_end(TK_ATTN_WEIGH, stream);
    SC_HIP(hipGetLastError());
  }
  return SC_OK;
}

// the attention's partials, then the splits' sums of the weights | the rows'
// logarithmic sums [head][row]
static size_t partial_bytes(const sc_plan* p, const sc_cache* c) {
  return (std::max(attention_lse_workspace_bytes(p, c), weigh_launches(p, c)->part_bytes) + 255) & ~size_t(255);
}

size_t weigh_attention_bytes(const sc_plan* p, const sc_cache* c) {
  return partial_bytes(p, c) + (size_t)p->nodes.size() * p->nq * c->d.n_heads * sizeof(float);
}

int launch_attention_weigh(const sc_plan* p, const sc_cache* c, int32_t layer, const void* q, void* o, float scale,
                           float* weights, void* ws, hipStream_t stream) {
  const size_t part = partial_bytes(p, c);
  if (weigh_merges(p, c)) {
    ShareMerge left;
    std::memset(static_cast<void*>(&left), 0, sizeof left);
    const int rc = launch_attention_partials(p, c, layer, q, scale, ws, &left, stream);
    return rc != SC_OK ? rc : launch_weigh(p, c, layer, q, nullptr, scale, weights, nullptr, o, &left, stream);
  }
  float* lse = reinterpret_cast<float*>(static_cast<char*>(ws) + part);
  const int rc = launch_attention_lse(p, c, layer, q, o, lse, scale, ws, part, stream);
  return rc != SC_OK ? rc
                     : launch_weigh(p, c, layer, q, lse, scale, weights, static_cast<float*>(ws), nullptr, nullptr, stream);
}

int launch_weights_clear(const sc_cache* c, const int32_t* slots, int32_t n, float* weights, hipStream_t stream) {
  for (int32_t at = 0; at < n; at += 64) {
    SlotList s;
    const int32_t m = std::min(n - at, 64);
    std::memset(&s, 0, sizeof s);
    std::copy(slots + at, slots + at + m, s.slot);
    for (int32_t l0 = 0; l0 < c->d.n_layers; l0 += 65535) {
      const size_t slot_floats = (size_t)c->d.n_heads * c->d.tokens_per_page;
      hipLaunchKernelGGL(weights_clear_kernel, dim3((uint32_t)m, (uint32_t)std::min(c->d.n_layers - l0, 65535)), dim3(256), 0,
                         stream, weights + (size_t)l0 * c->d.n_slots * slot_floats, slot_floats, c->d.n_slots, s);
    }
    SC_HIP(hipGetLastError());
  }
  return SC_OK;
}

}  // namespace sc
