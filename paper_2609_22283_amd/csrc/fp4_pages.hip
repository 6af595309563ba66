// Pages: moved as they are, held in 4 bits, and taken back out.
#include <algorithm>
#include <cstring>

#include "fp4.h"

namespace sc {

constexpr int kPairs = 448;  // of a launch: they travel in its arguments
struct PairList {
  int32_t src[kPairs], dst[kPairs];
};

static PairList pair_list(const PagePairs& p, int32_t first, int32_t n) {
  PairList l;
  std::memset(&l, 0, sizeof l);
  std::copy(p.src + first, p.src + first + n, l.src);
  std::copy(p.dst + first, p.dst + first + n, l.dst);
  return l;
}

// A work-group copies 16 KB of a page: four loads of a thread are out before the
// first is stored, and read past the caches.  x: pieces of a page, y: pairs, z: layers.
// Bound by memory: six pages of 1560 tokens x 12 heads in eight layers (920 MB read and
// written) 153 us, 6.0 TB/s.
constexpr int MV_T = 256, MV_N = 4;
__global__ __launch_bounds__(MV_T) void page_move_kernel(const char* from, char* to, uint64_t from_layer,
                                                         uint64_t to_layer, uint64_t bytes, PairList pairs) {
  const char* src = from + blockIdx.z * from_layer + (uint64_t)pairs.src[blockIdx.y] * bytes;
  char* dst = to + blockIdx.z * to_layer + (uint64_t)pairs.dst[blockIdx.y] * bytes;
  const uint64_t at = (uint64_t)blockIdx.x * (MV_T * MV_N * 16) + threadIdx.x * 16;
  u32x4u v[MV_N];
#pragma unroll
  for (int i = 0; i < MV_N; ++i)
    if (at + i * MV_T * 16 < bytes) v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4u*>(src + at + i * MV_T * 16));
#pragma unroll
  for (int i = 0; i < MV_N; ++i)
    if (at + i * MV_T * 16 < bytes) *reinterpret_cast<u32x4u*>(dst + at + i * MV_T * 16) = v[i];
}

// launch(the pairs, how many, first layer, layers) for grids that hold them all.
template <class F>
static int in_launches(const PagePairs& pairs, int32_t layers, hipStream_t stream, F launch) {
  for (int32_t l = 0; l < layers; l += 65535)
    for (int32_t p = 0; p < pairs.n; p += kPairs) {
      const int32_t n = std::min(kPairs, pairs.n - p);
      timer_begin(TK_PAGES, stream);
      launch(pair_list(pairs, p, n), n, l, std::min(65535, layers - l));
      timer_end(TK_PAGES, stream);
      SC_HIP(hipGetLastError());
    }
  return SC_OK;
}

int launch_page_moves(const PoolView& from, const PoolView& to, uint64_t bytes, const PagePairs& pairs, int32_t layers,
                      hipStream_t stream) {
  const uint32_t pieces = (uint32_t)((bytes + MV_T * MV_N * 16 - 1) / (MV_T * MV_N * 16));
  return in_launches(pairs, layers, stream, [&](const PairList& l, int32_t n, int32_t layer, int32_t m) {
    hipLaunchKernelGGL(page_move_kernel, dim3(pieces, n, m), dim3(MV_T), 0, stream,
                       from.base + layer * from.layer_bytes, to.base + layer * to.layer_bytes, from.layer_bytes,
                       to.layer_bytes, bytes, l);
  });
}

// Pages of both kinds, and the waves' items in a page: blocks, or pairs of them.
struct ConvertGeom {
  const char* from;
  char* to;
  uint64_t from_layer, to_layer, from_slot, to_slot;
  int32_t heads, tpp, blocks;
  DivMagic blocks_div;
};

// Lanes and passes over K of a block: pass i takes the tokens k_token(i) + lane / 16, eight
// channels a lane, so that four neighbouring lanes hold a group and a lane's passes fill its
// scales' words.
__device__ __forceinline__ int k_token(int i) { return 16 * (i >> 2) + 4 * (i & 3); }
__device__ __forceinline__ uint32_t k_codes_at(int i, int32_t lane) {
  return 512 * (i & 3) + 256 * (i >> 2) + (lane >> 2 & 3) * 64 + (lane >> 4) * 16 + (lane & 3) * 4;
}
__device__ __forceinline__ uint32_t k_scales_at(int32_t lane) { return kFp4KScale + (lane >> 4) * 16 + (lane >> 2 & 3) * 4; }
__device__ __forceinline__ uint32_t group_scale(const u32x4& v) {
  return fp4_scale(quad_max(umax(umax(bf16x2_top(v[0]), bf16x2_top(v[1])), umax(bf16x2_top(v[2]), bf16x2_top(v[3])))));
}
// Codes and scales of K of half a block, 16 tokens, whose four passes' values are given.
__device__ __forceinline__ void pack_keys(const u32x4 (&k)[4], int half, char* block, int32_t lane) {
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t s = group_scale(k[i]);
    *reinterpret_cast<uint32_t*>(block + k_codes_at(4 * half + i, lane)) = fp4_codes(k[i], s);
    w |= s << (8 * i);
  }
  if ((lane & 3) == 0) *reinterpret_cast<uint32_t*>(block + k_scales_at(lane) + 64 * half) = w;
}

// One wave per two blocks: of V, pass n takes the channels 8 n + lane / 8 of both, eight
// tokens a lane, 128 bytes of a channel (pairs of waves with a block each wait for each
// other's lines).  Read past the caches, which the pages it reads would only push others out of:
// 20 states of 64 tokens, 12 heads, 30 layers 79 us, 54 so.
__global__ __launch_bounds__(256) void page_pack_kernel(ConvertGeom g, PairList pairs) {
  const int32_t lane = threadIdx.x & 63;
  const int32_t item = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (item >= g.heads * g.blocks) return;  // g.blocks: pairs of blocks of a page
  const int32_t h = (int32_t)fast_div((uint32_t)item, g.blocks_div), b = 2 * (item - h * g.blocks), t0 = b * kFp4Tokens;
  const int32_t all = (g.tpp + kFp4Tokens - 1) / kFp4Tokens, left = g.tpp - t0;  // blocks of a page; its tokens from t0 on
  const char* page = g.from + blockIdx.z * g.from_layer + (uint64_t)pairs.src[blockIdx.y] * g.from_slot;
  char* block = g.to + blockIdx.z * g.to_layer + (uint64_t)pairs.dst[blockIdx.y] * g.to_slot + ((uint64_t)h * all + b) * kFp4Block;
  const char* krow = page + ((uint64_t)h * g.tpp + t0 + (lane >> 4)) * 256 + (lane & 15) * 16;
  const char* vrow = page + (uint64_t)g.heads * g.tpp * 256 + ((uint64_t)h * 128 + (lane >> 3)) * g.tpp * 2 + (t0 + 8 * (lane & 7)) * 2;
  const bool two = b + 1 < all, mine = two || (lane & 4) == 0;
  char* vcodes = block + (lane >> 2 & 1) * kFp4Block + kFp4V + (lane >> 3) * 16 + (lane & 3) * 4;
  u32x2 vw[2] = {};
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    u32x4 k[2][4], v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      k[i >> 2][i & 3] = v[i] = u32x4{};
      if (32 * half + k_token(i) + (lane >> 4) < left)
        k[i >> 2][i & 3] = __builtin_nontemporal_load(reinterpret_cast<const u32x4u*>(krow + (uint64_t)(32 * half + k_token(i)) * 256));
      if (8 * (lane & 7) < left) v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4u*>(vrow + (uint64_t)(8 * half + i) * 8 * g.tpp * 2));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {  // channel 64 half + 8 i + lane / 8: byte 4 half + i / 2 of the scales of channel % 16
      const uint32_t s = group_scale(v[i]);
      if (mine) *reinterpret_cast<uint32_t*>(vcodes + (8 * half + i) * 128) = fp4_codes(v[i], s);
      vw[i & 1][half] |= s << (8 * (i >> 1));
    }
    if (half == 0 || two) {
      pack_keys(k[0], 0, block + half * kFp4Block, lane);
      pack_keys(k[1], 1, block + half * kFp4Block, lane);
    }
  }
  if ((lane & 3) == 0 && mine) {
    char* vs = block + (lane >> 2 & 1) * kFp4Block + kFp4VScale + (lane >> 3) * 8;
    *reinterpret_cast<u32x2*>(vs) = vw[0];
    *reinterpret_cast<u32x2*>(vs + 64) = vw[1];
  }
}

// One wave per block: of V, pass n takes the channels 16 n + lane / 4, eight tokens a lane.
// Read past the caches like the pages of page_pack_kernel: with them out of 4 bits again these
// 20 states take 112 us in all (534 MB, 4.8 TB/s, as a plain copy runs), 127 with loads that stay.
__global__ __launch_bounds__(256) void page_unpack_kernel(ConvertGeom g, PairList pairs) {
  const int32_t lane = threadIdx.x & 63;
  const int32_t item = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (item >= g.heads * g.blocks) return;
  const int32_t h = (int32_t)fast_div((uint32_t)item, g.blocks_div), b = item - h * g.blocks, t0 = b * kFp4Tokens;
  const int32_t left = g.tpp - t0;  // tokens of the page from t0 on
  char* page = g.to + blockIdx.z * g.to_layer + (uint64_t)pairs.dst[blockIdx.y] * g.to_slot;
  const char* block = g.from + blockIdx.z * g.from_layer + (uint64_t)pairs.src[blockIdx.y] * g.from_slot + (uint64_t)item * kFp4Block;
  char* krow = page + ((uint64_t)h * g.tpp + t0 + (lane >> 4)) * 256 + (lane & 15) * 16;
  char* vrow = page + (uint64_t)g.heads * g.tpp * 256 + ((uint64_t)h * 128 + (lane >> 2)) * g.tpp * 2 + (t0 + 8 * (lane & 3)) * 2;
  const char* ks = block + k_scales_at(lane);
  uint32_t k[8], v[8];
  const uint32_t kw[2] = {*reinterpret_cast<const uint32_t*>(ks), *reinterpret_cast<const uint32_t*>(ks + 64)};
  const u32x2 vw = *reinterpret_cast<const u32x2*>(block + kFp4VScale + (lane >> 2) * 8);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    k[i] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(block + k_codes_at(i, lane)));
    v[i] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(block + kFp4V + i * 256 + lane * 4));
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (k_token(i) + (lane >> 4) < left)
      *reinterpret_cast<u32x4u*>(krow + (uint64_t)k_token(i) * 256) = fp4_values(k[i], kw[i >> 2] >> (8 * (i & 3)) & 255u);
    if (8 * (lane & 3) < left)
      *reinterpret_cast<u32x4u*>(vrow + (uint64_t)i * 16 * g.tpp * 2) = fp4_values(v[i], vw[i >> 2] >> (8 * (i & 3)) & 255u);
  }
}

int launch_page_convert(bool pack, const PoolView& from, const PoolView& to, const sc_cache_desc& d,
                        const PagePairs& pairs, int32_t layers, hipStream_t stream) {
  ConvertGeom g;
  std::memset(&g, 0, sizeof g);
  g.heads = d.n_heads;
  g.tpp = d.tokens_per_page;
  g.blocks = pack ? (fp4_blocks(g.tpp) + 1) / 2 : fp4_blocks(g.tpp);
  g.blocks_div = magic_div((uint32_t)g.blocks);
  const uint64_t wide = 4ull * d.n_heads * d.tokens_per_page * 128, held = (uint64_t)d.n_heads * fp4_blocks(g.tpp) * kFp4Block;
  g.from_slot = pack ? wide : held;
  g.to_slot = pack ? held : wide;
  g.from_layer = from.layer_bytes;
  g.to_layer = to.layer_bytes;
  const uint32_t groups = (uint32_t)((g.heads * g.blocks + 3) / 4);
  return in_launches(pairs, layers, stream, [&](const PairList& l, int32_t n, int32_t layer, int32_t m) {
    g.from = from.base + layer * from.layer_bytes;
    g.to = to.base + layer * to.layer_bytes;
    if (pack)
      hipLaunchKernelGGL(page_pack_kernel, dim3(groups, n, m), dim3(256), 0, stream, g, l);
    else
      hipLaunchKernelGGL(page_unpack_kernel, dim3(groups, n, m), dim3(256), 0, stream, g, l);
  });
}

// ------------------------------------------------------------------- append
struct AppendArgs {
  const uint16_t *k, *v;
  char* layer_base;
  uint64_t slot_bytes;
  int32_t heads, tpp, blocks;
  const float2* table;  // NULL: no rotation
  int32_t grid_w, pairs_t, pairs_h;
  int64_t off_h, off_w;
  int32_t pairs_w, frame0;
  DivMagic gw_div;
  int32_t slot[32];
};

// A wave takes half of K (z 0 and 1) or V (z 2) of a block: x the blocks of the state's pages, four
// to a work-group, y the head.  Keys as in pack_keys, rotated before; of V a lane takes eight
// channels of the tokens 8 (lane / 16) .. + 7, finds each channel's largest magnitude with the
// three lanes that hold its other tokens, and the codes cross LDS, so that they leave in
// 16-byte runs.  A chain of latencies: a frame of 64 tokens, 12 heads, rotated, takes 4.8 us
// (6.2 with K in one wave, 9.7 with V in the same one and rotations loaded one by one), a chunk
// of 3 x 1560 tokens (36 MB) 11.2 (12.4 with K in one).
template <bool ROPE>
__global__ __launch_bounds__(256) void fp4_append_kernel(AppendArgs g, int32_t items) {
  __shared__ __attribute__((aligned(16))) char lds[4][2048 + 128];
  const int32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = blockIdx.y;
  const int32_t item = blockIdx.x * 4 + wave;
  if (item >= items) return;  // a wave's LDS is its own: there is no barrier to miss
  const int32_t page = item / g.blocks, b = item - page * g.blocks, t0 = b * kFp4Tokens, left = g.tpp - t0;
  char* block = g.layer_base + (uint64_t)g.slot[page] * g.slot_bytes + ((uint64_t)h * g.blocks + b) * kFp4Block;
  const uint64_t row = (uint64_t)g.heads * 128, src = ((uint64_t)page * g.tpp + t0) * row + (uint64_t)h * 128 + 8 * (lane & 15);
  if (blockIdx.z < 2) {
    const int32_t t1 = 16 * blockIdx.z + (lane >> 4);  // of pass i: token t1 + 4 i
    u32x4 k[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int32_t t = t1 + 4 * i;
      k[i] = u32x4{};
      if (t < left) k[i] = *reinterpret_cast<const u32x4u*>(g.k + src + t * row);
    }
    if constexpr (ROPE) {
      // the rotations of this lane's channel pairs: the axis and its table are fixed, the
      // position changes with the token; all are out before the first is used
      const float2* table[4];
      int32_t ax[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int32_t p = 4 * (lane & 15) + j;
        ax[j] = p < g.pairs_t ? 0 : p < g.pairs_t + g.pairs_h ? 1 : 2;
        table[j] = g.table + (ax[j] == 0 ? (int64_t)(g.frame0 + page) * g.pairs_t + p
                              : ax[j] == 1 ? g.off_h + p - g.pairs_t : g.off_w + p - g.pairs_t - g.pairs_h);
      }
      float2 cs[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int32_t tok = min(t0 + t1 + 4 * i, g.tpp - 1);
        const int32_t hh = (int32_t)fast_div((uint32_t)tok, g.gw_div), ww = tok - hh * g.grid_w;
#pragma unroll
        for (int j = 0; j < 4; ++j) cs[i][j] = table[j][ax[j] == 0 ? 0 : ax[j] == 1 ? hh * g.pairs_h : ww * g.pairs_w];
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool there = t1 + 4 * i < left;  // behind the page's end zeros stay +0
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t w = k[i][j];
          const float x0 = __uint_as_float(w << 16), x1 = __uint_as_float(w & 0xffff0000u);
          // as the bf16 cache rotates and rounds them
          const uint32_t y = pack_bf16x2(fmaf(x0, cs[i][j].x, -(x1 * cs[i][j].y)), fmaf(x0, cs[i][j].y, x1 * cs[i][j].x));
          k[i][j] = there ? y : 0u;
        }
      }
    }
    pack_keys(k, blockIdx.z, block, lane);
    return;
  }
  u32x4 v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int32_t t = 8 * (lane >> 4) + i;
    v[i] = u32x4{};
    if (t < left) v[i] = *reinterpret_cast<const u32x4u*>(g.v + src + t * row);
  }
  char* stage = lds[wave];
#pragma unroll
  for (int j = 0; j < 8; ++j) {  // channel c = 8 (lane & 15) + j
    const int sel = j & 1;
    u32x4 x;
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t a = v[2 * e][j >> 1], c = v[2 * e + 1][j >> 1];
      x[e] = sel ? (a >> 16) | (c & 0xffff0000u) : (a & 0xffffu) | (c << 16);
      top = umax(top, bf16x2_top(x[e]));
    }
    u32x2 other = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(top, top, false, false));
    top = umax(other[0], other[1]);
    other = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(top, top, false, false));
    top = umax(other[0], other[1]);
    const uint32_t s = fp4_scale(top), c = 8 * (lane & 15) + j;
    *reinterpret_cast<uint32_t*>(stage + c * 16 + 4 * (lane >> 4)) = fp4_codes(x, s);
    if (lane < 16) stage[2048 + (c & 15) * 8 + (c >> 4)] = (char)s;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int i = 0; i < 2; ++i)
    *reinterpret_cast<u32x4*>(block + kFp4V + (i * 64 + lane) * 16) = *reinterpret_cast<const u32x4*>(stage + (i * 64 + lane) * 16);
  if (lane < 8)
    *reinterpret_cast<u32x4*>(block + kFp4VScale + lane * 16) = *reinterpret_cast<const u32x4*>(stage + 2048 + lane * 16);
}

int launch_fp4_append(const sc_cache* c, int32_t layer, const int32_t* slots, int32_t chunk, const void* k,
                      const void* v, const sc_rope* rope, hipStream_t stream) {
  const sc_cache_desc& d = c->d;
  AppendArgs g;
  std::memset(&g, 0, sizeof g);
  g.k = static_cast<const uint16_t*>(k);
  g.v = static_cast<const uint16_t*>(v);
  g.layer_base = c->pool + (size_t)layer * d.n_slots * c->slot_bytes;
  g.slot_bytes = c->slot_bytes;
  g.heads = d.n_heads;
  g.tpp = d.tokens_per_page;
  g.blocks = fp4_blocks(g.tpp);
  std::copy(slots, slots + d.pages_per_chunk, g.slot);
  if (rope) {
    const RopeLayout L = rope_layout(&rope->desc);
    g.table = static_cast<const float2*>(rope->dev_table);
    g.grid_w = rope->desc.grid_w;
    g.pairs_t = L.pairs_t;
    g.pairs_h = L.pairs_h;
    g.pairs_w = L.pairs_w;
    g.off_h = L.off_h;
    g.off_w = L.off_w;
    g.frame0 = chunk * d.pages_per_chunk;
    g.gw_div = magic_div((uint32_t)rope->desc.grid_w);
  }
  const int32_t items = d.pages_per_chunk * g.blocks;
  const dim3 grid((items + 3) / 4, d.n_heads, 3);
  timer_begin(TK_APPEND, stream);
  if (rope)
    hipLaunchKernelGGL(fp4_append_kernel<true>, grid, dim3(256), 0, stream, g, items);
  else
    hipLaunchKernelGGL(fp4_append_kernel<false>, grid, dim3(256), 0, stream, g, items);
  timer_end(TK_APPEND, stream);
  SC_HIP(hipGetLastError());
  return SC_OK;
}

}  // namespace sc
