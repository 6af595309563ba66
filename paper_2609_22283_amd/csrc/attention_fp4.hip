// Packed attention over pages held in 4 bits (their layout: fp4.h).
//
// For every pack node i and head h: O = softmax(Q K^T * scale) V over the keys of node i's
// pages, K and V the values that the codes stand for; q and o are bf16.
//
// The scaled matrix instructions take codes and their shared scales as a block holds them
// (fp4.h), so K and V are never taken apart: S^T = K Q^T and O^T = V^T P^T have them as the A
// operand, over 128 channels of four scales and over 128 keys of four blocks.  The other
// operand comes in 8 bits at most.  A bf16 number has 8 significant bits, which are two e4m3
// numbers of 4: q is split once per row, the exponentials of a chunk where they are made, and each
// product is two instructions, which is what 128 channels of bf16 cost as well (64 cycles of
// the matrix core), but without the codes' conversion, and over a quarter of the bytes in
// cache and registers.
#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>
#include <cstring>
#include <map>
#include <new>
#include <vector>

#include "attention_core.h"
#include "fp4.h"

namespace sc {

constexpr int64_t kFp4Groups = UINT32_MAX / 256;  // work-groups of a launch (256 threads each, numbered in 32 bits)

// A plan's pages (no more than attention_check lets through): the prefix that all nodes read first,
// then the nodes' own.
struct Fp4List {
  int32_t shared;
  int32_t off[kMaxNodes + 1];
  int32_t slot[kMaxPages];
};
struct Fp4Geom {
  const char* layer_base;
  uint64_t slot_bytes;
  int32_t heads, nodes, tpp, blocks, nq, rows;
  DivMagic blocks_div, nq_div;
  float unit;       // |scale| log2(e), a normal number
  uint32_t q_flip;  // sign bits of a negative scale
  // The items, first those of the prefix (none where the nodes read it by themselves, joined),
  // then the nodes' own: row tiles fastest, then heads, then (own) nodes, then pieces of so many
  // chunks.
  int32_t joined, p_items, p_tiles, p_pieces, p_len, o_tiles, o_len;
  float *part_o, *part_ml;  // [piece][head][row][128], [piece][head][row][2], or NULL: one piece
};

static size_t align256(size_t n) { return (n + 255) & ~size_t(255); }

static void fp4_fill(const sc_plan* p, const sc_cache* c, int32_t layer, float scale, Fp4List& l, Fp4Geom& g) {
  const sc_cache_desc& d = c->d;
  const int32_t n = (int32_t)p->nodes.size();
  std::memset(&l, 0, sizeof l);
  std::memset(&g, 0, sizeof g);
  l.shared = p->shared;
  std::copy(p->page_slot.begin(), p->page_slot.begin() + p->shared, l.slot);
  int32_t at = p->shared;
  for (int32_t i = 0; i < n; ++i) {
    l.off[i] = at;
    for (int32_t k = p->page_off[i] + p->shared; k < p->page_off[i + 1]; ++k) l.slot[at++] = p->page_slot[k];
  }
  for (int32_t i = n; i <= kMaxNodes; ++i) l.off[i] = at;
  g.layer_base = c->pool + (size_t)layer * d.n_slots * c->slot_bytes;
  g.slot_bytes = c->slot_bytes;
  g.heads = d.n_heads;
  g.nodes = n;
  g.rows = n * p->nq;
  g.tpp = d.tokens_per_page;
  g.blocks = fp4_blocks(d.tokens_per_page);
  g.nq = p->nq;
  g.blocks_div = magic_div((uint32_t)g.blocks);
  g.nq_div = magic_div((uint32_t)p->nq);
  g.unit = std::min(std::max(std::fabs(scale) * 1.4426950408889634f, FLT_MIN), FLT_MAX);
  g.q_flip = std::signbit(scale) ? 0x80008000u : 0u;
}

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));

constexpr float kFp4Rise = 40.f;  // sums of 2^31 keys in units of 2^m stay below 2^(40 + 31)
constexpr float kFp4Far = 4194304.f;  // 2^22: steps of fp32 below it are a quarter at most
constexpr int FA_ROW = 132;   // floats of a row of partial outputs in LDS

// The scaled instruction's operands: c + A B over 128: A 16 rows of codes (a lane: row lane % 16, the 32 columns of group lane / 16)
// whose scales are byte SA of the lanes' sa, B 16 columns of e4m3 (a lane: column lane % 16, rows 16 g ..
// + 15 and 64 + 16 g .. + 15 with g = lane / 16), in two parts with their scales in the first two
// bytes of sb.
template <int SA>
__device__ __forceinline__ f32x4 mx(const u32x4& a, const i32x8& hi, const i32x8& lo, const f32x4& c, uint32_t sa, uint32_t sb) {
  const i32x8 a8 = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  const f32x4 d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, hi, c, 4, 0, SA, (int)sa, 0, (int)sb);
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, lo, d, 4, 0, SA, (int)sa, 1, (int)sb);
}

__device__ __forceinline__ i32x8 join(const u32x4& a, const u32x4& b) {
  return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
}

// The largest of the values of lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ float quarters_max(float x) {
  u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// Four fp32 numbers of at most 448 as e4m3, and what that leaves of them, over `unit` (a power of
// two), in e4m3 again: 8 significant bits together, which is all that bf16 has, and half a step
// 2^-9 of the number.  One e4m3 number alone (half a step 2^-4) would take half of the
// products, and leave outputs with the error of a format that the caller did not choose.
__device__ __forceinline__ void split_e4m3(float a, float b, float c, float d, float unit, int& hi, int& lo) {
  int h, y;  // the conversions write half a register at a time: whatever is in it first
  asm volatile("" : "=v"(h));
  asm volatile("" : "=v"(y));
  h = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, h, false);
  h = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, h, true);
  const f32x2 ab = __builtin_amdgcn_cvt_pk_f32_fp8(h, false), cd = __builtin_amdgcn_cvt_pk_f32_fp8(h, true);
  i16x2 l = __builtin_bit_cast(i16x2, y);
  l = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(l, a - ab[0], b - ab[1], unit, false);
  l = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(l, c - cd[0], d - cd[1], unit, true);
  hi = h;
  lo = __builtin_bit_cast(int, l);
}

// 16 query rows as the B operand, in two parts with a scale each.
struct Fp4Rows {
  i32x8 hi, lo;
  uint32_t scale;  // of hi, of lo << 8
};
__device__ __forceinline__ Fp4Rows load_rows(const uint16_t* row, int32_t quarter, uint32_t flip) {
  u32x4 v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const u32x4*>(row + 64 * (i >> 1) + 16 * quarter + 8 * (i & 1));
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      top = umax(top, bf16x2_top(v[i][j]));
      v[i][j] ^= flip;
    }
  top = umax(top, (uint32_t)__shfl_xor((int)top, 16));
  top = umax(top, (uint32_t)__shfl_xor((int)top, 32));
  const uint32_t e = top >> 23, s = e > 7u ? e - 7u : 0u;  // the largest becomes 2^7 .. 2^8
  const float by = __uint_as_float((e > 7u ? 261u - e : 254u) << 23);
  Fp4Rows r;
  const uint32_t s_lo = s > 4u ? s - 4u : 0u;
  r.scale = (e == 255u ? 255u : s) | s_lo << 8;
  const float unit = __uint_as_float((127u + s_lo - s) << 23);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t a = v[i >> 1][2 * (i & 1)], b = v[i >> 1][2 * (i & 1) + 1];
    int h, l;
    split_e4m3(__uint_as_float(a << 16) * by, __uint_as_float(a & 0xffff0000u) * by, __uint_as_float(b << 16) * by,
               __uint_as_float(b & 0xffff0000u) * by, unit, h, l);
    r.hi[i] = e == 255u ? 0 : h;
    r.lo[i] = e == 255u ? 0 : l;
  }
  return r;
}

// What a work-group does: rows [row0, row0 + rows) of a head over the chunks [c0, c1) of 128
// keys (four blocks) of a list of pages; `slot` its place among the partials.
struct Fp4Item {
  int32_t head, row0, rows, node, pages, first, blocks, c0, c1, slot;
};
template <int R>
__device__ __forceinline__ Fp4Item fp4_item(const Fp4Geom& g, const Fp4List& list, int32_t b) {
  Fp4Item it;
  const bool prefix = b < g.p_items;
  const int32_t tiles = prefix ? g.p_tiles : g.o_tiles;
  if (!prefix) b -= g.p_items;
  const int32_t tile = b % tiles;
  b /= tiles;
  it.head = b % g.heads;
  b /= g.heads;
  it.node = prefix ? 0 : b % g.nodes;
  const int32_t piece = prefix ? b : b / g.nodes, len = prefix ? g.p_len : g.o_len;
  it.row0 = (prefix ? 0 : it.node * g.nq) + tile * 16 * R;
  it.rows = min(16 * R, (prefix ? g.rows : g.nq) - tile * 16 * R);
  it.first = prefix ? 0 : list.off[it.node];
  it.pages = prefix ? list.shared : list.off[it.node + 1] - it.first + (g.joined ? list.shared : 0);
  it.blocks = it.pages * g.blocks;
  it.c0 = piece * len;
  it.c1 = min(it.c0 + len, (it.blocks + 3) / 4);
  it.slot = prefix ? piece : g.p_pieces + piece;
  return it;
}

// A work-group has 16 R rows of a head; its NW waves take every NW-th chunk of 128 keys, each
// with a softmax of its own (running power of two, sums, outputs), and join them in LDS at the
// end.  Nothing is shared between the waves' loops, so there is no barrier in them:
// K and V go from the cache straight to the registers that the products read, K of the next
// chunk under the exponentials of this one, V in K's registers.  The rows' sums come from one
// more product, with ones, which has the exponentials as they were rounded.
//
// What bounds it: single tokens, reading the pages (16 x 16384 keys x 12 heads, 428 MB, 72.8
// us, 5.9 TB/s); many rows, the vector unit, busy for 75 % of the time with 28 cycles for
// each exponential and its two parts and 16 for each of the products' issue, the matrix core for
// half of it (four nodes of 4680 rows over 21 x 1560 keys 3.28 ms, 1148 TFLOP/s, in tiles of 32
// rows: the products of one half of the rows stand between the exponentials of the other; 3.54 ms and
// 1064 in tiles of 16, whose work-groups are three to a CU).  Tried on the same nodes: 32x32x64
// products of 64 keys 3.66 ms, with their loads further ahead 3.71; the waves on rows of their
// own, 128 in all, over the same keys 3.25, but slower at every shorter one (58 us become 144 at
// four nodes of 256 rows); the blocks' addresses on the scalar unit, no change.
template <int R, int NW>
__global__ __launch_bounds__(64 * NW, R == 1 && NW == 4 ? 3 : 2) void fp4_attention_kernel(
    const uint16_t* __restrict__ q, uint16_t* __restrict__ o, Fp4Geom g, Fp4List list) {
  __shared__ __attribute__((aligned(16))) float part[NW][16 * FA_ROW];
  __shared__ float ml[NW][2][16];
  __shared__ uint64_t base[kMaxPages];
  __shared__ u32x4 qs[R][4][64];         // the queries' operands: halves of hi, halves of lo
  __shared__ uint32_t q_scale[R][16];
  const int32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Fp4Item it = fp4_item<R>(g, list, (int32_t)xcd_remap(blockIdx.x, gridDim.x));
  if (it.c0 >= it.c1) return;
  const int32_t j0 = 4 * it.c0 / g.blocks, j1 = min(it.pages, (4 * it.c1 + g.blocks - 1) / g.blocks);
  for (int32_t j = j0 + (int32_t)threadIdx.x; j < j1; j += 64 * NW) {
    const int32_t s = !g.joined ? it.first + j : j < list.shared ? j : it.first + j - list.shared;
    base[j - j0] = (uint64_t)list.slot[s] * g.slot_bytes + (uint64_t)it.head * g.blocks * kFp4Block;
  }
  if (wave < R) {
    const Fp4Rows x = load_rows(q + ((size_t)(it.row0 + min(16 * wave + (lane & 15), it.rows - 1)) * g.heads + it.head) * 128,
                                lane >> 4, g.q_flip);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      qs[wave][i][lane] = u32x4{(uint32_t)x.hi[4 * i], (uint32_t)x.hi[4 * i + 1], (uint32_t)x.hi[4 * i + 2], (uint32_t)x.hi[4 * i + 3]};
      qs[wave][2 + i][lane] = u32x4{(uint32_t)x.lo[4 * i], (uint32_t)x.lo[4 * i + 1], (uint32_t)x.lo[4 * i + 2], (uint32_t)x.lo[4 * i + 3]};
    }
    if (lane < 16) q_scale[wave][lane] = x.scale;
  }
  __syncthreads();
  const auto block_at = [&](int32_t b) {
    b = min(b, it.blocks - 1);
    const int32_t j = (int32_t)fast_div((uint32_t)b, g.blocks_div);
    return g.layer_base + base[j - j0] + (uint32_t)(b - j * g.blocks) * kFp4Block;
  };
  const auto tokens_of = [&](int32_t b) {  // keys of a block
    const int32_t j = (int32_t)fast_div((uint32_t)min(b, it.blocks - 1), g.blocks_div);
    return b < it.blocks ? g.tpp - (b - j * g.blocks) * kFp4Tokens : 0;
  };
  // K rows: row 4 x + i of product b is token 16 (x % 2) + 4 (b % 4) + i of the chunk's block
  // 2 (b / 4) + x / 2, so that the rows a lane gets of S^T (x = lane / 16) are the columns it
  // has to give of P^T
  const uint32_t k_at = (lane >> 2 & 1) * 256 + (lane >> 4) * 64 + (lane & 3) * 16;
  const uint32_t ks_at = kFp4KScale + (lane >> 2 & 1) * 64 + (lane & 3) * 16 + (lane >> 4) * 4;
  const uint32_t v_at = kFp4V + (lane & 15) * 16, vs_at = kFp4VScale + (lane & 15) * 8;
  const bool ragged = (g.tpp & 31) != 0 || (it.blocks & 3) != 0;

  f32x4 acc[R][8], sum[R];  // sum: of a row's exponentials, as they enter the products
  float m[R];
  uint32_t qsc[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = -INFINITY;
    sum[r] = f32x4{};
    qsc[r] = q_scale[r][lane & 15];
#pragma unroll
    for (int n = 0; n < 8; ++n) acc[r][n] = f32x4{};
  }
  const u32x4 ones = {0x22222222u, 0x22222222u, 0x22222222u, 0x22222222u};
  u32x4 k[8];
  uint32_t ks[2];
  const auto load_k = [&](int32_t c) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const char* p = block_at(4 * c + 2 * h + (lane >> 3 & 1));
#pragma unroll
      for (int i = 0; i < 4; ++i) k[4 * h + i] = *reinterpret_cast<const u32x4*>(p + k_at + 512 * i);
      ks[h] = *reinterpret_cast<const uint32_t*>(p + ks_at);
    }
  };
  if (it.c0 + wave < it.c1) load_k(it.c0 + wave);
  for (int32_t c = it.c0 + wave; c < it.c1; c += NW) {
    bool cut = false;  // a block of the chunk ends early, or is not there
    int32_t left[2];
    if (ragged) {
      left[0] = tokens_of(4 * c + (lane >> 5)) - 16 * (lane >> 4 & 1);
      left[1] = tokens_of(4 * c + 2 + (lane >> 5)) - 16 * (lane >> 4 & 1);
      cut = __any(min(left[0], left[1]) < 16);
    }
    i32x8 hi[R], lo[R];
    uint32_t psc[R];
    u32x4 v[8];
    u32x2 vs;
    const auto load_v = [&]() __attribute__((always_inline)) {
      const char* vp = block_at(4 * c + (lane >> 4));
#pragma unroll
      for (int n = 0; n < 8; ++n) v[n] = *reinterpret_cast<const u32x4*>(vp + v_at + 256 * n);
      vs = *reinterpret_cast<const u32x2*>(vp + vs_at);
    };
    const auto logits = [&](int r, f32x4 (&s)[8]) __attribute__((always_inline)) {
      const f32x4 zero = {};
      const i32x8 q_hi = join(qs[r][0][lane], qs[r][1][lane]), q_lo = join(qs[r][2][lane], qs[r][3][lane]);
#define SC_QK(b) s[b] = mx<(b) & 3>(k[b], q_hi, q_lo, zero, ks[(b) >> 2], qsc[r])
      SC_QK(0); SC_QK(1); SC_QK(2); SC_QK(3); SC_QK(4); SC_QK(5); SC_QK(6); SC_QK(7);
#undef SC_QK
    };
    // what the exponentials of a chunk are relative to: a power of two no less than its
    // largest, 2^8 of it, which is a change of the scale of P alone.  The row's sums are
    // in units of 2^m, m the first chunk's power until one is far above it (were m to follow
    // every rise, some row of 16 would have its sums multiplied in most chunks).
    const auto shift_of = [&](int r, f32x4 (&s)[8]) __attribute__((always_inline)) {
      if (cut) {
#pragma unroll
        for (int b = 0; b < 8; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (4 * (b & 3) + i >= left[b >> 2]) s[b][i] = -INFINITY;
      }
      float top = s[0][0];
#pragma unroll
      for (int b = 0; b < 8; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[b][i]);
      top = quarters_max(top);
      const float t = top * g.unit, e = fmaxf(ceilf(t), -FLT_MAX);
      float shift = 8.f - e;
      if (__any(e - m[r] > kFp4Rise || fabsf(t) > kFp4Far)) {
        const float to = fmaxf(m[r], e), keep = __builtin_amdgcn_exp2f(m[r] - to);
        sum[r] *= keep;
#pragma unroll
        for (int n = 0; n < 8; ++n) acc[r][n] *= keep;
        m[r] = to;
        // From there on neither 8 - e nor how far t is below e is exact enough for exponentials of
        // 2^8 at most: the logits' distances from the chunk's largest are (which counts as the
        // fp32 number t, 2^-24 of it).  Without a number for t, above them all, the rows are NaN, and
        // below them all the chunk has no weight.
        const bool far = fabsf(t) > kFp4Far;
        const float from = far && top > -INFINITY ? top : 0.f;
        if (far) shift = 8.f - (e - t);
#pragma unroll
        for (int b = 0; b < 8; ++b) s[b] -= from;
      }
      const int32_t d = (int32_t)fminf(fmaxf(e - m[r], -300.f), 100.f);
      psc[r] = (uint32_t)max(d + 119, 0) | (uint32_t)max(d + 115, 0) << 8;
      return shift;
    };
    const auto exponentials = [&](int r, f32x4 (&s)[8], float shift) __attribute__((always_inline)) {
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(s[b][i], g.unit, shift));
        int h, l;
        split_e4m3(p[0], p[1], p[2], p[3], 0.0625f, h, l);
        asm volatile("" : "+v"(h), "+v"(l));  // here, and not where the products need them
        hi[r][b] = h;
        lo[r][b] = l;
      }
    };
    const auto products = [&](int r) __attribute__((always_inline)) {
#define SC_PV(n) acc[r][n] = mx<(n) & 3>(v[n], hi[r], lo[r], acc[r][n], vs[(n) >> 2], psc[r])
      SC_PV(0); SC_PV(1); SC_PV(2); SC_PV(3); SC_PV(4); SC_PV(5); SC_PV(6); SC_PV(7);
#undef SC_PV
      sum[r] = mx<0>(ones, hi[r], lo[r], sum[r], 0x7f7f7f7fu, psc[r]);
    };
    const int32_t next = c + NW < it.c1 ? c + NW : c;  // at the end the same again: no branch
    f32x4 s0[8];
    logits(0, s0);
    if constexpr (R == 1) {
      __builtin_amdgcn_sched_barrier(0);  // V takes the registers of K, whose last product this was
      load_v();
      exponentials(0, s0, shift_of(0, s0));
      __builtin_amdgcn_sched_barrier(0);
      load_k(next);
      __builtin_amdgcn_sched_barrier(0);
      products(0);
    } else {
      // the products of one half of the rows run under the exponentials of the other
      f32x4 s1[8];
      float shift = shift_of(0, s0);
      __builtin_amdgcn_sched_barrier(0);
      logits(1, s1);
      exponentials(0, s0, shift);
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 10, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
      load_v();
      shift = shift_of(1, s1);
      __builtin_amdgcn_sched_barrier(0);
      load_k(next);
      exponentials(1, s1, shift);
      products(0);
      __builtin_amdgcn_sched_group_barrier(0x020, 10, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, 40, 0);
#pragma unroll
      for (int i = 0; i < 18; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 8, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
      products(1);
    }
  }
  // the waves' parts of 16 rows at a time: thread t has eight channels of row t / 16
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (16 * r >= it.rows) break;
    if (r) __syncthreads();
#pragma unroll
    for (int n = 0; n < 8; ++n)
      *reinterpret_cast<f32x4*>(&part[wave][(lane & 15) * FA_ROW + 16 * n + 4 * (lane >> 4)]) = acc[r][n];
    if (lane < 16) {
      ml[wave][0][lane] = m[r];
      ml[wave][1][lane] = sum[r][0];
    }
    __syncthreads();
    const int32_t x = threadIdx.x >> 4, ch = 8 * (threadIdx.x & 15), row = it.row0 + 16 * r + x;
    if (x < 16 && 16 * r + x < it.rows) {
      float to = ml[0][0][x];
#pragma unroll
      for (int w = 1; w < NW; ++w) to = fmaxf(to, ml[w][0][x]);
      f32x4 y[2] = {};
      float l = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float keep = exp2f(ml[w][0][x] - to);
        l += keep * ml[w][1][x];
        y[0] += keep * *reinterpret_cast<const f32x4*>(&part[w][x * FA_ROW + ch]);
        y[1] += keep * *reinterpret_cast<const f32x4*>(&part[w][x * FA_ROW + ch + 4]);
      }
      if (g.part_o) {
        const size_t at = ((size_t)it.slot * g.heads + it.head) * g.rows + row;
        *reinterpret_cast<f32x4*>(g.part_o + at * 128 + ch) = y[0];
        *reinterpret_cast<f32x4*>(g.part_o + at * 128 + ch + 4) = y[1];
        if (ch == 0) {
          g.part_ml[2 * at] = to;
          g.part_ml[2 * at + 1] = l;
        }
      } else {
        const float by = 1.f / l;
        u32x4 z;
        z[0] = pack_bf16x2(y[0][0] * by, y[0][1] * by);
        z[1] = pack_bf16x2(y[0][2] * by, y[0][3] * by);
        z[2] = pack_bf16x2(y[1][0] * by, y[1][1] * by);
        z[3] = pack_bf16x2(y[1][2] * by, y[1][3] * by);
        *reinterpret_cast<u32x4u*>(o + ((size_t)row * g.heads + it.head) * 128 + ch) = z;
      }
    }
  }
}

// A wave per row and head joins the pieces that its node has, the prefix's and its own, N at
// a time, whose loads are independent: four, or eight of more pieces (one row over 16384 keys in
// 12 pieces 11.1 us in all, 11.5 four at a time; 256 rows in four 37.8, 38.6 by eight).  Bound by
// latency, then by the partials: 4 us for 256 rows of 12 heads in four pieces (6.4 MB).
template <int N>
__global__ __launch_bounds__(256) void fp4_combine_kernel(uint16_t* __restrict__ o, Fp4Geom g, Fp4List list) {
  const int32_t lane = threadIdx.x & 63, row = blockIdx.x * 4 + (threadIdx.x >> 6), h = blockIdx.y;
  if (row >= g.rows) return;
  const int32_t node = (int32_t)fast_div((uint32_t)row, g.nq_div);
  const int32_t blocks = (list.off[node + 1] - list.off[node] + (g.joined ? list.shared : 0)) * g.blocks;
  const int32_t pieces = g.p_pieces + ((blocks + 3) / 4 + g.o_len - 1) / g.o_len;
  const size_t step = (size_t)g.heads * g.rows, at = (size_t)h * g.rows + row;
  float m = -INFINITY, l = 0.f, y[2] = {0.f, 0.f};
  for (int32_t p = 0; p < pieces; p += N) {
    f32x2 x[N], ml[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const size_t from = (size_t)min(p + i, pieces - 1) * step + at;
      ml[i] = *reinterpret_cast<const f32x2*>(g.part_ml + 2 * from);
      x[i] = *reinterpret_cast<const f32x2*>(g.part_o + from * 128 + 2 * lane);
    }
    float to = m;
#pragma unroll
    for (int i = 0; i < N; ++i) to = fmaxf(to, ml[i][0]);  // past the end the last one again
    const float keep = __builtin_amdgcn_exp2f(m - to);
    m = to;
    l *= keep;
    y[0] *= keep;
    y[1] *= keep;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (p + i < pieces) {
        const float by = __builtin_amdgcn_exp2f(ml[i][0] - to);
        l = fmaf(by, ml[i][1], l);
        y[0] = fmaf(by, x[i][0], y[0]);
        y[1] = fmaf(by, x[i][1], y[1]);
      }
  }
  const float by = 1.f / l;
  *reinterpret_cast<uint32_t*>(o + ((size_t)row * g.heads + h) * 128 + 2 * lane) = pack_bf16x2(y[0] * by, y[1] * by);
}

// The same attention over bf16 pages: a plan over a cache of its distinct pages alone, which are
// taken out of their 4 bits into the workspace first.
struct Fp4Wide {
  sc_cache cache;
  sc_plan plan;
  std::vector<int32_t> src, dst;  // slots that are taken out, and where to
  size_t page_bytes = 0;
};

// How a plan runs within so many bytes of workspace.
struct Fp4Schedule {
  size_t room = 0;
  std::shared_ptr<Fp4Wide> wide;  // over bf16 pages; else by tiles of so many rows:
  int32_t tile = 16, waves = 4;
  int32_t joined = 1, p_len = 1, p_pieces = 0, o_len = 1, o_pieces = 1;  // chunks of a piece, pieces (own: the most of a node)
  size_t bytes = 0;
  double us = 1e30;
};

static int64_t fp4_chunks(const sc_cache* c, int64_t pages) {
  return (pages * fp4_blocks(c->d.tokens_per_page) + 3) / 4;
}

// NULL where the bf16 kernels do not take the plan (their pages hold a key tile).
static std::shared_ptr<Fp4Wide> fp4_wide(const sc_plan* p, const sc_cache* c) {
  if (c->d.tokens_per_page < (p->shared || p->nq <= 64 ? 32 : 64)) return nullptr;
  auto w = std::make_shared<Fp4Wide>();
  const auto last = std::max_element(p->page_slot.begin(), p->page_slot.end());
  std::vector<int32_t> place(last == p->page_slot.end() ? 0 : *last + 1, -1);
  const auto put = [&](int32_t s) {
    if (place[s] < 0) {
      place[s] = (int32_t)w->src.size();
      w->src.push_back(s);
      w->dst.push_back(place[s]);
    }
    return place[s];
  };
  w->plan.page_slot.reserve(p->page_slot.size());
  for (size_t i = 0; i + 1 < p->page_off.size(); ++i) {
    size_t k = p->page_off[i];
    for (int32_t s = 0; i && s < p->shared; ++s, ++k) w->plan.page_slot.push_back(w->plan.page_slot[s]);
    for (; k < (size_t)p->page_off[i + 1]; ++k) w->plan.page_slot.push_back(put(p->page_slot[k]));
  }
  w->cache.d = c->d;
  w->cache.d.dtype = SC_DTYPE_BF16;
  w->cache.d.n_layers = 1;
  w->cache.d.n_slots = (int32_t)w->src.size();
  w->cache.pool = nullptr;
  w->cache.slot_bytes = 4ull * c->d.n_heads * c->d.tokens_per_page * 128;
  w->cache.kv_half = w->cache.slot_bytes / 2;
  w->page_bytes = w->src.size() * w->cache.slot_bytes;
  w->plan.nodes = p->nodes;
  w->plan.page_off = p->page_off;
  if (p->page_slot.size() <= (size_t)kMaxPages) w->plan.page_state = p->page_state;  // of lists that one launch reads whole
  w->plan.cache = &w->cache;
  w->plan.nq = p->nq;
  w->plan.shared = p->shared;
  return attention_check(&w->plan, &w->cache) == SC_OK ? w : nullptr;
}

// The time in us at which `slots` work-groups at once have done items of the given number
// and time each, dealt out in this order.
struct Fp4Items {
  double count, us;
};
static double fp4_makespan(double slots, const std::vector<Fp4Items>& items) {
  std::vector<std::pair<double, double>> level{{0.0, slots}};  // from this time on, so many slots
  double end = 0.0;
  for (const Fp4Items& it : items)
    for (double left = it.count; left > 0;) {
      std::sort(level.begin(), level.end());
      if (left >= 2 * slots && level.back().first - level.front().first <= it.us) {  // whole rounds move all alike
        const double rounds = std::floor(left / slots) - 1;
        for (auto& l : level) l.first += rounds * it.us;
        left -= rounds * slots;
      }
      const double at = level.front().first + it.us, take = std::min(left, level.front().second);
      end = std::max(end, at);
      left -= take;
      level.front().second -= take;
      if (level.front().second <= 0) level.erase(level.begin());
      auto same = std::find_if(level.begin(), level.end(), [&](const auto& l) { return std::fabs(l.first - at) < 1e-3; });
      if (same != level.end())
        same->second += take;
      else
        level.emplace_back(at, take);
    }
  return end;
}

// The cheapest way within `room` bytes, by estimated time in us.  Measured (2 .. 12 heads, 1 ..
// 1024 rows a node, 512 .. 262144 keys, 2000 ways of cutting them; what is chosen is within
// 6 % of the best of them): four chunks, one to each wave of a work-group, take
//   tiles of 16 rows  1.45 with one work-group to a CU, 2.0 with two, 3.05 with three
//   tiles of 32 rows  2.3 with one, 3.75 with two
// and eight chunks, one to each of eight waves, of which a CU has room for one work-group, 2.1
// (the last four or fewer 1.45).  An item is 1 more, 1.6 with eight waves, a launch 3, no less
// than the pages take from HBM at 5.6 MB per us; joining pieces 3.5, 0.13 per piece and the
// partials at 2.2 MB per us.  So nodes that fill their tiles
// read a shared prefix each by itself (sixteen of 16 rows over 128 x 128 keys 38 us, 49 with
// the rows of all nodes in one matrix; 32 of one row over 256 x 64 keys 26 against 20), and
// where there are fewer work-groups than CUs, eight waves take what four would over more
// pieces (256 rows over 17 x 512 keys 21.6 us, 25.3; one frame of 64 rows over 21 x 64 8.5,
// 9.2; one row over 8 x 64 keys 6.6, 6.3).
// Over bf16 pages: the time of that attention, 8 and 0.17 per MB of them (four nodes of 4680
// rows over 21 x 1560 keys 2.94 to 3.07 ms, 3.28 by tiles; four of 256 over 21 x 256 59 us, 41 by
// tiles): 32 rows read K and V from cache once, 256 of the bf16 form's eight waves.
static Fp4Schedule find_fp4_schedule(const sc_plan* p, const sc_cache* c, size_t room) {
  const int32_t n = (int32_t)p->nodes.size(), H = c->d.n_heads;
  const int64_t rows = (int64_t)n * p->nq;
  std::map<int64_t, int32_t> own;  // pages of a node's own, and nodes with so many
  int64_t own_all = 0;
  for (int32_t i = 0; i < n; ++i) {
    const int64_t pages = p->page_off[i + 1] - p->page_off[i] - p->shared;
    ++own[pages];
    own_all += pages;
  }
  const int64_t own_max = own.rbegin()->first;
  Fp4Schedule best;
  best.room = room;
  const int64_t piece = rows * H * (128 + 2) * (int64_t)sizeof(float);
  const double from_hbm = (double)(p->shared + own_all) * c->slot_bytes / 5.6e6;
  const int64_t prefix = fp4_chunks(c, p->shared);
  std::vector<Fp4Items> items;
  struct Form {
    int32_t tile, waves;
  };
  for (const auto [tile, waves] : {Form{16, 4}, Form{16, 8}, Form{32, 4}})
    for (const int32_t joined : {1, 0}) {
      if (!joined && !p->shared) continue;
      const int64_t own_tiles = (int64_t)H * ((p->nq + tile - 1) / tile), p_tiles = (int64_t)H * ((rows + tile - 1) / tile);
      const int64_t own_chunks = fp4_chunks(c, own_max + (joined ? p->shared : 0)), cut = std::max(own_chunks, joined ? 0 : prefix);
      for (int64_t pieces = 1, last = 0; pieces <= std::min<int64_t>(cut, 256); pieces += 1 + pieces / 8) {
        const int64_t len = (cut + pieces - 1) / pieces, o_len = std::min(len, own_chunks), p_len = joined ? 1 : std::min(len, prefix);
        if (len == last) continue;
        last = len;
        Fp4Schedule s;
        s.room = room;
        s.tile = tile;
        s.waves = waves;
        s.joined = joined;
        s.o_len = (int32_t)o_len;
        s.o_pieces = (int32_t)((own_chunks + o_len - 1) / o_len);
        if (!joined) {
          s.p_len = (int32_t)p_len;
          s.p_pieces = (int32_t)((prefix + p_len - 1) / p_len);
        }
        const int64_t all = s.p_pieces + s.o_pieces;
        if (all > 1 && ((double)all * piece > (double)room || rows > 4 * kFp4Groups)) break;
        s.bytes = all > 1 ? (size_t)(all * piece) : 0;
        items.clear();
        double total = 0;
        const auto add = [&](double units, int64_t chunks, int64_t of) {
          if (chunks >= of) items.push_back({units * (double)(chunks / of), (double)of});
          if (chunks % of) items.push_back({units, (double)(chunks % of)});
          total += units * (double)((chunks + of - 1) / of);
        };
        if (!joined) add((double)p_tiles, prefix, p_len);
        for (const auto& o : own) add((double)own_tiles * o.second, fp4_chunks(c, o.first + (joined ? p->shared : 0)), o_len);
        if (total > (double)kFp4Groups) continue;
        const int32_t per = total <= kCUs || waves == 8 ? 1 : total <= 2 * kCUs || tile == 32 ? 2 : 3;  // work-groups to a CU
        const auto step = [&](int32_t k) { return tile == 32 ? (k == 1 ? 2.3 : 3.75) : k == 1 ? 1.45 : k == 2 ? 2.0 : 3.05; };
        // items of a last round that leaves a CU fewer work-groups run as those do
        const double rest = std::fmod(total, (double)kCUs * per);
        const int32_t rest_per = std::max(1, (int32_t)std::ceil(rest / kCUs));
        const size_t at_full = items.size();
        if (rest > 0 && rest < total && rest_per < per) {
          items.push_back({std::min(rest, items.back().count), items.back().us});
          items[at_full - 1].count -= items.back().count;
        }
        for (size_t i = 0; i < items.size(); ++i) {  // from chunks to us
          const double n = items[i].us, left = std::fmod(n, 8.0), one = step(i < at_full ? per : rest_per);
          items[i].us = waves == 4 ? std::ceil(n / 4) * one + 1.0
                                   : std::floor(n / 8) * 2.1 + (left > 4 ? 2.1 : left > 0 ? one : 0.0) + 1.6;
        }
        s.us = std::max(fp4_makespan((double)kCUs * per, items), from_hbm) + 3.0;
        if (s.bytes) s.us += 3.5 + 0.13 * (double)all + (double)s.bytes / 2.2e6;
        if (s.us < best.us) best = s;
      }
    }
  // no less than the products at 1400 TFLOP/s and the longest list's pages taken out
  double flops = 0;
  for (const auto& o : own) flops += 512.0 * p->nq * H * (double)(o.first + p->shared) * c->d.tokens_per_page * o.second;
  const double least = 8.0 + flops / 1.4e9 + 0.17e-6 * 512.0 * H * c->d.tokens_per_page * (double)(own_max + p->shared);
  if (auto w = least < best.us ? fp4_wide(p, c) : nullptr) {
    const size_t bytes = align256(w->page_bytes) + attention_exact_workspace_bytes(&w->plan, &w->cache);
    const double us = attention_exact_us(&w->plan, &w->cache) + 8.0 + 0.17e-6 * (double)w->page_bytes;
    if (bytes <= room && us < best.us) {
      best.wide = w;
      best.bytes = bytes;
      best.us = us;
    }
  }
  return best;
}

// Found once per plan, for any room, the no-allocation call's and a block's.
static const Fp4Schedule* fp4_schedule(const sc_plan* p, const sc_cache* c, size_t room) {
  for (const auto& s : p->fp4)
    if (s->room == room) return s.get();
  try {
    p->fp4.push_back(std::make_shared<Fp4Schedule>(find_fp4_schedule(p, c, room)));
  } catch (const std::bad_alloc&) {
    return nullptr;
  }
  return p->fp4.back().get();
}

size_t fp4_attention_workspace_bytes(const sc_plan* p, const sc_cache* c) {
  const Fp4Schedule* s = fp4_schedule(p, c, SIZE_MAX);
  return s ? s->bytes : 0;
}

int launch_fp4_attention(const sc_plan* p, const sc_cache* c, int32_t layer, const void* q, void* o, float scale,
                         void* ws, size_t room, hipStream_t stream) {
  if (!std::isfinite(scale)) return fail(SC_EINVAL, "scale must be finite");
  if (reinterpret_cast<uintptr_t>(q) & 15) return fail(SC_EINVAL, "q must be 16-byte aligned");
  if (reinterpret_cast<uintptr_t>(ws) & 15) return fail(SC_EINVAL, "workspace must be 16-byte aligned");
  const int64_t rows = (int64_t)p->nodes.size() * p->nq;
  if (rows > INT32_MAX) return fail(SC_EUNSUPPORTED, "%lld query rows", (long long)rows);
  const Fp4Schedule* s = fp4_schedule(p, c, SIZE_MAX);
  if (s && s->bytes > room) s = fp4_schedule(p, c, room);
  if (!s) return fail(SC_EINVAL, "out of host memory");
  if (s->wide) {
    Fp4Wide& w = *s->wide;
    w.cache.pool = static_cast<char*>(ws);
    const PagePairs pairs{w.src.data(), w.dst.data(), (int32_t)w.src.size()};
    const int rc = launch_page_convert(false, PoolView{c->pool + (size_t)layer * c->d.n_slots * c->slot_bytes, 0},
                                       PoolView{w.cache.pool, 0}, c->d, pairs, 1, stream);
    if (rc != SC_OK) return rc;
    // times log2(e) it has to be a number, or rows of zeros come out NaN
    const float by = std::min(std::max(scale, -2.35e38f), 2.35e38f);
    return launch_attention_exact(&w.plan, &w.cache, 0, q, o, by, w.cache.pool + align256(w.page_bytes), stream);
  }
  Fp4List l;
  Fp4Geom g;
  fp4_fill(p, c, layer, scale, l, g);
  g.joined = s->joined;
  g.o_tiles = (p->nq + s->tile - 1) / s->tile;
  g.o_len = s->o_len;
  if (!s->joined) {
    g.p_tiles = (g.rows + s->tile - 1) / s->tile;
    g.p_pieces = s->p_pieces;
    g.p_len = s->p_len;
    g.p_items = g.p_tiles * g.heads * g.p_pieces;
  }
  const int64_t items = (int64_t)g.p_items + (int64_t)g.o_tiles * g.heads * g.nodes * s->o_pieces;
  if (items > kFp4Groups) return fail(SC_EUNSUPPORTED, "%lld query tiles", (long long)items);
  if (s->bytes) {
    g.part_o = static_cast<float*>(ws);
    g.part_ml = g.part_o + (size_t)(g.p_pieces + s->o_pieces) * g.heads * g.rows * 128;
  }
  const uint16_t* qb = static_cast<const uint16_t*>(q);
  uint16_t* ob = static_cast<uint16_t*>(o);
  timer_begin(TK_ATTENTION, stream);
  if (s->waves == 8)
    hipLaunchKernelGGL((fp4_attention_kernel<1, 8>), dim3((uint32_t)items), dim3(512), 0, stream, qb, ob, g, l);
  else if (s->tile == 16)
    hipLaunchKernelGGL((fp4_attention_kernel<1, 4>), dim3((uint32_t)items), dim3(256), 0, stream, qb, ob, g, l);
  else
    hipLaunchKernelGGL((fp4_attention_kernel<2, 4>), dim3((uint32_t)items), dim3(256), 0, stream, qb, ob, g, l);
  timer_end(TK_ATTENTION, stream);
  if (s->bytes) {
    timer_begin(TK_ATTN_COMBINE, stream);
    const dim3 grid((uint32_t)(g.rows + 3) / 4, (uint32_t)g.heads);
    if (g.p_pieces + s->o_pieces <= 4)
      hipLaunchKernelGGL(fp4_combine_kernel<4>, grid, dim3(256), 0, stream, ob, g, l);
    else
      hipLaunchKernelGGL(fp4_combine_kernel<8>, grid, dim3(256), 0, stream, ob, g, l);
    timer_end(TK_ATTN_COMBINE, stream);
  }
  SC_HIP(hipGetLastError());
  return SC_OK;
}

int fp4_attention_form(const sc_plan* p, const sc_cache* c, int32_t* queries, int32_t* ring, int32_t* pieces) {
  const int rc = plan_current(p, c);
  if (rc != SC_OK) return rc;
  const Fp4Schedule* s = fp4_schedule(p, c, SIZE_MAX);
  if (!s) return fail(SC_EINVAL, "out of host memory");
  *queries = s->wide ? 0 : s->tile;
  *ring = s->wide ? 1 : s->waves;
  *pieces = s->wide ? 1 : s->joined ? s->o_pieces : -s->p_pieces;
  return SC_OK;
}

}  // namespace sc
