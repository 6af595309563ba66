// Several states folded into one: per layer and head the n tokens of the sources
// with the largest weights (of equal ones the first), in their order, gathered into
// the new state's pages.
//
// Two launches, or one for few tokens.  condense_select_kernel finds each head's tokens: the n-th largest
// weight by radix selection over the weights' bits (11 + 11 + 10), then one pass
// that gives every kept token its place.  One work-group per layer and head: a
// selection is a chain of counts over all of a head's tokens, which stay in
// registers meanwhile (12 heads of 14040 tokens: 11 us; 360 of 1344: 6.8).
// condense_gather_kernel moves the data: K rows whole, V^T rows element by element
// (their tokens are adjacent), eight tokens of a row to a store.  What bounds it: the
// lines of V^T, of which a kept token or two among 64 fetch the whole (from 21
// states of 64 tokens in 30 layers, 142 MB: 33 us from HBM, 4.3 TB/s, and 22 from the
// memory-side cache), and where the states are
// few its passes of latency (three of 4680 tokens, 12 heads: 17 us).  V^T staged through
// LDS in whole rows was slower on dense picks (two states of 4680 tokens in eight
// layers 170 us against 141) and faster on sparse ones of few layers (twelve of 224
// tokens in three, fp32: 21 against 39), with no rule on sizes that told them apart.
#include <algorithm>
#include <cstring>
#include <type_traits>

#include "device.h"
#include "internal.h"

namespace sc {

constexpr int kCondensePages = 800;

struct CondenseGeom {
  char* pool;          // of the first layer
  float* weights;      // of the first layer
  int32_t* kept;       // [layer][head][n]
  uint64_t slot_bytes, kv_half;
  int32_t n_heads, tpp, n_slots, n_src;  // n_src: source pages
  int32_t n;                             // tokens kept
  DivMagic tpp_div;
};
struct CondenseSlots {
  int32_t slot[kCondensePages];  // the sources', then the new state's
};

// Weights as unsigned keys of the same order; a NaN is lighter than anything, -0 is 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int CS_BINS = 2048;

// Inclusive sum over the lanes of a wave.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
#define SC_STEP(ctrl, rows) x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, rows, 0xf, false)
  SC_STEP(0x111, 0xf);  // row_shr 1, 2, 4, 8: within 16 lanes
  SC_STEP(0x112, 0xf);
  SC_STEP(0x114, 0xf);
  SC_STEP(0x118, 0xf);
  SC_STEP(0x142, 0xa);  // lane 15 of a row to the next, lane 31 to the upper half
  SC_STEP(0x143, 0xc);
#undef SC_STEP
  return x;
}

// The same over the T threads of a work-group (sums: T / 64 words of LDS, its own).
template <int T>
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t* sums, int32_t tid) {
  x = wave_scan(x);
  if ((tid & 63) == 63) sums[tid >> 6] = x;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < T / 64 - 1; ++w) x += w < (tid >> 6) ? sums[w] : 0u;
  return x;
}

// T threads hold R tokens each, in order (R a multiple of 8: eight tokens lie in
// one page); R 0: any number of tokens, read again in each pass.  C copies of a
// counter: fewer lanes of a wave meet in one.
// kept: where the numbers go (LDS or memory).
template <int T, int R, int C>
__device__ __forceinline__ void select_tokens(const CondenseGeom& g, const CondenseSlots& slots, int32_t head, int32_t layer,
                                              int32_t* kept) {
  constexpr int BPT = CS_BINS / T;    // bins of a thread, counted together by it:
  constexpr int ROW = BPT * C + 4;    // their counters, and a gap that spreads the threads over the banks
  __shared__ __attribute__((aligned(16))) uint32_t hist[T * ROW];
  __shared__ uint32_t sums[5][T / 64];
  __shared__ uint32_t found[3][2];
  const int32_t tid = threadIdx.x, N = g.n_src * g.tpp;
  const float* w = g.weights + ((size_t)layer * g.n_slots * g.n_heads + head) * g.tpp;
  const int32_t per = R ? R : ((N + T - 1) / T + 7) / 8 * 8, i0 = tid * per;
  constexpr int RR = R ? R : 8;
  uint32_t keys[RR];
  // eight tokens from i on (past the end: of the lowest key, and counted by nothing)
  const auto load = [&](int32_t i, uint32_t* k) __attribute__((always_inline)) {
    const int32_t p = (int32_t)fast_div((uint32_t)min(i, N - 8), g.tpp_div);
    const float* from = w + (size_t)slots.slot[p] * g.n_heads * g.tpp + (min(i, N - 8) - p * g.tpp);
#pragma unroll
    for (int e = 0; e < 8; ++e) k[e] = weight_key(from[e]);
  };
  // f(key) for this thread's tokens in order
  const auto each = [&](auto f) __attribute__((always_inline)) {
    if constexpr (R > 0) {
#pragma unroll
      for (int e = 0; e < R; ++e)
        if (i0 + e < N) f(keys[e], i0 + e);
    } else {
      for (int32_t i = i0; i < min(i0 + per, N); i += 8) {
        load(i, keys);
#pragma unroll
        for (int e = 0; e < 8; ++e) f(keys[e], i + e);
      }
    }
  };
  for (int32_t b = tid; b < T * ROW; b += T) hist[b] = 0;
  if constexpr (R > 0)
#pragma unroll
    for (int e = 0; e < R; e += 8) load(i0 + e, keys + e);
  __syncthreads();
  // the n-th largest key: `prefix` its bits found so far, `want` its rank among the
  // keys that share them
  uint32_t prefix = 0, want = (uint32_t)g.n;
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int sh = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    each([&](uint32_t k, int32_t) __attribute__((always_inline)) {
      if (pass == 0 || k >> (sh + bits) == prefix)
      {
        const uint32_t bin = CS_BINS - 1 - (k >> sh & ((1u << bits) - 1));  // from the top
        atomicAdd(&hist[bin / BPT * ROW + bin % BPT * C + (tid & (C - 1))], 1u);
      }
    });
    __syncthreads();
    // this thread's bins, and zeros in their place for the next pass
    uint32_t count[BPT], all = 0;
    u32x4* mine = reinterpret_cast<u32x4*>(hist + tid * ROW);
#pragma unroll
    for (int b = 0; b < BPT; ++b) count[b] = 0;
#pragma unroll
    for (int v = 0; v < BPT * C / 4; ++v) {
      const u32x4 c = mine[v];
      if (pass < 2) mine[v] = u32x4{};
#pragma unroll
      for (int e = 0; e < 4; ++e) count[(4 * v + e) / C] += c[e];
    }
#pragma unroll
    for (int b = 0; b < BPT; ++b) all += count[b];
    const uint32_t upto = block_scan<T>(all, sums[pass], tid);
    uint32_t before = upto - all;
    if (before < want && want <= upto)
#pragma unroll
      for (int b = 0; b < BPT; ++b) {
        if (before < want && want <= before + count[b]) {
          found[pass][0] = (uint32_t)(CS_BINS - 1 - BPT * tid - b);
          found[pass][1] = want - before;
        }
        before += count[b];
      }
    __syncthreads();
    prefix = prefix << bits | found[pass][0];
    want = found[pass][1];
  }
  // every key above `prefix` is kept, and the first `want` that equal it
  uint32_t above = 0, equal = 0;
  each([&](uint32_t k, int32_t) __attribute__((always_inline)) {
    above += k > prefix;
    equal += k == prefix;
  });
  const uint32_t own_above = above, own_equal = equal;
  above = block_scan<T>(above, sums[3], tid) - own_above;
  equal = block_scan<T>(equal, sums[4], tid) - own_equal;
  each([&](uint32_t k, int32_t i) __attribute__((always_inline)) {
    if (k > prefix || (k == prefix && equal < want)) kept[above + min(equal, want)] = i;
    above += k > prefix;
    equal += k == prefix;
  });
}

template <int T, int R, int C>
__global__ __launch_bounds__(T) void condense_select_kernel(CondenseGeom g, CondenseSlots slots) {
  const int32_t head = blockIdx.x, layer = blockIdx.y;
  select_tokens<T, R, C>(g, slots, head, layer, g.kept + ((size_t)layer * g.n_heads + head) * g.n);
}

// The gather's units of a head and layer, E the elements' type (uint16_t or uint32_t), HD
// the head dim: 16 bytes of a K row (its first unit the weight too), and CG_D rows of
// eight V^T columns.
constexpr int CG_T = 256, CG_D = 4;
template <class E, int HD>
struct Gather {
  static constexpr int U = HD * sizeof(E) / 16;  // units of a K row
  const CondenseGeom& g;
  const CondenseSlots& slots;
  const int32_t* kept;
  char* pool;
  float* w;
  size_t head_off;
  __device__ __forceinline__ Gather(const CondenseGeom& g_, const CondenseSlots& s, int32_t head, int32_t layer,
                                    const int32_t* k)
      : g(g_), slots(s), kept(k), pool(g_.pool + (size_t)layer * g_.n_slots * g_.slot_bytes),
        w(g_.weights + ((size_t)layer * g_.n_slots * g_.n_heads + head) * g_.tpp),
        head_off((size_t)head * g_.tpp * HD * sizeof(E)) {}
  __device__ __forceinline__ int32_t page_of(int32_t i) const { return (int32_t)fast_div((uint32_t)i, g.tpp_div); }
  __device__ __forceinline__ void k_unit(int32_t row, int32_t u) const {
    const int32_t from = kept[row], p = page_of(from), t = from - p * g.tpp, f = page_of(row), to = row - f * g.tpp;
    const int32_t src = slots.slot[p], dst = slots.slot[g.n_src + f];
    *reinterpret_cast<u32x4u*>(pool + (size_t)dst * g.slot_bytes + head_off + (size_t)to * HD * sizeof(E) + 16 * u) =
        *reinterpret_cast<const u32x4u*>(pool + (size_t)src * g.slot_bytes + head_off + (size_t)t * HD * sizeof(E) + 16 * u);
    if (u == 0) {
      const size_t stride = (size_t)g.n_heads * g.tpp;
      w[dst * stride + to] = w[src * stride + t];
    }
  }
  __device__ __forceinline__ void v_unit(int32_t run, int32_t d0) const {
    const char* src[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int32_t from = kept[8 * run + e], p = page_of(from);
      src[e] = pool + (size_t)slots.slot[p] * g.slot_bytes + g.kv_half + head_off +
               ((size_t)d0 * g.tpp + (from - p * g.tpp)) * sizeof(E);
    }
    const int32_t f = page_of(8 * run), to = 8 * run - f * g.tpp;
    char* dst = pool + (size_t)slots.slot[g.n_src + f] * g.slot_bytes + g.kv_half + head_off +
                ((size_t)d0 * g.tpp + to) * sizeof(E);
    E v[CG_D][8];
#pragma unroll
    for (int d = 0; d < CG_D; ++d)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[d][e] = *reinterpret_cast<const E*>(src[e] + (size_t)d * g.tpp * sizeof(E));
#pragma unroll
    for (int d = 0; d < CG_D; ++d) {
      u32x4u* out = reinterpret_cast<u32x4u*>(dst + (size_t)d * g.tpp * sizeof(E));
      if constexpr (sizeof(E) == 2) {
        u32x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (uint32_t)v[d][2 * e] | (uint32_t)v[d][2 * e + 1] << 16;
        *out = x;
      } else {
        out[0] = u32x4{v[d][0], v[d][1], v[d][2], v[d][3]};
        out[1] = u32x4{v[d][4], v[d][5], v[d][6], v[d][7]};
      }
    }
  }
};

// A work-group's share of a head's gather: the first k_blocks work-groups have the K
// units, the others the V^T ones.
template <class E, int HD>
__device__ __forceinline__ void gather_block(const Gather<E, HD>& gt, int32_t block, int32_t k_blocks) {
  constexpr int U = Gather<E, HD>::U;
  static_assert(CG_T % U == 0, "a work-group copies whole rows");
  const CondenseGeom& g = gt.g;
  if (block < k_blocks) {
    const int32_t row = block * (CG_T / U) + (int32_t)threadIdx.x / U;
    if (row < g.n) gt.k_unit(row, (int32_t)threadIdx.x % U);
    return;
  }
  const int32_t runs = g.n / 8;
  const int32_t i = (block - k_blocks) * CG_T + (int32_t)threadIdx.x, d0 = i / runs * CG_D;
  if (d0 < HD) gt.v_unit(i % runs, d0);
}

template <class E, int HD>
__global__ __launch_bounds__(CG_T) void condense_gather_kernel(CondenseGeom g, CondenseSlots slots, int32_t k_blocks) {
  gather_block(Gather<E, HD>(g, slots, (int32_t)blockIdx.y % g.n_heads, (int32_t)blockIdx.y / g.n_heads,
                             g.kept + (size_t)blockIdx.y * g.n),
               (int32_t)blockIdx.x, k_blocks);
}

// Both in one launch, for few tokens: every work-group of the gather selects for itself,
// which costs nothing where all of them are resident at once (seven to a CU, 20 KB of
// LDS each).  12 heads, apart against so: four states of 64 tokens in 12 layers 14.8 us
// against 11.9, 21 in 29 layers (1740 work-groups) 37.9 against 36.2; fp32, two of 312
// in three layers 15.2 against 13.2, two of 64 in 20 (2160) 16.1 against 19.3.
constexpr int CS_FEW = 256 * 8;
template <class E, int HD>
__global__ __launch_bounds__(CG_T) void condense_few_kernel(CondenseGeom g, CondenseSlots slots, int32_t k_blocks) {
  __shared__ int32_t kept[CS_FEW];
  const int32_t head = (int32_t)blockIdx.y % g.n_heads, layer = (int32_t)blockIdx.y / g.n_heads;
  select_tokens<CG_T, CS_FEW / CG_T, 1>(g, slots, head, layer, kept);
  __syncthreads();
  if (blockIdx.x == 0)
    for (int32_t i = threadIdx.x; i < g.n; i += CG_T) g.kept[(size_t)blockIdx.y * g.n + i] = kept[i];
  gather_block(Gather<E, HD>(g, slots, head, layer, kept), (int32_t)blockIdx.x, k_blocks);
}

int condense_check(const sc_cache* c, int32_t n_sources) {
  const int64_t pages = (int64_t)(n_sources + 1) * c->d.pages_per_chunk;
  if (pages > kCondensePages)
    return fail(SC_EUNSUPPORTED, "%d sources and their fold hold %lld pages, at most %d", n_sources, (long long)pages,
                kCondensePages);
  return SC_OK;
}

int launch_condense(const sc_cache* c, int32_t layer, int32_t n_layers, const int32_t* slots, int32_t n_src,
                    float* weights, int32_t* kept, hipStream_t stream) {
  const sc_cache_desc& d = c->d;
  CondenseGeom g;
  CondenseSlots s;
  std::memset(&g, 0, sizeof g);
  std::memset(&s, 0, sizeof s);
  std::copy(slots, slots + n_src + d.pages_per_chunk, s.slot);
  g.kept = kept;
  g.slot_bytes = c->slot_bytes;
  g.kv_half = c->kv_half;
  g.n_heads = d.n_heads;
  g.tpp = d.tokens_per_page;
  g.n_slots = d.n_slots;
  g.n_src = n_src;
  g.n = d.pages_per_chunk * d.tokens_per_page;
  g.tpp_div = magic_div((uint32_t)g.tpp);
  const int32_t N = n_src * g.tpp;
  const int32_t row_units = d.head_dim * (int32_t)dtype_size(d.dtype) / 16;
  const int32_t k_blocks = (int32_t)(((int64_t)g.n * row_units + CG_T - 1) / CG_T);
  const int32_t v_blocks = (int32_t)(((int64_t)g.n / 8 * (d.head_dim / CG_D) + CG_T - 1) / CG_T);
  const int32_t step = std::max(1, 65535 / d.n_heads);  // layers of a launch
  for (int32_t l = 0; l < n_layers; l += step) {
    const int32_t m = std::min(step, n_layers - l);
    g.pool = c->pool + (size_t)(layer + l) * d.n_slots * c->slot_bytes;
    g.weights = weights + (size_t)(layer + l) * d.n_slots * d.n_heads * g.tpp;
    g.kept = kept + (size_t)l * d.n_heads * g.n;
    const dim3 heads((uint32_t)d.n_heads, (uint32_t)m), grid((uint32_t)(k_blocks + v_blocks), (uint32_t)(m * d.n_heads));
    timer_begin(TK_CONDENSE, stream);
    const auto by_type = [&](auto launch) {
      if (d.dtype == SC_DTYPE_F32 && d.head_dim == 64)
        launch(uint32_t{}, std::integral_constant<int, 64>{});
      else if (d.dtype == SC_DTYPE_F32)
        launch(uint32_t{}, std::integral_constant<int, 128>{});
      else if (d.head_dim == 64)
        launch(uint16_t{}, std::integral_constant<int, 64>{});
      else
        launch(uint16_t{}, std::integral_constant<int, 128>{});
    };
    if (N <= CS_FEW && (int64_t)grid.x * grid.y <= 7 * kCUs) {
      by_type([&](auto e, auto hd) {
        hipLaunchKernelGGL((condense_few_kernel<decltype(e), decltype(hd)::value>), grid, dim3(CG_T), 0, stream, g, s, k_blocks);
      });
      timer_end(TK_CONDENSE, stream);
      SC_HIP(hipGetLastError());
      continue;
    }
    // few tokens: fewer waves meet at each barrier
    if (N <= 256 * 8)
      hipLaunchKernelGGL((condense_select_kernel<256, 8, 1>), heads, dim3(256), 0, stream, g, s);
    else if (N <= 1024 * 8)
      hipLaunchKernelGGL((condense_select_kernel<1024, 8, 4>), heads, dim3(1024), 0, stream, g, s);
    else if (N <= 1024 * 16)
      hipLaunchKernelGGL((condense_select_kernel<1024, 16, 4>), heads, dim3(1024), 0, stream, g, s);
    else if (N <= 1024 * 40)
      hipLaunchKernelGGL((condense_select_kernel<1024, 40, 4>), heads, dim3(1024), 0, stream, g, s);
    else
      hipLaunchKernelGGL((condense_select_kernel<1024, 0, 4>), heads, dim3(1024), 0, stream, g, s);
    by_type([&](auto e, auto hd) {
      hipLaunchKernelGGL((condense_gather_kernel<decltype(e), decltype(hd)::value>), grid, dim3(CG_T), 0, stream, g, s, k_blocks);
    });
    timer_end(TK_CONDENSE, stream);
    SC_HIP(hipGetLastError());
  }
  return SC_OK;
}

}  // namespace sc
