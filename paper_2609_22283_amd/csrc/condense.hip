// Several states folded into one: per layer and head the n tokens of the sources
// with the largest weights (of equal ones the first), in their order, gathered into
// the new state's pages.
//
// Two launches.  condense_select_kernel finds each head's tokens: the n-th largest
// weight by radix selection over the weights' bits (11 + 11 + 10), then one pass
// that gives every kept token its place.  One work-group per layer and head: a
// selection is a chain of counts over all of a head's tokens, and the tokens lie in
// LDS meanwhile.  condense_gather_kernel moves the data: K rows whole, V^T rows
// element by element (their tokens are adjacent), eight tokens of a row to a store.
#include <algorithm>
#include <cstring>

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

constexpr int CS_T = 1024, CS_BINS = 2048;

// Inclusive sums over the work-group's threads of two counts packed in 64 bits.
__device__ __forceinline__ uint64_t block_scan(uint64_t x, uint64_t* sums, int32_t tid) {
  const int32_t lane = tid & 63, wave = tid >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  if (lane == 63) sums[wave] = x;
  __syncthreads();
  uint64_t before = 0;
  for (int32_t w = 0; w < wave; ++w) before += sums[w];
  __syncthreads();
  return x + before;
}

// MAX: tokens kept in LDS (0: read again from memory in each pass).
template <int MAX>
__global__ __launch_bounds__(CS_T) void condense_select_kernel(CondenseGeom g, CondenseSlots slots) {
  __shared__ uint32_t keys[MAX ? MAX : 1];
  __shared__ uint32_t hist[CS_BINS];
  __shared__ uint64_t sums[CS_T / 64];
  __shared__ uint32_t found[2];
  const int32_t tid = threadIdx.x, head = blockIdx.x, layer = blockIdx.y, N = g.n_src * g.tpp;
  const float* w = g.weights + ((size_t)layer * g.n_slots * g.n_heads + head) * g.tpp;
  const auto load = [&](int32_t i) {
    const int32_t p = (int32_t)fast_div((uint32_t)i, g.tpp_div);
    return weight_key(w[(size_t)slots.slot[p] * g.n_heads * g.tpp + (i - p * g.tpp)]);
  };
  if constexpr (MAX > 0)
    for (int32_t i = tid; i < N; i += CS_T) keys[i] = load(i);
  const auto key = [&](int32_t i) {
    if constexpr (MAX > 0) return keys[i];
    return load(i);
  };
  // the n-th largest key, `prefix` its bits found so far, `want` its rank among the
  // keys that share them
  uint32_t prefix = 0, want = (uint32_t)g.n;
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int sh = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    for (int32_t b = tid; b < CS_BINS; b += CS_T) hist[b] = 0;
    __syncthreads();
    for (int32_t i = tid; i < N; i += CS_T) {
      const uint32_t k = key(i);
      if (pass == 0 || k >> (sh + bits) == prefix) atomicAdd(&hist[k >> sh & ((1u << bits) - 1)], 1u);
    }
    __syncthreads();
    // bins from the top, two to a thread
    const uint32_t hi = hist[CS_BINS - 1 - 2 * tid], lo = hist[CS_BINS - 2 - 2 * tid];
    const uint32_t upto = (uint32_t)block_scan(hi + lo, sums, tid), before = upto - hi - lo;
    if (before < want && want <= upto) {
      const bool first = want <= before + hi;
      found[0] = (uint32_t)(CS_BINS - 1 - 2 * tid) - (first ? 0u : 1u);
      found[1] = want - before - (first ? 0u : hi);
    }
    __syncthreads();
    prefix = prefix << bits | found[0];
    want = found[1];
    __syncthreads();
  }
  // every key above `prefix` is kept, and the first `want` that equal it; a thread
  // takes a run of tokens (of odd length: LDS banks)
  const int32_t run = (N + CS_T - 1) / CS_T | 1;
  const int32_t i0 = min(tid * run, N), i1 = min(i0 + run, N);
  uint32_t above = 0, equal = 0;
  for (int32_t i = i0; i < i1; ++i) {
    const uint32_t k = key(i);
    above += k > prefix;
    equal += k == prefix;
  }
  const uint64_t own = (uint64_t)equal << 32 | above, upto = block_scan(own, sums, tid) - own;
  above = (uint32_t)upto;
  equal = (uint32_t)(upto >> 32);
  int32_t* kept = g.kept + ((size_t)layer * g.n_heads + head) * g.n;
  for (int32_t i = i0; i < i1; ++i) {
    const uint32_t k = key(i);
    if (k > prefix) {
      kept[above + min(equal, want)] = i;
      ++above;
    } else if (k == prefix) {
      if (equal < want) kept[above + equal] = i;
      ++equal;
    }
  }
}

// E: the elements' type (uint16_t or uint32_t), HD the head dim.
constexpr int CG_T = 256, CG_D = 4;  // CG_D: V^T rows of a thread
template <class E, int HD>
__global__ __launch_bounds__(CG_T) void condense_gather_kernel(CondenseGeom g, CondenseSlots slots, int32_t k_blocks) {
  const int32_t head = blockIdx.y % g.n_heads, layer = blockIdx.y / g.n_heads;
  const int32_t* kept = g.kept + (size_t)blockIdx.y * g.n;
  char* pool = g.pool + (size_t)layer * g.n_slots * g.slot_bytes;
  const size_t head_off = (size_t)head * g.tpp * HD * sizeof(E);
  const auto page_of = [&](int32_t i) { return (int32_t)fast_div((uint32_t)i, g.tpp_div); };
  if ((int32_t)blockIdx.x < k_blocks) {
    constexpr int U = HD * sizeof(E) / 16;  // 16-byte units of a K row
    const int32_t i = (int32_t)blockIdx.x * CG_T + (int32_t)threadIdx.x, row = i / U, u = i % U;
    if (row >= g.n) return;
    const int32_t from = kept[row], p = page_of(from), t = from - p * g.tpp, f = page_of(row), to = row - f * g.tpp;
    const int32_t src = slots.slot[p], dst = slots.slot[g.n_src + f];
    *reinterpret_cast<u32x4u*>(pool + (size_t)dst * g.slot_bytes + head_off + (size_t)to * HD * sizeof(E) + 16 * u) =
        *reinterpret_cast<const u32x4u*>(pool + (size_t)src * g.slot_bytes + head_off + (size_t)t * HD * sizeof(E) + 16 * u);
    if (u == 0) {
      float* w = g.weights + ((size_t)layer * g.n_slots * g.n_heads + head) * g.tpp;
      const size_t stride = (size_t)g.n_heads * g.tpp;
      w[dst * stride + to] = w[src * stride + t];
    }
    return;
  }
  const int32_t runs = g.n / 8;
  const int32_t i = ((int32_t)blockIdx.x - k_blocks) * CG_T + (int32_t)threadIdx.x, run = i % runs, d0 = i / runs * CG_D;
  if (d0 >= HD) return;
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
    if (N <= 8192)
      hipLaunchKernelGGL((condense_select_kernel<8192>), heads, dim3(CS_T), 0, stream, g, s);
    else if (N <= 36864)
      hipLaunchKernelGGL((condense_select_kernel<36864>), heads, dim3(CS_T), 0, stream, g, s);
    else
      hipLaunchKernelGGL((condense_select_kernel<0>), heads, dim3(CS_T), 0, stream, g, s);
    if (d.dtype == SC_DTYPE_F32 && d.head_dim == 64)
      hipLaunchKernelGGL((condense_gather_kernel<uint32_t, 64>), grid, dim3(CG_T), 0, stream, g, s, k_blocks);
    else if (d.dtype == SC_DTYPE_F32)
      hipLaunchKernelGGL((condense_gather_kernel<uint32_t, 128>), grid, dim3(CG_T), 0, stream, g, s, k_blocks);
    else if (d.head_dim == 64)
      hipLaunchKernelGGL((condense_gather_kernel<uint16_t, 64>), grid, dim3(CG_T), 0, stream, g, s, k_blocks);
    else
      hipLaunchKernelGGL((condense_gather_kernel<uint16_t, 128>), grid, dim3(CG_T), 0, stream, g, s, k_blocks);
    timer_end(TK_CONDENSE, stream);
    SC_HIP(hipGetLastError());
  }
  return SC_OK;
}

}  // namespace sc
