// Packed attention over pages held in 4 bits (their layout: fp4.h).
//
// For every pack node i and head h: O = softmax(Q K^T * scale) V over the keys of node i's
// pages, K and V the values that the codes stand for; q and o are bf16.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "fp4.h"

namespace sc {

constexpr int kFp4Nodes = 64, kFp4Pages = 800;  // of a plan (attention_check)

// A plan's pages: the prefix that all nodes read first, then the nodes' own.
struct Fp4List {
  int32_t shared;
  int32_t off[kFp4Nodes + 1];
  int32_t slot[kFp4Pages];
};
struct Fp4Geom {
  const char* layer_base;
  uint64_t slot_bytes;
  int32_t heads, tpp, blocks, nq;
  DivMagic blocks_div, nq_div;
  float scale_log2;
};

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
  for (int32_t i = n; i <= kFp4Nodes; ++i) l.off[i] = at;
  g.layer_base = c->pool + (size_t)layer * d.n_slots * c->slot_bytes;
  g.slot_bytes = c->slot_bytes;
  g.heads = d.n_heads;
  g.tpp = d.tokens_per_page;
  g.blocks = fp4_blocks(d.tokens_per_page);
  g.nq = p->nq;
  g.blocks_div = magic_div((uint32_t)g.blocks);
  g.nq_div = magic_div((uint32_t)p->nq);
  g.scale_log2 = scale * 1.4426950408889634f;
}

__device__ __forceinline__ float fp4_value(uint32_t code) {  // of the code in the low bits
  const float m[8] = {0.f, 0.5f, 1.f, 1.5f, 2.f, 3.f, 4.f, 6.f};
  const float v = m[code & 7u];
  return code & 8u ? -v : v;
}
__device__ __forceinline__ float fp4_power(uint32_t s) {
  return s == 255u ? __uint_as_float(0x7fc00000u) : ldexpf(1.f, (int)s - 127);
}

// A wave per row and head: a lane takes half the channels of one key of a block, and
// two channels of the output.
__global__ __launch_bounds__(64) void fp4_attention_plain_kernel(const uint16_t* __restrict__ q, uint16_t* __restrict__ o,
                                                                 Fp4Geom g, Fp4List list) {
  __shared__ float qs[128], ps[32];
  const int32_t lane = threadIdx.x, row = blockIdx.x, h = blockIdx.y;
  const int32_t node = (int32_t)fast_div((uint32_t)row, g.nq_div);
  const uint16_t* qr = q + ((size_t)row * g.heads + h) * 128;
  qs[2 * lane] = bf16_to_f32(qr[2 * lane]);
  qs[2 * lane + 1] = bf16_to_f32(qr[2 * lane + 1]);
  __syncthreads();
  const int32_t own = list.off[node], pages = list.shared + list.off[node + 1] - own;
  float m = -INFINITY, sum = 0.f, acc[2] = {0.f, 0.f};
  const int32_t t = lane & 31, half = lane >> 5;
  for (int32_t j = 0; j < pages; ++j) {
    const char* page = g.layer_base + (uint64_t)list.slot[j < list.shared ? j : own + j - list.shared] * g.slot_bytes +
                       (uint64_t)h * g.blocks * kFp4Block;
    for (int32_t b = 0; b < g.blocks; ++b) {
      const uint8_t* blk = reinterpret_cast<const uint8_t*>(page) + (uint64_t)b * kFp4Block;
      float s = 0.f;
      for (int32_t c = 64 * half; c < 64 * half + 64; c += 32) {
        float d = 0.f;
        for (int32_t e = 0; e < 32; ++e) d += qs[c + e] * fp4_value(blk[t * 64 + (c + e) / 2] >> (4 * (e & 1)));
        s += d * fp4_power(blk[kFp4KScale + (t >> 4) * 64 + (t & 3) * 16 + (c >> 5) * 4 + (t >> 2 & 3)]);
      }
      s = (s + __shfl_xor(s, 32)) * g.scale_log2;
      if (t >= g.tpp - b * kFp4Tokens) s = -INFINITY;
      float top = s;
      for (int x = 1; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor(top, x));
      const float to = fmaxf(m, top), keep = m == to ? 1.f : exp2f(m - to);
      const float p = s == -INFINITY && t >= g.tpp - b * kFp4Tokens ? 0.f : exp2f(s - to);
      m = to;
      float all = p;
      for (int x = 1; x < 32; x <<= 1) all += __shfl_xor(all, x);
      sum = sum * keep + all;
      __syncthreads();
      if (half == 0) ps[t] = p;
      __syncthreads();
      for (int i = 0; i < 2; ++i) {
        const int32_t c = 2 * lane + i;
        float d = 0.f;
        for (int32_t e = 0; e < 32; ++e) d += ps[e] * fp4_value(blk[kFp4V + c * 16 + e / 2] >> (4 * (e & 1)));
        acc[i] = acc[i] * keep + d * fp4_power(blk[kFp4VScale + (c & 15) * 8 + (c >> 4)]);
      }
    }
  }
  *reinterpret_cast<uint32_t*>(o + ((size_t)row * g.heads + h) * 128 + 2 * lane) = pack_bf16x2(acc[0] / sum, acc[1] / sum);
}

size_t fp4_attention_workspace_bytes(const sc_plan*, const sc_cache*) { return 0; }

int launch_fp4_attention(const sc_plan* p, const sc_cache* c, int32_t layer, const void* q, void* o, float scale,
                         void* ws, size_t room, hipStream_t stream) {
  if (!std::isfinite(scale)) return fail(SC_EINVAL, "scale must be finite");
  const int64_t rows = (int64_t)p->nodes.size() * p->nq;
  if (rows > INT32_MAX) return fail(SC_EUNSUPPORTED, "%lld query rows", (long long)rows);
  Fp4List l;
  Fp4Geom g;
  fp4_fill(p, c, layer, scale, l, g);
  timer_begin(TK_ATTENTION, stream);
  hipLaunchKernelGGL(fp4_attention_plain_kernel, dim3((uint32_t)rows, (uint32_t)g.heads), dim3(64), 0, stream,
                     static_cast<const uint16_t*>(q), static_cast<uint16_t*>(o), g, l);
  timer_end(TK_ATTENTION, stream);
  SC_HIP(hipGetLastError());
  return SC_OK;
}

int fp4_attention_form(const sc_plan*, const sc_cache*, int32_t* queries, int32_t* ring, int32_t* pieces) {
  *queries = *ring = *pieces = 1;
  return SC_OK;
}

}  // namespace sc
