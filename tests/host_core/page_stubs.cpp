// Stand-ins for the launchers of csrc/fp4_pages.hip: pages move in host memory, so that
// a test can look where they went.  A conversion copies what both kinds of page have room
// for.  They fail with SC_EDEVICE, having done nothing, while g_page_fail is set.
#include <algorithm>
#include <cstring>

#include "../../paper_2609_22283_amd/csrc/internal.h"

bool g_page_fail = false;

namespace sc {

static int copy(const PoolView& from, const PoolView& to, uint64_t src_bytes, uint64_t dst_bytes, const PagePairs& p,
                int32_t layers) {
  if (g_page_fail) return fail(SC_EDEVICE, "page launch failed (forced)");
  for (int32_t l = 0; l < layers; ++l)
    for (int32_t i = 0; i < p.n; ++i)
      std::memcpy(to.base + l * to.layer_bytes + p.dst[i] * dst_bytes, from.base + l * from.layer_bytes + p.src[i] * src_bytes,
                  std::min(src_bytes, dst_bytes));
  return SC_OK;
}

int launch_page_moves(const PoolView& from, const PoolView& to, uint64_t bytes, const PagePairs& pairs, int32_t layers,
                      hipStream_t) {
  return copy(from, to, bytes, bytes, pairs, layers);
}
int launch_page_convert(bool pack, const PoolView& from, const PoolView& to, const sc_cache_desc& d,
                        const PagePairs& pairs, int32_t layers, hipStream_t) {
  const uint64_t wide = 4ull * d.n_heads * d.tokens_per_page * d.head_dim,
                 held = (uint64_t)d.n_heads * fp4_blocks(d.tokens_per_page) * kFp4Block;
  return copy(from, to, pack ? wide : held, pack ? held : wide, pairs, layers);
}

}  // namespace sc
