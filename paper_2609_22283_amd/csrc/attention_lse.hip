// Attention with the rows' logarithmic sums, and over a prefix shared by the pack:
// the kernels of attention_core.h in these forms (attention.hip chooses).
#include "attention_core.h"

namespace sc {

template <class M>
static void launch_main(const AttnShape& sh, uint32_t items, const typename M::Geom& g, const typename M::Plan& plan,
                        const void* q, void* o, int32_t dtype, int32_t head_dim, hipStream_t stream) {
  timer_begin(TK_ATTENTION, stream);
  if (dtype == SC_DTYPE_F32) {
    const float* qf = static_cast<const float*>(q);
    float* of = static_cast<float*>(o);
    // a pool that is only element-aligned: the copies into LDS move 16 bytes at a time
    const bool staged = (reinterpret_cast<uintptr_t>(g.layer_base) & 15) == 0;
    if (head_dim == 64 && staged)
      hipLaunchKernelGGL((attn_f32_kernel<64, M, true>), dim3(items), dim3(64 * F32_NW), 0, stream, qf, of, g, plan);
    else if (head_dim == 64)
      hipLaunchKernelGGL((attn_f32_kernel<64, M>), dim3(items), dim3(64 * F32_NW), 0, stream, qf, of, g, plan);
    else if (staged)
      hipLaunchKernelGGL((attn_f32_kernel<128, M, true>), dim3(items), dim3(64 * F32_NW), 0, stream, qf, of, g, plan);
    else
      hipLaunchKernelGGL((attn_f32_kernel<128, M>), dim3(items), dim3(64 * F32_NW), 0, stream, qf, of, g, plan);
    timer_end(TK_ATTENTION, stream);
    return;
  }
  const uint16_t* qb = static_cast<const uint16_t*>(q);
  uint16_t* ob = static_cast<uint16_t*>(o);
  if (sh.bq == WV_BQ) {
    hipLaunchKernelGGL((attn_waves_kernel<NoAhead, M>), dim3(items), dim3(64 * WV_NW), 0, stream, qb, ob, g, plan,
                       NoAhead{});
  } else if (sh.bq == BQ_TINY && (M::kShare || sh.ring == 4)) {  // a SharePlan's ring is 4 always
    hipLaunchKernelGGL((attn_bf16_kernel<2, 1, 4, M>), dim3(items), dim3(128), 0, stream, qb, ob, g, plan);
  } else if (sh.bq == BQ_TINY) {
    if constexpr (!M::kShare)
      hipLaunchKernelGGL((attn_bf16_kernel<2, 1, 3, M>), dim3(items), dim3(128), 0, stream, qb, ob, g, plan);
  } else if (sh.bq == BQ_SMALL) {
    hipLaunchKernelGGL((attn_bf16_kernel<4, 2, 2, M>), dim3(items), dim3(256), 0, stream, qb, ob, g, plan);
  } else {
    hipLaunchKernelGGL((attn_bf16_kernel<8, 2, 2, M>), dim3(items), dim3(512), 0, stream, qb, ob, g, plan);
  }
  timer_end(TK_ATTENTION, stream);
}

template <>
void launch_form<LseAttn>(const AttnShape& sh, uint32_t items, const LseGeom& g, const AttnPlan& plan, const void* q,
                          void* o, int32_t dtype, int32_t head_dim, hipStream_t stream) {
  launch_main<LseAttn>(sh, items, g, plan, q, o, dtype, head_dim, stream);
  if (!g.tail_units) return;
  uint16_t* ob = static_cast<uint16_t*>(o);
  timer_begin(TK_ATTN_COMBINE, stream);
  const dim3 grid((uint32_t)g.tail_units, (uint32_t)sh.bq / 8);
  if (sh.bq == BQ_TINY)
    hipLaunchKernelGGL((attn_combine_kernel<BQ_TINY, 1, LseAttn>), grid, dim3(256), 0, stream, ob, g, plan);
  else if (sh.bq == BQ_SMALL)
    hipLaunchKernelGGL((attn_combine_kernel<BQ_SMALL, 2, LseAttn>), grid, dim3(256), 0, stream, ob, g, plan);
  else
    hipLaunchKernelGGL((attn_combine_kernel<BQ_MAX, 2, LseAttn>), grid, dim3(256), 0, stream, ob, g, plan);
  timer_end(TK_ATTN_COMBINE, stream);
}

void launch_share_pieces(const AttnShape& sh, uint32_t items, const LseGeom& g, const SharePlan& plan, const void* q,
                         int32_t dtype, int32_t head_dim, hipStream_t stream) {
  launch_main<ShareAttn>(sh, items, g, plan, q, nullptr, dtype, head_dim, stream);
}

template <>
void launch_form<ShareAttn>(const AttnShape& sh, uint32_t items, const LseGeom& g, const SharePlan& plan,
                            const void* q, void* o, int32_t dtype, int32_t head_dim, hipStream_t stream) {
  launch_main<ShareAttn>(sh, items, g, plan, q, o, dtype, head_dim, stream);
  timer_begin(TK_ATTN_COMBINE, stream);
  // many: the chain of a row's loads, split over eight groups of lanes
  const bool many = g.p_pieces + g.o_pieces > 8, f32 = dtype == SC_DTYPE_F32;
  const dim3 grid(many ? (uint32_t)g.rows : (uint32_t)(g.rows + 7) / 8, (uint32_t)g.n_heads);
  if (f32 && head_dim == 64 && many)
    hipLaunchKernelGGL((attn_share_combine_kernel<64, 8, 0>), grid, dim3(256), 0, stream, o, g, plan);
  else if (f32 && head_dim == 64)
    hipLaunchKernelGGL((attn_share_combine_kernel<64, 1, 0>), grid, dim3(256), 0, stream, o, g, plan);
  else if (f32 && many)
    hipLaunchKernelGGL((attn_share_combine_kernel<128, 8, 0>), grid, dim3(256), 0, stream, o, g, plan);
  else if (f32)
    hipLaunchKernelGGL((attn_share_combine_kernel<128, 1, 0>), grid, dim3(256), 0, stream, o, g, plan);
  else if (sh.kh == 1 && many)
    hipLaunchKernelGGL((attn_share_combine_kernel<128, 8, 1>), grid, dim3(256), 0, stream, o, g, plan);
  else if (sh.kh == 1)
    hipLaunchKernelGGL((attn_share_combine_kernel<128, 1, 1>), grid, dim3(256), 0, stream, o, g, plan);
  else if (many)
    hipLaunchKernelGGL((attn_share_combine_kernel<128, 8, 2>), grid, dim3(256), 0, stream, o, g, plan);
  else
    hipLaunchKernelGGL((attn_share_combine_kernel<128, 1, 2>), grid, dim3(256), 0, stream, o, g, plan);
  timer_end(TK_ATTN_COMBINE, stream);
}

}  // namespace sc
