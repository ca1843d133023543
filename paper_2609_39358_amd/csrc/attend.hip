// tl_attend: every row over its request's keys up to its own, a window of them, or all.
#include "attend.h"

namespace tl {

size_t attend_needs(const tl_ctx* ctx, uint32_t n_q_heads, uint64_t n_reqs, uint64_t n_rows) {
  return layout_of(shape_of(ctx, n_q_heads, n_reqs, n_rows), ctx->D).end;
}

// The layout follows from the number of wavefronts alone, and fewer requests or
// rows may take any that no more than all rows of one request ask for.
size_t attend_workspace(const tl_ctx* ctx, uint32_t n_q_heads, uint64_t n_rows) {
  const uint64_t most = std::min<uint64_t>(n_rows, 1u << 24) * (n_q_heads / ctx->H);
  uint64_t need = 0;
  for (uint32_t waves : {0u, 4u, 8u})
    if (waves <= waves_of(ctx, most)) need = std::max(need, layout_of(shape_of(ctx, n_q_heads, 1, n_rows, waves), ctx->D).end);
  return need;
}

int launch_attend(const tl_ctx* ctx, void* stream, uint32_t layer, const tl_batch* batch, uint32_t n_q_heads, const tl_rows* q,
                  const tl_cache* cache, float scale, uint32_t flags, const tl_rows* out, float* d_lse, void* d_ws) {
  AttendArgs a = {};
  a.all = (flags & TL_ATTEND_ALL) != 0;
  const Shape sh = shape_of(ctx, n_q_heads, batch->n_reqs, batch->n_rows);
  fill(a, sh, ctx, layer, batch, n_q_heads, q, cache, scale, out, d_lse, d_ws);
  hipStream_t s = (hipStream_t)stream;
  (void)hipGetLastError();
  by_cache(ctx, [&](auto D, auto fp8, auto even) {
    {
      TimedLaunch timed(TL_KERNEL_ATTEND, s);
      if (sh.waves)
        launch_many<D(), fp8(), even(), kText>(sh, s, a);
      else
        hipLaunchKernelGGL((k_attend16<D(), fp8(), even()>), dim3(sh.workers), dim3(256), 0, s, a);
    }
    launch_join<D()>(sh, s, a);
  });
  return hipGetLastError() == hipSuccess ? TL_OK : TL_EDEVICE;
}

}  // namespace tl
