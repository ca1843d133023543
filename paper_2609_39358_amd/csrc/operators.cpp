// Argument validation of the operators on a paged cache (tl_append, tl_attend),
// in front of their launches.
#include <math.h>

#include "internal.h"

namespace {

constexpr uint32_t kMaxHeads = 1u << 16;  // query heads

// Caches that the operators read and write: bf16 pages, or scaled 8-bit ones.
int check_layer(const tl_ctx* ctx, uint32_t layer, const tl_cache* c) {
  if (layer >= ctx->L) return TL_EINVAL;
  if (ctx->dtype != TL_DTYPE_BF16 && ctx->dtype != TL_DTYPE_FP8_SCALED) return TL_ELAYOUT;
  if (ctx->D != 64 && ctx->D != 128 && ctx->D != 256) return TL_ELAYOUT;
  if (!c || !c->d_layer_k || !c->d_layer_v) return TL_EINVAL;
  if (c->page_stride < (int64_t)ctx->geo.slab_bytes || c->page_stride % 16) return TL_EINVAL;
  if (c->n_pages < 0 || c->n_pages > 0x7fffffff) return TL_EINVAL;
  if (((uintptr_t)c->d_layer_k | (uintptr_t)c->d_layer_v) & 7) return TL_EINVAL;
  return TL_OK;
}

int check_batch(const tl_batch* b) {
  if (!b) return TL_EINVAL;
  if (b->n_rows >= (1ull << 24) || b->n_reqs >= (1ull << 20) || b->table_width >= (1ull << 28)) return TL_ERANGE;
  if (!b->n_rows || !b->n_reqs) return TL_OK;
  if (!b->d_row_off || !b->d_kv_len || (b->table_width && !b->d_tables)) return TL_EINVAL;
  if (((uintptr_t)b->d_row_off | (uintptr_t)b->d_kv_len | (uintptr_t)b->d_tables) & 3) return TL_EINVAL;
  return TL_OK;
}

// Rows are moved 16 bytes at a time.
bool rows_ok(const tl_rows* r) {
  if (!r || !r->d_rows || ((uintptr_t)r->d_rows & 15)) return false;
  const int64_t lim = 1ll << 40;
  if (r->row_stride % 8 || r->head_stride % 8) return false;
  if (r->row_stride < -lim || r->row_stride > lim || r->head_stride < -lim || r->head_stride > lim) return false;
  return true;
}

// Results: no two of them in one place.
bool result_ok(const tl_rows* r, uint64_t n_rows, uint32_t n_heads, uint32_t dim) {
  if (!rows_ok(r)) return false;
  // strides of up to 2^40 times rows of up to 2^24 pass 64 bits
  const __int128 row = r->row_stride, head = r->head_stride, d = dim, rows = n_rows, heads = n_heads;
  if (row < 0 || head < 0) return false;
  const bool rows_outside = (heads == 1 || head >= d) && (rows == 1 || row >= (heads - 1) * head + d);
  const bool heads_outside = (rows == 1 || row >= d) && (heads == 1 || head >= (rows - 1) * row + d);
  return rows_outside || heads_outside;
}

bool heads_ok(const tl_ctx* ctx, uint32_t n_q_heads) {
  return n_q_heads && n_q_heads % ctx->H == 0 && n_q_heads <= kMaxHeads;
}

}  // namespace

extern "C" {

int tl_append(const tl_ctx* ctx, void* stream, uint32_t layer, const tl_batch* batch, const tl_rope* rope,
              const tl_rows* k, const tl_rows* v, uint32_t n_q_heads, const tl_rows* q, const tl_rows* q_out,
              const tl_cache* cache, uint8_t* d_status) {
  if (!ctx) return TL_EINVAL;
  int r = check_layer(ctx, layer, cache);
  if (r) return r;
  if ((r = check_batch(batch))) return r;
  if (!q != !q_out || !q != !n_q_heads || n_q_heads > kMaxHeads) return TL_EINVAL;
  if (rope) {
    if (rope->rot_dim > ctx->D || rope->rot_dim % 16 || !rope->rot_dim) return TL_EINVAL;
    if (!rope->d_cos_sin || ((uintptr_t)rope->d_cos_sin & 15) || rope->n_angles < 1) return TL_EINVAL;
    if (rope->flags & ~uint32_t(TL_ROPE_ADJACENT)) return TL_EINVAL;
    if (rope->n_axes < 1 || rope->n_axes > TL_ROPE_MAX_AXES || ((uintptr_t)rope->d_pos & 3)) return TL_EINVAL;
    if (rope->n_axes > 1 && (!rope->d_pos || !rope->pair_axis)) return TL_EINVAL;
    for (uint32_t i = 0; rope->pair_axis && i < rope->rot_dim / 2; ++i)
      if (rope->pair_axis[i] >= rope->n_axes) return TL_EINVAL;
  }
  if (batch->n_rows == 0 || batch->n_reqs == 0) return TL_OK;
  if (!rows_ok(k) || !rows_ok(v)) return TL_EINVAL;
  if (q) {
    if (!rows_ok(q) || !result_ok(q_out, batch->n_rows, n_q_heads, ctx->D))
      return TL_EINVAL;
    // in place, or elsewhere
    if (q->d_rows == q_out->d_rows && (q->row_stride != q_out->row_stride || q->head_stride != q_out->head_stride))
      return TL_EINVAL;
  }
  return tl::launch_append(ctx, stream, layer, batch, rope, k, v, n_q_heads, q, q_out, cache, d_status);
}

size_t tl_attend_workspace_bytes(const tl_ctx* ctx, uint32_t n_q_heads, size_t /*n_reqs*/, size_t n_rows) {
  if (!ctx || !heads_ok(ctx, n_q_heads)) return 0;
  return tl::attend_workspace(ctx, n_q_heads, n_rows);
}

int tl_attend(const tl_ctx* ctx, void* stream, uint32_t layer, const tl_batch* batch, uint32_t n_q_heads,
              const tl_rows* q, const tl_cache* cache, float scale, uint32_t flags, const tl_rows* out,
              float* d_lse, void* d_workspace, size_t workspace_bytes) {
  if (!ctx) return TL_EINVAL;
  int r = check_layer(ctx, layer, cache);
  if (r) return r;
  if ((r = check_batch(batch))) return r;
  if (!heads_ok(ctx, n_q_heads) || (flags & ~uint32_t(TL_ATTEND_ALL)) || !isfinite(scale)) return TL_EINVAL;
  if (batch->n_rows == 0 || batch->n_reqs == 0) return TL_OK;
  if (!rows_ok(q) || !result_ok(out, batch->n_rows, n_q_heads, ctx->D)) return TL_EINVAL;
  if (!d_workspace || ((uintptr_t)d_workspace & 15) || ((uintptr_t)d_lse & 3)) return TL_EINVAL;
  if (workspace_bytes < tl::attend_needs(ctx, n_q_heads, batch->n_reqs, batch->n_rows)) return TL_ERANGE;
  return tl::launch_attend(ctx, stream, layer, batch, n_q_heads, q, cache, scale, flags, out, d_lse, d_workspace);
}

}  // extern "C"
