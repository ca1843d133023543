// Argument validation of the operators on a paged cache (tl_append, tl_attend
// and their variants, tl_pages_*, tl_keep), in front of their launches.
#include <float.h>
#include <math.h>

#include <algorithm>
#include <initializer_list>

#include "internal.h"

namespace {

constexpr uint32_t kMaxHeads = 1u << 16;  // query heads

int check_cache(const tl_ctx* ctx, const tl_cache* c) {
  if (!c || !c->d_layer_k || !c->d_layer_v) return TL_EINVAL;
  if (c->page_stride < (int64_t)ctx->geo.slab_bytes || c->page_stride % 16) return TL_EINVAL;
  if (c->n_pages < 0 || c->n_pages > 0x7fffffff) return TL_EINVAL;
  if (((uintptr_t)c->d_layer_k | (uintptr_t)c->d_layer_v) & 7) return TL_EINVAL;
  return TL_OK;
}

// Caches whose values the operators read and write: bf16 pages, or scaled 8-bit ones.
int check_values(const tl_ctx* ctx) {
  if (ctx->dtype != TL_DTYPE_BF16 && ctx->dtype != TL_DTYPE_FP8_SCALED) return TL_ELAYOUT;
  if (ctx->D != 64 && ctx->D != 128 && ctx->D != 256) return TL_ELAYOUT;
  return TL_OK;
}

int check_layer(const tl_ctx* ctx, uint32_t layer, const tl_cache* c) {
  if (layer >= ctx->L) return TL_EINVAL;
  const int r = check_values(ctx);
  return r ? r : check_cache(ctx, c);
}

// A page's bytes are counted in 32 bits.
int check_pages(const tl_ctx* ctx, const tl_cache* c) {
  if (ctx->geo.slab_bytes >= (1ull << 31)) return TL_ELAYOUT;
  return check_cache(ctx, c);
}

bool words_ok(const void* p) { return p && !((uintptr_t)p & 3); }
bool maybe_words(const void* p) { return !((uintptr_t)p & 3); }
// Arrays of a call. What a kernel writes may share no byte with another one: its threads
// read and write in no particular order.
struct Bytes {
  const void* p;
  uint64_t n;
};
bool apart(std::initializer_list<Bytes> written, std::initializer_list<Bytes> read) {
  auto share = [](const Bytes& a, const Bytes& b) {
    return a.p && b.p && a.n && b.n && (uintptr_t)a.p < (uintptr_t)b.p + b.n && (uintptr_t)b.p < (uintptr_t)a.p + a.n;
  };
  for (const Bytes* a = written.begin(); a != written.end(); ++a) {
    for (const Bytes* b = a + 1; b != written.end(); ++b)
      if (share(*a, *b)) return false;
    for (const Bytes& b : read)
      if (share(*a, b)) return false;
  }
  return true;
}

int check_pool(const tl_pool* p) {
  if (!p || !words_ok(p->d_refs) || p->n_pages < 0 || p->n_pages > 0x7fffffff) return TL_EINVAL;
  return TL_OK;
}

Bytes pool_bytes(const tl_ctx* ctx, const tl_pool* p) { return {p->d_refs, 4ull * ctx->geo.n_groups * (uint64_t)p->n_pages}; }

// Table rows of a call: their entries are counted in 32 bits.
int check_table_rows(uint64_t n, uint64_t width) {
  if (n >= (1ull << 20) || width >= (1ull << 28) || n * width >= (1ull << 31)) return TL_ERANGE;
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

// Weights of a norm are read 16 bytes at a time.
bool weights_ok(int64_t stride) { return stride % 4 == 0 && stride >= -(1ll << 40) && stride <= 1ll << 40; }

bool heads_ok(const tl_ctx* ctx, uint32_t n_q_heads) {
  return n_q_heads && n_q_heads % ctx->H == 0 && n_q_heads <= kMaxHeads;
}

}  // namespace

extern "C" {

int tl_append(const tl_ctx* ctx, void* stream, uint32_t layer, const tl_batch* batch, const tl_rope* rope,
              const tl_rows* k, const tl_rows* v, uint32_t n_q_heads, const tl_rows* q, const tl_rows* q_out,
              const tl_cache* cache, uint8_t* d_status) {
  return tl_append_norm(ctx, stream, layer, batch, nullptr, rope, k, v, n_q_heads, q, q_out, cache, d_status);
}

int tl_append_norm(const tl_ctx* ctx, void* stream, uint32_t layer, const tl_batch* batch, const tl_norm* norm,
                   const tl_rope* rope, const tl_rows* k, const tl_rows* v, uint32_t n_q_heads, const tl_rows* q,
                   const tl_rows* q_out, const tl_cache* cache, uint8_t* d_status) {
  if (!ctx) return TL_EINVAL;
  int r = check_layer(ctx, layer, cache);
  if (r) return r;
  if ((r = check_batch(batch))) return r;
  if (!q != !q_out || !q != !n_q_heads || n_q_heads > kMaxHeads) return TL_EINVAL;
  if (norm) {
    if (!(norm->eps >= FLT_MIN) || !isfinite(norm->eps) || (norm->flags & ~uint32_t(TL_NORM_CENTER))) return TL_EINVAL;
    if (((uintptr_t)norm->d_q_weight | (uintptr_t)norm->d_k_weight) & 15) return TL_EINVAL;
    if (!weights_ok(norm->q_stride) || !weights_ok(norm->k_stride)) return TL_EINVAL;
  }
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
  return tl::launch_append(ctx, stream, layer, batch, norm, rope, k, v, n_q_heads, q, q_out, cache, d_status);
}

size_t tl_attend_workspace_bytes(const tl_ctx* ctx, uint32_t n_q_heads, size_t /*n_reqs*/, size_t n_rows) {
  if (!ctx || !heads_ok(ctx, n_q_heads)) return 0;
  return std::max(tl::attend_workspace(ctx, n_q_heads, n_rows), tl::attend_tree_workspace(ctx, n_q_heads));
}

// What tl_attend and tl_attend_tree check alike (`fine`: what each has besides); *go:
// whether there is something to do.
static int check_attend(const tl_ctx* ctx, uint32_t layer, const tl_batch* batch, uint32_t n_q_heads, const tl_rows* q,
                        const tl_cache* cache, float scale, const tl_rows* out, const float* d_lse, const void* d_workspace,
                        size_t workspace_bytes, size_t (*needs)(const tl_ctx*, uint32_t, uint64_t, uint64_t), bool fine, bool* go) {
  *go = false;
  int r = check_layer(ctx, layer, cache);
  if (r) return r;
  if ((r = check_batch(batch))) return r;
  if (!heads_ok(ctx, n_q_heads) || !fine || !isfinite(scale)) return TL_EINVAL;
  if (batch->n_rows == 0 || batch->n_reqs == 0) return TL_OK;
  if (!rows_ok(q) || !result_ok(out, batch->n_rows, n_q_heads, ctx->D)) return TL_EINVAL;
  if (!d_workspace || ((uintptr_t)d_workspace & 15) || ((uintptr_t)d_lse & 3)) return TL_EINVAL;
  if (workspace_bytes < needs(ctx, n_q_heads, batch->n_reqs, batch->n_rows)) return TL_ERANGE;
  *go = true;
  return TL_OK;
}

int tl_attend(const tl_ctx* ctx, void* stream, uint32_t layer, const tl_batch* batch, uint32_t n_q_heads,
              const tl_rows* q, const tl_cache* cache, float scale, uint32_t flags, const tl_rows* out,
              float* d_lse, void* d_workspace, size_t workspace_bytes) {
  if (!ctx) return TL_EINVAL;
  bool go;
  const int r = check_attend(ctx, layer, batch, n_q_heads, q, cache, scale, out, d_lse, d_workspace, workspace_bytes,
                             tl::attend_needs, !(flags & ~uint32_t(TL_ATTEND_ALL)), &go);
  if (!go) return r;
  return tl::launch_attend(ctx, stream, layer, batch, n_q_heads, q, cache, scale, flags, out, d_lse, d_workspace);
}

int tl_attend_tree(const tl_ctx* ctx, void* stream, uint32_t layer, const tl_batch* batch, const tl_tree* tree,
                   uint32_t n_q_heads, const tl_rows* q, const tl_cache* cache, float scale, const tl_rows* out,
                   float* d_lse, void* d_workspace, size_t workspace_bytes) {
  if (!ctx) return TL_EINVAL;
  bool go;
  const int r = check_attend(ctx, layer, batch, n_q_heads, q, cache, scale, out, d_lse, d_workspace, workspace_bytes,
                             tl::attend_tree_needs, tree && tree->words && tree->words <= 1u << 18, &go);
  if (!go) return r;
  if (!tree->d_seen || ((uintptr_t)tree->d_seen & 7) || !maybe_words(tree->d_pos)) return TL_EINVAL;
  if (ctx->window[layer] && !tree->d_pos) return TL_EINVAL;
  return tl::launch_attend_tree(ctx, stream, layer, batch, tree, n_q_heads, q, cache, scale, out, d_lse, d_workspace);
}

int tl_pages_copy(const tl_ctx* ctx, void* stream, const tl_cache* cache, size_t n, const int32_t* d_src,
                  const int32_t* d_dst, const uint32_t* d_rows) {
  if (!ctx) return TL_EINVAL;
  const int r = check_pages(ctx, cache);
  if (r) return r;
  if (n >= (1ull << 24)) return TL_ERANGE;
  if (!n) return TL_OK;
  if (!words_ok(d_src) || !words_ok(d_dst) || !maybe_words(d_rows)) return TL_EINVAL;
  return tl::launch_pages_copy(ctx, stream, cache, n, d_src, d_dst, d_rows);
}

size_t tl_pages_workspace_bytes(const tl_ctx* ctx, size_t n, size_t n_pages) {
  if (!ctx || n >= (1ull << 20) || n_pages > 0x7fffffff) return 0;
  return tl::pages_workspace(ctx, n, n_pages);
}

int tl_pages_fork(const tl_ctx* ctx, void* stream, const tl_pool* pool, const tl_cache* cache, size_t n_parents,
                  const uint32_t* d_kv_len, const int32_t* d_tables, size_t n, const int32_t* d_parent,
                  uint32_t* d_len_out, int32_t* d_tables_out, size_t table_width, uint8_t* d_status,
                  void* d_workspace, size_t workspace_bytes) {
  if (!ctx) return TL_EINVAL;
  int r = check_pages(ctx, cache);
  if (r || (r = check_pool(pool))) return r;
  if (pool->n_pages != cache->n_pages) return TL_EINVAL;
  if ((r = check_table_rows(n, table_width)) || (r = check_table_rows(n_parents, table_width))) return r;
  if (!n) return TL_OK;
  if (!words_ok(d_parent) || !words_ok(d_len_out) || (n_parents && !words_ok(d_kv_len))) return TL_EINVAL;
  const uint64_t row = 4ull * ctx->geo.n_groups * table_width;
  if (table_width && (!words_ok(d_tables_out) || (n_parents && !words_ok(d_tables)))) return TL_EINVAL;
  if (!d_workspace || ((uintptr_t)d_workspace & 15)) return TL_EINVAL;
  const uint64_t need = tl::pages_workspace(ctx, n, (uint64_t)pool->n_pages);
  if (!apart({{d_tables_out, n * row}, {d_len_out, 4 * n}, {d_status, n}, pool_bytes(ctx, pool), {d_workspace, need}},
             {{d_kv_len, 4 * n_parents}, {d_tables, n_parents * row}, {d_parent, 4 * n}}))
    return TL_EINVAL;
  if (workspace_bytes < need) return TL_ERANGE;
  return tl::launch_pages_fork(ctx, stream, pool, cache, n_parents, d_kv_len, d_tables, n, d_parent, d_len_out,
                               d_tables_out, table_width, d_status, d_workspace);
}

int tl_pages_take(const tl_ctx* ctx, void* stream, const tl_pool* pool, size_t n, const uint32_t* d_have,
                  const uint32_t* d_want, int32_t* d_tables, size_t table_width, uint8_t* d_status,
                  void* d_workspace, size_t workspace_bytes) {
  if (!ctx) return TL_EINVAL;
  int r = check_pool(pool);
  if (r || (r = check_table_rows(n, table_width))) return r;
  if (!n) return TL_OK;
  if (!words_ok(d_have) || !words_ok(d_want) || (table_width && !words_ok(d_tables))) return TL_EINVAL;
  if (!d_workspace || ((uintptr_t)d_workspace & 15)) return TL_EINVAL;
  const uint64_t need = tl::pages_workspace(ctx, n, (uint64_t)pool->n_pages), row = 4ull * ctx->geo.n_groups * table_width;
  if (!apart({{d_tables, n * row}, {d_status, n}, pool_bytes(ctx, pool), {d_workspace, need}}, {{d_have, 4 * n}, {d_want, 4 * n}}))
    return TL_EINVAL;
  if (workspace_bytes < need) return TL_ERANGE;
  return tl::launch_pages_take(ctx, stream, pool, n, d_have, d_want, d_tables, table_width, d_status, d_workspace);
}

int tl_pages_free(const tl_ctx* ctx, void* stream, const tl_pool* pool, size_t n, int32_t* d_tables,
                  size_t table_width, const uint32_t* d_first, const uint32_t* d_end) {
  if (!ctx) return TL_EINVAL;
  int r = check_pool(pool);
  if (r || (r = check_table_rows(n, table_width))) return r;
  if (!n || !table_width) return TL_OK;
  if (!words_ok(d_tables) || !maybe_words(d_first) || !maybe_words(d_end)) return TL_EINVAL;
  if (!apart({{d_tables, 4 * n * ctx->geo.n_groups * table_width}, pool_bytes(ctx, pool)}, {{d_first, 4 * n}, {d_end, 4 * n}})) return TL_EINVAL;
  return tl::launch_pages_free(ctx, stream, pool, n, d_tables, table_width, d_first, d_end);
}

int tl_keep(const tl_ctx* ctx, void* stream, const tl_batch* batch, const uint32_t* d_n_keep, const uint32_t* d_keep,
            const tl_cache* cache, uint32_t* d_len_out, uint8_t* d_status) {
  if (!ctx) return TL_EINVAL;
  int r = check_values(ctx);
  if (r || (r = check_pages(ctx, cache)) || (r = check_batch(batch))) return r;
  if (!batch->n_reqs) return TL_OK;
  if (!words_ok(batch->d_row_off) || !words_ok(batch->d_kv_len)) return TL_EINVAL;
  if (!words_ok(d_n_keep) || !words_ok(d_len_out) || (batch->n_rows && !words_ok(d_keep))) return TL_EINVAL;
  const uint64_t lens = 4 * batch->n_reqs;
  if (!apart({{d_len_out, lens}, {d_status, batch->n_reqs}},
             {{batch->d_kv_len, lens}, {batch->d_row_off, lens + 4}, {d_n_keep, lens}, {d_keep, 4 * batch->n_rows},
              {batch->d_tables, lens * ctx->geo.n_groups * batch->table_width}}))
    return TL_EINVAL;
  return tl::launch_keep(ctx, stream, batch, d_n_keep, d_keep, cache, d_len_out, d_status);
}

}  // extern "C"
