// tl_attend_tree: every row over its request's keys before the new tokens, and those new
// tokens that its mask names: a tree of drafted tokens, whose rows see their ancestors.
// The masks count only in the blocks of keys that hold new tokens; the others are the
// same work as tl_attend's.
#include "attend.h"

namespace tl {

int launch_attend_tree(const tl_ctx* ctx, void* stream, uint32_t layer, const tl_batch* batch, const tl_tree* tree, uint32_t n_q_heads,
                       const tl_rows* q, const tl_cache* cache, float scale, const tl_rows* out, float* d_lse, void* d_ws) {
  AttendArgs a = {};
  a.tree = tree->d_seen;
  a.tree_words = tree->words;
  a.tree_pos = tree->d_pos;
  return launch<true>(a, ctx, stream, layer, batch, n_q_heads, q, cache, scale, out, d_lse, d_ws);
}

}  // namespace tl
