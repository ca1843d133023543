// tl_attend_tree: every row over its request's keys before the new tokens, and those new
// tokens that its mask names: a tree of drafted tokens, whose rows see their ancestors.
// The masks count only in the blocks of keys that hold new tokens; the others are the
// same work as tl_attend's.
#include "attend.h"

namespace tl {
namespace {

// ---- 32 rows for each wavefront ------------------------------------------------------
// For trees of some tokens: up to some 32 to 64 rows (query heads of a K/V head times new
// tokens) per request. As in tiles of 16 rows, keys and values go from memory to
// registers in the layout that the matrix instructions take, two steps on their way, and
// a workgroup's four wavefronts take neighbouring heads of the same keys (where the
// number of heads is no multiple of four or two, keys that follow each other). What is
// widened and transposed there serves G runs of 16 rows, one or two (heads of 256: one): a
// wavefront has a SIMD, and its 512 registers, to itself (two on a SIMD with two runs each
// spill in the loop: 213 us where this takes 156). Queries are in shared memory. More runs
// do not pay: with four, whose registers spill, 64 rows took 261 us, two tiles of 32 242.
constexpr int kRowWaves = 4;

// Runs of 16 rows whose sums fit beside two steps of keys.
__host__ __device__ constexpr int most_runs(int dim) { return dim != 256 ? 2 : 1; }

template <int D>
union LdsRows {
  u32x4 q[kRowWaves][most_runs(D)][D / 32][64];  // a lane's part of each product's queries
  struct {                                            // a run's sums, of wavefronts that share its keys
    float m[kRowWaves][16], sum[kRowWaves][16];
    float o[kRowWaves][16][D];
  } s;
};

template <int D, int G>
struct RowsOf {
  f32x4 o[G][D / 16];
  Soft s[G];
  Place p[G];
};

// A step's keys for G runs of 16 rows.
template <int D, bool FP8, bool EVEN, int G>
__device__ __forceinline__ void block_rows(const AttendArgs& a, const u32x4 (*qs)[D / 32][64], Tile16<D, FP8>& t, uint32_t kv, int key0, int before,
                                           bool edge, uint32_t& odd, RowsOf<D, G>& r) {
  typedef Tile16<D, FP8> Tile;
  constexpr int N = 8 * Tile::kGroups, H = 2 * Tile::kGroups;
  const uint32_t lane = threadIdx.x & 63, c = lane % 16, quad = lane / 16;
  float k_scale[H], v_scale[EVEN ? H : N];
  if constexpr (FP8) {
    const uint32_t kb = scale_held(scale_of(t.ks, kv)), vb = scale_held(scale_of(t.vs, kv));
#pragma unroll
    for (int h = 0; h < H; ++h) {
      k_scale[h] = scale_value(EVEN ? __builtin_amdgcn_readlane(kb, h * 16) : __shfl(kb, h * 16 + c));
      if constexpr (EVEN) v_scale[h] = scale_value(__builtin_amdgcn_readlane(vb, h * 16));
    }
    if constexpr (!EVEN)
#pragma unroll
      for (int i = 0; i < N; ++i) v_scale[i] = scale_value(__shfl(vb, i / 4 * 16 + quad * 4 + i % 4));
  }
  float x[G][N];
  {
    f32x4 acc[G][H];
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int h = 0; h < H; ++h) acc[g][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
      u32x4 w[H];
#pragma unroll
      for (int h = 0; h < H; ++h) {
        if constexpr (FP8) {
          w[h][0] = widen(t.k[h][2 * k], k_scale[h], false);
          w[h][1] = widen(t.k[h][2 * k], k_scale[h], true);
          w[h][2] = widen(t.k[h][2 * k + 1], k_scale[h], false);
          w[h][3] = widen(t.k[h][2 * k + 1], k_scale[h], true);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) w[h][j] = t.k[h][4 * k + j];
        }
      }
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const bf16x8 q = as_bf16(qs[g][k][lane]);
#pragma unroll
        for (int h = 0; h < H; ++h) acc[g][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(w[h]), q, acc[g][h], 0, 0, 0);
      }
    }
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int i = 0; i < N; ++i) x[g][i] = acc[g][i / 4][i % 4];
  }
  if (edge || t.seen != ~0ull) {  // some row does not see some key
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const uint64_t sees = named(a, r.p[g].row, key0 - before) & t.seen;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int at = (i / 4) * 16 + quad * 4 + i % 4;
        x[g][i] = (sees >> at & 1) && key0 + at >= r.p[g].lo && key0 + at < r.p[g].hi ? x[g][i] : kNone;
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < Tile::kVWords; ++j) {
        // what a page holds where there is no key may be NaN; what only some rows see is
        // theirs at the end
        if (!(t.seen >> ((i / 4) * 16 + quad * 4 + i % 4) & 1)) t.v[i][j] = 0;
        if (edge) {
          const uint32_t bad = odd_bits<FP8>(t.v[i][j]);
          odd |= bad;
          t.v[i][j] &= ~bad;
        }
      }
  }
  bool more = false;
  float top[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    top[g] = x[g][0];
#pragma unroll
    for (int i = 1; i < N; ++i) top[g] = fmaxf(top[g], x[g][i]);
    top[g] *= a.scale;
    more |= top[g] > r.s[g].m + kSlack;
  }
  if (__any(more)) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      Soft& s = r.s[g];
      float y = fmaxf(top[g], __shfl_xor(top[g], 16));
      y = fmaxf(y, __shfl_xor(y, 32));
      const float m = fmaxf(s.m, y);
      const float now = m == kNone ? 0.f : m;
      const float by = s.m == kNone ? 0.f : exp2_(s.top - now);
      s.m = m;
      s.top = now;
      s.sum *= by;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) r.o[g][i] *= by;
    }
  }
  bf16x8 w[G][Tile::kGroups];
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float y = exp2_(__builtin_fmaf(x[g][i], a.scale, -r.s[g].top));
      r.s[g].sum += y;
      w[g][i / 8][i % 8] = (__bf16)y;  // for the product, which takes bf16; the result is no finer
    }
#pragma unroll
  for (int k = 0; k < Tile::kGroups; ++k)
#pragma unroll
    for (int n = 0; n < Tile::kElems; n += 2) {
      uint32_t e[8];  // elements n, n + 1 of each key
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (FP8)
          e[i] = widen(t.v[8 * k + i][n / 4], v_scale[EVEN ? 2 * k + i / 4 : 8 * k + i], n & 2);
        else
          e[i] = t.v[8 * k + i][n / 2];
      }
      u32x4 lo, hi;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lo[i] = __builtin_amdgcn_perm(e[2 * i + 1], e[2 * i], 0x05040100);
        hi[i] = __builtin_amdgcn_perm(e[2 * i + 1], e[2 * i], 0x07060302);
      }
#pragma unroll
      for (int g = 0; g < G; ++g) {
        r.o[g][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(lo), w[g][k], r.o[g][n], 0, 0, 0);
        r.o[g][n + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(hi), w[g][k], r.o[g][n + 1], 0, 0, 0);
      }
    }
}

// A segment of a tile, as one wavefront has it.
struct Segment {
  const int32_t* table;
  GlobalBytes kp, vp;
  uint32_t head0, hs;     // the workgroup's first run of heads, log2 of how many it takes
  uint32_t head, kv;      // this wavefront's run, and its K/V head
  int step;               // keys of a block
  int key0, last;         // first keys of this wavefront's first and last step
  int first_hi, last_lo;  // keys below and from these on are seen by all rows
  uint32_t rows;          // of the tile
  bool whole;
  uint64_t slot;
};

// A row's E elements from d0 on, its maximum and its sum, to where they belong.
template <int D>
__device__ __forceinline__ void give_row(const AttendArgs& a, const Segment& g, const Place& at, uint32_t row, uint32_t d0, const float* y, float top,
                                         float total, bool one) {
  constexpr int E = D / 16;
  if (g.whole) {
    const float inv = total == 0.f ? 0.f : 1.f / total;
    uint16_t* op = a.out + (int64_t)at.row * a.o_token + (int64_t)at.head * a.o_head + d0;
#pragma unroll
    for (int n = 0; n < E; n += 4) store_bf16x4(op + n, y[n] * inv, y[n + 1] * inv, y[n + 2] * inv, y[n + 3] * inv);
    if (one && a.lse) a.lse[(uint64_t)at.row * a.n_heads * a.group + at.head] = lse_of(top, total);
    return;
  }
  float* fp = a.part_o + (g.slot + row) * D + d0;
#pragma unroll
  for (int n = 0; n < E; n += 4) *(f32x4*)(fp + n) = f32x4{y[n], y[n + 1], y[n + 2], y[n + 3]};
  if (one) *(f32x2*)(a.part_ml + (g.slot + row) * 2) = f32x2{top, total};
}

template <int D, bool FP8, bool EVEN, int G>
__device__ __forceinline__ void segment_rows(const AttendArgs& a, LdsRows<D>& l, const Kind& kind, const Cursor& cur, const Request& q,
                                             const Span& s, const Segment& g) {
  typedef Tile16<D, FP8> Tile;
  constexpr int E = D / 16;
  const uint32_t tid = threadIdx.x, lane = tid & 63, c = lane % 16, quad = lane / 16, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  RowsOf<D, G> r;
#pragma unroll
  for (int i = 0; i < G; ++i) {
    r.s[i] = Soft{kNone, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < E; ++n) r.o[i][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    r.p[i] = place_of<kTree>(a, kind, q, g.head, cur.tile, i * 16 + c);
    const uint16_t* qp = a.q + (int64_t)r.p[i].row * a.q_token + (int64_t)r.p[i].head * a.q_head;
#pragma unroll
    for (int k = 0; k < D / 32; ++k)  // the elements that come with this product's keys
      l.q[wave][i][k][lane] =
          __builtin_bit_cast(u32x4, load_q(a, qp + (FP8 ? (k / 2) * 64 + quad * 16 + (k & 1) * 8 : k * 32 + quad * 8), r.p[i].there));
  }
  auto edge = [&](int key) { return key + Tile::kKeys > g.first_hi || key < g.last_lo; };
  uint32_t odd = 0;
  if (s.hi > s.lo) {
    const int mine = (int)(lane & (Tile::kKeys - 1));
    Tile ta, tb;
    // as in segment16: page ids two steps ahead, no keys to find past the last step
    auto ids = [&](int key) { return ids16<EVEN>(a, g.table, key <= g.last ? key + mine : 0x7fffff00, s); };
    Ids16 id = ids(g.key0), later = ids(g.key0 + g.step);
    load16<D, FP8, EVEN>(a, g.kp, g.vp, g.kv, id, ta);
    auto next = [&](int key, Tile& t) {
      id = later;
      later = ids(key + g.step);
      __builtin_amdgcn_sched_barrier(0);
      load16<D, FP8, EVEN>(a, g.kp, g.vp, g.kv, id, t);
      __builtin_amdgcn_sched_barrier(0);
    };
    int key = g.key0;
    for (; key + g.step <= g.last; key += 2 * g.step) {
      next(key + g.step, tb);
      block_rows<D, FP8, EVEN, G>(a, l.q[wave], ta, g.kv, key, q.before, edge(key), odd, r);
      next(key + 2 * g.step, ta);
      block_rows<D, FP8, EVEN, G>(a, l.q[wave], tb, g.kv, key + g.step, q.before, edge(key + g.step), odd, r);
    }
    if (key <= g.last) block_rows<D, FP8, EVEN, G>(a, l.q[wave], ta, g.kv, key, q.before, edge(key), odd, r);
  }
  if (__any(odd)) {
#pragma unroll 1
    for (int key = g.key0; key <= g.last; key += g.step) {
      if (!edge(key)) continue;
      odd_keys<D, FP8>(a, g.table, g.vp, g.kv, max(key, s.lo), min(key + Tile::kKeys, s.hi), [&](int at, GlobalBytes v) {
#pragma unroll
        for (int j = 0; j < G; ++j) {
          if (at < r.p[j].lo || at >= r.p[j].hi || !(named(a, r.p[j].row, at - q.before) & 1)) continue;
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int n = 0; n < E; n += 4) {
              const f32x4 y = odd4<FP8>(v + ((quad * 4 + i) * E + n) * (FP8 ? 1 : 2));
#pragma unroll
              for (int e = 0; e < 4; ++e) r.o[j][n + e][i] += y[e];
            }
        }
      });
    }
  }
  const uint32_t heads = 1u << g.hs;
#pragma unroll
  for (int j = 0; j < G; ++j) {
    float sum = r.s[j].sum;
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (heads == kRowWaves) {  // a run of heads for each wavefront
      if (!r.p[j].there) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float y[E];
#pragma unroll
        for (int n = 0; n < E; ++n) y[n] = r.o[j][n][i];
        give_row<D>(a, g, r.p[j], wave * kind.rows + j * 16 + c, (quad * 4 + i) * E, y, r.s[j].m, sum, i == 0 && quad == 0);
      }
      continue;
    }
    // the wavefronts' parts of a run, 16 rows at a time
    __syncthreads();
    if (quad == 0) {
      l.s.m[wave][c] = r.s[j].m;
      l.s.sum[wave][c] = sum;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int n = 0; n < E; ++n) l.s.o[wave][c][(quad * 4 + i) * E + n] = r.o[j][n][i];
    __syncthreads();
    // each thread: E elements of a row
    for (uint32_t f = tid / 16; f < heads * 16; f += 4 * kRowWaves) {
      const uint32_t head = f / 16, i = f % 16, d0 = tid % 16 * E, row = j * 16 + i;
      const Place p = place_of<kTree>(a, kind, q, g.head0 + head, cur.tile, row);
      if (!p.there) continue;
      float top = kNone, total = 0.f, y[E];
      for (uint32_t w = head; w < kRowWaves; w += heads) top = fmaxf(top, l.s.m[w][i]);
#pragma unroll
      for (int n = 0; n < E; ++n) y[n] = 0.f;
      for (uint32_t w = head; w < kRowWaves; w += heads) {
        const float m = l.s.m[w][i], by = m == kNone ? 1.f : exp2_(m - top);  // (a part without a maximum is zeros, or NaN)
        total += l.s.sum[w][i] * by;
#pragma unroll
        for (int n = 0; n < E; ++n) y[n] += l.s.o[w][i][d0 + n] * by;
      }
      give_row<D>(a, g, p, head * kind.rows + row, d0, y, top, total, tid % 16 == 0);
    }
  }
  if (heads != kRowWaves) __syncthreads();  // before the next segment's queries
}

template <int D, bool FP8, bool EVEN>
__device__ __forceinline__ void segment_rows(const AttendArgs& a, LdsRows<D>& l, const Cursor& cur, const Request& q, const Span& s,
                                             uint32_t k0, uint32_t k1) {
  const Kind& kind = a.kind[0];
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  Segment g;
  g.hs = kind.heads_shift;
  g.kp = layer_base(a.c.k);
  g.vp = layer_base(a.c.v);
  g.table = a.b.table + (uint64_t)cur.r * a.b.width;
  g.head0 = cur.head << g.hs;
  g.head = g.head0 + (wave & ((1u << g.hs) - 1));
  g.kv = g.head / kind.parts;
  const int sub = (int)(wave >> g.hs) * Tile16<D, FP8>::kKeys;
  g.step = 1 << kind.block_shift;
  g.key0 = (int)(s.b0 + k0) * g.step + sub;
  g.last = (int)(s.b0 + k1 - 1) * g.step + sub;
  g.first_hi = min(q.held, q.before);
  g.last_lo = a.window ? (int)max((int64_t)0, (int64_t)q.before + q.rows - (int64_t)a.window) : 0;
  g.rows = min(kind.tile_rows, q.rows - cur.tile * kind.tile_rows) * kind.part_heads;
  g.whole = k0 == 0 && k1 == s.n;
  g.slot = (2 * (uint64_t)cur.worker + (k0 > 0 ? 0 : 1)) * a.slot_rows;
  constexpr int most = most_runs(D);
  if (most == 1 || g.rows <= 16)
    segment_rows<D, FP8, EVEN, 1>(a, l, kind, cur, q, s, g);
  else
    segment_rows<D, FP8, EVEN, most>(a, l, kind, cur, q, s, g);
}

template <int D, bool FP8, bool EVEN>
__global__ __launch_bounds__(64 * kRowWaves, 1) void k_attend_rows(AttendArgs a) {
  __shared__ union {
    PlanLds plan;
    LdsRows<D> s;
  } l;
  Cursor cur;
  const bool any = plan<kTree>(a, l.plan, cur);
  if (!any) {
    if (threadIdx.x == 0) ((GlobalShare)a.share)[cur.worker].parts = 0;
    return;
  }
  __syncthreads();  // the plan has been read
  Request q = uniform(request_of(a, cur.r));
  for (bool first = true; cur.at < cur.end; first = false) {
    const Span s = span_of<kTree>(a, q, cur.tile);
    uint32_t k0, k1;
    const uint64_t tile_end = blocks_of<kTree>(a, cur, q, s, k0, k1);
    if (first && threadIdx.x == 0) note_share(a, cur, q, s, k0, k1);
    if (k0 < k1) segment_rows<D, FP8, EVEN>(a, l.s, cur, q, s, k0, k1);
    cur.at = min(cur.end, tile_end);
    if (cur.at == tile_end) {
      cur.first = tile_end;
      if (cur.at < cur.end) next_tile(a, q, cur);
    }
  }
}

// ---- launching ------------------------------------------------------------------------
// Whether a batch goes to k_attend_rows: by its rows (query heads of a K/V head times new
// tokens) per request, on average. us on k_attend_rows / on k_attend_many, 48 requests of
// 1,024 to 32,768 tokens:
//   heads of 64, scaled    32 rows   98 / 139     64 rows  159 / 258    96 rows  215 / 168
//   heads of 128, scaled   32 rows  156 / 240     40 rows  248 / 221    4 to 64 rows, 35 on average  205 / 273
//   heads of 256, scaled   16 rows  265 / 299     20 rows  492 / 309
// and 12 of 1,024 in bf16 on 16 heads of 128: 40 rows 55 / 60, 64 rows 62 / 63, 154 rows 94 / 93.
// (Whatever is left has more rows than what tl_attend takes in tiles of 16, so that shape_of
// gives it tiles of many rows.)
bool by_rows(const tl_ctx* ctx, uint32_t n_q_heads, uint64_t n_reqs, uint64_t n_rows) {
  const uint64_t per = n_rows * (n_q_heads / ctx->H) / (n_reqs ? n_reqs : 1);
  return per <= (ctx->D == 64 ? 64u : ctx->D == 256 ? 16u : ctx->dtype == TL_DTYPE_FP8_SCALED ? 36u : 64u);
}

Shape rows_shape(const tl_ctx* ctx, uint32_t n_q_heads, uint64_t n_reqs, uint64_t n_rows) {
  Shape s;
  const uint32_t group = n_q_heads / ctx->H, wide = ctx->dtype == TL_DTYPE_FP8_SCALED ? 1 : 2;
  s.waves = 0;
  s.workers = 256;
  Kind& k = s.kind[0];
  k = kind_of(ctx, group, 16 * most_runs((int)ctx->D));
  const uint32_t runs = ctx->H * k.parts;
  k.heads_shift = 0;
  while (k.heads_shift < 2 && runs % (2u << k.heads_shift) == 0) ++k.heads_shift;
  k.heads = runs >> k.heads_shift;
  k.block_shift = (ctx->D * wide < 128 ? 6 : 5) + 2 - k.heads_shift;
  k.weight = 1;
  k.cost = 1;
  s.kind[1] = k;
  s.few = ~0u;
  s.slot_rows = k.rows << k.heads_shift;
  s.joins = s.slot_rows / (1024 / ctx->D);
  const uint64_t rows = join_rows(s, k, ctx, n_reqs, n_rows);
  s.least = rows > 32 ? 3 : rows > 8 ? 2 : 1;  // as in shape_of
  return s;
}

// Whether each tile goes to one workgroup as a whole. Where a layer has a window, no tile has more
// keys than that and the new tokens, and if the tiles fill the workgroups, in some rounds, to a good
// part, there is little to even out: no tile is started and ended twice, no parts are written, and
// there is no join. us, cut / whole, window of 1,024, 16 heads of 128, bf16, requests of 77 tokens (16
// tiles each, 256 workgroups): 8 requests 75 / 68, 10 81 / 69, 12 93 / 73, 16 101 / 77, 17 108 / 133, 24 142 / 135, 32
// 172 / 143; of 30 tokens (512 workgroups) 32 requests 102 / 82, 44 166 / 156, 60 246 / 213; of 12
// (k_attend_rows, 4 tiles each) 44 104 / 88, 64 138 / 119, 110 220 / 201; 16 of 1 to 77 tokens 96 / 100.
// But the lengths, which only the device has, may differ by any factor, and then the longest tile
// is what a call waits for: so the window is a small one, of 2,048 keys with the new tokens. Where one
// request is longer than the window and all others have some tokens more than are new, 16 of 77 tokens
// take, with a window of 512 58 / 54, of 1,024 57 / 67, of 2,048 63 / 93, of 16,384 108 / 464 (64 of 12 tokens
// 42 / 36, 47 / 53, 47 / 87, 85 / 569); with lengths that differ less (log-normal, 1,500 in the middle) 75 / 55, 90 / 63,
// 104 / 88, 195 / 469 (79 / 58, 136 / 99, 181 / 157, 297 / 739).
constexpr uint64_t kWholeKeys = 2048;

bool whole_tiles(const tl_ctx* ctx, uint32_t layer, const Shape& s, const Kind& k, uint64_t n_reqs, uint64_t n_rows) {
  const uint64_t tokens = (n_rows + n_reqs - 1) / n_reqs, tiles = n_reqs * k.heads * ((tokens + k.tile_rows - 1) / k.tile_rows);
  const uint64_t rounds = (tiles + s.workers - 1) / s.workers;
  return ctx->window[layer] && ctx->window[layer] + tokens <= kWholeKeys && tiles * 5 >= rounds * s.workers * 3;
}

}  // namespace

size_t attend_tree_needs(const tl_ctx* ctx, uint32_t n_q_heads, uint64_t n_reqs, uint64_t n_rows) {
  if (!by_rows(ctx, n_q_heads, n_reqs, n_rows)) return layout_of(shape_of(ctx, n_q_heads, n_reqs, n_rows), ctx->D).end;
  return layout_of(rows_shape(ctx, n_q_heads, n_reqs, n_rows), ctx->D).end;
}

// Of any call: on k_attend_rows the layout does not depend on the batch.
size_t attend_tree_workspace(const tl_ctx* ctx, uint32_t n_q_heads) { return layout_of(rows_shape(ctx, n_q_heads, 1, 1), ctx->D).end; }

int launch_attend_tree(const tl_ctx* ctx, void* stream, uint32_t layer, const tl_batch* batch, const tl_tree* tree, uint32_t n_q_heads,
                       const tl_rows* q, const tl_cache* cache, float scale, const tl_rows* out, float* d_lse, void* d_ws) {
  AttendArgs a = {};
  a.tree = tree->d_seen;
  a.tree_words = tree->words;
  a.tree_pos = tree->d_pos;
  const bool rows = by_rows(ctx, n_q_heads, batch->n_reqs, batch->n_rows);
  const Shape sh = rows ? rows_shape(ctx, n_q_heads, batch->n_reqs, batch->n_rows) : shape_of(ctx, n_q_heads, batch->n_reqs, batch->n_rows);
  fill(a, sh, ctx, layer, batch, n_q_heads, q, cache, scale, out, d_lse, d_ws);
  if (whole_tiles(ctx, layer, sh, rows ? sh.kind[0] : sh.kind[1], batch->n_reqs, batch->n_rows)) a.tree_whole = a.least = 1;
  hipStream_t s = (hipStream_t)stream;
  (void)hipGetLastError();
  by_cache(ctx, [&](auto D, auto fp8, auto even) {
    {
      TimedLaunch timed(TL_KERNEL_ATTEND, s);
      if (rows)
        hipLaunchKernelGGL((k_attend_rows<D(), fp8(), even()>), dim3(sh.workers), dim3(64 * kRowWaves), 0, s, a);
      else
        launch_many<D(), fp8(), even(), kTree>(sh, s, a);
    }
    if (!a.tree_whole) launch_join<D()>(sh, s, a);
  });
  return hipGetLastError() == hipSuccess ? TL_OK : TL_EDEVICE;
}

}  // namespace tl
