// tl_attend: attention of a batch's new rows over a paged cache, whose pages hold
// bf16 values or 8-bit codes with a power-of-two scale per page and head.
//
// For a query q at one head: s_j = q . k_j * scale over the keys it sees,
// out = sum_j exp(s_j) v_j / sum_j exp(s_j), lse = log sum_j exp(s_j). Keys are
// taken in blocks; the running maximum m (in powers of two, as s is), the sum of
// 2^(s - m) and the products with v are held in 32 bits. m is raised only when a
// block exceeds it by more than 8, so that most blocks rescale nothing: 2^(s - m)
// then stays below 2^8, and the quotient does not depend on m.
//
// The matrix instructions take bf16. A code times its power-of-two scale is a
// bf16 value exactly; the weights 2^(s - m) are rounded to bf16 for the product
// with v (as accurate as the bf16 output), and not for the sum.
#include "paged.h"

namespace tl {

// The part of an item that one worker left to others: see k_attend_join.
struct Share {
  uint64_t first, end;  // units of the item
  uint64_t total;       // units of the call
  uint32_t workers;
  uint32_t r, head, tile;
  uint32_t open;        // the worker's first segment goes on with an item that another began
  uint32_t pad;
};

struct AttendArgs {
  Batch b;
  Pages c;
  const uint16_t* q;
  int64_t q_token, q_head;
  uint16_t* out;
  int64_t o_token, o_head;
  float* lse;  // [rows][query heads] or null
  uint32_t n_heads, group;      // K/V heads, query heads of each
  uint32_t parts, part_heads;   // a K/V head's query heads in `parts` runs of at most part_heads
  uint32_t tile_rows;           // batch rows of a tile: floor(M / part_heads)
  uint32_t all, window;
  float scale;                  // times log2(e)
  Share* share;                 // [workers]
  float* part_ml;               // [2 * workers][M][2]
  float* part_o;                // [2 * workers][M][D]
};

namespace {

constexpr int kThreads = 256;
constexpr float kNone = -__builtin_inff();
constexpr float kSlack = 8.f;  // how far a block's scores may exceed the running maximum

typedef const __attribute__((address_space(4))) uint32_t* ConstU32;

// ---- which keys a tile sees -----------------------------------------------------
struct Span {
  int lo, hi;      // keys [lo, hi) are seen by some row of the tile
  uint32_t b0, n;  // blocks of KT keys from b0 on; at least one, so that every tile has a worker
};

template <int KT>
__device__ __forceinline__ Span span_of(const AttendArgs& a, uint32_t rows, int held, int before, uint32_t tile) {
  Span s;
  s.lo = 0;
  s.hi = held;
  if (!a.all) {
    const int t0 = (int)(tile * a.tile_rows), t1 = (int)min(tile * a.tile_rows + a.tile_rows, rows);
    s.hi = min(held, before + t1);
    if (a.window) s.lo = (int)max((int64_t)0, (int64_t)before + t0 + 1 - (int64_t)a.window);
  }
  s.hi = max(s.hi, 0);
  s.lo = min(s.lo, s.hi);
  s.b0 = (uint32_t)s.lo / KT;
  s.n = max(1u, ((uint32_t)s.hi + KT - 1) / KT - s.b0);
  return s;
}

struct Request {
  uint32_t row0, rows, tiles;
  int held, before;  // keys, and keys before the first row's own
};

__device__ __forceinline__ Request request_of(const AttendArgs& a, uint32_t r) {
  Request q;
  q.row0 = a.b.first_row(r);
  const uint32_t row1 = a.b.first_row(r + 1);
  q.rows = row1 > q.row0 ? row1 - q.row0 : 0;
  q.tiles = (q.rows + a.tile_rows - 1) / a.tile_rows;
  q.held = a.c.n_pages ? (int)a.b.held(r) : 0;
  q.before = (int)min(a.b.kv_len[r], 0x7fffffffu) - (int)q.rows;
  return q;
}

// Blocks of a request's tiles tile0, tile0 + step, ...
template <int KT>
__device__ __forceinline__ uint64_t blocks_of(const AttendArgs& a, const Request& q, uint32_t tile0, uint32_t step) {
  uint64_t n = 0;
  for (uint32_t t = tile0; t < q.tiles; t += step) n += span_of<KT>(a, q.rows, q.held, q.before, t).n;
  return n;
}

// ---- work ------------------------------------------------------------------------
// Units of work are numbered: requests in order, a request's heads, a head's
// tiles, a tile's blocks of keys. A worker (a workgroup) takes an equal run of
// them, which it works out from the lengths on the device: requests of any
// lengths keep all workers busy to the end. A tile whose blocks fall to several
// workers is put together by k_attend_join.
struct Cursor {
  uint64_t at, end;  // units left
  uint64_t total;
  uint32_t workers;
  uint32_t r, head, tile;
  uint64_t first;  // first unit of the tile
};

struct PlanLds {
  uint64_t sum[kThreads + 1];
  uint64_t found_at, found_blocks;
  uint32_t found;
};

template <int KT>
__device__ bool plan(const AttendArgs& a, PlanLds& l, uint32_t worker, Cursor& c) {
  const uint32_t tid = threadIdx.x, n = a.b.n_reqs, heads = a.n_heads * a.parts;
  // threads for each request (few requests), or requests for each thread
  uint32_t split = 1;
  while (split < 64 && 2 * split * n <= kThreads) split *= 2;
  const uint32_t per = (n + kThreads - 1) / kThreads;
  uint64_t mine = 0;
  if (split > 1) {
    const uint32_t r = tid / split;
    if (r < n) mine = blocks_of<KT>(a, request_of(a, r), tid % split, split);
  } else {
    for (uint32_t r = tid * per; r < min(tid * per + per, n); ++r) mine += blocks_of<KT>(a, request_of(a, r), 0, 1);
  }
  mine *= heads;
  uint64_t incl = mine;
  for (uint32_t k = 1; k < 64; k *= 2) {
    const uint64_t up = __shfl_up(incl, k);
    if ((tid & 63) >= k) incl += up;
  }
  __shared__ uint64_t wave_sum[kThreads / 64];
  if ((tid & 63) == 63) wave_sum[tid / 64] = incl;
  __syncthreads();
  uint64_t before = 0;
  for (uint32_t w = 0; w < tid / 64; ++w) before += wave_sum[w];
  l.sum[tid] = before + incl - mine;
  if (tid == kThreads - 1) l.sum[kThreads] = before + incl;
  if (tid == 0) l.found = ~0u;
  __syncthreads();
  c.total = l.sum[kThreads];
  c.workers = (uint32_t)min((uint64_t)gridDim.x, c.total);
  // neighbouring runs of units on the same chiplet, whose workgroups share an L2
  if (c.workers == gridDim.x && gridDim.x % 8 == 0) worker = worker % 8 * (gridDim.x / 8) + worker / 8;
  c.at = c.end = 0;
  if (worker < c.workers) {
    c.at = c.total * worker / c.workers;
    c.end = c.total * (worker + 1) / c.workers;
  }
  const uint32_t step = split;
  if (c.at < c.end && tid % step == 0 && l.sum[tid] <= c.at && c.at < l.sum[tid + step]) {
    l.found = tid / step * (split > 1 ? 1 : per);
    l.found_at = l.sum[tid];
  }
  __syncthreads();
  if (l.found == ~0u) return false;
  c.r = l.found;
  c.first = l.found_at;
  while (c.r < n) {
    const Request q = request_of(a, c.r);
    const uint64_t blocks = split > 1 ? (l.sum[(c.r + 1) * split] - l.sum[c.r * split]) / heads : blocks_of<KT>(a, q, 0, 1);
    if (c.at < c.first + blocks * heads) {
      c.head = (uint32_t)((c.at - c.first) / blocks);
      c.first += c.head * blocks;
      c.tile = 0;
      for (;;) {
        const uint32_t k = span_of<KT>(a, q.rows, q.held, q.before, c.tile).n;
        if (c.at < c.first + k) return true;
        c.first += k;
        ++c.tile;
      }
    }
    c.first += blocks * heads;
    ++c.r;
  }
  return false;
}

// The tile after (r, head, tile); its first unit is c.first.
__device__ __forceinline__ void next_tile(const AttendArgs& a, Cursor& c) {
  if (++c.tile < request_of(a, c.r).tiles) return;
  c.tile = 0;
  if (++c.head < a.n_heads * a.parts) return;
  c.head = 0;
  while (++c.r < a.b.n_reqs && request_of(a, c.r).tiles == 0) {
  }
}

// ---- one row ------------------------------------------------------------------------
// Row m of a tile: batch row and query head.
struct Place {
  uint32_t row, head;
  bool there;
  int lo, hi;  // it sees keys [lo, hi)
};

__device__ __forceinline__ Place place_of(const AttendArgs& a, const Request& q, uint32_t head, uint32_t tile, uint32_t m) {
  Place p;
  const uint32_t part = head % a.parts, kv = head / a.parts;
  const uint32_t tok = m / a.part_heads, g = part * a.part_heads + m % a.part_heads;
  const uint32_t i = tile * a.tile_rows + tok;
  p.there = tok < a.tile_rows && i < q.rows && g < a.group;
  p.row = q.row0 + (p.there ? i : 0);
  p.head = kv * a.group + (p.there ? g : 0);
  p.lo = 0;
  p.hi = q.held;
  if (!a.all) {
    const int position = q.before + (int)i;
    p.hi = min(q.held, position + 1);
    if (a.window) p.lo = (int)max((int64_t)0, (int64_t)position + 1 - (int64_t)a.window);
  }
  if (!p.there) p.hi = p.lo;
  return p;
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// ---- tiles of 16 rows -----------------------------------------------------------------
// For few rows per request. Every key and value is used by 16 rows at most, so
// the cache's bytes are what it costs: they go from memory to registers in the
// layout that the matrix instructions take, with no stop in shared memory. Each
// of a workgroup's four wavefronts takes 32 of a block's 128 keys.
//
// S^T = K Q^T with mfma 16x16x32: lane l gives key l % 16 and takes row l % 16.
// Its result holds keys 4 * (l / 16) + i, i < 4, of each half of the 32: the
// eight weights that the lane gives to O^T = V^T P^T, whose sum over keys runs in
// that order. For V a lane loads D / 16 neighbouring elements of those eight
// keys and transposes them in registers: product n takes element n of each.
constexpr int kBlock16 = 128;

template <int D, bool FP8>
struct Tile16 {
  static constexpr int kElems = D / 16;                        // of V per lane and key
  static constexpr int kKWords = FP8 ? D / 16 : D / 8;         // 32-bit words of K per lane and key
  static constexpr int kVWords = FP8 ? kElems / 4 : kElems / 2;
  uint32_t k[2][kKWords];
  uint32_t v[8][kVWords];
  float k_scale[2], v_scale[8];
  uint32_t seen;  // which of the 32 keys are to be used
};

struct Ids16 {  // of one of 32 keys per lane
  uint32_t page;
  uint32_t row;
  bool in;
};

__device__ __forceinline__ Ids16 ids16(const AttendArgs& a, const int32_t* table, int key, const Span& s) {
  Ids16 x;
  x.in = key >= s.lo && key < s.hi;
  const uint32_t at = x.in ? (uint32_t)key : 0u, i = a.b.page.div(at);
  x.row = at - i * a.b.page.d;
  x.page = (uint32_t)table[i];
  return x;
}

template <int D, bool FP8>
__device__ __forceinline__ void load16(const AttendArgs& a, const uint8_t* kp, const uint8_t* vp, uint32_t kv, const Ids16& id,
                                       Tile16<D, FP8>& t) {
  constexpr int kRow = FP8 ? D : 2 * D;  // bytes of a head's row
  const uint32_t lane = threadIdx.x & 63, c = lane % 16, quad = lane / 16;
  const bool fine = id.in && id.page < a.c.n_pages;
  t.seen = (uint32_t)__ballot(fine);
  // keys that are not to be used are read from page 0
  const int64_t page = fine ? (int64_t)id.page * a.c.stride : 0;
  const int64_t off = page + (fine ? (int64_t)id.row * a.n_heads * kRow : 0) + (int64_t)kv * kRow;
  uint32_t scale = 127;
  if (FP8) scale = scale_held((lane < 32 ? kp : vp)[page + a.c.scale_off + kv]);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t at = __shfl(off, h * 16 + c);
    const uint8_t* p = kp + at + 16 * quad;
#pragma unroll
    for (int i = 0; i < Tile16<D, FP8>::kKWords / 4; ++i) {
      const u32x4 w = *(const u32x4*)(p + 64 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) t.k[h][4 * i + j] = w[j];
    }
    if (FP8) t.k_scale[h] = scale_value(__shfl(scale, h * 16 + c));
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t key = (i / 4) * 16 + quad * 4 + i % 4;
    const uint8_t* p = vp + __shfl(off, key) + kRow / 16 * c;
    constexpr int W = Tile16<D, FP8>::kVWords;
    if constexpr (W >= 4) {
#pragma unroll
      for (int k = 0; k < W / 4; ++k) {
        const u32x4 w = *(const u32x4*)(p + 16 * k);
#pragma unroll
        for (int j = 0; j < 4; ++j) t.v[i][4 * k + j] = w[j];
      }
    } else if constexpr (W == 2) {
      const u32x2 w = *(const u32x2*)p;
      t.v[i][0] = w[0];
      t.v[i][1] = w[1];
    } else {
      t.v[i][0] = *(const uint32_t*)p;
    }
    if (FP8) t.v_scale[i] = scale_value(__shfl(scale, 32 + key));
  }
}

__device__ __forceinline__ uint32_t widen(uint32_t codes, float scale, bool high) {
  const bf16x2 p = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true)
                        : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false);
  return __builtin_bit_cast(uint32_t, p);
}

__device__ __forceinline__ bf16x8 as_bf16(u32x4 w) { return __builtin_bit_cast(bf16x8, w); }

// The running state of one row, on every lane that works for it. `top` is m, or
// 0 while the row has seen nothing; `sum` a lane's own part.
struct Soft {
  float m, top, sum;
};

template <int D, bool FP8>
struct Rows16 {
  bf16x8 q[D / 32];
  f32x4 o[D / 16];
  Soft s;
};

template <int D, bool FP8>
__device__ __forceinline__ void block16(const AttendArgs& a, Tile16<D, FP8>& t, int key0, const Place& p, bool edge,
                                        Rows16<D, FP8>& r) {
  const uint32_t quad = (threadIdx.x & 63) / 16;
  float x[8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
      u32x4 w;
      if constexpr (FP8) {
        w[0] = widen(t.k[h][2 * k], t.k_scale[h], false);
        w[1] = widen(t.k[h][2 * k], t.k_scale[h], true);
        w[2] = widen(t.k[h][2 * k + 1], t.k_scale[h], false);
        w[3] = widen(t.k[h][2 * k + 1], t.k_scale[h], true);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = t.k[h][4 * k + j];
      }
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(w), r.q[k], acc, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) x[4 * h + i] = acc[i] * a.scale;
  }
  if (edge || t.seen != ~0u) {  // some row does not see some key
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = (i / 4) * 16 + quad * 4 + i % 4;
      const bool there = t.seen >> at & 1;
      x[i] = there && key0 + at >= p.lo && key0 + at < p.hi ? x[i] : kNone;
      if (!there) {  // whatever a page holds there, it may be NaN
#pragma unroll
        for (int j = 0; j < Tile16<D, FP8>::kVWords; ++j) t.v[i][j] = 0;
      }
    }
  }
  float top = x[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i]);
  if (__any(top > r.s.m + kSlack)) {
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float m = fmaxf(r.s.m, top);
    const float now = m == kNone ? 0.f : m;
    const float by = r.s.m == kNone ? 0.f : exp2_(r.s.top - now);
    r.s.m = m;
    r.s.top = now;
    r.s.sum *= by;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) r.o[i] *= by;
  }
  bf16x8 w;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float y = exp2_(x[i] - r.s.top);
    r.s.sum += y;
    w[i] = (__bf16)y;
  }
#pragma unroll
  for (int n = 0; n < Tile16<D, FP8>::kElems; n += 2) {
    uint32_t e[8];  // elements n, n + 1 of each key
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (FP8)
        e[i] = widen(t.v[i][n / 4], t.v_scale[i], n & 2);
      else
        e[i] = t.v[i][n / 2];
    }
    u32x4 lo, hi;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo[i] = __builtin_amdgcn_perm(e[2 * i + 1], e[2 * i], 0x05040100);
      hi[i] = __builtin_amdgcn_perm(e[2 * i + 1], e[2 * i], 0x07060302);
    }
    r.o[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(lo), w, r.o[n], 0, 0, 0);
    r.o[n + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(hi), w, r.o[n + 1], 0, 0, 0);
  }
}

__device__ __forceinline__ void store_bf16x4(uint16_t* p, float x, float y, float z, float w) {
  const bf16x2 lo = {(__bf16)x, (__bf16)y}, hi = {(__bf16)z, (__bf16)w};
  *(u32x2*)p = u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}

// A row's result from its sums: zeros and minus infinity for a row that saw nothing.
__device__ __forceinline__ float lse_of(float top, float sum) {
  return sum == 0.f ? kNone : (top + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
}

template <int D, bool FP8>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void k_attend16(AttendArgs a) {
  constexpr int M = 16;
  __shared__ union {
    PlanLds plan;
    struct {
      float m[4][M], sum[4][M];
      float o[4][M][D];
    } s;
  } l;
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid / 64, c = lane % 16, quad = lane / 16;
  Cursor cur;
  const bool any = plan<kBlock16>(a, l.plan, blockIdx.x, cur);
  uint32_t worker = blockIdx.x;
  if (cur.workers == gridDim.x && gridDim.x % 8 == 0) worker = worker % 8 * (gridDim.x / 8) + worker / 8;
  if (!any) {
    if (tid == 0) a.share[worker].open = 0;
    return;
  }
  const uint8_t* kp = (const uint8_t*)*a.c.k;
  const uint8_t* vp = (const uint8_t*)*a.c.v;
  bool first_segment = true;
  while (cur.at < cur.end) {
    const Request q = request_of(a, cur.r);
    const Span s = span_of<kBlock16>(a, q.rows, q.held, q.before, cur.tile);
    const uint32_t k0 = (uint32_t)(cur.at - cur.first), k1 = (uint32_t)min((uint64_t)s.n, cur.end - cur.first);
    const uint32_t kv = cur.head / a.parts;
    const int32_t* table = a.b.table + (uint64_t)cur.r * a.b.width;
    if (first_segment && tid == 0) {
      Share& sh = a.share[worker];
      sh.first = cur.first;
      sh.end = cur.first + s.n;
      sh.total = cur.total;
      sh.workers = cur.workers;
      sh.r = cur.r;
      sh.head = cur.head;
      sh.tile = cur.tile;
      sh.open = k0 > 0;
    }
    first_segment = false;

    const Place p = place_of(a, q, cur.head, cur.tile, c);
    Rows16<D, FP8> r;
    r.s = Soft{kNone, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < D / 16; ++i) r.o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    {
      const uint16_t* qp = a.q + (int64_t)p.row * a.q_token + (int64_t)p.head * a.q_head;
#pragma unroll
      for (int k = 0; k < D / 32; ++k) {
        // bf16 keys come 64 bytes at a time, codes too: the same elements of q
        const int at = FP8 ? (k / 2) * 64 + quad * 16 + (k & 1) * 8 : k * 32 + quad * 8;
        u32x4 w = {0, 0, 0, 0};
        if (p.there) w = *(const u32x4*)(qp + at);
        r.q[k] = as_bf16(w);
      }
    }
    // rows of a tile that do not all see the same keys: blocks that some row does not see whole
    const uint32_t rows_here = min(a.tile_rows, q.rows - cur.tile * a.tile_rows);
    const int first_hi = a.all ? q.held : min(q.held, q.before + (int)(cur.tile * a.tile_rows) + 1);
    const int last_lo = a.all || !a.window ? 0 : max(0, (int)min((int64_t)0x7fffffff, (int64_t)q.before + (int)(cur.tile * a.tile_rows + rows_here) - (int64_t)a.window));

    const int key0 = (int)((s.b0 + k0) * kBlock16 + wave * 32);
    const int last = (int)((s.b0 + k1 - 1) * kBlock16 + wave * 32);
    if (s.hi > s.lo) {
      Tile16<D, FP8> ta, tb;
      Ids16 id = ids16(a, table, key0 + (int)(lane & 31), s);
      load16<D, FP8>(a, kp, vp, kv, id, ta);
      id = ids16(a, table, min(key0 + kBlock16, last) + (int)(lane & 31), s);
      for (int key = key0; key <= last; key += 2 * kBlock16) {
        load16<D, FP8>(a, kp, vp, kv, id, tb);
        id = ids16(a, table, min(key + 2 * kBlock16, last) + (int)(lane & 31), s);
        block16<D, FP8>(a, ta, key, p, key + 32 > first_hi || key < last_lo, r);
        if (key + kBlock16 > last) break;
        load16<D, FP8>(a, kp, vp, kv, id, ta);
        id = ids16(a, table, min(key + 3 * kBlock16, last) + (int)(lane & 31), s);
        block16<D, FP8>(a, tb, key + kBlock16, p, key + kBlock16 + 32 > first_hi || key + kBlock16 < last_lo, r);
      }
    }

    // the four wavefronts' parts
    float sum = r.s.sum;
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    __syncthreads();
    if (quad == 0) {
      l.s.m[wave][c] = r.s.m;
      l.s.sum[wave][c] = sum;
    }
    __syncthreads();
    float top = kNone;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, l.s.m[w][c]);
    const float by = r.s.m == kNone ? 0.f : exp2_(r.s.m - top);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int n = 0; n < D / 16; ++n) l.s.o[wave][c][(quad * 4 + i) * (D / 16) + n] = r.o[n][i] * by;
    __syncthreads();
    // each thread: D / 16 elements of one row
    const uint32_t m = tid / 16, d0 = tid % 16 * (D / 16);
    float row_top = kNone, row_sum = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) row_top = fmaxf(row_top, l.s.m[w][m]);
#pragma unroll
    for (int w = 0; w < 4; ++w) row_sum += l.s.m[w][m] == kNone ? 0.f : l.s.sum[w][m] * exp2_(l.s.m[w][m] - row_top);
    const Place pm = place_of(a, q, cur.head, cur.tile, m);
    const bool whole = k0 == 0 && k1 == s.n;
    if (pm.there) {
      const float inv = row_sum == 0.f ? 0.f : 1.f / row_sum;
      const uint64_t slot = 2 * (uint64_t)worker + (k0 > 0 ? 0 : 1);
      uint16_t* op = a.out + (int64_t)pm.row * a.o_token + (int64_t)pm.head * a.o_head + d0;
      float* fp = a.part_o + (slot * M + m) * D + d0;
#pragma unroll
      for (int n = 0; n < D / 16; n += 4) {
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) y += *(const f32x4*)&l.s.o[w][m][d0 + n];
        if (whole)
          store_bf16x4(op + n, y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
        else
          *(f32x4*)(fp + n) = y;
      }
      if (tid % 16 == 0) {
        if (!whole) {
          a.part_ml[(slot * M + m) * 2] = row_top;
          a.part_ml[(slot * M + m) * 2 + 1] = row_sum;
        } else if (a.lse) {
          a.lse[(uint64_t)pm.row * a.n_heads * a.group + pm.head] = lse_of(row_top, row_sum);
        }
      }
    }
    cur.at = cur.first + k1;
    if (k1 == s.n) {
      cur.first += s.n;
      if (cur.at < cur.end) next_tile(a, cur);
    }
  }
}

// ---- tiles of 128 rows --------------------------------------------------------------
// For prompts. A block of 64 keys and values is widened to bf16 once, into shared
// memory, and used by the 32 rows of each of four wavefronts; the next block's
// bytes are on their way meanwhile.
//
// S^T = K Q^T with mfma 32x32x16: lane l takes row l % 32, and its result holds
// keys 8 * (i / 4) + 4 * (l / 32) + i % 4. Registers 8a .. 8a + 7 are what the
// lane gives to step a of O^T = V^T P^T, whose keys run in that order: V comes
// from shared memory through transposing reads of four keys each.
constexpr int kBlock128 = 64;

template <int D>
struct Lds128 {
  uint16_t k[kBlock128 * D], v[kBlock128 * D];
  int64_t off[2][kBlock128];       // byte offsets of the keys' rows
  uint32_t scale[2][kBlock128];    // scale bytes: K's, and V's in bits 8 to 15; 0: not to be used
  uint64_t seen[2];                // keys that are to be used
};

// Where 8 neighbouring elements, chunk c of key r, are kept: such that lanes
// that read together use all banks.
template <int D>
__device__ __forceinline__ uint32_t k_at(uint32_t r, uint32_t c) {
  return r * D + (c ^ (r & 7)) * 8;
}
template <int D>
__device__ __forceinline__ uint32_t v_at(uint32_t r, uint32_t elem) {  // elem: a multiple of 4
  const uint32_t sw = D == 64 ? (r >> 1 & 1) : (r & 3);
  return r * D + (elem ^ (sw * 32));
}

template <int D, bool FP8>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void k_attend128(AttendArgs a) {
  constexpr int M = 128, KT = kBlock128;
  constexpr int kRow = FP8 ? D : 2 * D;
  constexpr int kLoads = KT * kRow / 16 / kThreads;  // 16-byte pieces of K (and of V) per thread
  constexpr int kPieces = kRow / 16;                 // pieces of a key
  __shared__ union {
    PlanLds plan;
    Lds128<D> s;
  } l;
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid / 64, c = lane % 32, half = lane / 32;
  Cursor cur;
  const bool any = plan<KT>(a, l.plan, blockIdx.x, cur);
  uint32_t worker = blockIdx.x;
  if (cur.workers == gridDim.x && gridDim.x % 8 == 0) worker = worker % 8 * (gridDim.x / 8) + worker / 8;
  if (!any) {
    if (tid == 0) a.share[worker].open = 0;
    return;
  }
  const uint8_t* kp = (const uint8_t*)*a.c.k;
  const uint8_t* vp = (const uint8_t*)*a.c.v;
  bool first_segment = true;
  while (cur.at < cur.end) {
    const Request q = request_of(a, cur.r);
    const Span s = span_of<KT>(a, q.rows, q.held, q.before, cur.tile);
    const uint32_t k0 = (uint32_t)(cur.at - cur.first), k1 = (uint32_t)min((uint64_t)s.n, cur.end - cur.first);
    const uint32_t kv = cur.head / a.parts;
    const int32_t* table = a.b.table + (uint64_t)cur.r * a.b.width;
    if (first_segment && tid == 0) {
      Share& sh = a.share[worker];
      sh.first = cur.first;
      sh.end = cur.first + s.n;
      sh.total = cur.total;
      sh.workers = cur.workers;
      sh.r = cur.r;
      sh.head = cur.head;
      sh.tile = cur.tile;
      sh.open = k0 > 0;
    }
    first_segment = false;

    const uint32_t m = wave * 32 + c;
    const Place p = place_of(a, q, cur.head, cur.tile, m);
    bf16x8 qf[D / 16];
    {
      const uint16_t* qp = a.q + (int64_t)p.row * a.q_token + (int64_t)p.head * a.q_head;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        u32x4 w = {0, 0, 0, 0};
        if (p.there) w = *(const u32x4*)(qp + k * 16 + half * 8);
        qf[k] = as_bf16(w);
      }
    }
    // keys that some row of this wavefront sees, and keys that all of them see
    int wave_lo, wave_hi, all_lo, all_hi;
    {
      int lo = p.there ? p.lo : 0x7fffffff, hi = p.there ? p.hi : 0, lo2 = p.there ? p.lo : 0, hi2 = p.there ? p.hi : 0x7fffffff;
      for (uint32_t k = 1; k < 32; k *= 2) {
        lo = min(lo, __shfl_xor(lo, k));
        hi = max(hi, __shfl_xor(hi, k));
        lo2 = max(lo2, __shfl_xor(lo2, k));
        hi2 = min(hi2, __shfl_xor(hi2, k));
      }
      wave_lo = __builtin_amdgcn_readfirstlane(lo);
      wave_hi = __builtin_amdgcn_readfirstlane(hi);
      all_lo = __builtin_amdgcn_readfirstlane(lo2);
      all_hi = __builtin_amdgcn_readfirstlane(hi2);
    }
    f32x16 o[D / 32];
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
    Soft st = {kNone, 0.f, 0.f};

    const int block0 = (int)(s.b0 + k0) * KT, block_last = (int)(s.b0 + k1 - 1) * KT;
    u32x4 kr[kLoads], vr[kLoads];
    // wavefront 0: where the keys of a block are
    auto find = [&](int key0, Ids16& id) {
      if (wave == 0) id = ids16(a, table, key0 + (int)lane, s);
    };
    auto scales = [&](const Ids16& id, uint32_t& ks, uint32_t& vs) {
      if (!FP8 || wave != 0) return;
      const int64_t at = (id.in && id.page < a.c.n_pages ? (int64_t)id.page * a.c.stride : 0) + a.c.scale_off + kv;
      ks = kp[at];
      vs = vp[at];
    };
    auto note = [&](const Ids16& id, uint32_t ks, uint32_t vs, uint32_t slot) {
      if (wave != 0) return;
      const bool fine = id.in && id.page < a.c.n_pages;
      const int64_t page = fine ? (int64_t)id.page * a.c.stride : 0;
      uint32_t sc = 0x7f7f;
      if (FP8) sc = scale_held(ks) | scale_held(vs) << 8;
      l.s.off[slot][lane] = page + (fine ? (int64_t)id.row * a.n_heads * kRow : 0) + (int64_t)kv * kRow;
      l.s.scale[slot][lane] = fine ? sc : 0;
      const uint64_t seen = __ballot(fine);
      if (lane == 0) l.s.seen[slot] = seen;
    };
    auto fetch = [&](uint32_t slot) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const uint32_t at = tid + i * kThreads, row = at / kPieces, piece = at % kPieces;
        const int64_t off = l.s.off[slot][row] + piece * 16;
        kr[i] = *(const u32x4*)(kp + off);
        vr[i] = *(const u32x4*)(vp + off);
      }
    };
    auto keep = [&](uint32_t slot) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const uint32_t at = tid + i * kThreads, row = at / kPieces, piece = at % kPieces;
        const uint32_t sc = l.s.scale[slot][row];
        if constexpr (FP8) {
          const float ks = scale_value(sc & 0xff), vs = scale_value(sc >> 8);
          u32x4 w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            w[j / 2][j % 2 * 2] = widen(kr[i][j], ks, false);
            w[j / 2][j % 2 * 2 + 1] = widen(kr[i][j], ks, true);
            w[2 + j / 2][j % 2 * 2] = sc ? widen(vr[i][j], vs, false) : 0;
            w[2 + j / 2][j % 2 * 2 + 1] = sc ? widen(vr[i][j], vs, true) : 0;
          }
          *(u32x4*)(l.s.k + k_at<D>(row, 2 * piece)) = w[0];
          *(u32x4*)(l.s.k + k_at<D>(row, 2 * piece + 1)) = w[1];
          *(u32x4*)(l.s.v + v_at<D>(row, 16 * piece)) = w[2];
          *(u32x4*)(l.s.v + v_at<D>(row, 16 * piece + 8)) = w[3];
        } else {
          *(u32x4*)(l.s.k + k_at<D>(row, piece)) = kr[i];
          *(u32x4*)(l.s.v + v_at<D>(row, 8 * piece)) = sc ? vr[i] : u32x4{0, 0, 0, 0};
        }
      }
    };

    const bool some = s.hi > s.lo;
    if (some) {
      Ids16 id, later;
      uint32_t ks = 0, vs = 0;
      __syncthreads();
      find(block0, id);
      scales(id, ks, vs);
      note(id, ks, vs, 0);
      find(min(block0 + KT, block_last), id);
      scales(id, ks, vs);
      note(id, ks, vs, 1);
      find(min(block0 + 2 * KT, block_last), id);
      __syncthreads();
      fetch(0);
      uint32_t slot = 0;
      for (int key0 = block0; key0 <= block_last; key0 += KT, slot ^= 1) {
        keep(slot);
        const uint64_t seen = l.s.seen[slot];
        __syncthreads();
        fetch(slot ^ 1);
        scales(id, ks, vs);
        find(min(key0 + 3 * KT, block_last), later);
        if (key0 < wave_hi && key0 + KT > wave_lo) {
          float x[2][16];
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            f32x16 acc;
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[j] = 0.f;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
              const u32x4 w = *(const u32x4*)(l.s.k + k_at<D>(b * 32 + c, 2 * k + half));
              acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16(w), qf[k], acc, 0, 0, 0);
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) x[b][j] = acc[j] * a.scale;
          }
          if (seen != ~0ull || key0 < all_lo || key0 + KT > all_hi) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
              for (int j = 0; j < 16; ++j) {
                const int at = b * 32 + 8 * (j / 4) + 4 * half + j % 4;
                const bool there = (seen >> at & 1) && key0 + at >= p.lo && key0 + at < p.hi;
                x[b][j] = there ? x[b][j] : kNone;
              }
          }
          float top = x[0][0];
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int j = 0; j < 16; ++j) top = fmaxf(top, x[b][j]);
          if (__any(top > st.m + kSlack)) {
            top = fmaxf(top, __shfl_xor(top, 32));
            const float mm = fmaxf(st.m, top);
            const float now = mm == kNone ? 0.f : mm;
            const float by = st.m == kNone ? 0.f : exp2_(st.top - now);
            st.m = mm;
            st.top = now;
            st.sum *= by;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) o[i] *= by;
          }
          bf16x8 w[4];
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const float y = exp2_(x[b][j] - st.top);
              st.sum += y;
              w[2 * b + j / 8][j % 8] = (__bf16)y;
            }
#pragma unroll
          for (int st4 = 0; st4 < 4; ++st4) {
            const uint32_t i = lane % 16, key = st4 * 16 + half * 4 + i / 4;
#pragma unroll
            for (int d = 0; d < D / 32; ++d) {
              const uint32_t elem = d * 32 + (lane / 16 % 2) * 16 + i % 4 * 4;
              typedef short s16x4 __attribute__((ext_vector_type(4)));
              typedef __attribute__((address_space(3))) s16x4* Lds4;
              const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4)(l.s.v + v_at<D>(key, elem)));
              const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4)(l.s.v + v_at<D>(key + 8, elem)));
              const u32x2 lw = __builtin_bit_cast(u32x2, lo), hw = __builtin_bit_cast(u32x2, hi);
              o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16(u32x4{lw[0], lw[1], hw[0], hw[1]}), w[st4], o[d], 0, 0, 0);
            }
          }
        }
        note(id, ks, vs, slot);
        id = later;
        __syncthreads();
      }
    }

    float sum = st.sum + __shfl_xor(st.sum, 32);
    const bool whole = k0 == 0 && k1 == s.n;
    if (p.there) {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      const uint64_t slot = 2 * (uint64_t)worker + (k0 > 0 ? 0 : 1);
      uint16_t* op = a.out + (int64_t)p.row * a.o_token + (int64_t)p.head * a.o_head;
      float* fp = a.part_o + (slot * M + m) * D;
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
          const uint32_t at = d * 32 + 2 * j + 4 * half;
          if (whole)
            store_bf16x4(op + at, o[d][j] * inv, o[d][j + 1] * inv, o[d][j + 2] * inv, o[d][j + 3] * inv);
          else
            *(f32x4*)(fp + at) = f32x4{o[d][j], o[d][j + 1], o[d][j + 2], o[d][j + 3]};
        }
      if (half == 0) {
        if (!whole) {
          a.part_ml[(slot * M + m) * 2] = st.m;
          a.part_ml[(slot * M + m) * 2 + 1] = sum;
        } else if (a.lse) {
          a.lse[(uint64_t)p.row * a.n_heads * a.group + p.head] = lse_of(st.top, sum);
        }
      }
    }
    cur.at = cur.first + k1;
    if (k1 == s.n) {
      cur.first += s.n;
      if (cur.at < cur.end) next_tile(a, cur);
    }
  }
}

// ---- joining ---------------------------------------------------------------------------
// A tile that several workers share: the workgroup of the second of them (the
// first that goes on with it) adds up their parts, in the workers' order.
template <int M, int D>
__global__ __launch_bounds__(kThreads) void k_attend_join(AttendArgs a) {
  const uint32_t worker = blockIdx.x + 1;
  const Share sh = a.share[worker];
  if (!sh.open) return;
  auto start = [&](uint64_t w) { return sh.total * w / sh.workers; };
  if (start(worker - 1) > sh.first) return;  // the worker before goes on with it as well
  uint32_t last = worker;
  while (start(last + 1) < sh.end) ++last;
  const Request q = request_of(a, sh.r);
  constexpr int kLanes = D / 4;  // of a row
  for (uint32_t m = threadIdx.x / kLanes; m < M; m += kThreads / kLanes) {
    const Place p = place_of(a, q, sh.head, sh.tile, m);
    if (!p.there) continue;
    const uint32_t d = threadIdx.x % kLanes * 4;
    float top = kNone;
    for (uint32_t w = worker - 1; w <= last; ++w) {
      const uint64_t slot = 2 * (uint64_t)w + (w < worker ? 1 : 0);
      top = fmaxf(top, a.part_ml[(slot * M + m) * 2]);
    }
    float sum = 0.f;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    for (uint32_t w = worker - 1; w <= last; ++w) {
      const uint64_t slot = 2 * (uint64_t)w + (w < worker ? 1 : 0);
      const float pm = a.part_ml[(slot * M + m) * 2];
      const float by = pm == kNone ? 0.f : exp2_(pm - top);
      sum += a.part_ml[(slot * M + m) * 2 + 1] * by;
      y += *(const f32x4*)(a.part_o + (slot * M + m) * D + d) * by;
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    store_bf16x4(a.out + (int64_t)p.row * a.o_token + (int64_t)p.head * a.o_head + d, y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
    if (a.lse && d == 0) a.lse[(uint64_t)p.row * a.n_heads * a.group + p.head] = lse_of(top, sum);
  }
}

// ---- launching ----------------------------------------------------------------------------
struct Shape {
  uint32_t rows;     // of a tile
  uint32_t workers;  // workgroups: as many as the device holds at a time
};

Shape shape_of(const tl_ctx* ctx, uint32_t n_q_heads, uint64_t n_reqs, uint64_t n_rows) {
  Shape s;
  const uint64_t per = n_rows * (n_q_heads / ctx->H) / (n_reqs ? n_reqs : 1);
  s.rows = per <= 32 ? 16 : 128;
  s.workers = ctx->D == 256 ? 256 : 512;
  return s;
}

struct Layout {
  uint64_t ml, o, end;
};
Layout layout_of(const Shape& s, uint32_t D) {
  Layout l;
  l.ml = ((uint64_t)s.workers * sizeof(Share) + 255) / 256 * 256;
  l.o = l.ml + 2ull * s.workers * s.rows * 2 * 4;
  l.end = l.o + 2ull * s.workers * s.rows * D * 4;
  return l;
}

template <int D, bool FP8>
void launch(const Shape& sh, hipStream_t s, const AttendArgs& a) {
  {
    TimedLaunch timed(TL_KERNEL_ATTEND, s);
    if (sh.rows == 16)
      hipLaunchKernelGGL((k_attend16<D, FP8>), dim3(sh.workers), dim3(kThreads), 0, s, a);
    else
      hipLaunchKernelGGL((k_attend128<D, FP8>), dim3(sh.workers), dim3(kThreads), 0, s, a);
  }
  TimedLaunch timed(TL_KERNEL_ATTEND_JOIN, s);
  if (sh.rows == 16)
    hipLaunchKernelGGL((k_attend_join<16, D>), dim3(sh.workers - 1), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((k_attend_join<128, D>), dim3(sh.workers - 1), dim3(kThreads), 0, s, a);
}

}  // namespace

size_t attend_workspace(const tl_ctx* ctx, uint32_t n_q_heads, uint64_t n_reqs, uint64_t n_rows) {
  return (layout_of(shape_of(ctx, n_q_heads, n_reqs, n_rows), ctx->D).end + 255) / 256 * 256;
}

int launch_attend(const tl_ctx* ctx, void* stream, uint32_t layer, const tl_batch* batch, uint32_t n_q_heads, const tl_rows* q,
                  const tl_cache* cache, float scale, uint32_t flags, const tl_rows* out, float* d_lse, void* d_ws) {
  AttendArgs a = {};
  fill_batch(a.b, ctx, layer, batch);
  fill_pages(a.c, ctx, layer, cache);
  a.q = (const uint16_t*)q->d_rows;
  a.q_token = q->row_stride;
  a.q_head = q->head_stride;
  a.out = (uint16_t*)out->d_rows;
  a.o_token = out->row_stride;
  a.o_head = out->head_stride;
  a.lse = d_lse;
  a.n_heads = ctx->H;
  a.group = n_q_heads / ctx->H;
  const Shape sh = shape_of(ctx, n_q_heads, batch->n_reqs, batch->n_rows);
  a.parts = (a.group + sh.rows - 1) / sh.rows;
  a.part_heads = (a.group + a.parts - 1) / a.parts;
  a.tile_rows = sh.rows / a.part_heads;
  a.all = (flags & TL_ATTEND_ALL) != 0;
  a.window = a.all ? 0 : (uint32_t)ctx->window[layer];
  a.scale = scale * 1.4426950408889634f;
  const Layout lay = layout_of(sh, ctx->D);
  a.share = (Share*)d_ws;
  a.part_ml = (float*)((uint8_t*)d_ws + lay.ml);
  a.part_o = (float*)((uint8_t*)d_ws + lay.o);
  hipStream_t s = (hipStream_t)stream;
  (void)hipGetLastError();
  const bool fp8 = ctx->dtype == TL_DTYPE_FP8_SCALED;
  switch (ctx->D) {
    case 64: fp8 ? launch<64, true>(sh, s, a) : launch<64, false>(sh, s, a); break;
    case 128: fp8 ? launch<128, true>(sh, s, a) : launch<128, false>(sh, s, a); break;
    default: fp8 ? launch<256, true>(sh, s, a) : launch<256, false>(sh, s, a); break;
  }
  return hipGetLastError() == hipSuccess ? TL_OK : TL_EDEVICE;
}

}  // namespace tl
