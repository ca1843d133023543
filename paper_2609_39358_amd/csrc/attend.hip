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
#include <algorithm>
#include <type_traits>

#include "paged.h"

namespace tl {

// What the joining kernel has to know of a worker's first tile.
struct Share {
  uint32_t parts;  // workers of the tile, this one the second of them; 0: nothing to join here
  uint32_t kind, head, tile;
  uint32_t row0, rows;  // of the request
};

// Not a generic pointer: with such a store on its way, every wait for a load is
// for all of them.
typedef __attribute__((address_space(1))) Share* GlobalShare;

// How requests are cut into tiles: of 16 rows, or of 32 for each wavefront.
struct Kind {
  uint32_t rows;               // of a tile
  uint32_t parts, part_heads;  // a K/V head's query heads in `parts` runs of at most part_heads
  uint32_t tile_rows;          // batch rows of a tile: floor(rows / part_heads)
  uint32_t heads_shift;        // log2 of the runs that a workgroup takes together
  uint32_t heads;              // how many times it does so for a batch row's heads
  uint32_t block_shift;        // log2 of the keys of a block
  uint32_t weight;             // units of a block
  uint32_t cost;               // units that a tile takes besides: finding it, its queries, its result
};

struct AttendArgs {
  Batch b;
  Pages c;
  const uint16_t* q;
  int64_t q_token, q_head;
  uint16_t* out;
  int64_t o_token, o_head;
  float* lse;                // [rows][query heads] or null
  uint32_t n_heads, group;   // K/V heads, query heads of each
  Kind kind[2];
  uint32_t few;              // requests of at most this many rows are of kind 0
  uint32_t all, window;
  float scale;               // times log2(e), above 0
  uint32_t q_sign;           // flips the signs of q for scales below 0
  uint32_t slot_rows;        // rows of a worker's part
  uint32_t joins;            // workgroups that join a tile's parts
  uint32_t least;            // units that a worker has, at least
  Share* share;              // [workers]
  float* part_ml;            // [2 * workers][slot_rows][2]
  float* part_o;             // [2 * workers][slot_rows][D]
};

namespace {

constexpr int kPlan = 256;  // threads that make a plan
constexpr float kNone = -__builtin_inff();
constexpr float kSlack = 8.f;  // how far a block's scores may exceed the running maximum

// ---- which keys a tile sees -----------------------------------------------------
struct Request {
  uint32_t row0, rows, tiles;
  int held, before;  // keys, and keys before the first row's own
  uint32_t kind, tile_rows, heads, block_shift, weight, cost;  // as in Kind
};

__device__ __forceinline__ Request request_of(const AttendArgs& a, uint32_t r) {
  Request q;
  q.row0 = a.b.first_row(r);
  const uint32_t row1 = a.b.first_row(r + 1), kv_len = a.b.kv_len[r];
  q.rows = row1 > q.row0 ? row1 - q.row0 : 0;
  q.held = a.c.n_pages ? (int)min(kv_len, a.b.most) : 0;
  q.before = (int)min(kv_len, kMostTokens + (1u << 15)) - (int)q.rows;  // behind any table's end it does not matter how far
  q.kind = q.rows > a.few;
  q.tile_rows = q.kind ? a.kind[1].tile_rows : a.kind[0].tile_rows;
  q.heads = q.kind ? a.kind[1].heads : a.kind[0].heads;
  q.block_shift = q.kind ? a.kind[1].block_shift : a.kind[0].block_shift;
  q.weight = q.kind ? a.kind[1].weight : a.kind[0].weight;
  q.cost = q.kind ? a.kind[1].cost : a.kind[0].cost;
  q.tiles = (q.rows + q.tile_rows - 1) / q.tile_rows;
  return q;
}

// What a whole workgroup works on, in scalar registers.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint64_t uniform(uint64_t x) {
  return (uint64_t)uniform((uint32_t)(x >> 32)) << 32 | uniform((uint32_t)x);
}
__device__ __forceinline__ Request uniform(Request q) {
  return Request{uniform(q.row0), uniform(q.rows), uniform(q.tiles), uniform(q.held), uniform(q.before),
                 uniform(q.kind), uniform(q.tile_rows), uniform(q.heads), uniform(q.block_shift), uniform(q.weight), uniform(q.cost)};
}

struct Span {
  int lo, hi;      // keys [lo, hi) are seen by some row of the tile
  uint32_t b0, n;  // blocks of keys from b0 on; at least one, so that every tile has a worker
};

__device__ __forceinline__ Span span_of(const AttendArgs& a, const Request& q, uint32_t tile) {
  Span s;
  s.lo = 0;
  s.hi = q.held;
  if (!a.all) {
    const int t0 = (int)(tile * q.tile_rows), t1 = (int)min(tile * q.tile_rows + q.tile_rows, q.rows);
    s.hi = min(q.held, q.before + t1);
    if (a.window) s.lo = (int)max((int64_t)0, (int64_t)q.before + t0 + 1 - (int64_t)a.window);
  }
  s.hi = max(s.hi, 0);
  s.lo = min(s.lo, s.hi);
  s.b0 = (uint32_t)s.lo >> q.block_shift;
  s.n = s.hi > s.lo ? (((uint32_t)s.hi - 1) >> q.block_shift) + 1 - s.b0 : 1;
  return s;
}

// Units of a request's tiles tile0, tile0 + step, ...
__device__ __forceinline__ uint64_t units_of(const AttendArgs& a, const Request& q, uint32_t tile0, uint32_t step) {
  uint64_t n = 0;
  for (uint32_t t = tile0; t < q.tiles; t += step) n += q.cost + q.weight * span_of(a, q, t).n;
  return n;
}

// ---- work ------------------------------------------------------------------------
// Units of work are numbered: requests in order, a request's heads, a head's
// tiles, a tile's cost and its blocks of keys. A worker (a workgroup) takes an equal run of
// them, which it works out from the lengths on the device: requests of any
// lengths keep all workers busy to the end. A tile whose blocks fall to several
// workers is put together by k_attend_join.
struct Cursor {
  uint64_t at, end;  // units left
  uint64_t total;
  uint32_t workers, worker;
  uint32_t r, head, tile;
  uint64_t first;  // first unit of the tile
};

struct PlanLds {
  uint64_t sum[kPlan + 1];
  uint64_t found_at;
  uint32_t found;
};

__device__ bool plan(const AttendArgs& a, PlanLds& l, Cursor& c) {
  const uint32_t tid = threadIdx.x, n = a.b.n_reqs;
  // threads for each request (few requests), or requests for each thread
  uint32_t split = 1;
  while (split < 64 && 2 * split * n <= kPlan) split *= 2;
  const uint32_t per = (n + kPlan - 1) / kPlan;
  uint64_t mine = 0;
  if (split > 1) {
    if (tid / split < n) {
      const Request q = request_of(a, tid / split);
      mine = units_of(a, q, tid % split, split) * q.heads;
    }
  } else if (tid < kPlan) {
    for (uint32_t r = tid * per; r < min(tid * per + per, n); ++r) {
      const Request q = request_of(a, r);
      mine += units_of(a, q, 0, 1) * q.heads;
    }
  }
  uint64_t incl = mine;
  for (uint32_t k = 1; k < 64; k *= 2) {
    const uint64_t up = __shfl_up(incl, k);
    if ((tid & 63) >= k) incl += up;
  }
  __shared__ uint64_t wave_sum[kPlan / 64];
  if ((tid & 63) == 63 && tid < kPlan) wave_sum[tid / 64] = incl;
  __syncthreads();
  if (tid < kPlan) {
    uint64_t before = 0;
    for (uint32_t w = 0; w < tid / 64; ++w) before += wave_sum[w];
    l.sum[tid] = before + incl - mine;
    if (tid == kPlan - 1) l.sum[kPlan] = before + incl;
  }
  if (tid == 0) l.found = ~0u;
  __syncthreads();
  c.total = uniform(l.sum[kPlan]);
  c.workers = (uint32_t)min((uint64_t)gridDim.x, (c.total + a.least - 1) / a.least);
  // runs that follow each other go to workgroups of one chiplet, which share an L2
  c.worker = blockIdx.x;
  if (c.workers == gridDim.x && gridDim.x % 8 == 0) c.worker = c.worker % 8 * (gridDim.x / 8) + c.worker / 8;
  c.at = c.end = 0;
  if (c.worker < c.workers) {
    c.at = c.total * c.worker / c.workers;
    c.end = c.total * (c.worker + 1) / c.workers;
  }
  if (c.at < c.end && tid < kPlan && tid % split == 0 && l.sum[tid] <= c.at && c.at < l.sum[tid + split]) {
    l.found = tid / split * (split > 1 ? 1 : per);
    l.found_at = l.sum[tid];
  }
  __syncthreads();
  c.r = uniform(l.found);
  if (c.r == ~0u) return false;
  c.first = uniform(l.found_at);
  while (c.r < n) {
    const Request q = uniform(request_of(a, c.r));
    const uint64_t units = split > 1 ? uniform(l.sum[(c.r + 1) * split] - l.sum[c.r * split]) / q.heads : units_of(a, q, 0, 1);
    if (c.at < c.first + units * q.heads) {
      c.head = (uint32_t)((c.at - c.first) / units);
      c.first += c.head * units;
      c.tile = 0;
      for (;;) {
        const uint32_t k = q.cost + q.weight * span_of(a, q, c.tile).n;
        if (c.at < c.first + k) return true;
        c.first += k;
        ++c.tile;
      }
    }
    c.first += units * q.heads;
    ++c.r;
  }
  return false;
}

// The blocks [k0, k1) of the cursor's tile that begin in its run (none where the run
// ends within the tile's cost, or begins within its last block), and the tile's end.
__device__ __forceinline__ uint64_t blocks_of(const Cursor& c, const Request& q, const Span& s, uint32_t& k0, uint32_t& k1) {
  const int64_t n = (int64_t)s.n * q.weight;
  const uint64_t block0 = c.first + q.cost;
  const uint32_t u0 = (uint32_t)min(n, max((int64_t)0, (int64_t)(c.at - block0)));
  const uint32_t u1 = (uint32_t)min(n, max((int64_t)0, (int64_t)(c.end - block0)));
  k0 = (u0 + q.weight - 1) / q.weight;
  k1 = (u1 + q.weight - 1) / q.weight;
  return block0 + n;
}

// The tile after the cursor's; its first unit is c.first.
__device__ __forceinline__ void next_tile(const AttendArgs& a, Request& q, Cursor& c) {
  if (++c.tile < q.tiles) return;
  c.tile = 0;
  if (++c.head < q.heads) return;
  c.head = 0;
  while (++c.r < a.b.n_reqs && (q = uniform(request_of(a, c.r))).tiles == 0) {
  }
}

// A worker's first tile, for the joining kernel: worker w's run begins at
// floor(total * w / workers). The second worker of a tile sees to it.
__device__ void note_share(const AttendArgs& a, const Cursor& c, const Request& q, const Span& s, uint32_t k0, uint32_t k1) {
  Share sh = {0, q.kind, c.head, c.tile, q.row0, q.rows};
  const uint64_t block0 = c.first + q.cost, last = block0 + (uint64_t)(s.n - 1) * q.weight;  // where its first and last block begin
  if (k0 > 0 && k0 < k1 && c.total * (c.worker - 1) < (block0 + 1) * c.workers)  // this worker goes on with it, the one before begins it
    sh.parts = (uint32_t)(((last + 1) * c.workers - 1) / c.total) + 2 - c.worker;
  typedef __attribute__((address_space(1))) u32x2* Out;
  const Out to = (Out)(a.share + c.worker);
  to[0] = u32x2{sh.parts, sh.kind};
  to[1] = u32x2{sh.head, sh.tile};
  to[2] = u32x2{sh.row0, sh.rows};
}

// ---- one row ------------------------------------------------------------------------
// Row m of a tile: batch row and query head.
struct Place {
  uint32_t row, head;
  bool there;
  int lo, hi;  // it sees keys [lo, hi)
};

__device__ __forceinline__ Place place_of(const AttendArgs& a, const Kind& k, const Request& q, uint32_t head, uint32_t tile, uint32_t m) {
  Place p;
  const uint32_t part = head % k.parts, kv = head / k.parts;
  const uint32_t tok = m / k.part_heads, g = part * k.part_heads + m % k.part_heads;
  const uint32_t i = tile * k.tile_rows + tok;
  p.there = tok < k.tile_rows && i < q.rows && g < a.group;
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

__device__ __forceinline__ uint32_t widen(uint32_t codes, float scale, bool high) {
  const bf16x2 p = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true)
                        : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false);
  return __builtin_bit_cast(uint32_t, p);
}

__device__ __forceinline__ bf16x8 as_bf16(u32x4 w) { return __builtin_bit_cast(bf16x8, w); }

__device__ __forceinline__ bf16x8 load_q(const AttendArgs& a, const uint16_t* p, bool there) {
  u32x4 w = {0, 0, 0, 0};
  if (there) w = *(const u32x4*)p;
  return as_bf16(w ^ a.q_sign);
}

__device__ __forceinline__ void store_bf16x4(uint16_t* p, float x, float y, float z, float w) {
  const bf16x2 lo = {(__bf16)x, (__bf16)y}, hi = {(__bf16)z, (__bf16)w};
  *(u32x2*)p = u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}

// The running state of one row, on every lane that works for it. `top` is m, or
// 0 while the row has seen nothing; `sum` a lane's own part. Scores that are NaN
// raise no maximum: a row (or a part of one) that has none has sums of 0, or NaN,
// which count wherever parts are put together.
struct Soft {
  float m, top, sum;
};

// A row's result from its sums: minus infinity for a row that saw nothing.
__device__ __forceinline__ float lse_of(float top, float sum) {
  return sum == 0.f ? kNone : (top + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
}

// ---- values that are not finite ---------------------------------------------------------
// A row's weight for a key that it does not see is 0, but 0 times NaN is NaN: a
// value that is not finite would reach the rows of its tile that do not see it. In
// the blocks whose keys not all rows of a tile see, such values are taken out, and
// added at the tile's end to the rows that do see them.
//
// All bits of the elements of a word that are not finite.
template <bool FP8>
__device__ __forceinline__ uint32_t odd_bits(uint32_t w) {
  if (FP8) return (((w & 0x7f7f7f7fu) + 0x01010101u) >> 7 & 0x01010101u) * 0xffu;
  return (((w >> 7 & 0x00ff00ffu) + 0x00010001u) >> 8 & 0x00010001u) * 0xffffu;
}

// Four neighbouring elements, 0 in place of finite ones.
template <bool FP8>
__device__ __forceinline__ f32x4 odd4(GlobalBytes p) {
  f32x4 x;
  if constexpr (FP8) {
    const uint32_t bad = odd_bits<true>(*(GlobalU32)p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(bad >> (8 * i) & 1 ? 0x7fc00000u : 0u);
  } else {
    u32x2 w = *(GlobalU32x2)p;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      w[i] &= odd_bits<false>(w[i]);
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  return x;
}

__device__ __forceinline__ int64_t lane_value(int64_t x, uint32_t lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)x, lane), hi = __builtin_amdgcn_readlane((uint32_t)(x >> 32), lane);
  return (int64_t)((uint64_t)hi << 32 | lo);
}

// use(key, its values) for those keys of [lo, hi) whose values are not all
// finite, by a wavefront.
template <int D, bool FP8, class Use>
__device__ __forceinline__ void odd_keys(const AttendArgs& a, const int32_t* table, GlobalBytes vp, uint32_t kv, int lo, int hi, Use use) {
  constexpr uint32_t kRow = FP8 ? D : 2 * D;
#pragma unroll 1
  for (int k = lo; k < hi; k += 64) {
    const uint32_t key = (uint32_t)min(k + (int)(threadIdx.x & 63), hi - 1), at = a.b.page.div(key), page = (uint32_t)table[at];
    const bool fine = page < a.c.n_pages;
    const int64_t off = (fine ? (int64_t)page * a.c.stride : 0) + (int64_t)(key - at * a.b.page.d) * (a.n_heads * kRow) + (int64_t)kv * kRow;
    uint32_t bad = 0;
#pragma unroll 1
    for (uint32_t i = 0; i < kRow; i += 16) {
      const u32x4 w = *(GlobalU32x4)(vp + off + i);
      bad |= odd_bits<FP8>(w[0]) | odd_bits<FP8>(w[1]) | odd_bits<FP8>(w[2]) | odd_bits<FP8>(w[3]);
    }
    uint64_t some = __ballot(fine && bad && k + (int)(threadIdx.x & 63) < hi);
#pragma unroll 1
    for (; some; some &= some - 1) {
      const uint32_t i = (uint32_t)__builtin_ctzll(some);
      use(k + (int)i, vp + lane_value(off, i));
    }
  }
}

// ---- tiles of 16 rows -----------------------------------------------------------------
// For few rows per request. Every key and value is used by 16 rows at most, so
// the cache's bytes are what it costs: they go from memory to registers in the
// layout that the matrix instructions take, with no stop in shared memory. A
// workgroup's four wavefronts take neighbouring heads of the same keys, whose
// rows lie side by side (where the number of heads is not a multiple of four or
// two, keys that follow each other).
//
// S^T = K Q^T with mfma 16x16x32: lane l gives key l % 16 and takes row l % 16.
// Its result holds keys 4 * (l / 16) + i, i < 4, of each half of 32 keys: the
// eight weights that the lane gives to O^T = V^T P^T, whose sum over keys runs in
// that order. For V a lane loads D / 16 neighbouring elements of those eight
// keys and transposes them in registers: product n takes element n of each.
template <int D, bool FP8>
struct Tile16 {
  // keys of a wavefront's step: two steps in flight are what hides the memory's
  // latency, so short rows come in longer steps
  static constexpr int kGroups = D * (FP8 ? 1 : 2) < 128 ? 2 : 1;
  static constexpr int kKeys = 32 * kGroups;
  static constexpr int kElems = D / 16;                        // of V per lane and key
  static constexpr int kKWords = FP8 ? D / 16 : D / 8;         // 32-bit words of K per lane and key
  static constexpr int kVWords = FP8 ? kElems / 4 : kElems / 2;
  uint32_t k[2 * kGroups][kKWords];
  uint32_t v[8 * kGroups][kVWords];
  uint32_t ks, vs;  // a lane's key's (or sixteen keys') words of scale bytes
  uint64_t seen;  // which of the keys are to be used
};

// Where a step's keys are, a lane per key. Pages of whole sixteens of keys: a
// lane knows the first of its sixteen.
struct Ids16 {
  uint32_t page, row;
  bool in, some;
};

template <bool EVEN>
__device__ __forceinline__ Ids16 ids16(const AttendArgs& a, const int32_t* table, int key, const Span& s) {
  Ids16 x;
  x.in = key >= s.lo && key < s.hi;
  const int first = EVEN ? key & ~15 : key;
  x.some = EVEN ? first + 16 > s.lo && first < s.hi : x.in;
  const uint32_t at = x.some ? (uint32_t)first : 0u, i = a.b.page.div(at);
  x.row = at - i * a.b.page.d;
  x.page = (uint32_t)table[i];
  return x;
}

template <int N>
__device__ __forceinline__ void load_words(uint32_t* w, GlobalBytes p) {
  if constexpr (N >= 4) {
#pragma unroll
    for (int k = 0; k < N / 4; ++k) {
      const u32x4 x = *(GlobalU32x4)(p + 16 * k);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[4 * k + j] = x[j];
    }
  } else if constexpr (N == 2) {
    const u32x2 x = *(GlobalU32x2)p;
    w[0] = x[0];
    w[1] = x[1];
  } else {
    w[0] = *(GlobalU32)p;
  }
}

template <int D, bool FP8, bool EVEN>
__device__ __forceinline__ void load16(const AttendArgs& a, GlobalBytes kp, GlobalBytes vp, uint32_t kv, const Ids16& id,
                                       Tile16<D, FP8>& t) {
  typedef Tile16<D, FP8> Tile;
  constexpr uint32_t kRow = FP8 ? D : 2 * D;  // bytes of a head's row
  const uint32_t lane = threadIdx.x & 63, c = lane % 16, quad = lane / 16;
  const bool fine = id.some && id.page < a.c.n_pages;
  t.seen = __ballot(fine && id.in);
  // keys that are not to be used are read from page 0
  const int64_t page = fine ? (int64_t)id.page * a.c.stride : 0;
  const uint32_t step = a.n_heads * kRow;  // bytes from a key to the next
  const int64_t off = page + (fine ? (int64_t)id.row * step : 0) + (int64_t)kv * kRow;
  if (FP8) {
    t.ks = scale_word(kp + page, a.c.scale_off, kv);
    t.vs = scale_word(vp + page, a.c.scale_off, kv);
  }
#pragma unroll
  for (int h = 0; h < 2 * Tile::kGroups; ++h) {
    GlobalBytes p;
    if constexpr (EVEN)
      p = kp + lane_value(off, h * 16) + (c * step + 16 * quad);
    else
      p = kp + __shfl(off, h * 16 + c) + 16 * quad;
#pragma unroll
    for (int i = 0; i < Tile::kKWords / 4; ++i) load_words<4>(t.k[h] + 4 * i, p + 64 * i);
  }
#pragma unroll
  for (int i = 0; i < 8 * Tile::kGroups; ++i) {
    const uint32_t key = quad * 4 + i % 4, half = i / 4 * 16;
    GlobalBytes p;
    if constexpr (EVEN)
      p = vp + lane_value(off, half) + (key * step + kRow / 16 * c);
    else
      p = vp + __shfl(off, half + key) + kRow / 16 * c;
    load_words<Tile::kVWords>(t.v[i], p);
  }
}

template <int D, bool FP8>
struct Rows16 {
  bf16x8 q[D / 32];
  f32x4 o[D / 16];
  Soft s;
};

template <int D, bool FP8, bool EVEN>
__device__ __forceinline__ void block16(const AttendArgs& a, Tile16<D, FP8>& t, uint32_t kv, int key0, const Place& p, bool edge,
                                        bool several, uint32_t& odd, Rows16<D, FP8>& r) {
  typedef Tile16<D, FP8> Tile;
  constexpr int N = 8 * Tile::kGroups;
  const uint32_t lane = threadIdx.x & 63, c = lane % 16, quad = lane / 16;
  float k_scale[2 * Tile::kGroups], v_scale[EVEN ? 2 * Tile::kGroups : N];
  if constexpr (FP8) {
    const uint32_t kb = scale_held(scale_of(t.ks, kv)), vb = scale_held(scale_of(t.vs, kv));
#pragma unroll
    for (int h = 0; h < 2 * Tile::kGroups; ++h) {
      k_scale[h] = scale_value(EVEN ? __builtin_amdgcn_readlane(kb, h * 16) : __shfl(kb, h * 16 + c));
      if constexpr (EVEN) v_scale[h] = scale_value(__builtin_amdgcn_readlane(vb, h * 16));
    }
    if constexpr (!EVEN)
#pragma unroll
      for (int i = 0; i < N; ++i) v_scale[i] = scale_value(__shfl(vb, i / 4 * 16 + quad * 4 + i % 4));
  }
  float x[N];
#pragma unroll
  for (int h = 0; h < 2 * Tile::kGroups; ++h) {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
      u32x4 w;
      if constexpr (FP8) {
        w[0] = widen(t.k[h][2 * k], k_scale[h], false);
        w[1] = widen(t.k[h][2 * k], k_scale[h], true);
        w[2] = widen(t.k[h][2 * k + 1], k_scale[h], false);
        w[3] = widen(t.k[h][2 * k + 1], k_scale[h], true);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = t.k[h][4 * k + j];
      }
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(w), r.q[k], acc, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) x[4 * h + i] = acc[i];
  }
  if (edge || t.seen != ~0ull) {  // some row does not see some key
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = (i / 4) * 16 + quad * 4 + i % 4;
      const bool there = t.seen >> at & 1;
      x[i] = there && key0 + at >= p.lo && key0 + at < p.hi ? x[i] : kNone;
      if (!there) {  // whatever a page holds there, it may be NaN
#pragma unroll
        for (int j = 0; j < Tile::kVWords; ++j) t.v[i][j] = 0;
      }
    }
  }
  if (edge && several)
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < Tile::kVWords; ++j) {
        const uint32_t bad = odd_bits<FP8>(t.v[i][j]);
        odd |= bad;
        t.v[i][j] &= ~bad;
      }
  float top = x[0];
#pragma unroll
  for (int i = 1; i < N; ++i) top = fmaxf(top, x[i]);
  top *= a.scale;
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
#pragma unroll
  for (int g = 0; g < Tile::kGroups; ++g) {
    bf16x8 w;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float y = exp2_(__builtin_fmaf(x[8 * g + i], a.scale, -r.s.top));
      r.s.sum += y;
      w[i] = (__bf16)y;
    }
#pragma unroll
    for (int n = 0; n < Tile::kElems; n += 2) {
      uint32_t e[8];  // elements n, n + 1 of each key
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (FP8)
          e[i] = widen(t.v[8 * g + i][n / 4], v_scale[EVEN ? 2 * g + i / 4 : 8 * g + i], n & 2);
        else
          e[i] = t.v[8 * g + i][n / 2];
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
}

template <int D, int WAVES>
struct Lds16 {
  float m[WAVES][16], sum[WAVES][16];
  float o[WAVES][16][D];
};

// The cursor's blocks of one tile of 16 rows for each of a workgroup's runs of
// heads, up to the cursor's end or the tile's.
template <int D, bool FP8, bool EVEN, int WAVES>
__device__ __forceinline__ void segment16(const AttendArgs& a, Lds16<D, WAVES>& l, const Cursor& cur, const Request& q, const Span& s,
                                          uint32_t k0, uint32_t k1) {
  constexpr int M = 16, E = D / 16;
  typedef Tile16<D, FP8> Tile;
  const Kind& kind = a.kind[0];
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64), c = lane % 16, quad = lane / 16;
  const uint32_t hs = kind.heads_shift, heads = 1u << hs;
  const int step = 1 << kind.block_shift;  // keys of a block
  const GlobalBytes kp = layer_base(a.c.k), vp = layer_base(a.c.v);
  const int32_t* table = a.b.table + (uint64_t)cur.r * a.b.width;
  const uint32_t head = (cur.head << hs) + (wave & (heads - 1)), sub = wave >> hs;
  const uint32_t kv = head / kind.parts;
  const Place p = place_of(a, kind, q, head, cur.tile, c);
  Rows16<D, FP8> r;
  r.s = Soft{kNone, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < E; ++i) r.o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  {
    const uint16_t* qp = a.q + (int64_t)p.row * a.q_token + (int64_t)p.head * a.q_head;
#pragma unroll
    for (int k = 0; k < D / 32; ++k)  // the elements that come with this product's keys
      r.q[k] = load_q(a, qp + (FP8 ? (k / 2) * 64 + quad * 16 + (k & 1) * 8 : k * 32 + quad * 8), p.there);
  }
  // keys below first_hi and from last_lo on are seen by all rows of the tile
  const int t0 = (int)(cur.tile * kind.tile_rows), t1 = (int)min(cur.tile * kind.tile_rows + kind.tile_rows, q.rows);
  const int first_hi = a.all ? q.held : min(q.held, q.before + t0 + 1);
  const int last_lo = a.window ? (int)max((int64_t)0, (int64_t)q.before + t1 - (int64_t)a.window) : 0;

  const int key0 = (int)(s.b0 + k0) * step + (int)sub * Tile::kKeys, last = (int)(s.b0 + k1 - 1) * step + (int)sub * Tile::kKeys;
  const bool several = !a.all && t1 - t0 > 1;  // rows that see different keys
  auto edge = [&](int key) { return key + Tile::kKeys > first_hi || key < last_lo; };
  uint32_t odd = 0;
  if (s.hi > s.lo) {
    const int mine = (int)(lane & (Tile::kKeys - 1));
    Tile ta, tb;
    // Page ids are asked for two steps ahead and before the keys of the step
    // between: who waits for them does not wait for those.
    // Past the last step there are no keys to find: the same row is read, from near.
    auto ids = [&](int key) { return ids16<EVEN>(a, table, key <= last ? key + mine : 0x7fffff00, s); };
    Ids16 id = ids(key0), later = ids(key0 + step);
    load16<D, FP8, EVEN>(a, kp, vp, kv, id, ta);
    auto next = [&](int key, Tile& t) {  // the step from `key` on is on its way, into t
      id = later;
      later = ids(key + step);
      __builtin_amdgcn_sched_barrier(0);
      load16<D, FP8, EVEN>(a, kp, vp, kv, id, t);
      __builtin_amdgcn_sched_barrier(0);
    };
    int key = key0;
    for (; key + step <= last; key += 2 * step) {  // no way out in between: it would have every load waited for
      next(key + step, tb);
      block16<D, FP8, EVEN>(a, ta, kv, key, p, edge(key), several, odd, r);
      next(key + 2 * step, ta);
      block16<D, FP8, EVEN>(a, tb, kv, key + step, p, edge(key + step), several, odd, r);
    }
    if (key <= last) block16<D, FP8, EVEN>(a, ta, kv, key, p, edge(key), several, odd, r);
  }

  if (several && __any(odd)) {
#pragma unroll 1
    for (int key = key0; key <= last; key += step) {
      if (!edge(key)) continue;
      odd_keys<D, FP8>(a, table, vp, kv, max(key, s.lo), min(key + Tile::kKeys, s.hi), [&](int at, GlobalBytes v) {
        if (at < p.lo || at >= p.hi) return;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int n = 0; n < E; n += 4) {
            const f32x4 y = odd4<FP8>(v + ((quad * 4 + i) * E + n) * (FP8 ? 1 : 2));
#pragma unroll
            for (int j = 0; j < 4; ++j) r.o[n + j][i] += y[j];
          }
      });
    }
  }
  float sum = r.s.sum;
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  const bool whole = k0 == 0 && k1 == s.n;
  const uint64_t slot = (2 * (uint64_t)cur.worker + (k0 > 0 ? 0 : 1)) * a.slot_rows;
  // a row's E elements from d0 on, its maximum and its sum, to where they belong
  auto give = [&](const Place& at, uint32_t m, uint32_t d0, const float* y, float top, float total, bool one) {
    if (whole) {
      const float inv = total == 0.f ? 0.f : 1.f / total;
      uint16_t* op = a.out + (int64_t)at.row * a.o_token + (int64_t)at.head * a.o_head + d0;
#pragma unroll
      for (int n = 0; n < E; n += 4) store_bf16x4(op + n, y[n] * inv, y[n + 1] * inv, y[n + 2] * inv, y[n + 3] * inv);
      if (one && a.lse) a.lse[(uint64_t)at.row * a.n_heads * a.group + at.head] = lse_of(top, total);
      return;
    }
    float* fp = a.part_o + (slot + m) * D + d0;
#pragma unroll
    for (int n = 0; n < E; n += 4) *(f32x4*)(fp + n) = f32x4{y[n], y[n + 1], y[n + 2], y[n + 3]};
    if (one) *(f32x2*)(a.part_ml + (slot + m) * 2) = f32x2{top, total};
  };
  if (heads == WAVES) {  // a run of heads for each wavefront
    if (p.there) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float y[E];
#pragma unroll
        for (int n = 0; n < E; ++n) y[n] = r.o[n][i];
        give(p, wave * M + c, (quad * 4 + i) * E, y, r.s.m, sum, i == 0 && quad == 0);
      }
    }
    return;
  }
  // the wavefronts' parts of a run
  __syncthreads();
  if (quad == 0) {
    l.m[wave][c] = r.s.m;
    l.sum[wave][c] = sum;
  }
  __syncthreads();
  float top = kNone;
  for (uint32_t w = wave & (heads - 1); w < WAVES; w += heads) top = fmaxf(top, l.m[w][c]);
  const float by = r.s.m == kNone ? 0.f : exp2_(r.s.m - top);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int n = 0; n < E; ++n) l.o[wave][c][(quad * 4 + i) * E + n] = r.o[n][i] * by;
  __syncthreads();
  // each thread: E elements of a row
  for (uint32_t f = tid / 16; f < heads * M; f += 4 * WAVES) {
    const uint32_t h = f / M, m = f % M, d0 = tid % 16 * E;
    const Place pm = place_of(a, kind, q, (cur.head << hs) + h, cur.tile, m);
    if (!pm.there) continue;
    float row_top = kNone, row_sum = 0.f, y[E];
    for (uint32_t w = h; w < WAVES; w += heads) row_top = fmaxf(row_top, l.m[w][m]);
    for (uint32_t w = h; w < WAVES; w += heads) row_sum += l.m[w][m] == kNone ? l.sum[w][m] : l.sum[w][m] * exp2_(l.m[w][m] - row_top);
#pragma unroll
    for (int n = 0; n < E; ++n) y[n] = 0.f;
    for (uint32_t w = h; w < WAVES; w += heads)
#pragma unroll
      for (int n = 0; n < E; ++n) y[n] += l.o[w][m][d0 + n];
    give(pm, f, d0, y, row_top, row_sum, tid % 16 == 0);
  }
}

// Tiles of 16 rows for all requests. One token over 97,000 in scaled pages of 16
// heads of 128: 78 us, 5.1 TB/s (a large copy reaches 4.7); 64 requests of up to
// 32,768 164 us, 5.2 TB/s.
template <int D, bool FP8, bool EVEN>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void k_attend16(AttendArgs a) {
  __shared__ union {
    PlanLds plan;
    Lds16<D, 4> s;
  } l;
  Cursor cur;
  const bool any = plan(a, l.plan, cur);
  if (!any) {
    if (threadIdx.x == 0) ((GlobalShare)a.share)[cur.worker].parts = 0;
    return;
  }
  Request q = uniform(request_of(a, cur.r));
  for (bool first = true; cur.at < cur.end; first = false) {
    const Span s = span_of(a, q, cur.tile);
    uint32_t k0, k1;
    const uint64_t tile_end = blocks_of(cur, q, s, k0, k1);
    if (first && threadIdx.x == 0) note_share(a, cur, q, s, k0, k1);
    if (k0 < k1) segment16<D, FP8, EVEN, 4>(a, l.s, cur, q, s, k0, k1);
    cur.at = min(cur.end, tile_end);
    if (cur.at == tile_end) {
      cur.first = tile_end;
      if (cur.at < cur.end) next_tile(a, q, cur);
    }
  }
}

// ---- tiles of many rows ---------------------------------------------------------------------
// For prompts. A block of 64 keys and values is widened to bf16 once, into shared
// memory, and used by the R rows of each wavefront.
//
// S^T = K Q^T with mfma 32x32x16 (R = 32) or 16x16x32 (R = 16, for heads of 256,
// whose 32 rows would not fit two wavefronts' registers on a SIMD): lane l takes
// row l % R, and its result holds keys 8 * (i / 4) + 4 * (l / R) + i % 4 of R.
// Eight of those registers at a time are what the lane gives to a step of
// O^T = V^T P^T, whose keys run in that order: V comes from shared memory
// through transposing reads of four keys each.
//
// With eight wavefronts two share a SIMD. They work in opposite phases, with a
// barrier after each: while one wavefront's products (P V of this block, Q K of the
// next) use the matrix unit, the other's exponentials use the vector unit.
template <int D>
struct LdsMany {
  static constexpr int KT = 64;  // keys of a block
  alignas(1024) uint16_t k[2][KT * D];
  uint16_t v[2][KT * D];
};

typedef __attribute__((address_space(3))) const char* LdsAddress;
typedef __attribute__((address_space(3))) u32x4* LdsU32x4;
// (the low half of a generic address is the one in shared memory)
__device__ __forceinline__ uint32_t lds_of(const void* p) { return (uint32_t)(uintptr_t)p; }

template <int R>
struct Products;
template <>
struct Products<32> {
  typedef f32x16 Sum;
  static __device__ __forceinline__ Sum add(bf16x8 a, bf16x8 b, Sum c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Products<16> {
  typedef f32x4 Sum;
  static __device__ __forceinline__ Sum add(bf16x8 a, bf16x8 b, Sum c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
__host__ __device__ constexpr int rows_of_wave(int dim) { return dim == 256 ? 16 : 32; }

// Where an element is kept: such that lanes that read or write together use all
// banks. K: 8 neighbouring elements, chunk c of key r.
template <int D>
__device__ __forceinline__ constexpr uint32_t k_swap(uint32_t r) {
  return D == 64 ? r >> 1 & 7 : r & 15;
}
template <int D>
__device__ __forceinline__ uint32_t k_at(uint32_t r, uint32_t c) {
  return r * D + (c ^ k_swap<D>(r)) * 8;
}
// V: elem a multiple of 4.
template <int D>
__device__ __forceinline__ uint32_t v_swap(uint32_t r) {
  return (D == 64 ? (r >> 1 & 1) : (r & 3)) * 32 + (D == 256 ? (r >> 2 & 1) : 0) * 16 + (r & 1) * 8;
}
template <int D>
__device__ __forceinline__ uint32_t v_at(uint32_t r, uint32_t elem) {
  return r * D + (elem ^ v_swap<D>(r));
}

template <int D, bool FP8, int WAVES>
__device__ __forceinline__ void segment_many(const AttendArgs& a, LdsMany<D>& l, const Cursor& cur, const Request& q, const Span& s,
                                          uint32_t k0, uint32_t k1) {
  constexpr int R = rows_of_wave(D), KT = LdsMany<D>::KT, kThreads = 64 * WAVES;
  constexpr int NB = KT / R, S = R * R / 64;       // scores: blocks of R keys, and of each so many to a lane
  constexpr int DB = D / R;                        // output: blocks of R elements, so many to a lane as well
  constexpr int kParts = 64 / R;                   // lanes of a row
  constexpr int kDepth = 8 * kParts;               // elements (or keys) of a product
  typedef Products<R> Mfma;
  constexpr int kRow = FP8 ? D : 2 * D;                    // bytes of a head's row
  constexpr int kPieces = kRow / 16;                       // 16-byte pieces of a key
  constexpr int kKeys = kThreads / kPieces;                // keys that the threads bring at a time
  constexpr int kLoads = KT < kKeys ? 1 : KT / kKeys;      // pieces of K (and of V) per thread
  constexpr int kWaveKeys = 64 / kPieces;                  // keys of a wavefront at a time
  constexpr uint32_t kBatch = 4, kDs = D == 64 ? 2 : 4;  // products whose operands are read at a time
  const Kind& kind = a.kind[1];
  const uint32_t tid = threadIdx.x, lane = tid & 63, c = lane % R, part = lane / R;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const GlobalBytes kp = layer_base(a.c.k), vp = layer_base(a.c.v);
  const int32_t* table = a.b.table + (uint64_t)cur.r * a.b.width;
  const uint32_t kv = cur.head / kind.parts;

  const uint32_t m = wave * R + c;
  bf16x8 qf[D / kDepth];
  int row_lo, row_hi;  // keys that this lane's row sees
  {
    const Place p = place_of(a, kind, q, cur.head, cur.tile, m);
    const uint16_t* qp = a.q + (int64_t)p.row * a.q_token + (int64_t)p.head * a.q_head;
#pragma unroll
    for (int k = 0; k < D / kDepth; ++k) qf[k] = load_q(a, qp + k * kDepth + part * 8, p.there);
    row_lo = p.lo;
    row_hi = p.hi;
  }
  // keys that some row of this wavefront sees, and keys that all of them see: its
  // first token's and its last's
  int wave_lo = 0x7fffffff, wave_hi = 0, all_lo = 0, all_hi = 0x7fffffff;
  {
    const uint32_t tokens = min(kind.tile_rows, q.rows - cur.tile * kind.tile_rows);
    const uint32_t t0 = wave * R / kind.part_heads, t1 = min((wave * R + R - 1) / kind.part_heads, tokens - 1);
    if (t0 < tokens) {
      const Place p0 = place_of(a, kind, q, cur.head, cur.tile, t0 * kind.part_heads);
      const Place p1 = place_of(a, kind, q, cur.head, cur.tile, t1 * kind.part_heads);
      wave_lo = uniform(p0.lo);
      wave_hi = uniform(p1.hi);
      all_lo = uniform(p1.lo);
      all_hi = uniform(p0.hi);
    }
  }
  typename Mfma::Sum o[DB];
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int j = 0; j < S; ++j) o[i][j] = 0.f;
  Soft st = {kNone, 0.f, 0.f};

  const int blocks = (int)(k1 - k0), block0 = (int)(s.b0 + k0) * KT;
  const uint32_t step = a.n_heads * kRow;  // bytes from a key to the next
  bool holes = false;  // whether a page of these blocks is missing (rare: then every key is asked)
  // What a thread brings: a 16-byte piece of K and V of kLoads keys of a block.
  // Keys that no row sees are read from the nearest one that some row does.
  const uint32_t piece = lane / kWaveKeys, my_key = wave * kWaveKeys + lane % kWaveKeys;
  const bool brings = my_key < KT;
  static_assert(kKeys % (D == 64 ? 16 : 8) == 0, "a later key's place differs by an exclusive or alone");
  const uint32_t k_to = lds_of(l.k[0]) + k_at<D>(my_key, FP8 ? 2 * piece : piece) * 2;
  const uint32_t v_to = lds_of(l.v[0]) + v_at<D>(my_key, (FP8 ? 16 : 8) * piece) * 2;
  u32x4 kr[kLoads], vr[kLoads];
  uint32_t page[kLoads], row[kLoads];       // of a block to come
  int64_t k_off[kLoads];                    // of the block whose K is on its way
  uint32_t k_word[kLoads], v_word[kLoads], v_next[kLoads];  // of scale bytes: V's of the block before K's, and of K's
  uint32_t v_gone = 0, v_gone_next = 0;                     // whether its keys' pages are missing, a bit each
  auto find = [&](int n) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const uint32_t key = (uint32_t)max(s.lo, min(block0 + n * KT + (int)my_key + i * kKeys, s.hi - 1)), at = a.b.page.div(key);
      row[i] = key - at * a.b.page.d;
      page[i] = (uint32_t)table[at];
    }
  };
  // K of the block that find() looked up, and its scales
  auto fetch_k = [&]() {
    v_gone = v_gone_next;
    v_gone_next = 0;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const bool fine = page[i] < a.c.n_pages;
      const int64_t base = fine ? (int64_t)page[i] * a.c.stride : 0;
      k_off[i] = base + (int64_t)row[i] * step + (int64_t)kv * kRow + piece * 16;
      kr[i] = *(GlobalU32x4)(kp + k_off[i]);
      if (!fine) v_gone_next |= 1u << i;
      if constexpr (FP8) {
        v_word[i] = v_next[i];
        k_word[i] = scale_word(kp + base, a.c.scale_off, kv);
        v_next[i] = scale_word(vp + base, a.c.scale_off, kv);
      }
    }
  };
  // V of the block whose K was fetched last
  auto fetch_v = [&]() {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) vr[i] = *(GlobalU32x4)(vp + k_off[i]);
  };
  auto keep_k = [&](uint32_t n) {
    if (!brings) return;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const uint32_t to = (k_to + ((n & 1) * KT + i * kKeys) * D * 2) ^ (k_swap<D>(i * kKeys) * 16);
      if constexpr (FP8) {
        const float by = scale_value(scale_held(scale_of(k_word[i], kv)));
        u32x4 w[2];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          w[j / 2][j % 2 * 2] = widen(kr[i][j], by, false);
          w[j / 2][j % 2 * 2 + 1] = widen(kr[i][j], by, true);
        }
        *(LdsU32x4)(uintptr_t)to = w[0];
        *(LdsU32x4)(uintptr_t)(to ^ 16) = w[1];
      } else {
        *(LdsU32x4)(uintptr_t)to = kr[i];
      }
    }
  };
  // Blocks [plain_lo, plain_hi) hold keys that all rows of the tile see, no copies of
  // others (whose weight is 0, but 0 times infinity is NaN), and no page is missing:
  // their values are kept as they are.
  int all_from = s.lo, all_to = s.hi;
  if (!a.all) {
    const int t1 = (int)min(cur.tile * kind.tile_rows + kind.tile_rows, q.rows);
    all_to = min(all_to, q.before + (int)(cur.tile * kind.tile_rows) + 1);
    if (a.window) all_from = max(all_from, (int)max((int64_t)0, (int64_t)q.before + t1 - (int64_t)a.window));
  }
  const int plain_lo = max(0, all_from - block0 + KT - 1) / KT;
  int plain_hi = max(0, all_to - block0) / KT;
  uint32_t odd = 0;
  auto keep_v = [&](uint32_t n) {
    if (!brings) return;
    if ((int)n < plain_lo || (int)n >= plain_hi) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        if (v_gone >> i & 1) vr[i] = u32x4{0, 0, 0, 0};  // whatever page 0 holds there, it may be NaN
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t bad = odd_bits<FP8>(vr[i][j]);
          odd |= bad;
          vr[i][j] &= ~bad;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const uint32_t to = v_to + ((n & 1) * KT + i * kKeys) * D * 2;
      const u32x4 x = vr[i];
      if constexpr (FP8) {
        const float by = scale_value(scale_held(scale_of(v_word[i], kv)));
        u32x4 w[2];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          w[j / 2][j % 2 * 2] = widen(x[j], by, false);
          w[j / 2][j % 2 * 2 + 1] = widen(x[j], by, true);
        }
        *(LdsU32x4)(uintptr_t)to = w[0];
        *(LdsU32x4)(uintptr_t)(to ^ 16) = w[1];
      } else {
        *(LdsU32x4)(uintptr_t)to = x;
      }
    }
  };

  // Where this lane finds its part of a product's K and V, in bytes of shared
  // memory. The product's number goes in by an exclusive or, at the read itself:
  // one register each, not one for each product.
  const uint32_t k_lane = lds_of(l.k[0]) + c * D * 2 + (part ^ k_swap<D>(c)) * 16;
  auto v_lane = [&]() {
    // the lane's number, asked for at every use: kept, this would be spilled, and
    // waited for together with the loads on their way
    uint32_t i;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=&v"(i));
    const uint32_t v_row = i / R * 4 + i % 16 / 4;
    return lds_of(l.v[0]) + v_row * D * 2 + ((i % R / 16 * 16 + i % 4 * 4) ^ v_swap<D>(v_row)) * 2;
  };
  typename Mfma::Sum x[NB];    // a block's scores
  bf16x8 w[KT / kDepth];       // and weights

  auto used = [&](int n) { return block0 + n * KT < wave_hi && block0 + n * KT + KT > wave_lo; };
  // x = K Q^T of block n, the operands read a batch ahead
  auto scores = [&](uint32_t n) {
    const uint32_t from = k_lane + (n & 1) * KT * D * 2;
    u32x4 kf[2][kBatch];
    auto read = [&](uint32_t i) {
#pragma unroll
      for (uint32_t j = 0; j < kBatch; ++j) {
        const uint32_t at = i * kBatch + j, b = at / (D / kDepth), k = at % (D / kDepth);
        kf[i & 1][j] = *(LdsU32x4)((LdsAddress)(uintptr_t)(from ^ k * kDepth * 2) + b * R * D * 2);
      }
    };
    read(0);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int j = 0; j < S; ++j) x[b][j] = 0.f;
#pragma unroll
    for (uint32_t i = 0; i < NB * D / kDepth / kBatch; ++i) {
      if (i + 1 < NB * D / kDepth / kBatch) read(i + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (uint32_t j = 0; j < kBatch; ++j) {
        const uint32_t at = i * kBatch + j, b = at / (D / kDepth), k = at % (D / kDepth);
        x[b] = Mfma::add(as_bf16(kf[i & 1][j]), qf[k], x[b]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // w = the weights of block n
  auto weigh = [&](uint32_t n) {
    const int key0 = block0 + (int)n * KT;
    if (holes || key0 < all_lo || key0 + KT > all_hi) {  // some row may not see some key
      const int first = key0 + 4 * (int)part;
      uint32_t bits = ~0u;
      if (holes)
#pragma unroll 1
        for (uint32_t t = 0; t < S * NB; ++t) {
          const int key = first + (int)(t / S * R + t % S / 4 * 8 + t % 4);
          const bool in = key >= row_lo && key < row_hi;
          if (!in || (uint32_t)table[a.b.page.div((uint32_t)key)] >= a.c.n_pages) bits &= ~(1u << t);
        }
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < S; ++j) {
          const int key = first + R * b + 8 * (j / 4) + j % 4;
          const bool there = (bits >> (S * b + j) & 1) && key >= row_lo && key < row_hi;
          x[b][j] = there ? x[b][j] : kNone;
        }
    }
    float top = x[0][0];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int j = 0; j < S; ++j) top = fmaxf(top, x[b][j]);
    top *= a.scale;
    if (__any(top > st.m + kSlack)) {
      if constexpr (R == 16) top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float mm = fmaxf(st.m, top);
      const float now = mm == kNone ? 0.f : mm;
      const float by = st.m == kNone ? 0.f : exp2_(st.top - now);
      st.m = mm;
      st.top = now;
      st.sum *= by;
#pragma unroll
      for (int i = 0; i < DB; ++i) o[i] *= by;
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int j = 0; j < S; ++j) {
        const float y = exp2_(__builtin_fmaf(x[b][j], a.scale, -st.top));
        st.sum += y;
        w[(S * b + j) / 8][(S * b + j) % 8] = (__bf16)y;
      }
  };
  // o += V^T w of block n, the operands read a batch ahead
  auto values = [&](uint32_t n) {
    const uint32_t from = v_lane() + (n & 1) * KT * D * 2;
    constexpr uint32_t kSteps = KT / kDepth * DB / kDs;
    u32x2 vf[2][2 * kDs];
    auto read = [&](uint32_t i) {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s16x4* Lds4;
#pragma unroll
      for (uint32_t j = 0; j < kDs; ++j) {
        const uint32_t t = i / (DB / kDs), d = i % (DB / kDs) * kDs + j;
        const LdsAddress v = (LdsAddress)(uintptr_t)(from ^ d * R * 2) + t * kDepth * D * 2;
        vf[i & 1][2 * j] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4)v));
        vf[i & 1][2 * j + 1] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4)(v + kDepth / 2 * D * 2)));
      }
    };
    read(0);
#pragma unroll
    for (uint32_t i = 0; i < kSteps; ++i) {
      if (i + 1 < kSteps) read(i + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (uint32_t j = 0; j < kDs; ++j) {
        const uint32_t t = i / (DB / kDs), d = i % (DB / kDs) * kDs + j;
        const u32x2 lo = vf[i & 1][2 * j], hi = vf[i & 1][2 * j + 1];
        o[d] = Mfma::add(as_bf16(u32x4{lo[0], lo[1], hi[0], hi[1]}), w[t], o[d]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  if (s.hi > s.lo) {
    // Block n is kept in buffers n % 2. Past the last block its last key is read
    // again. Page ids are looked up a step before they are used.
    find(0);
    int gone = 0;
    {
      const uint32_t first = a.b.page.div((uint32_t)max(s.lo, block0)), end = a.b.page.div((uint32_t)min(s.hi, block0 + blocks * KT) - 1);
      for (uint32_t i = first + tid; i <= end; i += kThreads) gone |= (uint32_t)table[i] >= a.c.n_pages;
    }
    fetch_k();
    find(1);
    holes = __syncthreads_or(gone);
    if (holes) plain_hi = 0;
    if constexpr (WAVES == 8) {
      // Wavefronts 0 to 3 are a phase ahead. A step of theirs keeps K of the next
      // block and V of this one; the others', a phase later, those of the block
      // after, so that all of it is there a phase before its use.
      const uint32_t behind = wave / 4;
      fetch_v();
      keep_k(0);
      fetch_k();
      find(2);
      __syncthreads();
      if (used(0)) scores(0);
      auto bring = [&](uint32_t n) {
        keep_k(n + 1);
        keep_v(n);
        fetch_v();
        fetch_k();
        find((int)n + 3);
      };
      if (behind) {
        bring(0);
        __syncthreads();
      }
      for (int n = 0; n < blocks; ++n) {
        if (used(n)) weigh(n);
        bring(n + behind);
        __syncthreads();
        if (used(n)) values(n);
        if (n + 1 < blocks && used(n + 1)) scores(n + 1);
        __syncthreads();
      }
      if (!behind) __syncthreads();
    } else {
      // A step uses one block, keeps the next and fetches the one after.
      auto bring = [&](uint32_t n) {
        keep_k(n);
        v_gone = v_gone_next;
#pragma unroll
        for (int i = 0; i < kLoads && FP8; ++i) v_word[i] = v_next[i];
        keep_v(n);
        fetch_k();
        fetch_v();
        find((int)n + 2);
      };
      fetch_v();
      bring(0);
      __syncthreads();
      for (int n = 0; n < blocks; ++n) {
        const bool use = used(n);
        if (use) scores(n);
        bring(n + 1);
        if (use) {
          weigh(n);
          values(n);
        }
        __syncthreads();
      }
    }
  }

  if (__syncthreads_or(odd))
#pragma unroll 1
    for (int n = 0; n < blocks; ++n) {
      if (n >= plain_lo && n < plain_hi) continue;
      const int key0 = block0 + n * KT;
      odd_keys<D, FP8>(a, table, vp, kv, max(key0, s.lo), min(key0 + KT, s.hi), [&](int key, GlobalBytes v) {
        if (key < row_lo || key >= row_hi) return;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int j = 0; j < S; j += 4) {
            const f32x4 y = odd4<FP8>(v + (d * R + 2 * j + 4 * part) * (FP8 ? 1 : 2));
#pragma unroll
            for (int i = 0; i < 4; ++i) o[d][j + i] += y[i];
          }
      });
    }

  float sum = st.sum;
  if constexpr (R == 16) sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  const bool whole = k0 == 0 && k1 == s.n;
  const Place p = place_of(a, kind, q, cur.head, cur.tile, m);
  if (p.there) {
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const uint64_t slot = (2 * (uint64_t)cur.worker + (k0 > 0 ? 0 : 1)) * a.slot_rows;
    uint16_t* op = a.out + (int64_t)p.row * a.o_token + (int64_t)p.head * a.o_head;
    float* fp = a.part_o + (slot + m) * D;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int j = 0; j < S; j += 4) {
        const uint32_t at = d * R + 2 * j + 4 * part;
        if (whole)
          store_bf16x4(op + at, o[d][j] * inv, o[d][j + 1] * inv, o[d][j + 2] * inv, o[d][j + 3] * inv);
        else
          *(f32x4*)(fp + at) = f32x4{o[d][j], o[d][j + 1], o[d][j + 2], o[d][j + 3]};
      }
    if (part == 0) {
      if (!whole)
        *(f32x2*)(a.part_ml + (slot + m) * 2) = f32x2{st.m, sum};
      else if (a.lse)
        a.lse[(uint64_t)p.row * a.n_heads * a.group + p.head] = lse_of(st.top, sum);
    }
  }
}

// 8,192 new tokens behind 8,192, 32 heads of 128 over 16 in scaled pages: 1.7 ms, 960
// TFLOP/s (a large bf16 product of the library reaches 1,603). The matrix units are
// busy for 46 % of its cycles, the vector units for 52 %, shared memory for 37 %: the
// phases of a SIMD's two wavefronts overlap little. Heads of 256 (203 tokens over
// 1,500 states: 430 TFLOP/s) have them busy for 18, 28 and 26 %: a workgroup has about
// one tile, and its start, its end and the barriers of some 20 blocks are what it waits for.
// Registers that the compiler spills (heads of 128: 48 to 78 a lane) are used where a
// tile starts and ends, not in the loop over blocks.
//
// Tiles of many rows, and of 16 for requests of few (heads of 256: their 16-row
// tiles want the registers of one wavefront on a SIMD, and stay in k_attend16).
template <int D, bool FP8, bool EVEN, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void k_attend_many(AttendArgs a) {
  __shared__ union {
    PlanLds plan;
    Lds16<D, D == 256 ? 1 : WAVES> few;
    LdsMany<D> many;
  } l;
  Cursor cur;
  const bool any = plan(a, l.plan, cur);
  if (!any) {
    if (threadIdx.x == 0) ((GlobalShare)a.share)[cur.worker].parts = 0;
    return;
  }
  Request q = uniform(request_of(a, cur.r));
  for (bool first = true; cur.at < cur.end; first = false) {
    const Span s = span_of(a, q, cur.tile);
    uint32_t k0, k1;
    const uint64_t tile_end = blocks_of(cur, q, s, k0, k1);
    if (first && threadIdx.x == 0) note_share(a, cur, q, s, k0, k1);
    if (k0 == k1) {
      // none
    } else if (D == 256 || q.kind) {
      segment_many<D, FP8, WAVES>(a, l.many, cur, q, s, k0, k1);
    } else if constexpr (D != 256) {
      segment16<D, FP8, EVEN, WAVES>(a, l.few, cur, q, s, k0, k1);
    }
    cur.at = min(cur.end, tile_end);
    if (cur.at == tile_end) {
      cur.first = tile_end;
      if (cur.at < cur.end) next_tile(a, q, cur);
    }
  }
}

// ---- joining ---------------------------------------------------------------------------
// A tile that several workers share: the workgroups of the second of them add up
// its parts, each those of some of its rows. A run of D / 4 threads takes a row;
// where there are fewer rows than runs, several take every so manieth of a row's
// parts. The order of the sums follows from the sizes alone.
template <int D>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a) {
  constexpr uint32_t kLanes = D / 4, kRuns = 256 / kLanes;
  constexpr int kAhead = 8;  // parts on their way at a time
  __shared__ struct {
    float top[kRuns], sum[kRuns];
    f32x4 y[kRuns][kLanes];
  } l;
  const uint32_t worker = blockIdx.x / a.joins + 1;
  const Share sh = a.share[worker];
  if (!sh.parts) return;
  const Kind& kind = a.kind[sh.kind];
  Request q = {};
  q.row0 = sh.row0;
  q.rows = sh.rows;
  // the tile's rows, one run of heads after another
  const uint32_t rows = min(kind.tile_rows, sh.rows - sh.tile * kind.tile_rows) * kind.part_heads, all = rows << kind.heads_shift;
  const uint32_t mine = (all + a.joins - 1) / a.joins, f0 = blockIdx.x % a.joins * mine, end = min(f0 + mine, all);
  uint32_t slices = kRuns;  // of a row's parts
  while (slices > 1 && mine * slices > kRuns) slices /= 2;
  const uint32_t run = threadIdx.x / kLanes, d = threadIdx.x % kLanes, i = run / slices, slice = run % slices;
  for (uint32_t f = f0; f < end; f += kRuns) {
    const bool there = f + i < end;
    const uint32_t at_head = min(f + i, end - 1) / rows, m = min(f + i, end - 1) % rows, row = at_head * kind.rows + m;
    const Place p = place_of(a, kind, q, (sh.head << kind.heads_shift) + at_head, sh.tile, m);
    float top = kNone, sum = 0.f;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    for (uint32_t w0 = slice; there && w0 < sh.parts; w0 += slices * kAhead) {
      f32x2 ml[kAhead];
      f32x4 o[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const uint32_t w = min(w0 + k * slices, sh.parts - 1);
        const uint64_t at = (2 * (uint64_t)(worker - 1 + w) + (w == 0 ? 1 : 0)) * a.slot_rows + row;
        ml[k] = *(const f32x2*)(a.part_ml + at * 2);
        o[k] = *(const f32x4*)(a.part_o + at * D + 4 * d);
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (w0 + k * slices >= sh.parts) continue;
        if (ml[k][0] == kNone) {  // zeros, or NaN
          sum += ml[k][1];
          y += o[k];
          continue;
        }
        const float now = fmaxf(top, ml[k][0]);
        const float old = top == kNone ? 0.f : exp2_(top - now), by = exp2_(ml[k][0] - now);
        sum = sum * old + ml[k][1] * by;
        y = y * old + o[k] * by;
        top = now;
      }
    }
    if (slices > 1) {  // then these are all of the workgroup's rows
      if (d == 0) {
        l.top[run] = top;
        l.sum[run] = sum;
      }
      l.y[run][d] = y;
      __syncthreads();
      if (slice) return;
      const float own = top;
      for (uint32_t k = 1; k < slices; ++k) top = fmaxf(top, l.top[run + k]);
      const float by0 = own == kNone ? 0.f : exp2_(own - top);
      sum *= by0;
      y *= by0;
      for (uint32_t k = 1; k < slices; ++k) {
        const float by = l.top[run + k] == kNone ? 0.f : exp2_(l.top[run + k] - top);
        sum += l.sum[run + k] * by;
        y += l.y[run + k][d] * by;
      }
    }
    if (!there || !p.there) continue;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    store_bf16x4(a.out + (int64_t)p.row * a.o_token + (int64_t)p.head * a.o_head + 4 * d, y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
    if (a.lse && d == 0) a.lse[(uint64_t)p.row * a.n_heads * a.group + p.head] = lse_of(top, sum);
  }
}

// ---- launching ----------------------------------------------------------------------------
struct Shape {
  uint32_t waves;      // of a workgroup; 0: k_attend16, else k_attend_many with so many
  uint32_t workers;    // workgroups: as many as the device holds at a time
  uint32_t slot_rows, joins, least;
  Kind kind[2];
  uint32_t few;
};

Kind kind_of(const tl_ctx* ctx, uint32_t group, uint32_t rows) {
  Kind k;
  k.rows = rows;
  k.parts = (group + rows - 1) / rows;
  k.part_heads = (group + k.parts - 1) / k.parts;
  k.tile_rows = rows / k.part_heads;
  return k;
}

// Wavefronts of a workgroup for requests of `per` rows on average.
uint32_t waves_of(const tl_ctx* ctx, uint64_t per) {
  // Rows (query heads of a K/V head times new tokens) per request from which tiles
  // of many rows are faster, and from which eight wavefronts beat four. us, 64 requests of about 1,024 keys,
  // with tiles of 16 rows / four wavefronts / eight:
  //   heads of 64    64 rows  34.7 / 37.1 / 47.6    96 rows  44.6 / 37.8 / 47.2    (two of 4,096 rows 101.0 with four,
  //                  102.5 with eight; one of 16,384 332 and 320)
  //   heads of 128   32 rows  65.8 / 75.1 / 75.6    48 rows  87.2 / 84.7 / 97.9    192 rows  272 / 154 / 145
  //   heads of 256   12 rows   122 /   -  / 123     16 rows   128 /   -  / 124     32 rows   217 /  -  / 128
  const uint32_t many = ctx->D == 64 ? 64 : ctx->D == 128 ? 32 : 12, eight = ctx->D == 64 ? 4096 : ctx->D == 128 ? 128 : 0;
  return per <= many ? 0 : per > eight ? 8 : 4;
}

Shape shape_of(const tl_ctx* ctx, uint32_t n_q_heads, uint64_t n_reqs, uint64_t n_rows, uint32_t waves) {
  Shape s;
  const uint32_t group = n_q_heads / ctx->H, wide = ctx->dtype == TL_DTYPE_FP8_SCALED ? 1 : 2;
  s.waves = waves;
  s.workers = ctx->D == 256 || s.waves == 8 ? 256 : 512;
  // In the kernel that holds both kinds, requests with up to 32 rows take tiles of 16.
  // us, two prompts of 330 tokens beside 60 requests of 4 / 8 / 16 tokens, 4 query heads a
  // K/V head, 4,096 keys each: all in tiles of many rows 249 / 251 / 253, up to 16 rows
  // in tiles of 16 179 / 251 / 253, up to 32 179 / 272 / 253, up to 64 179 / 272 / 422; beside 6 of
  // 4 tokens 109, 88, 88, 88.
  s.few = !s.waves ? ~0u : ctx->D == 256 ? 0 : 32 / group;
  Kind& f = s.kind[0];
  f = kind_of(ctx, group, 16);
  const uint32_t runs = ctx->H * f.parts;
  f.heads_shift = 0;
  while ((2u << f.heads_shift) <= (s.waves ? s.waves : 4) && runs % (2u << f.heads_shift) == 0) ++f.heads_shift;
  f.heads = runs >> f.heads_shift;
  // keys of a wavefront's step, and how many wavefronts take steps of one run
  f.block_shift = (ctx->D * wide < 128 ? 6 : 5) + (s.waves == 8 ? 3 : 2) - f.heads_shift;
  // A block of many rows counts for 1.5 of few. us with 1 / 1.5 / 2: two prompts of 330 beside
  // 6 requests of 1 token 91 / 89 / 106, beside 60 169 / 173 / 186 (heads of 64, 8 of each: 164 / 194 / 231).
  f.weight = s.waves ? 2 : 1;
  f.cost = f.weight;
  Kind& m = s.kind[1];
  m = kind_of(ctx, group, rows_of_wave(ctx->D) * (s.waves ? s.waves : 4));
  m.heads_shift = 0;
  m.heads = ctx->H * m.parts;
  m.block_shift = 6;
  m.weight = s.waves ? 3 : 1;
  // Finding a tile, its queries and its result count for 4 blocks. us with 1 / 4 / 8: 8 prompts of
  // 200 tokens behind 100 51 / 35 / 35, 30 of 300 behind 500 198 / 192 / 187, the two of 330 91 / 89 / 91.
  m.cost = 4 * m.weight;
  s.slot_rows = 16u << f.heads_shift;
  if (s.waves && s.slot_rows < m.rows) s.slot_rows = m.rows;
  // Tiles of many rows have few parts: a run of threads for each row. Tiles of few
  // rows may have many, if there are few tiles: so many runs for a row that each
  // has about 8 parts, which are on their way together. Four tiles of 8 rows of 128
  // parts: 8.2 us, with 2 of a workgroup's 8 runs for each row 12.1.
  const uint32_t runs_of_block = 1024 / ctx->D;
  const uint64_t reqs = n_reqs ? n_reqs : 1, tokens = (n_rows + reqs - 1) / reqs;
  const uint64_t rows = (tokens < f.tile_rows ? tokens : f.tile_rows) * f.part_heads << f.heads_shift;
  s.joins = s.slot_rows / runs_of_block;
  if (!s.waves) {
    uint64_t slices = s.workers / (reqs * f.heads) / 8;
    slices = slices < 1 ? 1 : slices > runs_of_block ? runs_of_block : slices;
    const uint64_t wanted = (rows * slices + runs_of_block - 1) / runs_of_block;
    if (wanted < s.joins) s.joins = (uint32_t)wanted;
    if (!s.joins) s.joins = 1;
  }
  // A part costs the join more the more rows it has, so a worker of a small batch
  // has to have some blocks. us with 1 / 2 / 3, 8 rows: 13 / 13 / 14 (1,024 keys),
  // 13 / 13 / 14 (4,096); 32 rows: 13 / 13 / 13, 25 / 21 / 18; 64 rows: 18 / 16 / 15, 36 / 25 / 21.
  s.least = (s.waves || rows > 32 ? 3 : rows > 8 ? 2 : 1) * m.weight;
  return s;
}

Shape shape_of(const tl_ctx* ctx, uint32_t n_q_heads, uint64_t n_reqs, uint64_t n_rows) {
  return shape_of(ctx, n_q_heads, n_reqs, n_rows, waves_of(ctx, n_rows * (n_q_heads / ctx->H) / (n_reqs ? n_reqs : 1)));
}

struct Layout {
  uint64_t ml, o, end;
};
Layout layout_of(const Shape& s, uint32_t D) {
  Layout l;
  const uint64_t rows = 2ull * s.workers * s.slot_rows;
  l.ml = ((uint64_t)s.workers * sizeof(Share) + 255) / 256 * 256;
  l.o = l.ml + rows * 2 * 4;
  l.end = (l.o + rows * D * 4 + 255) / 256 * 256;
  return l;
}

template <int D, bool FP8, bool EVEN>
void launch(const Shape& sh, hipStream_t s, const AttendArgs& a) {
  {
    TimedLaunch timed(TL_KERNEL_ATTEND, s);
    const dim3 grid(sh.workers);
    if (!sh.waves)
      hipLaunchKernelGGL((k_attend16<D, FP8, EVEN>), grid, dim3(256), 0, s, a);
    else if (sh.waves == 8)
      hipLaunchKernelGGL((k_attend_many<D, FP8, EVEN, 8>), grid, dim3(512), 0, s, a);
    else if constexpr (D != 256)
      hipLaunchKernelGGL((k_attend_many<D, FP8, EVEN, 4>), grid, dim3(256), 0, s, a);
  }
  TimedLaunch timed(TL_KERNEL_ATTEND_JOIN, s);
  hipLaunchKernelGGL((k_attend_join<D>), dim3((sh.workers - 1) * sh.joins), dim3(256), 0, s, a);
}

template <int D>
void launch(bool fp8, bool even, const Shape& sh, hipStream_t s, const AttendArgs& a) {
  if (fp8)
    even ? launch<D, true, true>(sh, s, a) : launch<D, true, false>(sh, s, a);
  else
    even ? launch<D, false, true>(sh, s, a) : launch<D, false, false>(sh, s, a);
}

}  // namespace

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
  a.kind[0] = sh.kind[0];
  a.kind[1] = sh.kind[1];
  a.few = sh.few;
  a.slot_rows = sh.slot_rows;
  a.joins = sh.joins;
  a.least = sh.least;
  a.all = (flags & TL_ATTEND_ALL) != 0;
  a.window = a.all ? 0 : (uint32_t)ctx->window[layer];
  const float by = scale * 1.4426950408889634f;
  a.scale = fmaxf(fabsf(by), 1e-37f);
  a.q_sign = by < 0.f ? 0x80008000u : 0u;
  const Layout lay = layout_of(sh, ctx->D);
  a.share = (Share*)d_ws;
  a.part_ml = (float*)((uint8_t*)d_ws + lay.ml);
  a.part_o = (float*)((uint8_t*)d_ws + lay.o);
  hipStream_t s = (hipStream_t)stream;
  (void)hipGetLastError();
  const bool fp8 = ctx->dtype == TL_DTYPE_FP8_SCALED, even = ctx->P % 16 == 0;
  switch (ctx->D) {
    case 64: launch<64>(fp8, even, sh, s, a); break;
    case 128: launch<128>(fp8, even, sh, s, a); break;
    default: launch<256>(fp8, even, sh, s, a); break;
  }
  return hipGetLastError() == hipSuccess ? TL_OK : TL_EDEVICE;
}

}  // namespace tl
