// Pages of a cache as a whole: copied (tl_pages_copy), shared and copied by new
// branches of a request (tl_pages_fork), taken from and given back to a pool
// (tl_pages_take, tl_pages_free), and the rows of a request that stay moved
// together in them (tl_keep). All layers in one call.
#include <algorithm>

#include "paged.h"

namespace tl {
namespace {

// All layers' pages. A slab is one layer's K (2 * layer) or V (2 * layer + 1).
struct Slabs {
  const uint64_t* k;
  const uint64_t* v;
  int64_t stride;
  uint32_t n_pages, n_slabs;
  uint32_t page_tokens, row_bytes;
  uint32_t code_bytes, n_scales;  // of a page; scale bytes follow its codes
  uint32_t n_groups;
  uint8_t group[TL_MAX_LAYERS];

  __device__ __forceinline__ uint8_t* base(uint32_t slab) const { return (uint8_t*)(slab & 1 ? v : k)[slab >> 1]; }
};

typedef __attribute__((address_space(1))) uint8_t* Bytes;
typedef __attribute__((address_space(1))) u32x4* Granules;

constexpr uint32_t kThreads = 256;
constexpr uint32_t kFlight = 4;                               // 16-byte pieces of a thread on their way
constexpr uint32_t kPiece = kThreads * kFlight * 16;          // bytes that a workgroup copies at a time
constexpr uint32_t kMostGroups = 1u << 22;                    // workgroups of a launch; further work is looped over

// ---- copying ---------------------------------------------------------------------
// One workgroup's pieces of a page's first `rows` rows (every `pieces`th from `piece` on),
// and the page's scales with the first. Bounded by memory: every byte is read and written
// once, and not expected back soon.
__device__ __forceinline__ void copy_pieces(const Slabs& c, uint32_t slab, uint32_t src, uint32_t dst, uint32_t rows, uint32_t piece, uint32_t pieces) {
  const Bytes base = (Bytes)c.base(slab);
  const Bytes from = base + (int64_t)src * c.stride, to = base + (int64_t)dst * c.stride;
  const uint32_t bytes = rows * c.row_bytes, whole = bytes & ~15u, tid = threadIdx.x;
  for (uint32_t at = piece * kPiece + tid * 16; at < whole; at += pieces * kPiece) {
    u32x4 x[kFlight];
#pragma unroll
    for (uint32_t i = 0; i < kFlight; ++i)
      if (at + i * kThreads * 16 < whole) x[i] = __builtin_nontemporal_load((Granules)(from + at + i * kThreads * 16));
#pragma unroll
    for (uint32_t i = 0; i < kFlight; ++i)
      if (at + i * kThreads * 16 < whole) __builtin_nontemporal_store(x[i], (Granules)(to + at + i * kThreads * 16));
  }
  if (piece) return;
  if (whole + tid < bytes) to[whole + tid] = from[whole + tid];  // rows that end within sixteen bytes
  for (uint32_t i = tid; i < c.n_scales; i += kThreads) to[c.code_bytes + i] = from[c.code_bytes + i];
}

struct CopyArgs {
  Slabs c;
  const int32_t* src;
  const int32_t* dst;  // [n_groups][n]
  const uint32_t* rows;
  uint32_t n, pieces;
};

__global__ __launch_bounds__(kThreads) void k_pages_copy(CopyArgs a) {
  const uint64_t per = (uint64_t)a.c.n_slabs * a.pieces, items = a.n * per;
  for (uint64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const uint32_t i = (uint32_t)(item / per), rest = (uint32_t)(item % per), slab = rest / a.pieces, piece = rest % a.pieces;
    const uint64_t at = (uint64_t)a.c.group[slab >> 1] * a.n + i;
    const uint32_t src = (uint32_t)a.src[at], dst = (uint32_t)a.dst[at];
    if (src >= a.c.n_pages || dst >= a.c.n_pages || src == dst) continue;
    const uint32_t rows = a.rows ? min(a.rows[i], a.c.page_tokens) : a.c.page_tokens;
    copy_pieces(a.c, slab, src, dst, rows, piece, a.pieces);
  }
}

// ---- whose pages are whose ---------------------------------------------------------
// A pool counts each page's owners; one that has none is free. Of the lowest free
// pages each request is meant to have those behind what the requests before it want,
// whether they are served or not: a prefix sum, which does not depend on when a
// kernel's threads run, and by which none overtakes one that has to be refused.
// Counts change by atomic additions, whose order does not matter to their sum.
struct PoolArgs {
  int32_t* refs;  // [n_groups][n_pages]
  uint32_t n_pages, n_groups, page_tokens;
  uint32_t n;      // requests that want pages
  uint32_t width;  // of a table row
  uint8_t* status;
  uint32_t* start;  // workspace: [n_groups][n + 1] pages that the requests before want
  int32_t* list;    // workspace: [n_groups][n_pages] free pages, as many as are wanted
  uint8_t* served;  // workspace: [n] status of each request
  // tl_pages_fork
  const int32_t* parent;
  const int32_t* tables;  // [n_groups][n_parents][width]
  const uint32_t* kv_len;
  uint32_t n_parents;
  int32_t* out_tables;  // [n_groups][n][width]; also what tl_pages_take fills
  uint32_t* out_len;
  // tl_pages_take
  const uint32_t* have;
  const uint32_t* want;
};

constexpr uint32_t kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;
constexpr uint32_t kScan = 16;  // rounds of a pool's pages that are looked at together

// A parent's last page, if it is partly filled and there.
struct Fork {
  uint32_t parent, kv, full, part;
  bool fine;
};
__device__ __forceinline__ Fork fork_of(const PoolArgs& a, uint32_t r) {
  Fork f;
  f.parent = (uint32_t)a.parent[r];
  f.fine = f.parent < a.n_parents;
  f.kv = f.fine ? a.kv_len[f.parent] : 0;
  f.full = f.kv / a.page_tokens;
  f.part = f.kv - f.full * a.page_tokens;
  if (f.full + (f.part ? 1 : 0) > a.width) f.fine = false;
  return f;
}
__device__ __forceinline__ uint32_t last_page(const PoolArgs& a, const Fork& f, uint32_t g) {
  return (uint32_t)a.tables[((uint64_t)g * a.n_parents + f.parent) * a.width + f.full];
}

// A table's entry that names no page.
__device__ __forceinline__ bool lacks(const PoolArgs& a, int32_t id) { return (uint32_t)id >= a.n_pages; }

// Entries [c0, c1) of a table row: the ones in them that name no page are wanted.
__device__ __forceinline__ void range_of(const PoolArgs& a, uint32_t r, uint32_t& c0, uint32_t& c1, bool& fine) {
  const uint32_t have = a.have[r], want = a.want[r], P = a.page_tokens;
  c0 = have / P + (have % P ? 1 : 0);
  c1 = want / P + (want % P ? 1 : 0);
  fine = c1 <= a.width;
  if (!fine || c1 < c0) c1 = c0;
}

__device__ __forceinline__ uint32_t lanes_below(uint64_t mask) { return __popcll(mask & ((1ull << (threadIdx.x & 63)) - 1)); }

// A lane walks its own request's range of a table row where that is short; a longer one is
// walked by the whole wavefront, 64 entries at a time.
constexpr uint32_t kShort = 4;

// Pages that request r (a lane each) wants in group g.
template <bool FORK>
__device__ uint32_t wanted(const PoolArgs& a, uint32_t r, uint32_t g) {
  if constexpr (FORK) {
    if (r >= a.n) return 0;
    const Fork f = fork_of(a, r);
    return f.fine && f.part && last_page(a, f, g) < a.n_pages ? 1 : 0;
  } else {
    uint32_t c0 = 0, c1 = 0, n = 0;
    bool fine = true;
    if (r < a.n) range_of(a, r, c0, c1, fine);
    const int32_t* row = a.out_tables + ((uint64_t)g * a.n + min(r, a.n - 1)) * a.width;
    if (c1 - c0 <= kShort) {
#pragma unroll
      for (uint32_t i = 0; i < kShort; ++i)
        if (c0 + i < c1) n += lacks(a, row[c0 + i]);
    }
    for (uint64_t m = __ballot(c1 - c0 > kShort); m; m &= m - 1) {
      const uint32_t lane = (uint32_t)__builtin_ctzll(m), who = __shfl(r, lane), b0 = __shfl(c0, lane), b1 = __shfl(c1, lane);
      const int32_t* theirs = a.out_tables + ((uint64_t)g * a.n + who) * a.width;
      uint32_t k = 0;
      for (uint32_t c = b0 + (threadIdx.x & 63); c < b1; c += 64) k += lacks(a, theirs[c]);
      for (uint32_t d = 1; d < 64; d *= 2) k += __shfl_xor(k, d);
      if ((threadIdx.x & 63) == lane) n = k;
    }
    return n;
  }
}

// One workgroup: what every request wants, the lowest free pages, who is served, and
// tl_pages_take's entries. A chain of loads that wait for each other (some 1 us each), so
// the first pages' counts are asked for before the requests' wishes, and what a thread
// knows of its request stays in registers where there is a thread for each.
template <bool FORK>
__global__ __launch_bounds__(kPlanThreads) void k_pool_plan(PoolArgs a) {
  __shared__ uint32_t sums[kPlanWaves], before_of[kScan * kPlanWaves], found_now, found[TL_MAX_GROUPS];
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid / 64;
  const bool one = a.n <= kPlanThreads;  // a thread for each request
  uint32_t at[TL_MAX_GROUPS], mine[TL_MAX_GROUPS];
  int32_t held[kScan];
  auto ask = [&](const int32_t* refs, uint64_t p0) {
#pragma unroll
    for (uint32_t k = 0; k < kScan; ++k) {
      const uint64_t p = p0 + k * kPlanThreads + tid;
      held[k] = p < a.n_pages ? refs[p] : 1;
    }
  };
#pragma unroll
  for (uint32_t g = 0; g < TL_MAX_GROUPS; ++g) {
    if (g >= a.n_groups) break;
    const int32_t* refs = a.refs + (uint64_t)g * a.n_pages;
    ask(refs, 0);
    uint32_t* start = a.start + (uint64_t)g * (a.n + 1);
    uint32_t total = 0;
    for (uint32_t r0 = 0; r0 < a.n; r0 += kPlanThreads) {
      const uint32_t r = r0 + tid, n = wanted<FORK>(a, r, g);
      uint32_t incl = n;
      for (uint32_t k = 1; k < 64; k *= 2) {
        const uint32_t up = __shfl_up(incl, k);
        if (lane >= k) incl += up;
      }
      __syncthreads();  // the last round's sums have been read
      if (lane == 63) sums[wave] = incl;
      __syncthreads();
      uint32_t before = total;
      const uint32_t s = lane < kPlanWaves ? sums[lane] : 0;
      for (uint32_t w = 0; w < kPlanWaves; ++w) {
        const uint32_t x = __builtin_amdgcn_readlane(s, w);
        if (w < wave) before += x;
        total += x;
      }
      at[g] = before + incl - n;
      mine[g] = n;
      if (r < a.n) start[r] = at[g];
    }
    if (tid == 0) start[a.n] = total;
    // the lowest free pages
    int32_t* list = a.list + (uint64_t)g * a.n_pages;
    uint32_t have = 0;
    for (uint64_t p0 = 0; p0 < a.n_pages && have < total; p0 += kScan * kPlanThreads) {
      if (p0) ask(refs, p0);
      uint64_t free[kScan];
#pragma unroll
      for (uint32_t k = 0; k < kScan; ++k) free[k] = __ballot(held[k] <= 0);
      __syncthreads();  // the last round's numbers have been read
      if (lane == 0)
#pragma unroll
        for (uint32_t k = 0; k < kScan; ++k) before_of[k * kPlanWaves + wave] = __popcll(free[k]);
      __syncthreads();
      if (wave == 0) {  // how many there are before each wavefront's of each round
        constexpr uint32_t kEach = kScan * kPlanWaves / 64;
        uint32_t n[kEach], sum = 0;
#pragma unroll
        for (uint32_t k = 0; k < kEach; ++k) n[k] = before_of[lane * kEach + k];
#pragma unroll
        for (uint32_t k = 0; k < kEach; ++k) {
          const uint32_t x = n[k];
          n[k] = sum;
          sum += x;
        }
        uint32_t incl = sum;
        for (uint32_t k = 1; k < 64; k *= 2) {
          const uint32_t up = __shfl_up(incl, k);
          if (lane >= k) incl += up;
        }
#pragma unroll
        for (uint32_t k = 0; k < kEach; ++k) before_of[lane * kEach + k] = incl - sum + n[k];
        if (lane == 63) found_now = incl;
      }
      __syncthreads();
#pragma unroll
      for (uint32_t k = 0; k < kScan; ++k) {
        const uint32_t i = have + before_of[k * kPlanWaves + wave] + lanes_below(free[k]);
        if ((free[k] >> lane & 1) && i < total) list[i] = (int32_t)(p0 + k * kPlanThreads + tid);
      }
      have += found_now;
    }
    if (tid == 0) found[g] = have;
  }
  __syncthreads();
  // a request is served in all groups or in none
  for (uint32_t r0 = 0; r0 < a.n; r0 += kPlanThreads) {
    const uint32_t r = r0 + tid;
    uint8_t said = TL_ACCEPT;
    uint32_t c0 = 0, c1 = 0;
    bool fine = true;
#pragma unroll
    for (uint32_t g = 0; g < TL_MAX_GROUPS; ++g) {
      if (g >= a.n_groups) break;
      if (!one && r < a.n) {
        const uint32_t* start = a.start + (uint64_t)g * (a.n + 1);
        at[g] = start[r];
        mine[g] = start[r + 1] - at[g];
      }
      if (r < a.n && mine[g] && at[g] + mine[g] > found[g]) said = TL_MISSING;
    }
    if (r < a.n) {
      if constexpr (FORK)
        fine = fork_of(a, r).fine;
      else
        range_of(a, r, c0, c1, fine);
      if (!fine) said = TL_BADARG;
      a.served[r] = said;
      if (a.status) a.status[r] = said;
    }
    if constexpr (!FORK) {
      if (said != TL_ACCEPT) c1 = c0;
#pragma unroll
      for (uint32_t g = 0; g < TL_MAX_GROUPS; ++g) {
        if (g >= a.n_groups) break;
        const int32_t* list = a.list + (uint64_t)g * a.n_pages;
        int32_t* refs = a.refs + (uint64_t)g * a.n_pages;
        int32_t* row = a.out_tables + ((uint64_t)g * a.n + min(r, a.n - 1)) * a.width;
        if (c1 - c0 <= kShort) {
          uint32_t from = at[g];
#pragma unroll
          for (uint32_t i = 0; i < kShort; ++i)
            if (c0 + i < c1 && lacks(a, row[c0 + i])) {
              const int32_t p = list[from++];
              row[c0 + i] = p;
              refs[p] = 1;
            }
        }
        for (uint64_t m = __ballot(c1 - c0 > kShort); m; m &= m - 1) {
          const uint32_t who = (uint32_t)__builtin_ctzll(m), b0 = __shfl(c0, who), b1 = __shfl(c1, who);
          uint32_t from = __shfl(at[g], who);
          int32_t* theirs = a.out_tables + ((uint64_t)g * a.n + __shfl(r, who)) * a.width;
          for (uint32_t c = b0; c < b1; c += 64) {
            const bool wants = c + lane < b1 && lacks(a, theirs[c + lane]);
            const uint64_t all = __ballot(wants);
            if (wants) {
              const int32_t p = list[from + lanes_below(all)];
              theirs[c + lane] = p;
              refs[p] = 1;
            }
            from += __popcll(all);
          }
        }
      }
    }
  }
}

struct ForkArgs {
  Slabs c;
  PoolArgs p;
  uint32_t pieces;
};

// The first n * n_groups workgroups write a branch's table and count it among its
// pages' owners; the others copy pieces of last pages.
__global__ __launch_bounds__(kThreads) void k_pages_fork(ForkArgs a) {
  const PoolArgs& p = a.p;
  const uint64_t tables = (uint64_t)p.n * p.n_groups, per = (uint64_t)a.c.n_slabs * a.pieces, items = tables + p.n * per;
  for (uint64_t item = blockIdx.x; item < items; item += gridDim.x) {
    if (item < tables) {
      const uint32_t r = (uint32_t)(item / p.n_groups), g = (uint32_t)(item % p.n_groups);
      const bool served = p.served[r] == TL_ACCEPT;
      const Fork f = fork_of(p, r);
      const uint32_t* start = p.start + (uint64_t)g * (p.n + 1);
      int32_t* refs = p.refs + (uint64_t)g * p.n_pages;
      const bool own = served && start[r + 1] > start[r];
      for (uint32_t c = threadIdx.x; c < p.width; c += kThreads) {
        int32_t id = -1;
        if (served && c < f.full) {
          id = p.tables[((uint64_t)g * p.n_parents + f.parent) * p.width + c];
          if ((uint32_t)id < p.n_pages)
            atomicAdd(refs + id, 1);
          else
            id = -1;
        } else if (own && c == f.full) {
          id = p.list[(uint64_t)g * p.n_pages + start[r]];
          refs[id] = 1;
        }
        p.out_tables[((uint64_t)g * p.n + r) * p.width + c] = id;
      }
      if (g == 0 && threadIdx.x == 0) p.out_len[r] = served ? f.kv : 0;
      continue;
    }
    const uint64_t at = item - tables;
    const uint32_t r = (uint32_t)(at / per), rest = (uint32_t)(at % per), slab = rest / a.pieces, piece = rest % a.pieces;
    const uint32_t g = a.c.group[slab >> 1];
    const uint32_t* start = p.start + (uint64_t)g * (p.n + 1);
    if (p.served[r] != TL_ACCEPT || start[r + 1] == start[r]) continue;
    const Fork f = fork_of(p, r);
    copy_pieces(a.c, slab, last_page(p, f, g), (uint32_t)p.list[(uint64_t)g * p.n_pages + start[r]], f.part, piece, a.pieces);
  }
}

struct FreeArgs {
  int32_t* refs;
  uint32_t n_pages, page_tokens, width;
  uint64_t rows, n;  // table rows (n for each group)
  int32_t* tables;
  const uint32_t* first;
  const uint32_t* end;
};

__global__ __launch_bounds__(kThreads) void k_pages_free(FreeArgs a) {
  const uint64_t all = a.rows * a.width;
  for (uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x; i < all; i += (uint64_t)gridDim.x * kThreads) {
    const uint64_t row = i / a.width;
    const uint32_t c = (uint32_t)(i - row * a.width), r = (uint32_t)(row % a.n), P = a.page_tokens;
    const uint32_t c0 = a.first ? a.first[r] / P + (a.first[r] % P ? 1 : 0) : 0, c1 = a.end ? a.end[r] / P : a.width;
    if (c < c0 || c >= c1) continue;
    const uint32_t id = (uint32_t)a.tables[i];
    if (id < a.n_pages) atomicAdd(a.refs + row / a.n * a.n_pages + id, -1);
    a.tables[i] = -1;
  }
}

// ---- rows that stay --------------------------------------------------------------
struct KeepArgs {
  Slabs c;
  Batch b;  // table: of group 0
  const uint32_t* n_keep;
  const uint32_t* keep;
  uint32_t* len_out;
  uint8_t* status;
  uint32_t columns, blocks;  // 16-byte columns of a row, and workgroups (or wavefronts) that share them
  uint32_t slabs;            // of a wavefront
};

// Largest magnitude among 16 codes, as values; NaN codes do not count.
__device__ __forceinline__ float largest_code(u32x4 w) {
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[e], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[e], true);
    m = fmaxf(fmaxf(fabsf(lo[0]), fabsf(lo[1])), m);
    m = fmaxf(fmaxf(fabsf(hi[0]), fabsf(hi[1])), m);
  }
  return m;
}

// The smallest scale byte under which a code's value (above 0) of scale byte `from` is 448
// or less: 1.m * 2^e needs 2^(e - 8), twice that above 1.75.
__device__ __forceinline__ uint32_t scale_for(float value, uint32_t from) {
  const uint32_t bits = __float_as_uint(value);
  const int b = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0) + (int)from;
  return (uint32_t)max(b, (int)kScaleMin);
}

// Codes of scale byte `from`, rounded to scale byte `to`.
__device__ __forceinline__ u32x4 rescale(u32x4 w, uint32_t from, uint32_t to) {
  // 448 * 2^-40 rounds to 0, as less does; a page whose scale falls by over 2^20 holds zeros
  const int by = min(max((int)from - (int)to, -40), 20);
  const float f = __uint_as_float((uint32_t)(127 + by) << 23);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[e], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[e], true);
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0] * f, lo[1] * f, 0, false);
    w[e] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(hi[0] * f, hi[1] * f, c, true);
  }
  return w;
}

// A row only moves towards the front, and never past one that stays: the rows of a step
// are all read before the first of them is written, and then no later row's source has
// been written over. So a request's rows are moved in place, in steps that follow each
// other, and in parallel over columns, slabs and requests.
//
// Scaled pages: a step is whole pages of the rows' new places (or all rows that are left),
// whose scales follow from the codes' largest magnitudes; a page of more rows than a step
// holds is read twice.

// Rows of one request, and where they go.
struct Kept {
  uint32_t rows, before, n, P;
  bool sound;
  const uint32_t* keep;
  const int32_t* table;
  uint64_t group_stride;
};
__device__ __forceinline__ Kept kept_of(const KeepArgs& a, uint32_t r) {
  Kept k;
  const uint32_t row0 = a.b.first_row(r), row1 = a.b.first_row(r + 1), kv_len = a.b.kv_len[r];
  k.rows = row1 > row0 ? row1 - row0 : 0;
  k.sound = kv_len >= k.rows && kv_len <= a.b.most;
  k.before = kv_len - k.rows;
  k.n = k.sound ? min(a.n_keep[r], k.rows) : 0;
  k.P = a.c.page_tokens;
  k.keep = a.keep + row0;
  k.table = a.b.table + (uint64_t)r * a.b.width;
  k.group_stride = (uint64_t)a.b.n_reqs * a.b.width;
  return k;
}

// Rows in front that stay where they are: found by a whole wavefront.
__device__ __forceinline__ uint32_t rows_in_place(const Kept& k) {
  const uint32_t lane = threadIdx.x & 63;
  for (uint32_t i = 0; i < k.n; i += 64) {
    const uint64_t moves = __ballot(i + lane < k.n && k.keep[min(i + lane, k.n - 1)] != i + lane);
    if (moves) return i + (uint32_t)__builtin_ctzll(moves);
  }
  return k.n;
}

// Where row i is and where it goes; false: it cannot be kept, since it names no later row
// than the one before, or has no page in some group (every layer stops at the same row).
struct RowMove {
  int64_t from_page, to_page;
  uint32_t from_row, to_row, page;  // rows of those pages, and the new place's page in the table
};
__device__ __forceinline__ bool move_of(const KeepArgs& a, const Kept& k, uint32_t i, uint32_t own, RowMove& m) {
  const uint32_t at = k.keep[i], last = i ? k.keep[i - 1] : 0;
  if (at >= k.rows || (i && at <= last)) return false;
  const uint32_t ps = k.before + at, pd = k.before + i, cs = a.b.page.div(ps), cd = a.b.page.div(pd);
  bool fine = true;
  for (uint32_t g = 0; g < a.c.n_groups; ++g) {
    const uint32_t src = (uint32_t)k.table[g * k.group_stride + cs], dst = (uint32_t)k.table[g * k.group_stride + cd];
    if (src >= a.c.n_pages || dst >= a.c.n_pages) fine = false;
    if (g == own) {
      m.from_page = (int64_t)src * a.c.stride;
      m.to_page = (int64_t)dst * a.c.stride;
    }
  }
  m.from_row = ps - cs * k.P;
  m.to_row = pd - cd * k.P;
  m.page = cd;
  return fine;
}

__device__ __forceinline__ void say_kept(const KeepArgs& a, const Kept& k, uint32_t r, uint32_t done, bool bad) {
  a.len_out[r] = k.sound ? k.before + done : a.b.kv_len[r];
  if (a.status) a.status[r] = k.sound && !bad && a.n_keep[r] <= k.rows ? TL_ACCEPT : TL_BADARG;
}

// Few rows: a wavefront by itself takes L 16-byte columns (scaled pages: a head) of one
// request's rows in some slabs, one after another, and waits for no other. What it costs is
// instructions and one wait after another, not bytes: so a step's places are found once for
// all its slabs, a step has as many rows as the lanes hold once (accepted drafts are few; twice
// where requests bring many rows), and registers are few, for many wavefronts on a SIMD. 96
// requests that keep up to 7 of up to 48 rows, 32 layers of 8 heads of 128 in 8 bits: 23 us; with
// 32 rows a step and the next slab's asked for ahead 50 (186 registers and more), a workgroup for
// all heads and a slab 53.
template <int L, int U>
struct FewRows {
  static constexpr uint32_t R = 64 / L, N = R * U;  // rows at a time, rows of a step
};

__device__ __forceinline__ int64_t shuffled(int64_t x, uint32_t lane) {
  const uint32_t lo = __shfl((uint32_t)x, lane), hi = __shfl((uint32_t)((uint64_t)x >> 32), lane);
  return (int64_t)((uint64_t)hi << 32 | lo);
}

// Rows that have been asked for are there, before anything is written after this.
template <int U>
__device__ __forceinline__ void arrived(u32x4 (&x)[U]) {
#pragma unroll
  for (int u = 0; u < U; ++u) asm volatile("" : "+v"(x[u]) : : "memory");
}

template <bool FP8, int L, int U>
__device__ void keep_few(const KeepArgs& a, uint32_t r, uint32_t slab0, uint32_t slab1, uint32_t block) {
  typedef FewRows<L, U> F;
  const uint32_t lane = threadIdx.x & 63, j = lane % L, sub = lane / L, column = block * L + j;
  const bool there = column < a.columns;
  const Kept k = kept_of(a, r);
  const uint32_t own = a.c.group[slab0 >> 1];
  // the slabs' bases, a lane each: asked for once, and before all else
  const int64_t bases = (int64_t)a.c.base(min(slab0 + lane, slab1 - 1));
  uint32_t done = rows_in_place(k);
  bool bad = false;
  while (done < k.n && !bad) {
    const uint32_t pos = k.before + done, page0 = a.b.page.div(pos), o = pos - page0 * k.P;
    uint32_t ask = k.n - done;  // rows of the step
    if (ask > F::N) ask = !FP8 ? F::N : (uint32_t)min((uint64_t)ask, ((uint64_t)page0 + (k.P <= F::N ? F::N / k.P : 1)) * k.P - pos);
    const bool whole = ask <= F::N;  // they are held, not read again
    const uint32_t last = a.b.page.div(pos + ask - 1);
    // this lane's rows
    int64_t from[U], to[U], from_scale[U], to_scale[U];
    uint32_t page[U];
    auto find = [&](uint32_t i, uint32_t count) {
      RowMove m = {0, 0, 0, 0, 0};
      const bool fine = lane >= count || move_of(a, k, i + lane, own, m);
      const uint64_t none = ~__ballot(fine);
      const int64_t f = m.from_page + (int64_t)m.from_row * a.c.row_bytes, t = m.to_page + (int64_t)m.to_row * a.c.row_bytes;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t at = u * F::R + sub;
        from[u] = shuffled(f, at) + column * 16;
        to[u] = shuffled(t, at) + column * 16;
        if constexpr (FP8) {
          from_scale[u] = shuffled(m.from_page, at) + a.c.code_bytes + block;
          to_scale[u] = shuffled(m.to_page, at) + a.c.code_bytes + block;
          page[u] = __shfl(m.page, at);
        }
      }
      return none ? min(count, (uint32_t)__builtin_ctzll(none)) : count;
    };
    int64_t first_scale_at = 0;
    if (whole) {
      const uint32_t count = find(done, ask);
      bad = count < ask;
      ask = count;
      if (!ask) break;
      if constexpr (FP8) first_scale_at = shuffled(to_scale[0], 0);
    }
    u32x4 x[U] = {};
    uint32_t scale[U] = {};
#pragma unroll 1
    for (uint32_t slab = slab0; slab < slab1; ++slab) {
      const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)bases, slab - slab0);
      const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)((uint64_t)bases >> 32), slab - slab0);
      const Bytes base = (Bytes)((uint64_t)hi << 32 | lo);
      auto load = [&](uint32_t count) {
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (u * F::R + sub < count && there) {
            x[u] = *(Granules)(base + from[u]);
            if constexpr (FP8) scale[u] = base[from_scale[u]];
          }
      };
      if constexpr (!FP8) {
        load(ask);
        arrived(x);
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (u * F::R + sub < ask && there) *(Granules)(base + to[u]) = x[u];
      } else {
        uint32_t needs[U], first = kScaleMin, old = 0;  // scale bytes of a row's new page, and of the step's first one
        // what the pages of the rows that were read need
        auto needs_of = [&](uint32_t count) {
          uint32_t mine[U];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            scale[u] = scale_held(scale[u]);
            float m = u * F::R + sub < count && there ? largest_code(x[u]) : 0.f;
#pragma unroll
            for (int d = 1; d < L; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
            mine[u] = m > 0.f ? scale_for(m, scale[u]) : kScaleMin;
            needs[u] = kScaleMin;
          }
          for (uint32_t p = page0; p <= last; ++p) {  // two pages, mostly
            uint32_t m = kScaleMin;
#pragma unroll
            for (int u = 0; u < U; ++u)
              if (u * F::R + sub < count && page[u] == p) m = max(m, mine[u]);
#pragma unroll
            for (int d = L; d < 64; d *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, d));
            if (p == page0) first = max(first, m);
#pragma unroll
            for (int u = 0; u < U; ++u)
              if (page[u] == p) needs[u] = m;
          }
        };
        if (whole) {
          load(ask);
          if (o) old = base[first_scale_at];
          needs_of(ask);
        } else {
          for (uint32_t i = 0; i < ask; i += F::N) {
            const uint32_t want = min(F::N, ask - i), count = find(done + i, want);
            load(count);
            if (i == 0) {
              first_scale_at = shuffled(to_scale[0], 0);
              if (o && count) old = base[first_scale_at];
            }
            needs_of(count);
            if (count < want) {  // the same for every slab
              bad = true;
              ask = i + count;
            }
          }
          if (!ask) break;
        }
        if (o) {
          old = scale_held(old);
          if (first > old) {  // the page's scale rises: the rows before are rounded again
            for (uint32_t i = sub; i < o && there; i += F::R) {
              const Granules at = (Granules)(base + first_scale_at - a.c.code_bytes - block + (int64_t)i * a.c.row_bytes + column * 16);
              *at = rescale(*at, old, first);
            }
          } else {
            first = old;
          }
        }
        auto store = [&](uint32_t count) {
          arrived(x);
#pragma unroll
          for (int u = 0; u < U; ++u) {
            if (u * F::R + sub >= count || !there) continue;
            const uint32_t now = page[u] == page0 ? first : needs[u];
            *(Granules)(base + to[u]) = scale[u] == now ? x[u] : rescale(x[u], scale[u], now);
            if (j == 0 && whole) base[to_scale[u]] = (uint8_t)now;  // (each of a page's rows the same)
          }
        };
        if (whole) {
          store(ask);
        } else {
          for (uint32_t i = 0; i < ask; i += F::N) {
            const uint32_t count = find(done + i, min(F::N, ask - i));
            load(count);
#pragma unroll
            for (int u = 0; u < U; ++u) scale[u] = scale_held(scale[u]);
            store(count);
          }
          if (there && j == 0 && sub == 0) base[first_scale_at] = (uint8_t)first;  // no row asks for the one before any more
        }
      }
    }
    done += ask;
  }
  if (slab0 == 0 && block == 0 && lane == 0) say_kept(a, k, r, done, bad);
}

template <bool FP8, int L, int U>
__global__ __launch_bounds__(kThreads) void k_keep_few(KeepArgs a) {
  const uint64_t per = (uint64_t)((a.c.n_slabs + a.slabs - 1) / a.slabs) * a.blocks, items = a.b.n_reqs * per;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  for (uint64_t item = (uint64_t)blockIdx.x * (kThreads / 64) + wave; item < items; item += (uint64_t)gridDim.x * (kThreads / 64)) {
    const uint32_t rest = (uint32_t)(item % per), slab0 = rest / a.blocks * a.slabs;
    keep_few<FP8, L, U>(a, (uint32_t)(item / per), slab0, min(slab0 + a.slabs, a.c.n_slabs), rest % a.blocks);
  }
}

// Many rows: a workgroup takes C 16-byte columns of a slab, R rows at a time with U more
// behind each. In bf16 bounded by memory; with scales by what a step waits for, one thing
// after another.
template <bool FP8, int C, int U>
struct KeepLds {
  static constexpr uint32_t R = kThreads / C, N = R * U;  // rows at a time, rows of a step
  int64_t from[N], to[N];                                 // bytes from a slab's start
  int64_t from_page[FP8 ? N : 1], to_page[FP8 ? N : 1];
  uint32_t good[kThreads / 64];                           // of each wavefront's rows
  uint32_t slot[FP8 ? N : 1];                             // a row's new page, among the step's
  uint32_t need[FP8 ? N : 1][FP8 ? C / 4 : 1];            // scale bytes of those pages, of the workgroup's heads
};

template <bool FP8, int C, int U>
__device__ void keep_many(const KeepArgs& a, KeepLds<FP8, C, U>& l, uint32_t r, uint32_t slab, uint32_t block) {
  constexpr uint32_t R = kThreads / C, N = R * U;
  static_assert(N <= kThreads, "a thread for each row of a step");
  const uint32_t tid = threadIdx.x, lane = tid & 63, col = tid % C, sub = tid / C, column = block * C + col;
  const bool there = column < a.columns;
  const Kept k = kept_of(a, r);
  const uint32_t own = a.c.group[slab >> 1];
  const Bytes base = (Bytes)a.c.base(slab);
  uint32_t done = rows_in_place(k), page0 = 0;  // page0: the step's first page

  // The places of rows [i, i + count), and how many of them can be kept.
  auto find = [&](uint32_t i, uint32_t count) {
    __syncthreads();  // what was found last has been used
    bool fine = true;
    if (tid < count) {
      RowMove m = {0, 0, 0, 0, 0};
      fine = move_of(a, k, i + tid, own, m);
      l.from[tid] = m.from_page + (int64_t)m.from_row * a.c.row_bytes;
      l.to[tid] = m.to_page + (int64_t)m.to_row * a.c.row_bytes;
      if constexpr (FP8) {
        l.from_page[tid] = m.from_page;
        l.to_page[tid] = m.to_page;
        l.slot[tid] = m.page - page0;
      }
    }
    const uint64_t bad = ~__ballot(fine);
    if (lane == 0) l.good[tid / 64] = bad ? tid + (uint32_t)__builtin_ctzll(bad) : ~0u;
    __syncthreads();
    uint32_t good = count;
#pragma unroll
    for (uint32_t w = 0; w < kThreads / 64; ++w) good = min(good, l.good[w]);
    return good;
  };

  bool bad = false;
  u32x4 x[U];
  auto load = [&](uint32_t count) {
#pragma unroll
    for (uint32_t u = 0; u < U; ++u)
      if (there && u * R + sub < count) x[u] = *(Granules)(base + l.from[u * R + sub] + column * 16);
  };
  if constexpr (!FP8) {
    while (done < k.n && !bad) {
      const uint32_t want = min(N, k.n - done), count = find(done, want);
      bad = count < want;
      load(count);
      __syncthreads();  // all of the step's rows are read
#pragma unroll
      for (uint32_t u = 0; u < U; ++u)
        if (there && u * R + sub < count) *(Granules)(base + l.to[u * R + sub] + column * 16) = x[u];
      done += count;
    }
  } else {
    const uint32_t lanes = a.c.row_bytes / a.c.n_scales / 16;  // of a head
    const uint32_t head = min(column / lanes, a.c.n_scales - 1), mine = col / lanes;
    const bool leads = there && col % lanes == 0;
    while (done < k.n && !bad) {
      const uint32_t pos = k.before + done;
      page0 = a.b.page.div(pos);
      const uint32_t o = pos - page0 * k.P;  // of the first page, rows before
      const uint64_t end = k.n - done <= N ? ~0ull : ((uint64_t)page0 + (k.P <= N ? N / k.P : 1)) * k.P;
      uint32_t ask = (uint32_t)min((uint64_t)(k.n - done), end - pos);
      const bool whole = ask <= N;  // the rows are held, not read again
      uint32_t scale[U];
      auto load_scales = [&](uint32_t count) {
#pragma unroll
        for (uint32_t u = 0; u < U; ++u)
          if (u * R + sub < count) scale[u] = scale_held(base[l.from_page[u * R + sub] + a.c.code_bytes + head]);
      };
      __syncthreads();
      for (uint32_t t = tid; t < N * (C / 4); t += kThreads) l.need[t / (C / 4)][t % (C / 4)] = kScaleMin;
      int64_t first_page = 0;
      for (uint32_t i = 0; i < ask; i += N) {
        const uint32_t want = min(N, ask - i), count = find(done + i, want);
        if (i == 0 && count) first_page = l.to_page[0];
        load(count);
        load_scales(count);
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
          const uint32_t t = u * R + sub;
          float m = there && t < count ? largest_code(x[u]) : 0.f;
          for (uint32_t d = 1; d < lanes; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
          if (leads && m > 0.f) atomicMax(&l.need[l.slot[t]][mine], scale_for(m, scale[u]));
        }
        if (count < want) {
          bad = true;
          ask = i + count;
        }
      }
      __syncthreads();  // all rows are read (or will be again), and what their pages need is known
      if (!ask) break;
      uint32_t first_scale = l.need[0][mine];
      if (o) {
        const uint32_t old = scale_held(base[first_page + a.c.code_bytes + head]);
        if (first_scale > old) {  // the page's scale rises: the rows before are rounded again
          for (uint32_t i = sub; i < o && there; i += R) {
            const Granules at = (Granules)(base + first_page + (int64_t)i * a.c.row_bytes + column * 16);
            *at = rescale(*at, old, first_scale);
          }
        } else {
          first_scale = old;
        }
      }
      auto store = [&](uint32_t count) {
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
          const uint32_t t = u * R + sub;
          if (!there || t >= count) continue;
          const uint32_t to = l.slot[t] ? l.need[l.slot[t]][mine] : first_scale;
          *(Granules)(base + l.to[t] + column * 16) = scale[u] == to ? x[u] : rescale(x[u], scale[u], to);
          // a page's scale, with the first of its rows that move
          if (whole && leads && (t == 0 || l.slot[t] != l.slot[t - 1])) base[l.to_page[t] + a.c.code_bytes + head] = (uint8_t)to;
        }
      };
      if (whole) {
        __syncthreads();  // the first page's scale before has been read
        store(ask);
      } else {
        for (uint32_t i = 0; i < ask; i += N) {
          const uint32_t count = min(N, ask - i);
          find(done + i, count);
          load(count);
          load_scales(count);
          __syncthreads();  // all of these rows are read
          store(count);
        }
        __syncthreads();  // no row asks for the scale before any more
        if (leads && sub == 0) base[first_page + a.c.code_bytes + head] = (uint8_t)first_scale;
      }
      done += ask;
    }
  }
  if (slab == 0 && block == 0 && tid == 0) say_kept(a, k, r, done, bad);
}

template <bool FP8, int C, int U>
__global__ __launch_bounds__(kThreads) void k_keep(KeepArgs a) {
  __shared__ KeepLds<FP8, C, U> l;
  const uint64_t per = (uint64_t)a.c.n_slabs * a.blocks, items = a.b.n_reqs * per;
  for (uint64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const uint32_t rest = (uint32_t)(item % per);
    keep_many<FP8, C, U>(a, l, (uint32_t)(item / per), rest / a.blocks, rest % a.blocks);
  }
}

// ---- launching -------------------------------------------------------------------
void fill_slabs(Slabs& s, const tl_ctx* ctx, const tl_cache* c) {
  s.k = c->d_layer_k;
  s.v = c->d_layer_v;
  s.stride = c->page_stride;
  s.n_pages = (uint32_t)c->n_pages;
  s.n_slabs = 2 * ctx->L;
  s.page_tokens = ctx->P;
  const bool scaled = ctx->dtype == TL_DTYPE_FP8_SCALED;
  s.code_bytes = scaled ? ctx->P * ctx->H * ctx->D : (uint32_t)ctx->geo.slab_bytes;
  s.row_bytes = s.code_bytes / ctx->P;
  s.n_scales = scaled ? ctx->H : 0;
  s.n_groups = ctx->geo.n_groups;
  std::copy(ctx->geo.group, ctx->geo.group + ctx->L, s.group);
}

// Workgroups of each of `copies` pages: one for 64 KiB where that fills the device, else one
// for each piece. us, 301 pages of 64 KiB, about half of each, 24 slabs: 107 with one, 116 with
// four (whole pages 193 and 194); 30 of 1 MiB: 182 with one, 155 with 64; 8 pages of 4 slabs 4.7
// and 3.8.
uint32_t pieces_of(uint32_t bytes, uint64_t copies) {
  const uint32_t wide = (bytes + 4 * kPiece - 1) / (4 * kPiece);
  return copies * wide >= 2048 ? wide : (bytes + kPiece - 1) / kPiece;
}

uint32_t grid_of(uint64_t items) { return (uint32_t)std::min<uint64_t>(items, kMostGroups); }

struct PoolLayout {
  uint64_t start, list, end;
};
PoolLayout pool_layout(const tl_ctx* ctx, uint64_t n, uint64_t n_pages) {
  const uint64_t G = ctx->geo.n_groups;
  PoolLayout l;
  l.start = (n + 255) / 256 * 256;  // behind a status for each request
  l.list = l.start + 4 * G * (n + 1);
  l.end = (l.list + 4 * G * n_pages + 255) / 256 * 256;
  return l;
}

void fill_pool(PoolArgs& p, const tl_ctx* ctx, const tl_pool* pool, uint64_t n, uint64_t width, uint8_t* d_status, void* ws) {
  const PoolLayout l = pool_layout(ctx, n, (uint64_t)pool->n_pages);
  p.refs = pool->d_refs;
  p.n_pages = (uint32_t)pool->n_pages;
  p.n_groups = ctx->geo.n_groups;
  p.page_tokens = ctx->P;
  p.n = (uint32_t)n;
  p.width = (uint32_t)width;
  p.status = d_status;
  p.served = (uint8_t*)ws;
  p.start = (uint32_t*)((uint8_t*)ws + l.start);
  p.list = (int32_t*)((uint8_t*)ws + l.list);
}

int launched() { return hipGetLastError() == hipSuccess ? TL_OK : TL_EDEVICE; }

}  // namespace

uint64_t pages_workspace(const tl_ctx* ctx, uint64_t n, uint64_t n_pages) { return pool_layout(ctx, n, n_pages).end; }

int launch_pages_copy(const tl_ctx* ctx, void* stream, const tl_cache* cache, uint64_t n, const int32_t* d_src,
                      const int32_t* d_dst, const uint32_t* d_rows) {
  CopyArgs a = {};
  fill_slabs(a.c, ctx, cache);
  a.src = d_src;
  a.dst = d_dst;
  a.rows = d_rows;
  a.n = (uint32_t)n;
  a.pieces = pieces_of(a.c.code_bytes, n * a.c.n_slabs);
  (void)hipGetLastError();
  {
    TimedLaunch timed(TL_KERNEL_PAGES, stream);
    hipLaunchKernelGGL(k_pages_copy, dim3(grid_of((uint64_t)n * a.c.n_slabs * a.pieces)), dim3(kThreads), 0, (hipStream_t)stream, a);
  }
  return launched();
}

int launch_pages_fork(const tl_ctx* ctx, void* stream, const tl_pool* pool, const tl_cache* cache, uint64_t n_parents,
                      const uint32_t* d_kv_len, const int32_t* d_tables, uint64_t n, const int32_t* d_parent, uint32_t* d_len_out,
                      int32_t* d_tables_out, uint64_t width, uint8_t* d_status, void* ws) {
  ForkArgs a = {};
  fill_slabs(a.c, ctx, cache);
  fill_pool(a.p, ctx, pool, n, width, d_status, ws);
  a.p.parent = d_parent;
  a.p.tables = d_tables;
  a.p.kv_len = d_kv_len;
  a.p.n_parents = (uint32_t)n_parents;
  a.p.out_tables = d_tables_out;
  a.p.out_len = d_len_out;
  a.pieces = pieces_of(a.c.code_bytes, n * a.c.n_slabs);
  hipStream_t s = (hipStream_t)stream;
  (void)hipGetLastError();
  {
    TimedLaunch timed(TL_KERNEL_POOL, stream);
    hipLaunchKernelGGL((k_pool_plan<true>), dim3(1), dim3(kPlanThreads), 0, s, a.p);
  }
  {
    TimedLaunch timed(TL_KERNEL_PAGES, stream);
    const uint64_t items = n * (a.p.n_groups + (uint64_t)a.c.n_slabs * a.pieces);
    hipLaunchKernelGGL(k_pages_fork, dim3(grid_of(items)), dim3(kThreads), 0, s, a);
  }
  return launched();
}

int launch_pages_take(const tl_ctx* ctx, void* stream, const tl_pool* pool, uint64_t n, const uint32_t* d_have, const uint32_t* d_want,
                      int32_t* d_tables, uint64_t width, uint8_t* d_status, void* ws) {
  PoolArgs a = {};
  fill_pool(a, ctx, pool, n, width, d_status, ws);
  a.have = d_have;
  a.want = d_want;
  a.out_tables = d_tables;
  (void)hipGetLastError();
  {
    TimedLaunch timed(TL_KERNEL_POOL, stream);
    hipLaunchKernelGGL((k_pool_plan<false>), dim3(1), dim3(kPlanThreads), 0, (hipStream_t)stream, a);
  }
  return launched();
}

int launch_pages_free(const tl_ctx* ctx, void* stream, const tl_pool* pool, uint64_t n, int32_t* d_tables, uint64_t width,
                      const uint32_t* d_first, const uint32_t* d_end) {
  FreeArgs a = {pool->d_refs, (uint32_t)pool->n_pages, ctx->P, (uint32_t)width, n * ctx->geo.n_groups, n, d_tables, d_first, d_end};
  (void)hipGetLastError();
  {
    TimedLaunch timed(TL_KERNEL_POOL, stream);
    hipLaunchKernelGGL(k_pages_free, dim3(grid_of((a.rows * width + kThreads - 1) / kThreads)), dim3(kThreads), 0, (hipStream_t)stream, a);
  }
  return launched();
}

int launch_keep(const tl_ctx* ctx, void* stream, const tl_batch* batch, const uint32_t* d_n_keep, const uint32_t* d_keep,
                const tl_cache* cache, uint32_t* d_len_out, uint8_t* d_status) {
  KeepArgs a = {};
  fill_slabs(a.c, ctx, cache);
  fill_batch(a.b, ctx, 0, batch);
  a.b.table = batch->d_tables;
  a.n_keep = d_n_keep;
  a.keep = d_keep;
  a.len_out = d_len_out;
  a.status = d_status;
  a.columns = a.c.row_bytes / 16;
  // By the average, as the lengths are on the device only: a request of thousands of rows among
  // many of a few is walked by single wavefronts, some rows a step. One of 20,011 that keeps 8,003
  // beside 96 of up to 48, 24 slabs of 16 heads of 128 in 8 bits: 5.5 ms, in calls of their own 0.47 and 0.03.
  const bool many = batch->n_rows / batch->n_reqs > 256;
  hipStream_t s = (hipStream_t)stream;
  (void)hipGetLastError();
  {
    TimedLaunch timed(TL_KERNEL_KEEP, stream);
    const bool fp8 = ctx->dtype == TL_DTYPE_FP8_SCALED;
    if (many) {
      // Columns of a workgroup (a head's at least) and rows of a thread. Few columns make more
      // workgroups and longer steps; short steps make room for more workgroups at a time. us with
      // 16 columns and 8 rows / 8 and 4 / 8 and 8: in 8 bits, 16 heads of 128, 8,003 rows of one
      // request in 24 slabs 779 / 482 / 454, 1,443 in 4 slabs of 256-token pages 121 / 71 / 52, 1,500
      // of each of 8 requests in 24 slabs 540 / 440 / 548; the same in bf16 362 / 343 / 339, 31 / 24 / 19,
      // 494 / 531 / 533.
      const uint64_t rows = (uint64_t)batch->n_reqs * a.c.n_slabs, small = rows * ((a.columns + 7) / 8);
      const bool wide = fp8 ? ctx->D == 256 : small >= 2048;
      a.blocks = wide ? (a.columns + 15) / 16 : (a.columns + 7) / 8;
      const dim3 grid(grid_of(rows * a.blocks));
      if (fp8 && wide)
        hipLaunchKernelGGL((k_keep<true, 16, 8>), grid, dim3(kThreads), 0, s, a);
      else if (fp8 && small >= 1024)
        hipLaunchKernelGGL((k_keep<true, 8, 4>), grid, dim3(kThreads), 0, s, a);
      else if (fp8)
        hipLaunchKernelGGL((k_keep<true, 8, 8>), grid, dim3(kThreads), 0, s, a);
      else if (wide)
        hipLaunchKernelGGL((k_keep<false, 16, 8>), grid, dim3(kThreads), 0, s, a);
      else
        hipLaunchKernelGGL((k_keep<false, 8, 8>), grid, dim3(kThreads), 0, s, a);
    } else {
      const uint32_t L = fp8 ? ctx->D / 16 : 8;
      a.blocks = (a.columns + L - 1) / L;
      // A wavefront's slabs, of one group of layers (a layer's two, or any): as many as leave
      // work for six wavefronts on every SIMD, up to 8. us with 2 / 4 / 8 / 16: 96 requests of 64
      // slabs of 8 heads 30 / 26 / 24 / 31, 8 of them 7.1 / 9.3 / 14 / 23.
      const uint64_t all = (uint64_t)batch->n_reqs * a.c.n_slabs * a.blocks;
      a.slabs = a.c.n_groups == 1 ? (uint32_t)std::clamp<uint64_t>(all / 6144 & ~1ull, 2, 8) : 2;
      const uint64_t items = (uint64_t)batch->n_reqs * ((a.c.n_slabs + a.slabs - 1) / a.slabs) * a.blocks;
      const dim3 grid(grid_of((items + kThreads / 64 - 1) / (kThreads / 64)));
      // Rows of a step: once or twice what the lanes hold. us, 96 requests of 48 rows that keep 7 / 12
      // / 20 of them, heads of 128 in 8 bits 23 / 63 / 73 with 8 rows, 36 / 41 / 54 with 16; heads of 256 46 / 110
      // and 73 / 87; in bf16 35 / 58 and 35 / 48. Up to 64 rows most are drafts that were refused.
      const bool more = batch->n_rows / batch->n_reqs > 64;
      if (!fp8)
        hipLaunchKernelGGL((k_keep_few<false, 8, 2>), grid, dim3(kThreads), 0, s, a);
      else if (L == 4)
        hipLaunchKernelGGL((k_keep_few<true, 4, 1>), grid, dim3(kThreads), 0, s, a);
      else if (L == 8 && more)
        hipLaunchKernelGGL((k_keep_few<true, 8, 2>), grid, dim3(kThreads), 0, s, a);
      else if (L == 8)
        hipLaunchKernelGGL((k_keep_few<true, 8, 1>), grid, dim3(kThreads), 0, s, a);
      else if (more)
        hipLaunchKernelGGL((k_keep_few<true, 16, 4>), grid, dim3(kThreads), 0, s, a);
      else
        hipLaunchKernelGGL((k_keep_few<true, 16, 2>), grid, dim3(kThreads), 0, s, a);
    }
  }
  return launched();
}

}  // namespace tl
