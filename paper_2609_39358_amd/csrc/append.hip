// tl_append, tl_append_norm: the new tokens' keys and values into the pages of a cache,
// keys and queries normed and rotated on the way.
#include <float.h>

#include <algorithm>

#include "paged.h"

namespace tl {
namespace {

struct Rows {
  const uint16_t* p;
  int64_t token, head;  // strides in elements
};

struct AppendArgs {
  Batch b;
  Pages c;
  Rows k, v, q;
  uint16_t* q_out;
  int64_t qo_token, qo_head;
  uint32_t n_heads, n_q_heads;
  // rotation: pair i of the first `rot` elements by the angle in row
  // pos[axis(i)] of the table
  uint32_t rot, adjacent, n_axes;
  int64_t n_angles;
  const f32x2* cos_sin;  // [n_angles][rot / 2]
  const int32_t* pos;    // [n_axes][n_rows], or null: a token's place in its request
  uint32_t axis[8];      // two bits per pair
  // norms of queries (0) and keys (1): weights of a head, or null for ones
  const float* weight[2];
  int64_t weight_head[2];  // elements from one head's to the next's; 0: all heads' are the same
  float eps;
  uint32_t center;  // the mean is taken off first
  uint8_t* status;
  // the first part of the grid, with scaled pages
  uint32_t n_windows, step;  // windows of so many rows
  uint32_t splits, split_heads;  // workgroups of a window, and their heads
};

constexpr int kWaves = 4;
constexpr uint32_t kInfinite = 0x7f800000;

typedef __attribute__((address_space(1))) uint8_t* GlobalOut;
typedef __attribute__((address_space(1))) u32x2* GlobalOut2;
typedef __attribute__((address_space(1))) u32x4* GlobalOut4;

// A row of D elements is held by D / 16 lanes, 16 elements each: x[0..8) and
// x[8..16) are the two halves of eight pairs, or two runs of eight elements.
template <int D>
struct Row {
  static constexpr int kLanes = D / 16;
  static constexpr int kRows = 64 / kLanes;  // rows of a wavefront
};

__device__ __forceinline__ void unpack(u32x4 w, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

__device__ __forceinline__ u32x4 pack(const float* x) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    bf16x2 p = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
    w[i] = __builtin_bit_cast(uint32_t, p);
  }
  return w;
}

// Where lane j's two runs of eight elements start. Elements i and i + rot / 2
// make a pair unless pairs are adjacent; elements from rot on are not turned.
__device__ __forceinline__ void runs(const AppendArgs& a, bool turned, uint32_t j, uint32_t& first, uint32_t& second) {
  const bool halves = turned && !a.adjacent && 16 * j < a.rot;
  first = halves ? 8 * j : 16 * j;
  second = halves ? a.rot / 2 + 8 * j : 16 * j + 8;
}

struct Angles {
  float c[8], s[8];
  bool ok;
};

// The angles of lane j's eight pairs for row t at `position`. Not ok: a
// position has no row in the table.
__device__ __forceinline__ void load_angles(const AppendArgs& a, uint32_t t, int64_t position, uint32_t j, Angles& g) {
  g.ok = true;
  if (!a.rot) return;
  const uint32_t half = a.rot / 2, p0 = 16 * j < a.rot ? 8 * j : 0;
  if (a.n_axes == 1) {
    if (a.pos) position = a.pos[t];
    g.ok = position >= 0 && position < a.n_angles;
    const f32x4* p = (const f32x4*)(a.cos_sin + (g.ok ? position : 0) * half + p0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 w = p[i];
      g.c[2 * i] = w[0];
      g.s[2 * i] = w[1];
      g.c[2 * i + 1] = w[2];
      g.s[2 * i + 1] = w[3];
    }
    return;
  }
  int64_t row[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const int64_t at = (uint32_t)i < a.n_axes ? a.pos[(uint64_t)i * a.b.n_rows + t] : 0;
    const bool in = at >= 0 && at < a.n_angles;
    g.ok = g.ok && in;
    row[i] = in ? at : 0;
  }
  const uint32_t bits = a.axis[p0 >> 4] >> (2 * (p0 & 15));
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t ax = bits >> (2 * i) & 3;
    const f32x2 w = a.cos_sin[(ax == 0 ? row[0] : ax == 1 ? row[1] : row[2]) * half + p0 + i];
    g.c[i] = w[0];
    g.s[i] = w[1];
  }
}

// Each product and sum is rounded by itself: a row's values do not depend on
// what the compiler would have contracted in the kernel that wrote it.
__device__ __forceinline__ void turn(float& x, float& y, float c, float s) {
#pragma clang fp contract(off)
  const float u = x * c - y * s;
  y = y * c + x * s;
  x = u;
}

__device__ __forceinline__ void rotate(const AppendArgs& a, uint32_t j, const Angles& g, float* x) {
  if (16 * j >= a.rot) return;
  if (a.adjacent) {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn(x[2 * i], x[2 * i + 1], g.c[i], g.s[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn(x[i], x[8 + i], g.c[i], g.s[i]);
  }
}

// The sum over a row's lanes, the same on all of them.
template <int D>
__device__ __forceinline__ float row_sum(float s) {
#pragma unroll
  for (int k = 1; k < Row<D>::kLanes; k *= 2) s += __shfl_xor(s, k);
  return s;
}

// x / sqrt(mean(x^2) + eps) of a row of D elements, less its mean first where that is
// asked for (the mean before the squares: no difference of large sums). In 32 bits; each
// operation is rounded by itself, as in turn().
template <int D>
__device__ __forceinline__ float centered_squares(bool center, float* x) {
#pragma clang fp contract(off)
  if (center) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += x[i];
    s = row_sum<D>(s) * (1.f / D);
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] -= s;
  }
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) s += x[i] * x[i];
  return row_sum<D>(s) * (1.f / D);
}
template <int D>
__device__ __forceinline__ void norm(const AppendArgs& a, float* x) {
#pragma clang fp contract(off)
  float y[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) y[i] = x[i];
  float s = centered_squares<D>(a.center, y);
  float eps = a.eps;
  if (!(s < __uint_as_float(kInfinite))) {
    // Values of 2^60 and more: their squares pass 32 bits, but not those of 2^-70 times
    // them (and values that are not finite stay what they are). eps is lost beside these
    // squares, unless all of them are 0: equal values less their mean, which the smallest
    // normal number in its place leaves 0.
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = x[i] * 0x1p-70f;
    s = centered_squares<D>(a.center, y);
    eps = FLT_MIN;
  }
  const float r = 1.f / __builtin_sqrtf(s + eps);
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = y[i] * r;
}

// Lane j's weights of a head (of queries 0, of keys 1), at the elements that it holds.
struct Weights {
  f32x4 w[4];
};
__device__ __forceinline__ Weights load_weights(const AppendArgs& a, int which, uint32_t head, uint32_t first, uint32_t second) {
  Weights y;
  const float* p = a.weight[which];
  if (!p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) y.w[i] = f32x4{1.f, 1.f, 1.f, 1.f};
    return y;
  }
  p += (int64_t)head * a.weight_head[which];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    y.w[i] = *(const f32x4*)(p + first + 4 * i);
    y.w[2 + i] = *(const f32x4*)(p + second + 4 * i);
  }
  return y;
}

// Lane j's 16 elements of a row, as they were read, normed (w) and turned by the row's
// angles; a row that has none is kept as zeros, and reported.
template <int D, bool NORM>
__device__ __forceinline__ void values(const AppendArgs& a, const u32x4* raw, bool turned, uint32_t j, const Angles& g, const Weights* w, float* x) {
  unpack(raw[0], x);
  unpack(raw[1], x + 8);
  if constexpr (NORM) {
    if (turned) {
      norm<D>(a, x);
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] *= w->w[i / 4][i % 4];
    }
  }
  if (!g.ok) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.f;
  } else if (turned) {
    rotate(a, j, g, x);
  }
}

__device__ __forceinline__ uint32_t largest_bits(const float* x, uint32_t m) {
#pragma unroll
  for (int i = 0; i < 16; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
  return m;
}

__device__ __forceinline__ uint32_t largest_finite_bits(const float* x, uint32_t m) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t y = __float_as_uint(x[i]) & 0x7fffffffu;
    m = y < kInfinite ? max(m, y) : m;
  }
  return m;
}

__device__ __forceinline__ u32x2 codes8(const float* x, float inv) {
  u32x2 w;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * inv, x[4 * i + 1] * inv, 0, false);
    c = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * inv, x[4 * i + 3] * inv, c, true);
    w[i] = (uint32_t)c;
  }
  return w;
}

// Row t of a request: the page and row of its place, or false.
__device__ __forceinline__ bool place(const AppendArgs& a, uint32_t r, int64_t position, uint32_t& page, uint32_t& o) {
  if (position < 0 || position >= a.b.most) return false;
  const uint32_t i = a.b.page.div((uint32_t)position);
  o = (uint32_t)position - i * a.b.page.d;
  page = (uint32_t)a.b.table[(uint64_t)r * a.b.width + i];
  return page < a.c.n_pages;
}

// What wavefronts that share a head tell each other: the largest value and the
// page's scale before, of K and of V.
struct Shared {
  uint32_t m[2][kWaves][2], old[2][kWaves][2];
};

// n tokens of request r from row t on, which go to one page (if there is one), from
// position's row on: heads [head0, head1) of K and V, by the wavefronts of a workgroup. A wavefront takes one
// head's K and V of up to HELD * kRows tokens and keeps them until the page's
// scale is known; with fewer tokens it takes several heads, and up to all four
// share the tokens of one. Of more tokens than four can hold the earlier ones are
// read again.
template <int D, int HELD, bool NORM>
__device__ void put_fragment(const AppendArgs& a, Shared& l, uint32_t head0, uint32_t head1, uint32_t r, uint32_t t, uint32_t n,
                             int64_t position) {
  constexpr int L = Row<D>::kLanes, R = Row<D>::kRows;
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64, j = lane % L, row = lane / L;
  uint32_t span = 1, share = 1;
  while (span < n && span < R) span *= 2;
  while (share < kWaves && HELD * span * share < n) share *= 2;
  const uint32_t groups = kWaves / share, w = wave % share, heads = R / span, sub = w * span + (row & (span - 1));
  const uint32_t every = span * share, chunk = HELD * every, chunks = (n + chunk - 1) / chunk;
  const uint32_t packs = (head1 - head0 + heads - 1) / heads;
  uint32_t first[2], second[2];
  runs(a, true, j, first[0], second[0]);
  runs(a, false, j, first[1], second[1]);
  Angles g[HELD];
  u32x4 raw[2][HELD][2];
  float x[2][HELD][16];
  Weights weights;
  auto angles = [&](uint32_t c) {
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
      const uint32_t i = min(c * chunk + h * every + sub, n - 1);
      load_angles(a, t + i, position + i, j, g[h]);
    }
  };
  auto load = [&](uint32_t head, uint32_t c) {
    if constexpr (NORM) weights = load_weights(a, 1, min(head, head1 - 1), first[0], second[0]);
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
      const uint32_t i = min(c * chunk + h * every + sub, n - 1);
      const uint16_t* k = a.k.p + (int64_t)(t + i) * a.k.token + (int64_t)min(head, head1 - 1) * a.k.head;
      const uint16_t* v = a.v.p + (int64_t)(t + i) * a.v.token + (int64_t)min(head, head1 - 1) * a.v.head;
      raw[0][h][0] = *(const u32x4*)(k + first[0]);
      raw[0][h][1] = *(const u32x4*)(k + second[0]);
      raw[1][h][0] = *(const u32x4*)(v + first[1]);
      raw[1][h][1] = *(const u32x4*)(v + second[1]);
    }
  };
  auto convert = [&] {
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
      values<D, NORM>(a, raw[0][h], true, j, g[h], &weights, x[0][h]);
      values<D, NORM>(a, raw[1][h], false, j, g[h], nullptr, x[1][h]);
    }
  };

  const uint32_t mine = head0 + wave / share * heads + row / span;
  load(mine, 0);  // before the page is known: a decode step waits for one thing after another
  if (chunks == 1) angles(0);
  uint32_t page, o;
  if (!place(a, r, position, page, o)) return;
  const GlobalOut pages[2] = {(GlobalOut)*a.c.k + (int64_t)page * a.c.stride, (GlobalOut)*a.c.v + (int64_t)page * a.c.stride};
  for (uint32_t p = 0, flip = 0; p < packs; p += groups, flip ^= 1) {
    const uint32_t head = mine + p * heads;
    uint32_t m[2] = {0, 0}, old[2] = {0, 0};
    if (o)
#pragma unroll
      for (int s = 0; s < 2; ++s) old[s] = pages[s][a.c.scale_off + min(head, head1 - 1)];
    for (uint32_t c = 0; c < chunks; ++c) {
      if (chunks > 1) {
        angles(c);
        if (p + c) load(head, c);
      }
      convert();
      // the last rows are there more than once, which changes no maximum
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        uint32_t y = 0;
#pragma unroll
        for (int h = 0; h < HELD; ++h) y = largest_bits(x[s][h], y);
        if (y >= kInfinite) {
          y = 0;
#pragma unroll
          for (int h = 0; h < HELD; ++h) y = largest_finite_bits(x[s][h], y);
        }
        m[s] = max(m[s], y);
      }
    }
    if (chunks == 1 && p + groups < packs) load(head + groups * heads, 0);
#pragma unroll
    for (int s = 0; s < 2; ++s)
      for (uint32_t k = 1; k < L * span; k *= 2) m[s] = max(m[s], (uint32_t)__shfl_xor((int)m[s], k));
    if (share > 1) {  // then a wavefront has one head
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        l.m[flip][wave][s] = m[s];
        if (w == 0) l.old[flip][wave][s] = old[s];
      }
      __syncthreads();
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        for (uint32_t k = 0; k < share; ++k) m[s] = max(m[s], l.m[flip][wave - w + k][s]);
        old[s] = l.old[flip][wave - w][s];
      }
    }
    float inv[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      uint32_t b = scale_byte(__uint_as_float(m[s]));
      if (o && head < head1) {
        const uint32_t held = scale_held(old[s]);
        if (b > held) {
          // the page's scale rises: the rows before are rounded again
          const float by = scale_inverse(127 + min(b - held, 40u));  // 2^(held - b); 448 * 2^-40 rounds to 0 as well
          constexpr int kAhead = 4;
          for (uint32_t i0 = sub; i0 < o; i0 += kAhead * every) {
            GlobalOut4 at[kAhead];
            u32x4 q[kAhead];
#pragma unroll
            for (int f = 0; f < kAhead; ++f) {
              at[f] = (GlobalOut4)(pages[s] + ((uint64_t)(i0 + f * every) * a.n_heads + head) * D + 16 * j);
              if (i0 + f * every < o) q[f] = *at[f];
            }
#pragma unroll
            for (int f = 0; f < kAhead; ++f) {
              if (i0 + f * every >= o) continue;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(q[f][e], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(q[f][e], true);
                int c = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0] * by, lo[1] * by, 0, false);
                q[f][e] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(hi[0] * by, hi[1] * by, c, true);
              }
              *at[f] = q[f];
            }
          }
        } else {
          b = held;
        }
      }
      if (j == 0 && sub == 0 && head < head1) pages[s][a.c.scale_off + head] = (uint8_t)b;
      inv[s] = scale_inverse(b);
    }
    for (uint32_t c = chunks; c-- > 0;) {
      if (c + 1 < chunks) {
        angles(c);
        load(head, c);
        convert();
      }
#pragma unroll
      for (int h = 0; h < HELD; ++h) {
        const uint32_t i = c * chunk + h * every + sub;
        if (i >= n || head >= head1) continue;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const GlobalOut out = pages[s] + ((uint64_t)(o + i) * a.n_heads + head) * D;
          *(GlobalOut2)(out + first[s]) = codes8(x[s][h], inv[s]);
          *(GlobalOut2)(out + second[s]) = codes8(x[s][h] + 8, inv[s]);
        }
      }
    }
  }
}

// A wavefront's row t: its status, its queries, and with bf16 pages its K and V.
// They are lines of D elements that the same angles turn.
template <int D, bool FP8, bool NORM>
__device__ void put_row(const AppendArgs& a, uint32_t t) {
  constexpr int L = Row<D>::kLanes, R = Row<D>::kRows, kBatch = 4;
  const uint32_t lane = threadIdx.x & 63, j = lane % L, H = a.n_heads, nq = a.q.p ? a.n_q_heads : 0;
  const uint32_t lines = nq + (FP8 ? 0 : 2 * H);
  uint32_t first, second;
  runs(a, true, j, first, second);
  u32x4 raw[kBatch][2];
  auto load = [&](uint32_t u0) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const uint32_t u = u0 + i * R;
      if (u >= lines) continue;
      const uint16_t* p = a.q.p + (int64_t)t * a.q.token + (int64_t)u * a.q.head;
      uint32_t at = first, then = second;
      if (!FP8 && u >= nq) {
        p = a.k.p + (int64_t)t * a.k.token + (int64_t)(u - nq) * a.k.head;
        if (u >= nq + H) {
          p = a.v.p + (int64_t)t * a.v.token + (int64_t)(u - nq - H) * a.v.head;
          at = 16 * j;
          then = 16 * j + 8;
        }
      }
      raw[i][0] = *(const u32x4*)(p + at);
      raw[i][1] = *(const u32x4*)(p + then);
    }
  };
  load(lane / L);
  const uint32_t r = find_request(a.b, t);
  const int64_t position = r < a.b.n_reqs ? (int64_t)a.b.kv_len[r] - (a.b.first_row(r + 1) - t) : -1;
  uint32_t page = 0, o = 0;
  const bool has_place = r < a.b.n_reqs && place(a, r, position, page, o);
  Angles g;
  load_angles(a, t, position, j, g);
  if (a.status) {
    const bool fine = __all(has_place && g.ok);
    if (lane == 0) a.status[t] = fine ? TL_ACCEPT : TL_BADARG;
  }
  if (r == a.b.n_reqs && !(a.pos && __all(g.ok))) return;  // not a request's row, and at no position of its own
  const GlobalOut k_row = (GlobalOut)*a.c.k + (int64_t)page * a.c.stride + (uint64_t)o * H * (2 * D);
  const GlobalOut v_row = (GlobalOut)*a.c.v + (int64_t)page * a.c.stride + (uint64_t)o * H * (2 * D);
  for (uint32_t u0 = lane / L; u0 < lines; u0 += kBatch * R) {
    if (u0 >= kBatch * R) load(u0);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const uint32_t u = u0 + i * R;
      if (u >= lines) continue;
      const bool is_v = !FP8 && u >= nq + H;
      float x[16];
      Weights w;
      if constexpr (NORM) {
        const bool is_k = !FP8 && u >= nq;
        if (!is_v) w = load_weights(a, is_k, is_k ? u - nq : u, first, second);
      }
      values<D, NORM>(a, raw[i], !is_v, j, g, &w, x);
      GlobalOut out = (GlobalOut)(a.q_out + (int64_t)t * a.qo_token + (int64_t)u * a.qo_head);
      if (!FP8 && u >= nq) {
        if (!has_place) continue;
        out = is_v ? v_row + (uint64_t)(u - nq - H) * (2 * D) : k_row + (uint64_t)(u - nq) * (2 * D);
      }
      *(GlobalOut4)(out + 2 * (is_v ? 16 * j : first)) = pack(x);
      *(GlobalOut4)(out + 2 * (is_v ? 16 * j + 8 : second)) = pack(x + 8);
    }
  }
}

// The first n_windows * splits workgroups take a window of `step` rows and some heads
// of K and V each: those fragments (rows of one request that go to one scaled page)
// that begin there. The others take a row per wavefront.
template <int D, int HELD, bool NORM>
__global__ __launch_bounds__(64 * kWaves, NORM && HELD == 2 ? 2 : 1) void k_append(AppendArgs a) {
  constexpr bool FP8 = HELD > 0;
  uint32_t block = blockIdx.x;
  if constexpr (FP8) {
    __shared__ Shared l;
    if (block < a.n_windows * a.splits) {
      const uint32_t head0 = block % a.splits * a.split_heads, head1 = min(head0 + a.split_heads, a.n_heads);
      uint32_t t = block / a.splits * a.step;
      const uint32_t end = min(t + a.step, a.b.n_rows);
      uint32_t r = find_request(a.b, t);
      while (t < end && r < a.b.n_reqs) {
        const uint32_t row0 = a.b.first_row(r), row1 = a.b.first_row(r + 1);
        if (t >= row1 || t < row0) {
          if (++r == a.b.n_reqs) break;
          t = max(t, a.b.first_row(r));
          continue;
        }
        const int64_t position = (int64_t)a.b.kv_len[r] - (row1 - t);
        const uint32_t P = a.b.page.d;
        // rows that the table has no place for (before a request's own start, or
        // past the end of its table) make one run, which is refused
        uint32_t o = 0, n = row1 - t;
        if (position < 0) {
          n = (uint32_t)min((int64_t)n, -position);
        } else if (position < a.b.most) {
          o = (uint32_t)position - a.b.page.div((uint32_t)position) * P;
          n = min(P - o, n);
        }
        if (t == row0 || o == 0) {
          __syncthreads();  // what the last fragment shared has been read
          put_fragment<D, HELD, NORM>(a, l, head0, head1, r, t, n, position);
        }
        t += n;
      }
      return;
    }
    block -= a.n_windows * a.splits;
  }
  const uint32_t t = block * kWaves + threadIdx.x / 64;
  if (t < a.b.n_rows) put_row<D, FP8, NORM>(a, t);
}

template <int D, bool NORM>
void launch(bool fp8, uint32_t grid, hipStream_t s, const AppendArgs& a) {
  if (!fp8)
    hipLaunchKernelGGL((k_append<D, 0, NORM>), dim3(grid), dim3(64 * kWaves), 0, s, a);
  else if (a.step <= (uint32_t)Row<D>::kRows || (a.n_windows >= 256 && a.step <= (uint32_t)(kWaves * Row<D>::kRows)))
    // A lane holds one row: where one wavefront's lanes hold a window, or, with many
    // windows, four do. 24,573 tokens into pages of 16 rows of 16 heads of 128: 153 us,
    // 4.7 TB/s, with two rows held 170; 64 requests of 2 rows 7.6 and 9.5; 128
    // windows of 16 rows 17.7 and 14.9.
    // (With norms 24,573 tokens take 190 to 210 us, 40 more registers; in bf16 pages, a row a
    // wavefront, 167 to 187, where 811 MB at a large copy's rate take 174.)
    hipLaunchKernelGGL((k_append<D, 1, NORM>), dim3(grid), dim3(64 * kWaves), 0, s, a);
  else
    hipLaunchKernelGGL((k_append<D, 2, NORM>), dim3(grid), dim3(64 * kWaves), 0, s, a);
}

}  // namespace

void fill_batch(Batch& b, const tl_ctx* ctx, uint32_t layer, const tl_batch* batch) {
  b.row_off = batch->d_row_off;
  b.kv_len = batch->d_kv_len;
  b.n_reqs = (uint32_t)batch->n_reqs;
  b.n_rows = (uint32_t)batch->n_rows;
  b.width = (uint32_t)batch->table_width;
  b.table = batch->d_tables + (uint64_t)ctx->geo.group[layer] * batch->n_reqs * batch->table_width;
  const uint64_t most = batch->table_width * ctx->P;
  b.most = most < kMostTokens ? (uint32_t)most : kMostTokens;
  b.page.set(ctx->P);
}

void fill_pages(Pages& p, const tl_ctx* ctx, uint32_t layer, const tl_cache* c) {
  p.k = c->d_layer_k + layer;
  p.v = c->d_layer_v + layer;
  p.stride = c->page_stride;
  p.n_pages = (uint32_t)c->n_pages;
  p.scale_off = ctx->P * ctx->H * ctx->D;
}

int launch_append(const tl_ctx* ctx, void* stream, uint32_t layer, const tl_batch* batch, const tl_norm* norm, const tl_rope* rope,
                  const tl_rows* k, const tl_rows* v, uint32_t n_q_heads, const tl_rows* q, const tl_rows* q_out,
                  const tl_cache* cache, uint8_t* d_status) {
  AppendArgs a = {};
  fill_batch(a.b, ctx, layer, batch);
  fill_pages(a.c, ctx, layer, cache);
  auto rows = [](const tl_rows* r) { return Rows{(const uint16_t*)r->d_rows, r->row_stride, r->head_stride}; };
  a.k = rows(k);
  a.v = rows(v);
  if (q) {
    a.q = rows(q);
    a.q_out = (uint16_t*)q_out->d_rows;
    a.qo_token = q_out->row_stride;
    a.qo_head = q_out->head_stride;
  }
  a.n_heads = ctx->H;
  a.n_q_heads = n_q_heads;
  a.n_axes = 1;
  if (rope) {
    a.rot = rope->rot_dim;
    a.adjacent = (rope->flags & TL_ROPE_ADJACENT) != 0;
    a.n_axes = rope->n_axes;
    a.n_angles = rope->n_angles;
    a.cos_sin = (const f32x2*)rope->d_cos_sin;
    a.pos = rope->d_pos;
    for (uint32_t i = 0; rope->pair_axis && i < rope->rot_dim / 2; ++i)
      a.axis[i >> 4] |= (uint32_t)rope->pair_axis[i] << (2 * (i & 15));
  }
  if (norm) {
    a.weight[0] = norm->d_q_weight;
    a.weight[1] = norm->d_k_weight;
    a.weight_head[0] = norm->q_stride;
    a.weight_head[1] = norm->k_stride;
    a.eps = norm->eps;
    a.center = (norm->flags & TL_NORM_CENTER) != 0;
  }
  a.status = d_status;
  const bool fp8 = ctx->dtype == TL_DTYPE_FP8_SCALED;
  if (fp8) {
    // A workgroup of the first part takes about one fragment: a row of each
    // request where requests bring one row, a page's rows where they bring many;
    // with few of those, some of the heads.
    const uint64_t per = batch->n_rows / batch->n_reqs;
    a.step = (uint32_t)(per < 1 ? 1 : per < ctx->P ? per : ctx->P);
    // A launch has fewer than 2^32 threads: of millions of rows on pages of one token, a
    // window takes four, one after another.
    if (a.step == 1 && a.b.n_rows > (1u << 22)) a.step = 4;
    a.n_windows = (a.b.n_rows + a.step - 1) / a.step;
    // Heads that a fragment's workgroup takes at once, and not one round after another
    // (put_fragment).
    const uint32_t rows = a.step, R = 64 / (ctx->D / 16), whole = a.n_windows;
    auto at_once = [&](uint32_t step) {
      const uint32_t held = step <= R || (a.n_windows >= 256 && step <= kWaves * R) ? 1 : 2;
      uint32_t span = 1, share = 1;
      while (span < rows && span < R) span *= 2;
      while (share < kWaves && held * span * share < rows) share *= 2;
      return kWaves / share * (R / span);
    };
    auto split = [&](uint32_t workgroups, uint32_t heads) {
      a.splits = std::max(1u, std::min(workgroups / a.n_windows, (ctx->H + heads - 1) / heads));
      return (ctx->H + a.splits - 1) / a.splits;
    };
    // Fragments that begin in one window are written one after another. Shorter windows part them,
    // but each window that is left empty takes a workgroup the time to find that out, for each
    // share of the heads. So windows are either whole, and few of them give their heads to several
    // workgroups, at least four heads to each; or shorter, 256 or more of them, and each
    // workgroup takes as many heads as it can at once. us, whole / shorter, 8 heads of 128 and pages of 16
    // unless said. Shorter where all fragments are on the device at the same time:
    //   3 requests of 40 rows 11.1 / 6.1, 12 of 24 15.5 / 9.0, 12 of 8 8.6 / 8.5 (48 of 8 9.0 / 9.5);
    // where a fragment has more than 64 rows, and a workgroup much to do for it:
    //   pages of 128, 1 of 4,096 49 / 24, 1 of 8,192 51 / 42 (1 of 16,384 62 / 82); pages of 256, 16 heads,
    //   1 of 3,000 94 / 28, 24 of 300 115 / 57, 1 of 8,192 107 / 101 (1 of 16,384 152 / 241, 1 of 24,573 193 / 397);
    // and where several requests longer than a page begin and end inside pages, so that
    // there are a fifth more fragments than windows:
    //   48 of 40 17.7 / 14.7, 96 of 24 18.6 / 14.8, 130 of 20 18.5 / 17.3 (192 of 20 21.3 / 22.2; and 48 of 32 12.6 / 15.0).
    // Requests of up to 32 rows and no longer than a page are in between: of equal lengths one or
    // two begin in a window, of different lengths, which only the device has, many may. They get
    // windows of half of that, or where that leaves few a quarter: 96 of 1 to 24 rows 24.0 / 15.9 (as short as above
    // 13.1), 192 of 1 to 16 21.4 / 16.1, 96 of 12 each 12.2 / 13.1 (14.9), 130 of 16 each 14.2 / 15.8 (18.5).
    // Whole in all else: 1 of 3,200 15.4 / 18.7, 1 of 8,192 25.3 / 28.3; 16 heads, 1 of 512
    // 11.5 / 15.7, 1 of 1,552 14.5 / 22.5; pages of 64, 48 of 40 22.1 / 29.8, 16 heads, 1 of 4,096 31.9 / 52.2.
    const uint64_t fragments = (a.b.n_rows + batch->n_reqs * (ctx->P - 1)) / ctx->P;
    const uint32_t most = at_once(rows);
    const uint64_t shares = fragments * ((ctx->H + most - 1) / most);
    const bool few = shares < 128 || (rows > 64 && shares < 850 && whole < 128);
    const bool ragged = per > ctx->P && rows <= 64 && 5 * fragments >= 6 * (uint64_t)whole && whole < 256;
    const bool several = batch->n_reqs > 1 && per <= ctx->P && rows <= 32 && whole < 256;
    auto shorten = [&] {
      a.step = (a.step + 1) / 2;
      a.n_windows = (a.b.n_rows + a.step - 1) / a.step;
    };
    if (few || ragged) {
      while (a.step > (rows > 64 ? 64 : 2) && a.n_windows < 256) shorten();
      const uint32_t heads = at_once(a.step);
      a.split_heads = std::min(ctx->H, (split(1100, heads) + heads - 1) / heads * heads);
    } else {
      for (int i = 0; several && i < 2 && a.step > 2 && (i == 0 || a.n_windows < 150); ++i) shorten();
      const uint32_t many = rows > 64 ? 1024 : 512;
      a.split_heads = rows > 1 && a.n_windows < many ? split(many + a.n_windows - 1, std::max<uint32_t>(kWaves, most)) : ctx->H;
    }
    a.splits = (ctx->H + a.split_heads - 1) / a.split_heads;
  }
  const uint32_t single = !fp8 || q || d_status ? (a.b.n_rows + kWaves - 1) / kWaves : 0;
  const uint32_t grid = a.n_windows * a.splits + single;
  hipStream_t s = (hipStream_t)stream;
  (void)hipGetLastError();
  {
    TimedLaunch timed(TL_KERNEL_APPEND, stream);
    if (ctx->D == 64)
      norm ? launch<64, true>(fp8, grid, s, a) : launch<64, false>(fp8, grid, s, a);
    else if (ctx->D == 128)
      norm ? launch<128, true>(fp8, grid, s, a) : launch<128, false>(fp8, grid, s, a);
    else
      norm ? launch<256, true>(fp8, grid, s, a) : launch<256, false>(fp8, grid, s, a);
  }
  return hipGetLastError() == hipSuccess ? TL_OK : TL_EDEVICE;
}

}  // namespace tl
