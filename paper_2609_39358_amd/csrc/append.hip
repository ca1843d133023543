// tl_append: the new tokens' keys and values into the pages of a cache, keys and
// queries rotated on the way.
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
  uint8_t* status;
  uint32_t step;       // rows per workgroup of the first part of the grid
  uint32_t n_windows;  // workgroups of that part
};

constexpr int kWaves = 4;

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

// Lane j's part of row t of one head, rotated if `turned`.
__device__ __forceinline__ void load_row(const AppendArgs& a, const Rows& in, bool turned, uint32_t t, uint32_t head,
                                         int64_t position, uint32_t j, float* x) {
  uint32_t first, second;
  runs(a, turned, j, first, second);
  const uint16_t* p = in.p + (int64_t)t * in.token + (int64_t)head * in.head;
  const u32x4 lo = *(const u32x4*)(p + first), hi = *(const u32x4*)(p + second);
  unpack(lo, x);
  unpack(hi, x + 8);
  Angles g;
  load_angles(a, t, position, j, g);
  if (!g.ok) {  // no angle: the token is kept as zeros, and reported
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.f;
  } else if (turned && a.rot) {
    rotate(a, j, g, x);
  }
}

__device__ __forceinline__ float largest_finite(const float* x, float m) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float y = fabsf(x[i]);
    m = y < __builtin_inff() ? fmaxf(m, y) : m;
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

// n tokens from row t on, which go to rows [o, o + n) of one page, by the
// wavefronts of a workgroup: a wavefront takes one head's K or V of up to
// kRows tokens at a time, or with fewer tokens that of several heads.
template <int D, bool FP8>
__device__ void put_fragment(const AppendArgs& a, uint32_t t, uint32_t n, uint32_t page, uint32_t o, int64_t position) {
  constexpr int L = Row<D>::kLanes, R = Row<D>::kRows;
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64, j = lane % L, row = lane / L;
  uint32_t span = 1;
  while (span < n && span < R) span *= 2;
  const uint32_t heads = R / span, sub = row & (span - 1);
  const uint32_t packs = (a.n_heads + heads - 1) / heads;
  for (uint32_t job = wave; job < 2 * packs; job += kWaves) {
    const bool is_k = (job & 1) == 0;
    const uint32_t head = (job >> 1) * heads + row / span;
    const Rows& in = is_k ? a.k : a.v;
    GlobalOut base = (GlobalOut)*(is_k ? a.c.k : a.c.v) + (int64_t)page * a.c.stride;
    if (!FP8) {
      if (head < a.n_heads) {
        uint32_t first, second;
        runs(a, is_k, j, first, second);
        for (uint32_t i = sub; i < n; i += span) {
          float x[16];
          load_row(a, in, is_k, t + i, head, position + i, j, x);
          const GlobalOut out = base + ((uint64_t)(o + i) * a.n_heads + head) * (2 * D);
          *(GlobalOut4)(out + 2 * first) = pack(x);
          *(GlobalOut4)(out + 2 * second) = pack(x + 8);
        }
      }
      continue;
    }
    float m = 0.f;
    if (head < a.n_heads)
      for (uint32_t i = sub; i < n; i += span) {
        float x[16];
        load_row(a, in, is_k, t + i, head, position + i, j, x);
        m = largest_finite(x, m);
      }
    for (uint32_t k = 1; k < L * span; k *= 2) m = fmaxf(m, __shfl_xor(m, k));
    if (head >= a.n_heads) continue;
    uint32_t b = scale_byte(m);
    const GlobalOut scales = base + a.c.scale_off;
    if (o) {
      const uint32_t old = scale_held(scales[head]);
      if (b > old) {
        // the page's scale rises: the rows before are rounded again
        const float by = scale_inverse(127 + min(b - old, 40u));  // 2^(old - b); 448 * 2^-40 rounds to 0 as well
        for (uint32_t i = sub; i < o; i += span) {
          const GlobalOut4 p = (GlobalOut4)(base + ((uint64_t)i * a.n_heads + head) * D + 16 * j);
          u32x4 w = *p;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[q], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[q], true);
            int c = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0] * by, lo[1] * by, 0, false);
            w[q] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(hi[0] * by, hi[1] * by, c, true);
          }
          *p = w;
        }
      } else {
        b = old;
      }
    }
    if (j == 0 && sub == 0) scales[head] = (uint8_t)b;
    const float inv = scale_inverse(b);
    uint32_t first, second;
    runs(a, is_k, j, first, second);
    for (uint32_t i = sub; i < n; i += span) {
      float x[16];
      load_row(a, in, is_k, t + i, head, position + i, j, x);
      const GlobalOut out = base + ((uint64_t)(o + i) * a.n_heads + head) * D;
      *(GlobalOut2)(out + first) = codes8(x, inv);
      *(GlobalOut2)(out + second) = codes8(x + 8, inv);
    }
  }
}

// Row t of a request: the page and row of its place, or false.
__device__ __forceinline__ bool place(const AppendArgs& a, uint32_t r, int64_t position, uint32_t& page, uint32_t& o) {
  if (position < 0 || position >= a.b.most) return false;
  const uint32_t i = a.b.page.div((uint32_t)position);
  o = (uint32_t)position - i * a.b.page.d;
  page = (uint32_t)a.b.table[(uint64_t)r * a.b.width + i];
  return page < a.c.n_pages;
}

// The first n_windows workgroups take `step` rows each: those fragments (rows
// of one request that go to one page) that begin there. The others take a row
// per wavefront: its queries and its status.
template <int D, bool FP8>
__global__ __launch_bounds__(64 * kWaves) void k_append(AppendArgs a) {
  constexpr int L = Row<D>::kLanes, R = Row<D>::kRows;
  if (blockIdx.x < a.n_windows) {
    uint32_t t = blockIdx.x * a.step;
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
        uint32_t page, row;
        if (place(a, r, position, page, row)) put_fragment<D, FP8>(a, t, n, page, row, position);
      }
      t += n;
    }
    return;
  }
  const uint32_t t = (blockIdx.x - a.n_windows) * kWaves + threadIdx.x / 64;
  if (t >= a.b.n_rows) return;
  const uint32_t r = find_request(a.b, t), lane = threadIdx.x & 63, j = lane % L;
  const int64_t position = r < a.b.n_reqs ? (int64_t)a.b.kv_len[r] - (a.b.first_row(r + 1) - t) : -1;
  Angles g;
  load_angles(a, t, position, j, g);
  if (a.status) {
    uint32_t page, row;
    const bool fine = __all(r < a.b.n_reqs && place(a, r, position, page, row) && g.ok);
    if (lane == 0) a.status[t] = fine ? TL_ACCEPT : TL_BADARG;
  }
  if (!a.q.p) return;
  uint32_t first, second;
  runs(a, true, j, first, second);
  for (uint32_t head = lane / L; head < a.n_q_heads; head += R) {
    const uint16_t* p = a.q.p + (int64_t)t * a.q.token + (int64_t)head * a.q.head;
    float x[16];
    unpack(*(const u32x4*)(p + first), x);
    unpack(*(const u32x4*)(p + second), x + 8);
    if (!g.ok) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = 0.f;
    } else if (a.rot) {
      rotate(a, j, g, x);
    }
    uint16_t* out = a.q_out + (int64_t)t * a.qo_token + (int64_t)head * a.qo_head;
    *(u32x4*)(out + first) = pack(x);
    *(u32x4*)(out + second) = pack(x + 8);
  }
}

template <int D>
void launch(bool fp8, uint32_t grid, hipStream_t s, const AppendArgs& a) {
  if (fp8)
    hipLaunchKernelGGL((k_append<D, true>), dim3(grid), dim3(64 * kWaves), 0, s, a);
  else
    hipLaunchKernelGGL((k_append<D, false>), dim3(grid), dim3(64 * kWaves), 0, s, a);
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
  b.most = most < 0x7fffffff ? (uint32_t)most : 0x7fffffff;
  b.page.set(ctx->P);
}

void fill_pages(Pages& p, const tl_ctx* ctx, uint32_t layer, const tl_cache* c) {
  p.k = c->d_layer_k + layer;
  p.v = c->d_layer_v + layer;
  p.stride = c->page_stride;
  p.n_pages = (uint32_t)c->n_pages;
  p.scale_off = ctx->P * ctx->H * ctx->D;
}

int launch_append(const tl_ctx* ctx, void* stream, uint32_t layer, const tl_batch* batch, const tl_rope* rope,
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
  a.status = d_status;
  // A workgroup of the first part takes about one fragment: a row of each
  // request where requests bring one row, a page's rows where they bring many.
  const uint64_t per = batch->n_rows / batch->n_reqs;
  a.step = (uint32_t)(per < 1 ? 1 : per < ctx->P ? per : ctx->P);
  a.n_windows = (a.b.n_rows + a.step - 1) / a.step;
  const uint32_t single = q || d_status ? (a.b.n_rows + kWaves - 1) / kWaves : 0;
  hipStream_t s = (hipStream_t)stream;
  const bool fp8 = ctx->dtype == TL_DTYPE_FP8_SCALED;
  (void)hipGetLastError();
  {
    TimedLaunch timed(TL_KERNEL_APPEND, stream);
    if (ctx->D == 64)
      launch<64>(fp8, a.n_windows + single, s, a);
    else if (ctx->D == 128)
      launch<128>(fp8, a.n_windows + single, s, a);
    else
      launch<256>(fp8, a.n_windows + single, s, a);
  }
  return hipGetLastError() == hipSuccess ? TL_OK : TL_EDEVICE;
}

}  // namespace tl
