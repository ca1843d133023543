// Device code shared by the kernels that work on an engine's paged cache
// (append.hip, attend.hip): the ragged batch of one call, its page tables, and
// the scaled 8-bit pages. Not part of the ABI.
#pragma once
#include <hip/hip_runtime.h>

#include "internal.h"

namespace tl {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Scale bytes of scaled 8-bit pages: b stands for 2^(b - 127). From 2^-117 on
// every code times its scale is a normal bf16 value, so that a page's values
// are exactly what the matrix instructions are given.
constexpr uint32_t kScaleMin = 10;
constexpr uint32_t kScaleMax = 247;

// x / d for x < 2^31 and one d >= 1 of a whole launch: a multiplication.
struct FastDiv {
  uint32_t d, mul, shift;
  void set(uint32_t div) {
    d = div;
    mul = shift = 0;
    if (div == 1) return;
    uint32_t l = 1;
    while ((1ull << l) < div) ++l;
    mul = (uint32_t)((1ull << (31 + l)) / div + 1);
    shift = l - 1;
  }
  __device__ __forceinline__ uint32_t div(uint32_t x) const { return mul ? __umulhi(x, mul) >> shift : x; }
};

// Tokens of a request, at most: keys are numbered in 32 bits with a sign, and a
// kernel's steps look up to some blocks past the last one.
constexpr uint32_t kMostTokens = (1u << 31) - (1u << 16);

// One call's requests (tl_batch) for one layer.
struct Batch {
  const uint32_t* row_off;
  const uint32_t* kv_len;
  const int32_t* table;  // of the layer's group
  uint32_t n_reqs, n_rows, width;
  uint32_t most;         // tokens that a table row can address, up to kMostTokens
  FastDiv page;

  __device__ __forceinline__ uint32_t first_row(uint32_t r) const { return min(row_off[r], n_rows); }
  __device__ __forceinline__ uint32_t held(uint32_t r) const { return min(kv_len[r], most); }
};

// Pages of one layer. The bases are read on the device.
struct Pages {
  const uint64_t* k;
  const uint64_t* v;
  int64_t stride;
  uint32_t n_pages;
  uint32_t scale_off;  // bytes of a page's codes: its scale bytes follow
};

// The caches' bases are read from memory: they are told apart from other address
// spaces here, since a load that might be of shared memory is waited for with
// every access to that.
typedef __attribute__((address_space(1))) const uint8_t* GlobalBytes;
typedef __attribute__((address_space(1))) const uint32_t* GlobalU32;
typedef __attribute__((address_space(1))) const u32x2* GlobalU32x2;
typedef __attribute__((address_space(1))) const u32x4* GlobalU32x4;
__device__ __forceinline__ GlobalBytes layer_base(const uint64_t* p) { return (GlobalBytes)*p; }

// Request that row t belongs to (first_row(r) <= t < first_row(r + 1)), or
// n_reqs: found by the whole wavefront, 64 offsets at a time.
__device__ __forceinline__ uint32_t find_request(const Batch& b, uint32_t t) {
  uint32_t lo = 0, hi = b.n_reqs;
  const uint32_t lane = threadIdx.x & 63;
  while (hi - lo > 1) {
    const uint32_t step = (hi - lo + 63) / 64, at = lo + lane * step;
    const uint64_t below = __ballot(at < hi && b.row_off[at < hi ? at : lo] <= t);
    const uint32_t n = __popcll(below);
    if (n == 0) return b.n_reqs;
    lo += (n - 1) * step;
    hi = min(hi, lo + step);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  return b.first_row(lo) <= t && t < b.first_row(lo + 1) ? lo : b.n_reqs;
}

// Smallest scale byte that brings values up to `amax` (finite) to 448 or less.
__device__ __forceinline__ uint32_t scale_byte(float amax) {
  const uint32_t bits = __float_as_uint(amax);
  // amax = 1.m * 2^(E - 127); 448 = 1.75 * 2^8
  const int b = (int)(bits >> 23) - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0);
  return (uint32_t)max(b, (int)kScaleMin);
}
// The word that holds a head's scale byte, which starts at bit 8 * (head % 4): in
// a page the scales begin at a multiple of 64 bytes and end before its slab does.
__device__ __forceinline__ uint32_t scale_word(GlobalBytes page, uint32_t scale_off, uint32_t head) {
  return *(GlobalU32)(page + (scale_off + (head & ~3u)));
}
__device__ __forceinline__ uint32_t scale_of(uint32_t word, uint32_t head) { return word >> (8 * (head & 3)) & 0xff; }
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ float scale_inverse(uint32_t byte) { return __uint_as_float((254 - byte) << 23); }
// A page's scale byte as it is used: one that no append writes is brought into range.
__device__ __forceinline__ uint32_t scale_held(uint32_t byte) { return min(max(byte, kScaleMin), kScaleMax); }

// The device's view of a call's batch and of one layer's pages; append.hip.
void fill_batch(Batch& b, const tl_ctx* ctx, uint32_t layer, const tl_batch* batch);
void fill_pages(Pages& p, const tl_ctx* ctx, uint32_t layer, const tl_cache* c);

}  // namespace tl
