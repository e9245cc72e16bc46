// What the kernels of the paged cache share: shapes, per-layer pointers, where things lie in a page, and how an index that the
// device holds becomes an address that is in bounds.
#pragma once
#include "mixkv_stream.h"

namespace mixkv {

// Problem shape, identical for every layer of a call.
struct PShape {
  int32_t batch, hq, hkv, G, D, P, lp;   // lp: log2 of the rows of a page
  int32_t max_pages, n_pages;
  int32_t units_per_layer;               // batch * hkv
  int32_t q4;                            // pages hold 4-bit codes
  int64_t page_bytes;
  float scale_log2e;
};

struct PCache {
  char *K, *V;
  char *bounds;
  const int32_t *table, *lengths;
};

// A 4-bit page: the codes (rows * D / 2 bytes), then a step and a base, fp16 each, for every 32 elements (include/mixkv.h).
__host__ __device__ constexpr int64_t page_bytes_of(bool q4, int dtype, int P, int D) {
  return q4 ? (int64_t)P * D / 2 + (int64_t)P * (D / 32) * 4 : (int64_t)P * D * (dtype == MIXKV_BF16 ? 2 : 4);
}

mixkv_status make_pshape(const mixkv_paged_params *p, PShape *s);
mixkv_status check_caches(const mixkv_paged_cache *c, int n_layers, bool pages, bool bounds);
inline bool misaligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
// Dense rows with strides n (rows) and h (heads) in elements of eb bytes: whether the strides are none, the bytes from the first to the last.
inline bool bad_row_strides(const PShape &s, int eb, int64_t n_rows, int64_t n, int64_t h) {
  return n < s.D || h < 0 || n > INT64_MAX / 16 / (n_rows + 1) || h > (INT64_MAX >> 30) || (n * eb) % 16 || (h * eb) % 16;
}
inline uint64_t row_span(const PShape &s, int eb, int64_t n_rows, int64_t n, int64_t h, int heads) { return (uint64_t)((n_rows - 1) * n + (heads - 1) * h + s.D) * eb; }
inline bool regions_overlap(const void *a, uint64_t na, const void *b, uint64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

// Rows of unit u (sequence, head) of a layer.
__device__ __forceinline__ int head_rows(const PShape &s, const PCache &c, int u) {
  return min(max(c.lengths[u], 0), s.max_pages << s.lp);
}
// The page of place `i` of unit u's table, -1 if there is none.
__device__ __forceinline__ int page_at(const PShape &s, const PCache &c, int u, int i) {
  if ((uint32_t)i >= (uint32_t)s.max_pages) return -1;
  const int id = c.table[(int64_t)u * s.max_pages + i];
  return (uint32_t)id < (uint32_t)s.n_pages ? id : -1;
}

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// The unit of the workgroup number x + units * turn, x < units.  Workgroups go to the chip's eight dies in turn by their number, so a
// multiple of eight units would leave each of a unit's workgroups to one die, and units are of unequal length: the units move on with the turns.
__device__ __forceinline__ int dealt_unit(int x, int turn, int units) { return (int)(((uint32_t)x + (uint32_t)turn + ((uint32_t)turn >> 1)) % (uint32_t)units); }

__device__ __forceinline__ float f16_value(uint32_t bits) { return (float)__builtin_bit_cast(_Float16, (uint16_t)bits); }
__device__ __forceinline__ uint32_t f16_bits(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
// Bit position of element e of a word of eight codes.
__host__ __device__ constexpr int code_shift(int e) { return 4 * ((e >> 1) + 4 * (e & 1)); }
// The element that a code stands for: 1 + code / 16 is exact, its product with an fp16 too.
__device__ __forceinline__ float code_value(uint32_t code, float step, float base) { return fmaf(step, 1.f + (float)code * 0.0625f, base); }

}  // namespace mixkv
