// Queries of new rows within a window (mixkv_paged_window_attention, mixkv_paged_weights): which rows a launch has, what they see, where they lie.
#pragma once
#include <algorithm>

#include "mixkv_paged.h"

namespace mixkv {

// The queries of a layer; strides in bytes.
struct WinLayer {
  const char *Q;
  int64_t qsn, qsh;
  const int32_t *start, *count;
  char *out;
  float *lse;
};
struct WinTable { PCache c[kLayersPerLaunch]; WinLayer l[kLayersPerLaunch]; };
static_assert(sizeof(WinTable) <= 3500, "kernel arguments have to fit in 4 KB");

// A row at place p sees the places j <= p with j > p - window or j < first.
struct PWindow {
  int32_t window, first;                 // both at most 2^30
  int32_t max_count, n_rows;
};

__device__ __forceinline__ bool sees(const PWindow &w, int place, int j) { return j <= place && (j > place - w.window || j < w.first); }

// What neighbouring rows of a unit see, row i being query head i % G of new row i / G: of the head's 32-row tiles those that hold the first
// rows and those of the windows.
struct View {
  int len, ng;                           // rows of the cache, rows of the group
  int i0;                                // the group's first row
  int place0, start;                     // new row 0: its place (below 0: before the head's first row), its row among the queries
  int pa, pb;                            // last places that the group's first and last row see, -1: none
  int ns, w0, tiles;                     // tiles of the first rows, first tile of the windows behind those, tiles together
  // the last place that the group's row i sees
  __device__ __forceinline__ int place(const PShape &s, int i) const { return max(place0 + (i0 + i) / s.G, -1); }
  // whether any row of the group sees place j <= len
  __device__ __forceinline__ bool any_sees(const PWindow &w, int j) const { return j <= pb && (j > pa - w.window || j < w.first); }
  // the t-th of its tiles
  __device__ __forceinline__ int tile(int t) const { return t < ns ? t : w0 + (t - ns); }
  // the group's row i, in bounds; and its number among the outputs, -1 if it is none of them
  __device__ __forceinline__ const char *query(const PShape &s, const PWindow &w, const WinLayer &l, int h, int i) const {
    const int t = (i0 + i) / s.G, g = i0 + i - t * s.G;
    const int64_t row = min(max((int64_t)start + t, (int64_t)0), (int64_t)w.n_rows - 1);
    return l.Q + row * l.qsn + (int64_t)(h * s.G + g) * l.qsh;
  }
  __device__ __forceinline__ int64_t out_row(const PShape &s, const PWindow &w, int h, int i) const {
    const int t = (i0 + i) / s.G, g = i0 + i - t * s.G;
    const int64_t row = (int64_t)start + t;
    return row >= 0 && row < w.n_rows ? row * s.hq + h * s.G + g : -1;
  }
};
// The group of up to `size` rows from row i0 of unit u on.
__device__ __forceinline__ View view_of(const PShape &s, const PWindow &w, const PCache &c, const WinLayer &l, int u, int i0, int size) {
  View v;
  const int count = max(l.count[u], 0);
  v.start = l.start[u];
  v.len = head_rows(s, c, u);
  v.i0 = i0;
  v.place0 = v.len - count;
  v.ng = min(min(count, w.max_count) * s.G - i0, size);
  v.pa = max(v.place0 + i0 / s.G, -1);
  v.pb = max(v.place0 + (i0 + max(v.ng, 1) - 1) / s.G, -1);
  v.ns = (min(w.first, v.pb + 1) + 31) >> 5;
  v.w0 = max(v.ns, max(0, v.pa - w.window + 1) >> 5);
  v.tiles = v.ns + max(0, ((v.pb + 32) >> 5) - v.w0);
  return v;
}
// The most tiles that a group of up to `size` rows can have, in heads of up to max_rows.
inline int64_t most_tiles(const PShape &s, const PWindow &w, int max_rows, int size) {
  const int64_t all = ((int64_t)max_rows + 31) / 32, span = (size + s.G - 1) / s.G + 1;
  return std::min(all, ((int64_t)w.first + 31) / 32 + (w.window + span + 62) / 32);
}

// A weighted sum over its sum of weights; no rows give zeros, a NaN stays one.
__device__ __forceinline__ float row_result(float acc, float tot) { return tot == 0.f ? 0.f : acc / tot; }
// Log-sum-exp from the offset, in exponents of 2, and the sum; no rows give -infinity.
__device__ __forceinline__ float row_lse(float offset, float tot) { return tot == 0.f ? -INFINITY : (offset + __builtin_amdgcn_logf(tot)) * 0.69314718055994530942f; }

// 1 + code / 16 for the codes i and i + 4 of a word: the code on top of the mantissa of 1.0.
__device__ __forceinline__ f16x2 code_pair(uint32_t w, int i) {
  return __builtin_bit_cast(f16x2, ((i < 2 ? w << (6 - 4 * i) : w >> (4 * i - 6)) & 0x03c003c0u) | 0x3c003c00u);
}

// 16 bytes of LDS by their address.
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
__device__ __forceinline__ u32x4 lds_vec(uint32_t at) { return *(const lds_u32x4 *)(uintptr_t)at; }
__device__ __forceinline__ void store_lds(uint32_t at, u32x4 x) { *(lds_u32x4 *)(uintptr_t)at = x; }

// Whether a word holds an infinity or a NaN, and the word with zeros in their places.
template <int DT>
__device__ __forceinline__ bool no_number(uint32_t w) {
  if constexpr (DT == MIXKV_F32) return (w & 0x7f800000u) == 0x7f800000u;
  else return (w & 0x7f800000u) == 0x7f800000u || (w & 0x7f80u) == 0x7f80u;
}
template <int DT>
__device__ __forceinline__ uint32_t numbers_only(uint32_t w) {
  if constexpr (DT == MIXKV_F32) return no_number<MIXKV_F32>(w) ? 0u : w;
  else return ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u) | ((w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu);
}

mixkv_status make_window(const PShape &s, int n_rows, int window, int first, int max_count, int max_rows, PWindow *w);
mixkv_status check_queries(const PShape &s, int eb, const mixkv_paged_queries *q, int n_layers, int64_t n_rows, bool outputs);
// Whether rows go to the kernel of prompts (mixkv_pagedprompt.hip), its workspace and its launches.
constexpr int kFewRows = 64;
inline bool many_rows(const PShape &s, int dtype, const PWindow &w) { return dtype == MIXKV_BF16 && (int64_t)w.max_count * s.G > kFewRows; }
size_t prompt_bytes(const PShape &s, const PWindow &w, int n_layers, int max_rows);
mixkv_status launch_prompt(const PShape &s, const PWindow &w, const mixkv_paged_cache *caches, const mixkv_paged_queries *queries, int n_layers, int max_rows,
                           void *workspace, hipStream_t stream);
WinTable window_table(const mixkv_paged_cache *c, const mixkv_paged_queries *q, int nl, int eb);

}  // namespace mixkv
