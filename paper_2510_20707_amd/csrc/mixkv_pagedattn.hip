// Attention of one new token per sequence over the pages of its cache (mixkv_paged_attention).
//
// A head's rows are dealt to workgroups in chunks of whole 32-row tiles.  The number of chunks of a launch comes from the host's bound on
// the lengths, the chunks that a head has from its own length, so short heads of a ragged batch cost workgroups that end at once; the
// last chunk takes whatever lies beyond.  A workgroup leaves its running softmax (maximum, sum, weighted values) in the workspace
// unless its head has one chunk, and paged_merge_kernel folds the chunks in order.
#include <algorithm>

#include "mixkv_paged.h"

namespace mixkv {

struct AttnLayer { const char *Q; char *out; const int32_t *sel, *nsel; };
struct AttnTable { PCache c[kLayersPerLaunch]; AttnLayer l[kLayersPerLaunch]; };

struct AShape {
  int32_t nchunks, ctiles;     // chunks of a head in the launch, tiles of a chunk
  int32_t gchunks, gt;         // groups of up to kAttnHeads query heads, and the heads of a full one
  int32_t keep;                // entries of a head's list of selected pages, 0: all pages
};

constexpr int kAttnHeads = 16;

// Tiles of unit u, and where a tile lies: its first row in the pool as (page, row of the page), and how many of its rows exist.
__device__ __forceinline__ int head_tiles(const PShape &s, const AShape &a, const PCache &c, const AttnLayer &l, int u, int len) {
  if (a.keep == 0) return (len + 31) >> 5;
  return min(max(l.nsel[u], 0), a.keep) << (s.lp - 5);
}
struct Tile { int page, row, live; };
__device__ __forceinline__ Tile tile_at(const PShape &s, const AShape &a, const PCache &c, const AttnLayer &l, int u, int len, int t) {
  const int sub = s.lp - 5;
  int place = t >> sub;
  if (a.keep) place = l.sel[(int64_t)u * a.keep + place];
  Tile x;
  x.row = (t & ((1 << sub) - 1)) * 32;
  x.page = page_at(s, c, u, place);
  x.live = x.page < 0 ? 0 : min(max(len - ((place << s.lp) + x.row), 0), 32);   // a place with a page is one of the table
  return x;
}
// The tiles [t0, t1) of chunk `ch`.
__device__ __forceinline__ void chunk_of(const AShape &a, int tiles, int ch, int &t0, int &t1) {
  t0 = min((int64_t)tiles, (int64_t)ch * a.ctiles);
  t1 = ch == a.nchunks - 1 ? tiles : (int)min((int64_t)tiles, (int64_t)(ch + 1) * a.ctiles);
}
__device__ __forceinline__ int chunks_used(const AShape &a, int tiles) { return (int)min((int64_t)a.nchunks, ((int64_t)tiles + a.ctiles - 1) / a.ctiles); }

// ------------------------------------------------------------------------------------------------
// paged_plain_kernel: tiles of 32 rows as floats in LDS; 256 threads form the scores of up to 16 heads, then the weights, then the values.
// ------------------------------------------------------------------------------------------------
template <int DT, int D, bool Q4>
__global__ __launch_bounds__(256) void paged_plain_kernel(PShape s, AShape a, AttnTable tab, float *part, int64_t unit0) {
  constexpr int EB = DT == MIXKV_BF16 ? 2 : 4, H = kAttnHeads, NG = D / 32;
  __shared__ float kt[32][D + 1], vt[32][D], qs[H][D + 1], ws[H][33], ms[H], ls[H], fs[H];
  const int tid = threadIdx.x;
  const int ch = blockIdx.x % a.nchunks, ug = blockIdx.x / a.nchunks, gc = ug % a.gchunks, ul = ug / a.gchunks;
  const int layer = ul / s.units_per_layer, u = ul - layer * s.units_per_layer;
  const int b = u / s.hkv, h = u - b * s.hkv, ng = min(H, s.G - gc * H);
  const PCache c = tab.c[layer];
  const AttnLayer l = tab.l[layer];
  const int len = head_rows(s, c, u), tiles = head_tiles(s, a, c, l, u, len);
  int t0, t1;
  chunk_of(a, tiles, ch, t0, t1);
  if (t0 >= t1 && ch > 0) return;
  const int64_t q0 = (int64_t)b * s.hq + h * s.G + gc * H;           // first query row
  auto value = [&](const char *p, int64_t i) -> float {
    if constexpr (DT == MIXKV_BF16) return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(p)[i] << 16);
    else return reinterpret_cast<const float *>(p)[i];
  };
  for (int i = tid; i < H * D; i += 256) {
    const int g = i / D, d = i - g * D;
    qs[g][d] = g < ng ? value(l.Q, (q0 + g) * D + d) : 0.f;
  }
  if (tid < H) { ms[tid] = -INFINITY; ls[tid] = 0.f; }
  constexpr int OWN = H * D / 256;
  float o[OWN] = {};
  for (int t = t0; t < t1; ++t) {
    const Tile x = tile_at(s, a, c, l, u, len, t);
    const char *kp = c.K + (int64_t)max(x.page, 0) * s.page_bytes, *vp = c.V + (int64_t)max(x.page, 0) * s.page_bytes;
    const int64_t codes = (int64_t)s.P * D / 2;
    __syncthreads();
    for (int i = tid; i < 32 * D; i += 256) {
      const int rr = i / D, d = i - rr * D, r = x.row + rr;
      float k = 0.f, v = 0.f;
      if (rr < x.live) {
        if constexpr (Q4) {
          const int g = d >> 5, pl = D == 128 ? (g & 1) * 2 + (g >> 1) : g;
          const uint32_t kw = reinterpret_cast<const uint32_t *>(kp)[r * (D / 8) + ((d & 31) >> 3) * NG + pl];
          const uint16_t *ks = reinterpret_cast<const uint16_t *>(kp + codes) + 2 * (r * NG + pl);
          k = code_value((kw >> code_shift(d & 7)) & 15u, f16_value(ks[0]), f16_value(ks[1]));
          const int strip = (r >> 5) * 4 + ((r & 15) >> 2), e = 2 * (r & 3) + ((r >> 4) & 1);
          const uint32_t vw = reinterpret_cast<const uint32_t *>(vp)[strip * D + (d >> 6) * 64 + (d & 15) * 4 + ((d >> 4) & 3)];
          const uint16_t *vs = reinterpret_cast<const uint16_t *>(vp + codes) + (strip * NG + g) * 16 + e;
          v = code_value((vw >> code_shift(e)) & 15u, f16_value(vs[0]), f16_value(vs[8]));
        } else {
          k = value(kp, (int64_t)r * D + d);
          v = value(vp, (int64_t)r * D + d);
        }
      }
      kt[rr][d] = k; vt[rr][d] = v;
    }
    __syncthreads();
    for (int i = tid; i < H * 32; i += 256) {
      const int g = i >> 5, rr = i & 31;
      float x2 = 0.f;
      for (int d = 0; d < D; ++d) x2 = fmaf(qs[g][d], kt[rr][d], x2);
      ws[g][rr] = rr < x.live ? x2 * s.scale_log2e : -INFINITY;
    }
    __syncthreads();
    if (tid < H) {
      float m = ms[tid], sum = 0.f;
      for (int rr = 0; rr < 32; ++rr) m = fmaxf(m, ws[tid][rr]);
      const float mu = m == -INFINITY ? 0.f : m;
      for (int rr = 0; rr < 32; ++rr) {
        const float p = fast_exp2(ws[tid][rr] - mu);
        ws[tid][rr] = p;
        sum += p;
      }
      fs[tid] = fast_exp2(ms[tid] - mu);
      ls[tid] = ls[tid] * fs[tid] + sum;
      ms[tid] = m;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < OWN; ++j) {
      const int i = tid + 256 * j, g = i / D, d = i - g * D;
      float acc = o[j] * fs[g];
      for (int rr = 0; rr < 32; ++rr) acc = fmaf(ws[g][rr], vt[rr][d], acc);
      o[j] = acc;
    }
  }
  __syncthreads();
  const bool whole = chunks_used(a, tiles) <= 1;
#pragma unroll
  for (int j = 0; j < OWN; ++j) {
    const int i = tid + 256 * j, g = i / D, d = i - g * D;
    if (g >= ng) continue;
    if (!whole) {
      float *dst = part + ((((unit0 + ul) * a.gchunks + gc) * a.nchunks + ch) * a.gt + g) * (D + 2);
      dst[d] = o[j];
      if (d == 0) { dst[D] = ms[g]; dst[D + 1] = ls[g]; }
      continue;
    }
    const float res = ls[g] > 0.f ? o[j] / ls[g] : (ls[g] == 0.f ? 0.f : ls[g]);
    if constexpr (EB == 2) reinterpret_cast<uint16_t *>(l.out)[(q0 + g) * D + d] = f32_to_bf16_rne(res);
    else reinterpret_cast<float *>(l.out)[(q0 + g) * D + d] = res;
  }
}

// Folds the chunks of one (unit, group of query heads), in order: a thread per output element.
template <int DT, int D>
__global__ __launch_bounds__(256) void paged_merge_kernel(PShape s, AShape a, AttnTable tab, const float *part, int64_t unit0) {
  const int ug = blockIdx.x, gc = ug % a.gchunks, ul = ug / a.gchunks;
  const int layer = ul / s.units_per_layer, u = ul - layer * s.units_per_layer;
  const int b = u / s.hkv, h = u - b * s.hkv, ng = min(kAttnHeads, s.G - gc * kAttnHeads);
  const PCache c = tab.c[layer];
  const AttnLayer l = tab.l[layer];
  const int used = chunks_used(a, head_tiles(s, a, c, l, u, head_rows(s, c, u)));
  if (used <= 1) return;
  const int idx = blockIdx.y * 256 + threadIdx.x;
  if (idx >= ng * D) return;
  const int g = idx / D, d = idx - g * D;
  const float *src = part + (((unit0 + ul) * a.gchunks + gc) * a.nchunks * a.gt + g) * (D + 2);
  const int64_t step = (int64_t)a.gt * (D + 2);
  float m = -INFINITY;
  for (int i = 0; i < used; ++i) m = fmaxf(m, src[i * step + D]);
  const float mu = m == -INFINITY ? 0.f : m;
  float acc = 0.f, tot = 0.f;
  for (int i = 0; i < used; ++i) {
    const float f = fast_exp2(src[i * step + D] - mu);
    acc = fmaf(src[i * step + d], f, acc);
    tot = fmaf(src[i * step + D + 1], f, tot);
  }
  const float res = tot > 0.f ? acc / tot : (tot == 0.f ? 0.f : tot);
  const int64_t at = ((int64_t)b * s.hq + h * s.G + gc * kAttnHeads + g) * D + d;
  if constexpr (DT == MIXKV_BF16) reinterpret_cast<uint16_t *>(l.out)[at] = f32_to_bf16_rne(res);
  else reinterpret_cast<float *>(l.out)[at] = res;
}

// Tiles of a chunk and chunks of a head, from nothing but the arguments.
static void attn_config(const PShape &s, int n_layers, int max_rows, AShape *a) {
  a->gchunks = (s.G + kAttnHeads - 1) / kAttnHeads;
  a->gt = std::min(s.G, kAttnHeads);
  const int64_t groups = (int64_t)n_layers * s.units_per_layer * a->gchunks, tiles = ((int64_t)max_rows + 31) / 32;
  int64_t ct = (tiles * groups + 1023) / 1024;
  ct = std::max<int64_t>(8, std::min<int64_t>(ct, 256));
  a->ctiles = (int)((ct + 3) / 4 * 4);
  a->nchunks = (int)std::max<int64_t>(1, (tiles + a->ctiles - 1) / a->ctiles);
}
static size_t attn_bytes(const PShape &s, const AShape &a, int n_layers) {
  if (a.nchunks == 1) return 0;
  return (size_t)n_layers * s.units_per_layer * a.gchunks * a.nchunks * a.gt * (s.D + 2) * sizeof(float);
}
static int clamp_rows(const PShape &s, int max_rows) { return std::min(max_rows, s.max_pages * s.P); }

}  // namespace mixkv

extern "C" mixkv_status mixkv_paged_attention_workspace_size(const mixkv_paged_params *params, int32_t n_layers, int32_t max_rows, size_t *bytes) {
  using namespace mixkv;
  PShape s;
  const mixkv_status st = make_pshape(params, &s);
  if (st != MIXKV_OK) return st;
  if (!bytes || n_layers < 1 || n_layers > MIXKV_MAX_LAYERS || max_rows < 1) return MIXKV_ERR_INVALID_ARG;
  AShape a{};
  attn_config(s, n_layers, clamp_rows(s, max_rows), &a);
  *bytes = (attn_bytes(s, a, n_layers) + 255) / 256 * 256;
  return MIXKV_OK;
}

extern "C" mixkv_status mixkv_paged_attention(const mixkv_paged_params *params, const mixkv_paged_cache *caches, const mixkv_paged_attention_layer *layers,
                                              int32_t n_layers, int32_t max_selected, int32_t max_rows, void *workspace, size_t workspace_bytes,
                                              void *hip_stream) {
  using namespace mixkv;
  PShape s;
  mixkv_status st = make_pshape(params, &s);
  if (st != MIXKV_OK) return st;
  if (max_rows < 1) return MIXKV_ERR_INVALID_ARG;
  if ((st = check_caches(params, caches, n_layers, true, false)) != MIXKV_OK) return st;
  if (!layers) return MIXKV_ERR_INVALID_ARG;
  const bool sparse = layers[0].selected != nullptr;
  if (sparse && (max_selected < 1 || (int64_t)max_selected * s.P > (1 << 30))) return MIXKV_ERR_INVALID_ARG;
  for (int l = 0; l < n_layers; ++l) {
    const mixkv_paged_attention_layer &d = layers[l];
    if (!d.Q || !d.out || misaligned(d.Q, 16) || misaligned(d.out, 16)) return MIXKV_ERR_INVALID_ARG;
    if ((d.selected != nullptr) != sparse || (d.n_selected != nullptr) != sparse) return MIXKV_ERR_INVALID_ARG;
    if (misaligned(d.selected, 4) || misaligned(d.n_selected, 4)) return MIXKV_ERR_INVALID_ARG;
  }
  AShape a{};
  attn_config(s, n_layers, clamp_rows(s, max_rows), &a);
  a.keep = sparse ? max_selected : 0;
  if ((int64_t)std::min(n_layers, kLayersPerLaunch) * s.units_per_layer * a.gchunks * a.nchunks >= (1 << 24)) return MIXKV_ERR_UNSUPPORTED;
  const size_t need = attn_bytes(s, a, n_layers);
  if (need > 0) {
    if (!workspace || misaligned(workspace, 256)) return MIXKV_ERR_INVALID_ARG;
    if (workspace_bytes < need) return MIXKV_ERR_WORKSPACE_TOO_SMALL;
  }
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  float *part = static_cast<float *>(workspace);
  for (int l0 = 0; l0 < n_layers; l0 += kLayersPerLaunch) {
    const int nl = n_layers - l0 < kLayersPerLaunch ? n_layers - l0 : kLayersPerLaunch;
    AttnTable t;
    for (int l = 0; l < kLayersPerLaunch; ++l) {
      t.c[l] = PCache{};
      t.l[l] = AttnLayer{};
      if (l >= nl) continue;
      const mixkv_paged_cache &c = caches[l0 + l];
      const mixkv_paged_attention_layer &d = layers[l0 + l];
      t.c[l] = PCache{static_cast<char *>(c.K_pages), static_cast<char *>(c.V_pages), nullptr, c.page_table, c.lengths};
      t.l[l] = AttnLayer{static_cast<const char *>(d.Q), static_cast<char *>(d.out), d.selected, d.n_selected};
    }
    const int64_t groups = (int64_t)nl * s.units_per_layer * a.gchunks, unit0 = (int64_t)l0 * s.units_per_layer;
    auto go = [&](auto kern, auto merge) {
      hipLaunchKernelGGL(kern, dim3((unsigned)(groups * a.nchunks)), dim3(256), 0, stream, s, a, t, part, unit0);
      if (a.nchunks > 1)
        hipLaunchKernelGGL(merge, dim3((unsigned)groups, (unsigned)((a.gt * s.D + 255) / 256)), dim3(256), 0, stream, s, a, t, (const float *)part, unit0);
    };
    constexpr int B16 = MIXKV_BF16, F32 = MIXKV_F32;
    if (s.q4) { if (s.D == 128) go(paged_plain_kernel<B16, 128, true>, paged_merge_kernel<B16, 128>); else go(paged_plain_kernel<B16, 64, true>, paged_merge_kernel<B16, 64>); }
    else if (params->dtype == B16) { if (s.D == 128) go(paged_plain_kernel<B16, 128, false>, paged_merge_kernel<B16, 128>); else go(paged_plain_kernel<B16, 64, false>, paged_merge_kernel<B16, 64>); }
    else { if (s.D == 128) go(paged_plain_kernel<F32, 128, false>, paged_merge_kernel<F32, 128>); else go(paged_plain_kernel<F32, 64, false>, paged_merge_kernel<F32, 64>); }
    if (hipGetLastError() != hipSuccess) return MIXKV_ERR_HIP;
  }
  return MIXKV_OK;
}
