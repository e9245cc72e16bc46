// Pages worth attending to (mixkv_paged_select): scores of all pages from their key bounds, then the best of each head.
//
// With lo and hi a page's smallest and largest keys per element, max(q_d lo_d, q_d hi_d) = max(q_d, 0) hi_d + min(q_d, 0) lo_d, so the sum
// over a group's queries is one product of 2 D elements with Q+ = sum max(q, 0) and Q- = sum min(q, 0): as cheap for 16 query heads as for
// one.  It is formed in 64 bits, where the rounding to 32 bits that the pages are ranked by does not depend on the order of the sum.
#include "mixkv_paged.h"

namespace mixkv {

struct SelLayer { const void *Q; int32_t *selected, *n_selected; };
struct SelTable { PCache c[kLayersPerLaunch]; SelLayer l[kLayersPerLaunch]; };

constexpr int kSelThreads = 256;

// Order of the scores as unsigned numbers; the zeros are one.
__device__ __forceinline__ uint32_t score_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

template <int DT>
__device__ __forceinline__ double element_of(const void *p, int64_t i) {
  if constexpr (DT == MIXKV_BF16) return __uint_as_float((uint32_t)static_cast<const uint16_t *>(p)[i] << 16);
  else return static_cast<const float *>(p)[i];
}

// One workgroup per (layer, sequence, KV head) and worker; a wave per page.
template <int DT, int D>
__global__ __launch_bounds__(kSelThreads) void page_score_kernel(PShape s, SelTable tab, uint32_t *keys, int64_t unit0) {
  __shared__ double up[D], down[D];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int layer = blockIdx.x / s.units_per_layer, u = blockIdx.x - layer * s.units_per_layer;
  const int b = u / s.hkv, h = u - b * s.hkv;
  const PCache c = tab.c[layer];
  const int np = (head_rows(s, c, u) + s.P - 1) >> s.lp;
  for (int d = tid; d < D; d += kSelThreads) {
    double p = 0., m = 0.;
    for (int g = 0; g < s.G; ++g) {
      const double q = element_of<DT>(tab.l[layer].Q, (int64_t)(b * s.hq + h * s.G + g) * D + d);
      p += q > 0. ? q : 0.;
      m += q < 0. ? q : 0.;
    }
    up[d] = p; down[d] = m;
  }
  __syncthreads();
  uint32_t *out = keys + (unit0 + blockIdx.x) * s.max_pages;
  for (int i = blockIdx.y * 4 + wave; i < np; i += gridDim.y * 4) {
    const int id = page_at(s, c, u, i);
    double x = 0.;
    if (id >= 0)
      for (int d = lane; d < D; d += 64)
        x += (up[d] != 0. ? up[d] * element_of<DT>(c.bounds, ((int64_t)id * 2 + 1) * D + d) : 0.) +
             (down[d] != 0. ? down[d] * element_of<DT>(c.bounds, (int64_t)id * 2 * D + d) : 0.);
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) x += __shfl_xor(x, off);
    if (lane == 0) out[i] = id >= 0 ? score_key((float)x) : 0u;
  }
}

// The best `keep` pages of a head: the pages in between the forced ones are counted by their key, eight bits at a time, until the
// key of the last kept one is known; pages of that key are taken from the front.
__global__ __launch_bounds__(kSelThreads) void page_top_kernel(PShape s, SelTable tab, const uint32_t *keys, int64_t unit0, int keep, int first, int last) {
  __shared__ int count[256], wsum[4][2], found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int layer = blockIdx.x / s.units_per_layer, u = blockIdx.x - layer * s.units_per_layer;
  const PCache c = tab.c[layer];
  const SelLayer L = tab.l[layer];
  int32_t *sel = L.selected + (int64_t)u * keep;
  const int np = (head_rows(s, c, u) + s.P - 1) >> s.lp, kept = min(np, keep);
  if (tid == 0) L.n_selected[u] = kept;
  if (np <= keep) {
    for (int i = tid; i < keep; i += kSelThreads) sel[i] = i < np ? i : -1;
    return;
  }
  const uint32_t *in = keys + (unit0 + blockIdx.x) * s.max_pages;
  const int a = first, z = np - last;                  // pages [a, z) compete for `need` places
  int need = keep - first - last;
  uint32_t prefix = 0;
  for (int shift = 24; shift >= 0 && need > 0; shift -= 8) {
    for (int i = tid; i < 256; i += kSelThreads) count[i] = 0;
    __syncthreads();
    for (int i = a + tid; i < z; i += kSelThreads) {
      const uint32_t k = in[i];
      if (shift == 24 || k >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&count[(k >> shift) & 255], 1);
    }
    __syncthreads();
    if (tid == 0) {
      int above = 0, v = 255;
      while (above + count[v] < need) above += count[v--];
      found[0] = v; found[1] = need - above;
    }
    __syncthreads();
    prefix |= (uint32_t)found[0] << shift;
    need = found[1];
    __syncthreads();
  }
  // need of the pages with key == prefix, and all above it
  const bool any = keep > first + last;
  int at = 0, ties = 0;
  for (int i0 = 0; i0 < np; i0 += kSelThreads) {
    const int i = i0 + tid;
    bool take = i < np && (i < a || i >= z), tie = false;
    if (!take && i < np && any) {
      const uint32_t k = in[i];
      take = k > prefix;
      tie = k == prefix;
    }
    const uint64_t tb = __builtin_amdgcn_ballot_w64(tie), below = ((uint64_t)1 << lane) - 1;
    if (lane == 0) wsum[wave][0] = __popcll(tb);
    __syncthreads();
    int t = ties + __popcll(tb & below), t_all = 0;
    for (int w = 0; w < 4; ++w) { t_all += wsum[w][0]; if (w < wave) t += wsum[w][0]; }
    take |= tie && t < need;
    ties += t_all;
    const uint64_t kb = __builtin_amdgcn_ballot_w64(take);
    if (lane == 0) wsum[wave][1] = __popcll(kb);
    __syncthreads();
    int o = at + __popcll(kb & below), o_all = 0;
    for (int w = 0; w < 4; ++w) { o_all += wsum[w][1]; if (w < wave) o += wsum[w][1]; }
    if (take) sel[o] = i;
    at += o_all;
  }
}

static size_t select_bytes(const PShape &s, int n_layers) { return (size_t)n_layers * s.units_per_layer * s.max_pages * 4; }

}  // namespace mixkv

extern "C" mixkv_status mixkv_paged_select_workspace_size(const mixkv_paged_params *params, int32_t n_layers, size_t *bytes) {
  using namespace mixkv;
  PShape s;
  const mixkv_status st = make_pshape(params, &s);
  if (st != MIXKV_OK) return st;
  if (!bytes || n_layers < 1 || n_layers > MIXKV_MAX_LAYERS) return MIXKV_ERR_INVALID_ARG;
  *bytes = (select_bytes(s, n_layers) + 255) / 256 * 256;
  return MIXKV_OK;
}

extern "C" mixkv_status mixkv_paged_select(const mixkv_paged_params *params, const mixkv_paged_cache *caches, const mixkv_paged_select_layer *layers,
                                           int32_t n_layers, int32_t max_selected, int32_t keep_first, int32_t keep_last, void *workspace,
                                           size_t workspace_bytes, void *hip_stream) {
  using namespace mixkv;
  PShape s;
  mixkv_status st = make_pshape(params, &s);
  if (st != MIXKV_OK) return st;
  if (max_selected < 1 || keep_first < 0 || keep_last < 0 || (int64_t)keep_first + keep_last > max_selected) return MIXKV_ERR_INVALID_ARG;
  if ((st = check_caches(params, caches, n_layers, false, true)) != MIXKV_OK) return st;
  if (!layers) return MIXKV_ERR_INVALID_ARG;
  for (int l = 0; l < n_layers; ++l) {
    const mixkv_paged_select_layer &d = layers[l];
    if (!d.Q || !d.selected || !d.n_selected || misaligned(d.Q, 16) || misaligned(d.selected, 4) || misaligned(d.n_selected, 4)) return MIXKV_ERR_INVALID_ARG;
  }
  if (!workspace || misaligned(workspace, 256)) return MIXKV_ERR_INVALID_ARG;
  if (workspace_bytes < select_bytes(s, n_layers)) return MIXKV_ERR_WORKSPACE_TOO_SMALL;
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  uint32_t *keys = static_cast<uint32_t *>(workspace);
  for (int l0 = 0; l0 < n_layers; l0 += kLayersPerLaunch) {
    const int nl = n_layers - l0 < kLayersPerLaunch ? n_layers - l0 : kLayersPerLaunch;
    SelTable t;
    for (int l = 0; l < kLayersPerLaunch; ++l) {
      t.c[l] = PCache{};
      t.l[l] = SelLayer{};
      if (l >= nl) continue;
      const mixkv_paged_cache &c = caches[l0 + l];
      t.c[l] = PCache{nullptr, nullptr, static_cast<char *>(c.K_bounds), c.page_table, c.lengths};
      t.l[l] = SelLayer{layers[l0 + l].Q, layers[l0 + l].selected, layers[l0 + l].n_selected};
    }
    const int64_t units = (int64_t)nl * s.units_per_layer, unit0 = (int64_t)l0 * s.units_per_layer;
    int64_t w = (s.max_pages + 15) / 16, most = 8192 / units < 1 ? 1 : 8192 / units;
    if (w > most) w = most;
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3((unsigned)units, (unsigned)w), dim3(kSelThreads), 0, stream, s, t, keys, unit0); };
    if (params->dtype == MIXKV_BF16) { if (s.D == 128) go(page_score_kernel<MIXKV_BF16, 128>); else go(page_score_kernel<MIXKV_BF16, 64>); }
    else { if (s.D == 128) go(page_score_kernel<MIXKV_F32, 128>); else go(page_score_kernel<MIXKV_F32, 64>); }
    hipLaunchKernelGGL(page_top_kernel, dim3((unsigned)units), dim3(kSelThreads), 0, stream, s, t, (const uint32_t *)keys, unit0, max_selected, keep_first,
                       keep_last);
    if (hipGetLastError() != hipSuccess) return MIXKV_ERR_HIP;
  }
  return MIXKV_OK;
}
