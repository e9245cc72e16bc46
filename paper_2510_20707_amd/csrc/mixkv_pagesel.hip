// Pages worth attending to (mixkv_paged_select): order keys of all pages' scores from their key bounds, then the best of each head.
//
// With lo and hi a page's smallest and largest keys per element, max(q_d lo_d, q_d hi_d) = max(q_d, 0) hi_d + min(q_d, 0) lo_d, so the sum
// over a group's queries is one product of 2 D elements with Q+ = sum max(q, 0) and Q- = sum min(q, 0): as cheap for 16 query heads as for
// one.  It is formed in 64 bits: the order of the sum decides the rounding to 32 bits, by which pages are ranked, only within some 2^-45 of a tie, and it is the
// same order for every page, so that equal bounds have equal scores.
#include <algorithm>

#include "mixkv_paged.h"
#include "mixkv_topsel.h"

namespace mixkv {

struct SelLayer { const void *Q; int32_t *selected, *n_selected; };
struct SelTable { PCache c[kLayersPerLaunch]; SelLayer l[kLayersPerLaunch]; };

constexpr int kSelThreads = 256, kLongThreads = 1024;

// Sums of eight doubles over aligned groups of L lanes: in every step a lane hands half of what it has to its partner and adds the partner's
// other half, so that three steps leave it one of the eight (that of index 4 (lane & 1) + (lane & 2) + (lane / 4 & 1)).
template <int N, int OFF>
__device__ __forceinline__ void scatter_step(double (&v)[8], int lane) {
  const bool up = (lane & OFF) != 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const double keep = up ? v[N + i] : v[i], give = up ? v[i] : v[N + i];
    v[i] = keep + __shfl_xor(give, OFF);
  }
}
template <int L>
__device__ __forceinline__ double scatter_sum(double (&v)[8], int lane) {
  scatter_step<4, 1>(v, lane);
  scatter_step<2, 2>(v, lane);
  scatter_step<1, 4>(v, lane);
  double x = v[0];
#pragma unroll
  for (int off = 8; off < L; off <<= 1) x += __shfl_xor(x, off);
  return x;
}

// ------------------------------------------------------------------------------------------------
// page_score_kernel: order keys of the pages' scores.  A page's bounds are 2 D neighbouring elements: L lanes take 16 bytes each and keep
// their elements of (Q-, Q+) in registers; a wave has eight times 64 / L pages in flight.
// Bound: memory in long launches; in short ones the chain of table entry, bounds, the queries (fewer than eight to a KV head are loaded and waited for one
// after another), sums (4 heads of 2048 pages: 9.3 us with the choice).
// ------------------------------------------------------------------------------------------------
template <int DT, int D>
__global__ __launch_bounds__(kSelThreads) void page_score_kernel(PShape s, SelTable tab, uint32_t *keys, int64_t unit0, int stride, int steps) {
  constexpr int EB = DT == MIXKV_BF16 ? 2 : 4, E = 16 / EB, L = 2 * D * EB / 16, PPW = 64 / L, PAGES = 8 * PPW;
  static_assert(L >= 16 && L <= 64, "a page's bounds are read by a group of lanes");
  __shared__ double qsum[2][D];                           // Q-, Q+
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, u = blockIdx.x, layer = blockIdx.z;
  const int b = u / s.hkv, h = u - b * s.hkv;
  const PCache c = tab.c[layer];
  const int64_t begin = (int64_t)blockIdx.y * steps * 4 * PAGES;
  int page0 = (int)begin + wave * PAGES;                  // the wave's first page of its first step
  // lane i: the table's entry of page i of a step, asked for a step ahead; the first one does not wait for the head's length
  auto entry_of = [&](int first) { return lane < PAGES ? c.table[(int64_t)u * s.max_pages + min(first + lane, s.max_pages - 1)] : -1; };
  int entry = entry_of(page0);
  const int len = head_rows(s, c, u), np = (len + s.P - 1) >> s.lp;
  if (begin >= np) return;
  const int part = lane % L, group = lane / L;
  u32x4 r[8];
  auto load = [&]() {
    const int page = (uint32_t)entry < (uint32_t)s.n_pages ? entry : 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = load_vec<true>(c.bounds + (int64_t)__shfl(page, j * PPW + group) * (2 * D * EB) + part * 16);
  };
  load();
  int loaded = entry;                                     // the entries of what is loaded
  entry = entry_of(page0 + 4 * PAGES);
  for (int i = tid; i < 2 * D; i += kSelThreads) {
    const int side = i / D, d = i - side * D;
    const char *q = static_cast<const char *>(tab.l[layer].Q) + ((int64_t)(b * s.hq + h * s.G) * D + d) * EB;
    double x = 0.;
#pragma unroll 8
    for (int g = 0; g < s.G; ++g) {
      float v;
      if constexpr (DT == MIXKV_BF16) v = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t *>(q + g * D * EB) << 16);
      else v = *reinterpret_cast<const float *>(q + g * D * EB);
      x += side ? fmaxf(v, 0.f) : fminf(v, 0.f);
    }
    qsum[side][d] = x;
  }
  __syncthreads();
  double q[E];
#pragma unroll
  for (int e = 0; e < E; ++e) q[e] = (&qsum[0][0])[part * E + e];
  auto bound_of = [&](int j, int e) {
    if constexpr (DT == MIXKV_BF16) return __uint_as_float(e & 1 ? r[j][e >> 1] & 0xffff0000u : r[j][e >> 1] << 16);
    else return __uint_as_float(r[j][e]);
  };
  uint32_t *out = keys + (unit0 + (int64_t)layer * s.units_per_layer + u) * stride;
  for (int st = 0; st < steps && page0 < np; ++st, page0 += 4 * PAGES) {
    double v[8], all = 0.;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = 0.;
#pragma unroll
      for (int e = 0; e < E; ++e) v[j] = fma(q[e], (double)bound_of(j, e), v[j]);
      all += v[j];
    }
    if (__builtin_amdgcn_ballot_w64(all != all) != 0) {   // an infinity that may have met a zero: such a bound counts nothing
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        asm volatile("" : "+v"(r[j]));                      // not ahead of the branch
        v[j] = 0.;
#pragma unroll
        for (int e = 0; e < E; ++e) v[j] = fma(q[e], (double)(q[e] != 0. ? bound_of(j, e) : 0.f), v[j]);
      }
    }
    const int j = 4 * (lane & 1) + (lane & 2) + ((lane >> 2) & 1), i = page0 + j * PPW + group;   // the sum that the lane is left with
    const bool there = (uint32_t)__shfl(loaded, j * PPW + group) < (uint32_t)s.n_pages;
    if (st + 1 < steps && page0 + 4 * PAGES < np) {
      load();
      loaded = entry;
      entry = entry_of(page0 + 8 * PAGES);
    }
    const float x = (float)scatter_sum<L>(v, lane);
    if (part < 8 && i < np) out[i] = order_key_u(there && x == x ? x : -INFINITY);   // (no NaN: a key of zero means none)
  }
}

// The pages of a head that are kept whatever their score: [0, first) and [np - last, np) beside `need` of those in between; false: all are kept.
__device__ __forceinline__ bool forced_pages(const PShape &s, const PCache &c, const SelLayer &L, int u, int keep, int first, int last, int *np,
                                             int threads) {
  *np = (head_rows(s, c, u) + s.P - 1) >> s.lp;
  int32_t *sel = L.selected + (int64_t)u * keep;
  if (threadIdx.x == 0) L.n_selected[u] = min(*np, keep);
  if (*np <= keep) {
    for (int i = threadIdx.x; i < keep; i += threads) sel[i] = i < *np ? i : -1;
    return false;
  }
  for (int i = threadIdx.x; i < first; i += threads) sel[i] = i;
  for (int i = threadIdx.x; i < last; i += threads) sel[keep - last + i] = *np - last + i;
  return true;
}

// ------------------------------------------------------------------------------------------------
// page_top_kernel: the best pages of a head by the threshold search of mixkv_topsel.h, a thread to EPT neighbouring pages.
// ------------------------------------------------------------------------------------------------
template <int THREADS, int EPT>
__global__ __launch_bounds__(THREADS) void page_top_kernel(PShape s, SelTable tab, const uint32_t *keys, int64_t unit0, int stride, int keep, int first,
                                                           int last) {
  __shared__ MsScratch sc;
  const int u = blockIdx.x, layer = blockIdx.z, base = threadIdx.x * EPT;
  const PCache c = tab.c[layer];
  const SelLayer L = tab.l[layer];
  const uint32_t *in = keys + (unit0 + (int64_t)layer * s.units_per_layer + u) * stride;
  u32x4 raw[EPT / 4];
#pragma unroll
  for (int e = 0; e < EPT / 4; ++e) raw[e] = reinterpret_cast<const u32x4 *>(in)[min(base / 4 + e, stride / 4 - 1)];
  int np;
  if (!forced_pages(s, c, L, u, keep, first, last, &np, THREADS) || keep == first + last) return;
  uint32_t key[EPT];
  KeyRange range;
#pragma unroll
  for (int e = 0; e < EPT; ++e) {
    const bool in_between = base + e >= first && base + e < np - last;
    key[e] = in_between ? raw[e >> 2][e & 3] : 0u;
    range.add_or_none(key[e], in_between);
  }
  thresholds_begin<THREADS>(range, sc);
  __syncthreads();
  top_select_keys<THREADS, EPT>(key, keep - first - last, L.selected + (int64_t)u * keep + first, nullptr, 0, sc, [&](int e) { return base + e; });
}

// The same for more pages than a workgroup holds in registers, counted by their key, eight bits at a time, until the key of the last
// kept one is known; pages of that key are taken from the front.
__global__ __launch_bounds__(kLongThreads) void page_top_long_kernel(PShape s, SelTable tab, const uint32_t *keys, int64_t unit0, int stride, int keep,
                                                                    int first, int last) {
  __shared__ int count[256], wsum[kLongThreads / 64][2], found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, u = blockIdx.x, layer = blockIdx.z;
  const PCache c = tab.c[layer];
  const SelLayer L = tab.l[layer];
  int np;
  if (!forced_pages(s, c, L, u, keep, first, last, &np, kLongThreads) || keep == first + last) return;
  const uint32_t *in = keys + (unit0 + (int64_t)layer * s.units_per_layer + u) * stride;
  int32_t *sel = L.selected + (int64_t)u * keep + first;
  const int a = first, z = np - last;                  // pages [a, z) compete for `need` places
  int need = keep - first - last;
  uint32_t prefix = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) count[tid] = 0;
    __syncthreads();
#pragma unroll 4
    for (int i0 = a; i0 < z; i0 += kLongThreads) {
      const uint32_t k = i0 + tid < z ? in[i0 + tid] : 0u;
      hist_add(count, (k >> shift) & 255, i0 + tid < z && (shift == 24 || k >> (shift + 8) == prefix >> (shift + 8)));
    }
    __syncthreads();
    if (wave == 0) {                                    // the bin that the last kept key is in, from above, four bins a lane
      int n[4], sum = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) { n[k] = count[255 - 4 * lane - k]; sum += n[k]; }
      int upto = sum;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const int x = __shfl_up(upto, off);
        upto += lane >= off ? x : 0;
      }
      int above = upto - sum;
      if (above < need && need <= upto) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (above < need && need <= above + n[k]) { found[0] = 255 - 4 * lane - k; found[1] = need - above; }
          above += n[k];
        }
      }
    }
    __syncthreads();
    prefix |= (uint32_t)found[0] << shift;
    need = found[1];
    __syncthreads();
  }
  int at = 0, ties = 0;                                 // need of the pages with key == prefix, and all above it
  for (int i0 = a; i0 < z; i0 += kLongThreads) {
    const uint32_t k = i0 + tid < z ? in[i0 + tid] : 0u;
    const bool tie = i0 + tid < z && k == prefix;
    const uint64_t tb = __builtin_amdgcn_ballot_w64(tie), below = ((uint64_t)1 << lane) - 1;
    if (lane == 0) wsum[wave][0] = __popcll(tb);
    __syncthreads();
    int t = ties + __popcll(tb & below), t_all = 0;
    for (int w = 0; w < kLongThreads / 64; ++w) { t_all += wsum[w][0]; if (w < wave) t += wsum[w][0]; }
    const bool take = i0 + tid < z && (k > prefix || (tie && t < need));
    ties += t_all;
    const uint64_t kb = __builtin_amdgcn_ballot_w64(take);
    if (lane == 0) wsum[wave][1] = __popcll(kb);
    __syncthreads();
    int o = at + __popcll(kb & below), o_all = 0;
    for (int w = 0; w < kLongThreads / 64; ++w) { o_all += wsum[w][1]; if (w < wave) o += wsum[w][1]; }
    if (take) sel[o] = i0 + tid;
    at += o_all;
  }
}

static int key_stride(const PShape &s) { return (s.max_pages + 3) / 4 * 4; }
static size_t select_bytes(const PShape &s, int n_layers) { return (size_t)n_layers * s.units_per_layer * key_stride(s) * 4; }

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
  if ((int64_t)max_selected * s.P > (1 << 30)) return MIXKV_ERR_INVALID_ARG;             // as mixkv_paged_attention, which takes the list
  if ((st = check_caches(caches, n_layers, false, true)) != MIXKV_OK) return st;
  if (!layers) return MIXKV_ERR_INVALID_ARG;
  for (int l = 0; l < n_layers; ++l) {
    const mixkv_paged_select_layer &d = layers[l];
    if (!d.Q || !d.selected || !d.n_selected || misaligned(d.Q, 16) || misaligned(d.selected, 4) || misaligned(d.n_selected, 4)) return MIXKV_ERR_INVALID_ARG;
  }
  if (!workspace || misaligned(workspace, 256)) return MIXKV_ERR_INVALID_ARG;
  if (workspace_bytes < select_bytes(s, n_layers)) return MIXKV_ERR_WORKSPACE_TOO_SMALL;
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  uint32_t *keys = static_cast<uint32_t *>(workspace);
  const int per = std::min(kLayersPerLaunch, ((1 << 22) - 1) / s.units_per_layer);       // of up to a thousand threads a head: fewer than 2^32 in a launch
  for (int l0 = 0; l0 < n_layers; l0 += per) {
    const int nl = std::min(n_layers - l0, per);
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
    const int stride = key_stride(s), eb = params->dtype == MIXKV_BF16 ? 2 : 4;
    // A workgroup's pages a step, and steps: the sums over the queries come before them, so that in long launches several steps share them.  us for
    // 32 sequences of up to 1024 pages, 8 heads of 128, in at least 512, 1024 and 2048 workgroups: 25.5, 24.3, 23.6.
    const int pages = 4 * 8 * (64 / (2 * s.D * eb / 16));
    const int64_t all = (s.max_pages + pages - 1) / pages;
    const int64_t least = std::max<int64_t>(all / 65535, all * units >> 23) + 1;          // at most 65535 workgroups along a head, and fewer than 2^24 in all
    const int64_t steps = std::min<int64_t>(std::max<int64_t>((all * units + 2047) / 2048, least), std::max<int64_t>(8, least));
    const dim3 grid((unsigned)s.units_per_layer, (unsigned)((all + steps - 1) / steps), (unsigned)nl), one((unsigned)s.units_per_layer, 1, (unsigned)nl);
    auto score = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(kSelThreads), 0, stream, s, t, keys, unit0, stride, (int)steps); };
    if (params->dtype == MIXKV_BF16) { if (s.D == 128) score(page_score_kernel<MIXKV_BF16, 128>); else score(page_score_kernel<MIXKV_BF16, 64>); }
    else { if (s.D == 128) score(page_score_kernel<MIXKV_F32, 128>); else score(page_score_kernel<MIXKV_F32, 64>); }
    auto top = [&](auto kern, int threads) {
      hipLaunchKernelGGL(kern, one, dim3(threads), 0, stream, s, t, (const uint32_t *)keys, unit0, stride, max_selected, keep_first, keep_last);
    };
    // The smallest workgroup that holds the pages in registers.  us for the best 64 of 1000, 4000, 16 000 pages, 4 heads: 4 pages a thread of 256 4.2, 8 of
    // 512 4.8 4.8, 16 of 1024 6.8 6.8 7.2, from memory 6.9 12.8 36.
    if (stride <= 1024) top(page_top_kernel<256, 4>, 256);
    else if (stride <= 4096) top(page_top_kernel<512, 8>, 512);
    else if (stride <= 16384) top(page_top_kernel<1024, 16>, 1024);
    else top(page_top_long_kernel, kLongThreads);
    if (hipGetLastError() != hipSuccess) return MIXKV_ERR_HIP;
  }
  return MIXKV_OK;
}
