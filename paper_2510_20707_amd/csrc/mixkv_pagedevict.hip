// Eviction by accumulated attention weight (mixkv_paged_evict): the places that a head keeps, then its rows into the pages of another table.
#include <algorithm>

#include "mixkv_pagedrow.h"
#include "mixkv_topsel.h"

namespace mixkv {

struct EvictLayer {
  const float *weights;
  float *into;
  const int32_t *keep;
  int32_t *kept, *n_kept;
  char *K, *V, *bounds;                   // the pools and the table that the rows go to
  const int32_t *table;
};
constexpr int kEvictLayers = 24;          // pointer-table entries of a launch
struct EvictTable { PCache c[kEvictLayers]; EvictLayer l[kEvictLayers]; };
static_assert(sizeof(EvictTable) <= 3072, "kernel arguments have to fit in 4 KB");

struct EvictShape { int32_t max_keep, first, last; };

constexpr int kRankThreads = 1024, kMoveThreads = 256;

// The order key of row i of a head of `len` rows: 0 if it does not exist.
__device__ __forceinline__ uint32_t row_key(const PShape &s, const EvictShape &e, const PCache &c, const EvictLayer &l, int u, int len, int i) {
  const int id = page_at(s, c, u, i >> s.lp);
  if (id < 0) return 0u;
  if (i < e.first || i >= len - e.last) return order_key_u(INFINITY);
  const float x = l.weights[((int64_t)id << s.lp) + (i & (s.P - 1))];
  return order_key_u(x == x ? x : -INFINITY);
}

// ------------------------------------------------------------------------------------------------
// evict_rank_kernel: a workgroup to a head.  Rows are counted by their key, eight bits at a time, until the key of the last kept one is known;
// rows of that key are taken from the front.
// ------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(kRankThreads) void evict_rank_kernel(PShape s, EvictShape ev, EvictTable tab) {
  __shared__ int count[256], wsum[kRankThreads / 64][2], found[2], exist;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, u = blockIdx.x, layer = blockIdx.z;
  const PCache c = tab.c[layer];
  const EvictLayer l = tab.l[layer];
  const int len = head_rows(s, c, u);
  int32_t *kept = l.kept + (int64_t)u * ev.max_keep;
  if (tid == 0) exist = 0;
  __syncthreads();
  int mine = 0;
  for (int i = tid; i < len; i += kRankThreads) mine += page_at(s, c, u, i >> s.lp) >= 0 ? 1 : 0;
  mine = wave_reduce<WSum>(mine, 0);
  if (lane == 0) atomicAdd(&exist, mine);
  __syncthreads();
  const int keep = min(min(max(l.keep[u], 0), ev.max_keep), exist);
  if (tid == 0) l.n_kept[u] = keep;
  for (int i = keep + tid; i < ev.max_keep; i += kRankThreads) kept[i] = -1;
  if (keep == 0) return;                                // uniform
  int need = keep;
  uint32_t prefix = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) count[tid] = 0;
    __syncthreads();
    for (int i0 = 0; i0 < len; i0 += kRankThreads) {
      const uint32_t k = i0 + tid < len ? row_key(s, ev, c, l, u, len, i0 + tid) : 0u;
      hist_add(count, (k >> shift) & 255, k != 0 && (shift == 24 || k >> (shift + 8) == prefix >> (shift + 8)));
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
  int at = 0, ties = 0;                                 // need of the rows with key == prefix, and all above it
  for (int i0 = 0; i0 < len; i0 += kRankThreads) {
    const uint32_t k = i0 + tid < len ? row_key(s, ev, c, l, u, len, i0 + tid) : 0u;
    const bool tie = k == prefix;                       // (no key that is wanted is 0)
    const uint64_t tb = __builtin_amdgcn_ballot_w64(tie), below = ((uint64_t)1 << lane) - 1;
    if (lane == 0) wsum[wave][0] = __popcll(tb);
    __syncthreads();
    int t = ties + __popcll(tb & below), t_all = 0;
    for (int w = 0; w < kRankThreads / 64; ++w) { t_all += wsum[w][0]; if (w < wave) t += wsum[w][0]; }
    const bool take = k > prefix || (tie && t < need);
    ties += t_all;
    const uint64_t kb = __builtin_amdgcn_ballot_w64(take);
    if (lane == 0) wsum[wave][1] = __popcll(kb);
    __syncthreads();
    int o = at + __popcll(kb & below), o_all = 0;
    for (int w = 0; w < kRankThreads / 64; ++w) { o_all += wsum[w][1]; if (w < wave) o += wsum[w][1]; }
    if (take && o < keep) kept[o] = i0 + tid;
    at += o_all;
  }
}

// ------------------------------------------------------------------------------------------------
// evict_move_kernel: a workgroup to a page of `into`, D/16 lanes to a row.
// ------------------------------------------------------------------------------------------------
template <int DT, int D, bool Q4>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(PShape s, EvictShape ev, EvictTable tab) {
  constexpr int EB = DT == MIXKV_BF16 ? 2 : 4, LPR = D / 16, RS = kMoveThreads / LPR, RB = D * EB, RUNS = D / 8;
  __shared__ uint32_t words[Q4 ? RS * RUNS : 1];           // codes of the value rows of a pass, a word per eight elements
  __shared__ __align__(16) char red[4][2 * RB];
  const int tid = threadIdx.x, j = tid % LPR, slot = tid / LPR, u = blockIdx.x, layer = blockIdx.z;
  const PCache c = tab.c[layer];
  const EvictLayer l = tab.l[layer];
  const PCache to{l.K, l.V, l.bounds, l.table, nullptr};
  const int32_t *kept = l.kept + (int64_t)u * ev.max_keep;
  const int n = l.n_kept[u];
  for (int pg = blockIdx.y; (int64_t)pg << s.lp < n; pg += gridDim.y) {
    const int id = page_at(s, to, u, pg);
    if (id < 0) continue;                                  // uniform
    const int first = pg << s.lp, rows = min(n - first, s.P);
    char *kp = to.K + (int64_t)id * s.page_bytes, *vp = to.V + (int64_t)id * s.page_bytes;
    RunRange<DT> ra, rb;
    ra.none(); rb.none();
    for (int s0 = 0; s0 < rows; s0 += RS) {
      const int r = s0 + slot;
      const bool live = r < rows;
      const int i = live ? kept[first + r] : 0, from = page_at(s, c, u, i >> s.lp), fr = i & (s.P - 1);
      const bool there = live && from >= 0;                // (rows of no page are never kept)
      const char *ks = c.K + (int64_t)max(from, 0) * s.page_bytes, *vs = c.V + (int64_t)max(from, 0) * s.page_bytes;
      Run<DT> ka{}, kb{};
      if constexpr (!Q4) {
        if (there) {
          const int64_t src = (int64_t)fr * RB + 8 * EB * j, dst = (int64_t)r * RB + 8 * EB * j;
          Run<DT> va, vb;
          ka.load(ks + src); kb.load(ks + src + RB / 2);
          va.load(vs + src); vb.load(vs + src + RB / 2);
          ka.store(kp + dst); kb.store(kp + dst + RB / 2);
          va.store(vp + dst); vb.store(vp + dst + RB / 2);
        }
      } else {
        if (there) {
          const Place4<D> a(j, fr, s.P), z(j, r, s.P);
          char *ksm = const_cast<char *>(ks), *vsm = const_cast<char *>(vs);
          const u32x2 kw = *a.key_words(ksm), sc = *a.key_scales(ksm);
          *z.key_words(kp) = kw;
          if ((j & 3) == 0) *z.key_scales(kp) = sc;
          if (c.bounds) {
            float x0[8], x1[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              x0[e] = code_value((kw[0] >> code_shift(e)) & 15u, f16_value(sc[0] & 0xffffu), f16_value(sc[0] >> 16));
              x1[e] = code_value((kw[1] >> code_shift(e)) & 15u, f16_value(sc[1] & 0xffffu), f16_value(sc[1] >> 16));
            }
            ka.set(x0); kb.set(x1);
          }
          if ((j & 3) == 0) {
            const uint16_t *p0 = a.value_scale(vsm, a.ga()), *p1 = a.value_scale(vsm, a.gb());
            uint16_t *q0 = z.value_scale(vp, z.ga()), *q1 = z.value_scale(vp, z.gb());
            q0[0] = p0[0]; q0[8] = p0[8];
            q1[0] = p1[0]; q1[8] = p1[8];
          }
          const uint32_t *strip = a.strip_words(vsm), sh = code_shift(a.e);
          uint32_t w0 = 0, w1 = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            w0 |= ((strip[Place4<D>::word_of(8 * j + e)] >> sh) & 15u) << code_shift(e);
            w1 |= ((strip[Place4<D>::word_of(D / 2 + 8 * j + e)] >> sh) & 15u) << code_shift(e);
          }
          words[slot * RUNS + j] = w0;
          words[slot * RUNS + LPR + j] = w1;
        }
        __syncthreads();
        store_strips<D, RS, kMoveThreads>(vp, words, s0, 0, rows);
        __syncthreads();
      }
      if (there) {
        if (c.bounds && to.bounds) { ra.add(ka); rb.add(kb); }
        if (l.into && j == 0) l.into[((int64_t)id << s.lp) + r] = l.weights[((int64_t)from << s.lp) + fr];
      }
    }
    if (c.bounds && to.bounds) store_bounds<DT, D>(to.bounds + (int64_t)id * 2 * RB, ra, rb, red, false);   // uniform
  }
}

}  // namespace mixkv

extern "C" mixkv_status mixkv_paged_evict_workspace_size(const mixkv_paged_params *params, int32_t n_layers, int32_t max_rows, size_t *bytes) {
  using namespace mixkv;
  PShape s;
  const mixkv_status st = make_pshape(params, &s);
  if (st != MIXKV_OK) return st;
  if (!bytes || n_layers < 1 || n_layers > MIXKV_MAX_LAYERS || max_rows < 1) return MIXKV_ERR_INVALID_ARG;
  *bytes = 0;
  return MIXKV_OK;
}

extern "C" mixkv_status mixkv_paged_evict(const mixkv_paged_params *params, const mixkv_paged_cache *caches, const mixkv_paged_cache *into,
                                          const mixkv_paged_evict_layer *layers, int32_t n_layers, int32_t max_keep, int32_t keep_first, int32_t keep_last,
                                          int32_t max_rows, void *workspace, size_t workspace_bytes, void *hip_stream) {
  using namespace mixkv;
  (void)workspace; (void)workspace_bytes;
  PShape s;
  mixkv_status st = make_pshape(params, &s);
  if (st != MIXKV_OK) return st;
  if (max_keep < 1 || keep_first < 0 || keep_last < 0 || max_rows < 1) return MIXKV_ERR_INVALID_ARG;
  if (max_keep > s.max_pages * s.P) return MIXKV_ERR_INVALID_ARG;
  if ((st = check_caches(caches, n_layers, true, false)) != MIXKV_OK) return st;
  if (!into || !layers) return MIXKV_ERR_INVALID_ARG;
  for (int l = 0; l < n_layers; ++l) {
    const mixkv_paged_cache &t = into[l];
    const mixkv_paged_evict_layer &d = layers[l];
    if (!t.K_pages || !t.V_pages || t.K_pages == t.V_pages || misaligned(t.K_pages, 16) || misaligned(t.V_pages, 16) || misaligned(t.K_bounds, 16)) return MIXKV_ERR_INVALID_ARG;
    if (!t.page_table || misaligned(t.page_table, 4) || t.page_table == caches[l].page_table) return MIXKV_ERR_INVALID_ARG;
    if (!d.weights || !d.keep || !d.kept || !d.n_kept) return MIXKV_ERR_INVALID_ARG;
    if (misaligned(d.weights, 4) || misaligned(d.weights_into, 4) || misaligned(d.keep, 4) || misaligned(d.kept, 4) || misaligned(d.n_kept, 4)) return MIXKV_ERR_INVALID_ARG;
    if (d.n_kept == caches[l].lengths || d.n_kept == d.keep) return MIXKV_ERR_INVALID_ARG;
  }
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  const EvictShape ev{max_keep, keep_first, keep_last};
  for (int l0 = 0; l0 < n_layers; l0 += kEvictLayers) {
    const int nl = std::min(n_layers - l0, kEvictLayers);
    EvictTable t;
    for (int l = 0; l < kEvictLayers; ++l) {
      t.c[l] = PCache{};
      t.l[l] = EvictLayer{};
      if (l >= nl) continue;
      const mixkv_paged_cache &c = caches[l0 + l], &z = into[l0 + l];
      const mixkv_paged_evict_layer &d = layers[l0 + l];
      t.c[l] = PCache{static_cast<char *>(c.K_pages), static_cast<char *>(c.V_pages), static_cast<char *>(c.K_bounds), c.page_table, c.lengths};
      t.l[l] = EvictLayer{d.weights, d.weights_into, d.keep, d.kept, d.n_kept, static_cast<char *>(z.K_pages), static_cast<char *>(z.V_pages),
                          static_cast<char *>(z.K_bounds), z.page_table};
    }
    const dim3 heads((unsigned)s.units_per_layer, 1, (unsigned)nl);
    hipLaunchKernelGGL(evict_rank_kernel, heads, dim3(kRankThreads), 0, stream, s, ev, t);
    // a workgroup to a page, fewer than 2^32 threads
    const int64_t pages = ((int64_t)max_keep + s.P - 1) / s.P, most = std::max<int64_t>(1, std::min<int64_t>(65535, ((int64_t)1 << 23) / ((int64_t)s.units_per_layer * nl)));
    const dim3 grid((unsigned)s.units_per_layer, (unsigned)std::min(pages, most), (unsigned)nl);
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(kMoveThreads), 0, stream, s, ev, t); };
    if (s.q4) { if (s.D == 128) go(evict_move_kernel<MIXKV_BF16, 128, true>); else go(evict_move_kernel<MIXKV_BF16, 64, true>); }
    else if (params->dtype == MIXKV_BF16) { if (s.D == 128) go(evict_move_kernel<MIXKV_BF16, 128, false>); else go(evict_move_kernel<MIXKV_BF16, 64, false>); }
    else { if (s.D == 128) go(evict_move_kernel<MIXKV_F32, 128, false>); else go(evict_move_kernel<MIXKV_F32, 64, false>); }
    if (hipGetLastError() != hipSuccess) return MIXKV_ERR_HIP;
  }
  return MIXKV_OK;
}
