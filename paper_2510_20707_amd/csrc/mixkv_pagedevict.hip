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

// The order key of a row's weight: the first and the last rows are infinite, NaN ranks last.  (0 is left for rows that do not exist.)
__device__ __forceinline__ uint32_t weight_key(const EvictShape &e, int len, int i, float x) {
  return order_key_u(i < e.first || i >= len - e.last ? INFINITY : (x == x ? x : -INFINITY));
}
// The keys of four neighbouring rows (of one page) from row i on, a multiple of four.
__device__ __forceinline__ u32x4 four_keys(const EvictShape &e, int len, int i, int id, f32x4 w) {
  u32x4 k;
#pragma unroll
  for (int j = 0; j < 4; ++j) k[j] = id >= 0 && i + j < len ? weight_key(e, len, i + j, w[j]) : 0u;
  return k;
}
// The places of a head that are kept: how many, and what lies behind them in the list.
__device__ __forceinline__ int kept_rows(const EvictShape &e, const EvictLayer &l, int u, int exist, int32_t *kept, int threads) {
  const int keep = min(min(max(l.keep[u], 0), e.max_keep), exist);
  if (threadIdx.x == 0) l.n_kept[u] = keep;
  for (int i = keep + threadIdx.x; i < e.max_keep; i += threads) kept[i] = -1;
  return keep;
}

// ------------------------------------------------------------------------------------------------
// evict_rank_kernel: a workgroup to a head, its rows' keys in registers, a thread to EPT neighbouring ones; the best by the threshold search of mixkv_topsel.h.
// ------------------------------------------------------------------------------------------------
template <int THREADS, int EPT>
__global__ __launch_bounds__(THREADS) void evict_rank_kernel(PShape s, EvictShape ev, EvictTable tab) {
  __shared__ MsScratch sc;
  __shared__ int exist_s[THREADS / 64];
  const int tid = threadIdx.x, u = blockIdx.x, layer = blockIdx.z, base = tid * EPT;
  const PCache c = tab.c[layer];
  const EvictLayer l = tab.l[layer];
  const int id = page_at(s, c, u, base >> s.lp);           // (of all of the thread's rows)
  const float *w = l.weights + ((int64_t)max(id, 0) << s.lp) + (base & (s.P - 1));
  f32x4 raw[EPT / 4];
#pragma unroll
  for (int e = 0; e < EPT / 4; ++e) raw[e] = reinterpret_cast<const f32x4 *>(w)[e];
  const int len = head_rows(s, c, u);
  uint32_t key[EPT];
  KeyRange range;
  int mine = 0;
#pragma unroll
  for (int e = 0; e < EPT; e += 4) {
    const u32x4 k = four_keys(ev, len, base + e, id, raw[e / 4]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      key[e + j] = k[j];
      mine += k[j] != 0 ? 1 : 0;
      range.add_or_none(k[j], k[j] != 0);
    }
  }
  thresholds_begin<THREADS>(range, sc);
  mine = wave_reduce<WSum>(mine, 0);
  if ((tid & 63) == 0) exist_s[tid >> 6] = mine;
  __syncthreads();
  int exist = 0;
#pragma unroll
  for (int i = 0; i < THREADS / 64; ++i) exist += exist_s[i];
  int32_t *kept = l.kept + (int64_t)u * ev.max_keep;
  const int keep = kept_rows(ev, l, u, exist, kept, THREADS);
  if (keep == 0) return;                                // uniform
  top_select_keys<THREADS, EPT>(key, keep, kept, nullptr, 0, sc, [&](int e) { return base + e; });
}

// ------------------------------------------------------------------------------------------------
// Longer heads.  evict_keys_kernel writes their keys one after another, in as many workgroups as there is work for; evict_long_kernel, a workgroup to a head,
// counts them by eleven bits, eleven, and ten until the key of the last kept one is known, and lists the kept ones: each wave has a range of rows of its own, so that
// one fold over the waves gives all of them their places.
// ------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void evict_keys_kernel(PShape s, EvictShape ev, EvictTable tab, uint32_t *keys, int64_t stride) {
  const int u = blockIdx.x, layer = blockIdx.z;
  const PCache c = tab.c[layer];
  const EvictLayer l = tab.l[layer];
  const int len = head_rows(s, c, u);
  uint32_t *out = keys + (layer * (int64_t)s.units_per_layer + u) * stride;
  for (int64_t i = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 4; i < len; i += (int64_t)gridDim.y * 1024) {
    const int id = page_at(s, c, u, (int)i >> s.lp);
    const f32x4 w = *reinterpret_cast<const f32x4 *>(l.weights + ((int64_t)max(id, 0) << s.lp) + ((int)i & (s.P - 1)));
    *reinterpret_cast<u32x4 *>(out + i) = four_keys(ev, len, (int)i, id, w);
  }
}

constexpr int kLongBins = 2048, kLongWaves = kRankThreads / 64;

__global__ __launch_bounds__(kRankThreads) void evict_long_kernel(PShape s, EvictShape ev, EvictTable tab, const uint32_t *keys, int64_t stride) {
  __shared__ int hist[kLongBins], wsum[kLongWaves][2], found[2], total;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, u = blockIdx.x, layer = blockIdx.z;
  const PCache c = tab.c[layer];
  const EvictLayer l = tab.l[layer];
  const uint32_t *in = keys + (layer * (int64_t)s.units_per_layer + u) * stride;
  const int len = head_rows(s, c, u);
  int32_t *kept = l.kept + (int64_t)u * ev.max_keep;
  constexpr int U = 8;                                  // 16-byte loads of a thread under way
  // every key of the workgroup's, 4 a thread and turn
  auto each = [&](auto &&f) {
    for (int i0 = 0; i0 < len; i0 += 4 * U * kRankThreads) {
      u32x4 k[U];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int i = i0 + (j * kRankThreads + tid) * 4;
        k[j] = i < len ? *reinterpret_cast<const u32x4 *>(in + i) : u32x4{0u, 0u, 0u, 0u};
      }
#pragma unroll
      for (int j = 0; j < U; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) f(k[j][e]);
    }
  };
  // The bin that the need-th largest counted key is in, and how many of that bin are needed; `found` holds the bin and the keys above it.
  auto find = [&](int need) {
    const int hi = kLongBins - 1 - 2 * tid, a = hist[hi], b = hist[hi - 1];        // from above
    int wtot;
    const int inc = wave_scan_incl_add(a + b, &wtot);
    if (lane == 0) wsum[wave][0] = wtot;
    __syncthreads();
    int excl = inc - a - b, all = 0;
#pragma unroll
    for (int w = 0; w < kLongWaves; ++w) { excl += w < wave ? wsum[w][0] : 0; all += wsum[w][0]; }
    if (tid == 0) total = all;
    if (excl < need && need <= excl + a) { found[0] = hi; found[1] = excl; }
    else if (excl + a < need && need <= excl + a + b) { found[0] = hi - 1; found[1] = excl + a; }
    __syncthreads();
  };
  auto clear = [&]() {
    hist[tid] = 0;
    hist[tid + kRankThreads] = 0;
    __syncthreads();
  };
  clear();
  each([&](uint32_t k) { hist_add(hist, (int)(k >> 21), k != 0); });
  __syncthreads();
  find(0);
  const int keep = kept_rows(ev, l, u, total, kept, kRankThreads);
  if (keep == 0) return;                                // uniform
  find(keep);
  uint32_t prefix = (uint32_t)found[0] << 21;
  int need = keep - found[1];
#pragma unroll 1
  for (int shift = 10; shift >= 0; shift -= 10) {       // bits 20 ... 10, then 9 ... 0
    const int upper = shift == 10 ? 21 : 10;
    const uint32_t mask = shift == 10 ? 2047u : 1023u;
    __syncthreads();
    clear();
    each([&](uint32_t k) { hist_add(hist, (int)((k >> shift) & mask), k >> upper == prefix >> upper && k != 0); });
    __syncthreads();
    find(need);
    prefix |= (uint32_t)found[0] << shift;
    need -= found[1];
  }
  // ---- the keys above `prefix`, and the first `need` that are it: a wave's range of rows, 64 at a time, counted and then listed
  const int per = ((len + kLongWaves - 1) / kLongWaves + 63) / 64 * 64, r0 = min(wave * per, len), r1 = min(r0 + per, len);
  auto rows = [&](auto &&f) {
    constexpr int V = 16;
    for (int i0 = r0; i0 < r1; i0 += 64 * V) {
      uint32_t k[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int i = i0 + 64 * j + lane;
        k[j] = i < r1 ? in[i] : 0u;
      }
#pragma unroll
      for (int j = 0; j < V; ++j) f(k[j], i0 + 64 * j + lane);
    }
  };
  int above = 0, ties = 0;
  rows([&](uint32_t k, int) { above += __popcll(__builtin_amdgcn_ballot_w64(k > prefix)); ties += __popcll(__builtin_amdgcn_ballot_w64(k == prefix)); });
  __syncthreads();
  if (lane == 0) { wsum[wave][0] = above; wsum[wave][1] = ties; }
  __syncthreads();
  int at = 0, before = 0;
#pragma unroll
  for (int w = 0; w < kLongWaves; ++w) {
    if (w < wave) { at += wsum[w][0]; before += wsum[w][1]; }
  }
  at += min(before, need);
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  rows([&](uint32_t k, int i) {
    const uint64_t tb = __builtin_amdgcn_ballot_w64(k == prefix);
    const bool take = k > prefix || (k == prefix && before + __popcll(tb & below) < need);
    before += __popcll(tb);
    const uint64_t kb = __builtin_amdgcn_ballot_w64(take);
    const int o = at + __popcll(kb & below);
    if (take && o < keep) kept[o] = i;
    at += __popcll(kb);
  });
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

// Heads that a workgroup holds in registers; longer ones' keys lie in the workspace, a head's one after another.  (The rule goes by the page table's width: a head
// can be as long as that, whatever the host thinks.)
constexpr int kRankRows = 16384;
static int64_t key_stride(const PShape &s) { return (int64_t)s.max_pages * s.P; }
static size_t evict_bytes(const PShape &s, int n_layers, int max_rows) {
  (void)max_rows;
  return key_stride(s) <= kRankRows ? 0 : (size_t)std::min(n_layers, kEvictLayers) * s.units_per_layer * key_stride(s) * sizeof(uint32_t);
}

}  // namespace mixkv

extern "C" mixkv_status mixkv_paged_evict_workspace_size(const mixkv_paged_params *params, int32_t n_layers, int32_t max_rows, size_t *bytes) {
  using namespace mixkv;
  PShape s;
  const mixkv_status st = make_pshape(params, &s);
  if (st != MIXKV_OK) return st;
  if (!bytes || n_layers < 1 || n_layers > MIXKV_MAX_LAYERS || max_rows < 1) return MIXKV_ERR_INVALID_ARG;
  *bytes = (evict_bytes(s, n_layers, max_rows) + 255) / 256 * 256;
  return MIXKV_OK;
}

extern "C" mixkv_status mixkv_paged_evict(const mixkv_paged_params *params, const mixkv_paged_cache *caches, const mixkv_paged_cache *into,
                                          const mixkv_paged_evict_layer *layers, int32_t n_layers, int32_t max_keep, int32_t keep_first, int32_t keep_last,
                                          int32_t max_rows, void *workspace, size_t workspace_bytes, void *hip_stream) {
  using namespace mixkv;
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
    if (misaligned(d.weights, 16) || misaligned(d.weights_into, 4) || misaligned(d.keep, 4) || misaligned(d.kept, 4) || misaligned(d.n_kept, 4)) return MIXKV_ERR_INVALID_ARG;
    if (d.n_kept == caches[l].lengths || d.n_kept == d.keep) return MIXKV_ERR_INVALID_ARG;
  }
  const size_t need = evict_bytes(s, n_layers, max_rows);
  if (need > 0) {
    if (!workspace || misaligned(workspace, 256)) return MIXKV_ERR_INVALID_ARG;
    if (workspace_bytes < need) return MIXKV_ERR_WORKSPACE_TOO_SMALL;
  }
  uint32_t *keys = static_cast<uint32_t *>(workspace);
  const int64_t stride = key_stride(s);
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
    // fewer than 2^32 threads
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(65535, ((int64_t)1 << 23) / ((int64_t)s.units_per_layer * nl)));
    auto rank = [&](auto kern, int threads) { hipLaunchKernelGGL(kern, heads, dim3((unsigned)threads), 0, stream, s, ev, t); };
    if (stride <= 1024) rank(evict_rank_kernel<256, 4>, 256);
    else if (stride <= 4096) rank(evict_rank_kernel<512, 8>, 512);
    else if (stride <= kRankRows) rank(evict_rank_kernel<1024, 16>, 1024);
    else {
      const int64_t y = std::min(most, std::max<int64_t>(1, ((int64_t)std::min<int64_t>(max_rows, stride) + 1023) / 1024));
      hipLaunchKernelGGL(evict_keys_kernel, dim3((unsigned)s.units_per_layer, (unsigned)y, (unsigned)nl), dim3(256), 0, stream, s, ev, t, keys, stride);
      hipLaunchKernelGGL(evict_long_kernel, heads, dim3(kRankThreads), 0, stream, s, ev, t, (const uint32_t *)keys, stride);
    }
    const int64_t pages = ((int64_t)max_keep + s.P - 1) / s.P;
    const dim3 grid((unsigned)s.units_per_layer, (unsigned)std::min(pages, most), (unsigned)nl);
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(kMoveThreads), 0, stream, s, ev, t); };
    if (s.q4) { if (s.D == 128) go(evict_move_kernel<MIXKV_BF16, 128, true>); else go(evict_move_kernel<MIXKV_BF16, 64, true>); }
    else if (params->dtype == MIXKV_BF16) { if (s.D == 128) go(evict_move_kernel<MIXKV_BF16, 128, false>); else go(evict_move_kernel<MIXKV_BF16, 64, false>); }
    else { if (s.D == 128) go(evict_move_kernel<MIXKV_F32, 128, false>); else go(evict_move_kernel<MIXKV_F32, 64, false>); }
    if (hipGetLastError() != hipSuccess) return MIXKV_ERR_HIP;
  }
  return MIXKV_OK;
}
