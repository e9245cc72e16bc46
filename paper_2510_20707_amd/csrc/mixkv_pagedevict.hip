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
static_assert(sizeof(EvictTable) <= 3500, "kernel arguments have to fit in 4 KB");

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
__device__ __forceinline__ int kept_rows(const EvictShape &e, const EvictLayer &l, int u, int budget, int exist, int32_t *kept, int threads) {
  const int keep = min(min(max(budget, 0), e.max_keep), exist);
  if (threadIdx.x == 0) l.n_kept[u] = keep;
  for (int i = keep + threadIdx.x; i < e.max_keep; i += threads) kept[i] = -1;
  return keep;
}

// A head that is longer than the host said, by one workgroup from memory: its keys counted by eleven bits, eleven, and ten until the key of the last kept one is known, and then
// listed.  A wave has a range of rows of its own, so that one fold over the waves gives all of them their places.
constexpr int kLongBins = 2048;
struct LongScratch { int hist[kLongBins], wsum[kMsMaxWaves][2], found[2], total; };

template <int THREADS>
__device__ __forceinline__ void rank_long(const PShape &s, const PCache &c, const EvictShape &ev, const EvictLayer &l, int u, int len, int budget, LongScratch &sc) {
  constexpr int W = THREADS / 64, BPT = kLongBins / THREADS, U = 8;   // U: groups of four rows of a thread under way
  auto keys_at = [&](int i, bool there) {                             // of the rows i ... i + 3, i a multiple of four; 0 where !there
    const int at = page_at(s, c, u, i >> s.lp);
    const f32x4 x = *reinterpret_cast<const f32x4 *>(l.weights + ((int64_t)max(at, 0) << s.lp) + (i & (s.P - 1)));
    return four_keys(ev, len, i, there ? at : -1, x);
  };
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int32_t *kept = l.kept + (int64_t)u * ev.max_keep;
  // every key, 4 a thread and turn
  auto each = [&](auto &&f) {
    for (int i0 = 0; i0 < len; i0 += 4 * U * THREADS) {
      u32x4 k[U];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int i = i0 + (j * THREADS + tid) * 4;
        k[j] = keys_at(min(i, (len - 1) & ~3), i < len);
      }
#pragma unroll
      for (int j = 0; j < U; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) f(k[j][e]);
    }
  };
  // The bin that the need-th largest counted key is in, and the keys above it, to `found`; all that were counted to `total`.
  auto find = [&](int need) {
    int n[BPT], sum = 0;                                // bins from above
#pragma unroll
    for (int b = 0; b < BPT; ++b) {
      n[b] = sc.hist[kLongBins - 1 - tid * BPT - b];
      sum += n[b];
    }
    int wtot;
    const int inc = wave_scan_incl_add(sum, &wtot);
    if (lane == 0) sc.wsum[wave][0] = wtot;
    __syncthreads();
    int excl = inc - sum, all = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) { excl += w < wave ? sc.wsum[w][0] : 0; all += sc.wsum[w][0]; }
    if (tid == 0) sc.total = all;
#pragma unroll
    for (int b = 0; b < BPT; ++b) {
      if (excl < need && need <= excl + n[b]) { sc.found[0] = kLongBins - 1 - tid * BPT - b; sc.found[1] = excl; }
      excl += n[b];
    }
    __syncthreads();
  };
  auto clear = [&]() {
    for (int i = tid; i < kLongBins; i += THREADS) sc.hist[i] = 0;
    __syncthreads();
  };
  clear();
  each([&](uint32_t k) { if (k != 0) atomicAdd(&sc.hist[k >> 21], 1); });
  __syncthreads();
  find(0);
  const int keep = kept_rows(ev, l, u, budget, sc.total, kept, THREADS);
  if (keep == 0) return;                                // uniform
  find(keep);
  uint32_t prefix = (uint32_t)sc.found[0] << 21;
  int need = keep - sc.found[1];
#pragma unroll 1
  for (int shift = 10; shift >= 0; shift -= 10) {       // bits 20 ... 10, then 9 ... 0
    const int upper = shift == 10 ? 21 : 10;
    const uint32_t mask = shift == 10 ? 2047u : 1023u;
    __syncthreads();
    clear();
    each([&](uint32_t k) { if (k >> upper == prefix >> upper && k != 0) atomicAdd(&sc.hist[(k >> shift) & mask], 1); });
    __syncthreads();
    find(need);
    prefix |= (uint32_t)sc.found[0] << shift;
    need -= sc.found[1];
  }
  // ---- the keys above `prefix`, and the first `need` that are it: a wave's range of rows, 256 at a time, counted and then listed
  const int per = ((len + W - 1) / W + 255) / 256 * 256, r0 = min(wave * per, len), r1 = min(r0 + per, len);
  auto rows = [&](auto &&f) {
    constexpr int V = 4;
    for (int i0 = r0; i0 < r1; i0 += 256 * V) {
      u32x4 k[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int i = i0 + 256 * j + 4 * lane;
        k[j] = keys_at(min(i, (len - 1) & ~3), i < r1);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) f(k[j], i0 + 256 * j + 4 * lane);
    }
  };
  int above = 0, ties = 0;                              // the lane's
  rows([&](const u32x4 &k, int) {
#pragma unroll
    for (int e = 0; e < 4; ++e) { above += k[e] > prefix ? 1 : 0; ties += k[e] == prefix ? 1 : 0; }
  });
  above = wave_reduce<WSum>(above, 0);
  ties = wave_reduce<WSum>(ties, 0);
  __syncthreads();
  if (lane == 0) { sc.wsum[wave][0] = above; sc.wsum[wave][1] = ties; }
  __syncthreads();
  int at = 0, before = 0;                               // kept rows, and rows of the last key, in front of the wave's next ones
#pragma unroll
  for (int w = 0; w < W; ++w)
    if (w < wave) { at += sc.wsum[w][0]; before += sc.wsum[w][1]; }
  at += min(before, need);
  rows([&](const u32x4 &k, int i) {
    int a = 0, t = 0, wa, wt;
#pragma unroll
    for (int e = 0; e < 4; ++e) { a += k[e] > prefix ? 1 : 0; t += k[e] == prefix ? 1 : 0; }
    const int ia = wave_scan_incl_add(a, &wa), it = wave_scan_incl_add(t, &wt);
    int tie = before + it - t, o = at + (ia - a) + (min(tie, need) - min(before, need));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool last = k[e] == prefix, take = k[e] > prefix || (last && tie < need);
      tie += last ? 1 : 0;
      if (take && o < keep) kept[o] = i + e;
      o += take ? 1 : 0;
    }
    at += wa + (min(before + wt, need) - min(before, need));
    before += wt;
  });
}

// ------------------------------------------------------------------------------------------------
// evict_rank_kernel: a workgroup to a head, its rows' keys in registers, a thread to EPT neighbouring ones; the best by the threshold search of mixkv_topsel.h.  Heads that
// are longer than the host said are counted from memory.
// Bound: the search's barriers.  4 heads of 2112 rows 9 us (512 threads), 256 heads of up to 16 384 25 us (1024).
// ------------------------------------------------------------------------------------------------
template <int THREADS, int EPT>
__global__ __launch_bounds__(THREADS) void evict_rank_kernel(PShape s, EvictShape ev, EvictTable tab) {
  __shared__ union { MsScratch ms; LongScratch lg; } sc;
  __shared__ int exist_s[THREADS / 64];
  const int tid = threadIdx.x, u = blockIdx.x, layer = blockIdx.z, base = tid * EPT;
  const PCache c = tab.c[layer];
  const EvictLayer l = tab.l[layer];
  const int id = page_at(s, c, u, base >> s.lp);           // (of all of the thread's rows)
  const int len = head_rows(s, c, u), budget = l.keep[u];
  const float *w = l.weights + ((int64_t)max(id, 0) << s.lp) + (base & (s.P - 1));
  f32x4 raw[EPT / 4];
#pragma unroll
  for (int e = 0; e < EPT / 4; ++e) raw[e] = reinterpret_cast<const f32x4 *>(w)[e];
  if (len > THREADS * EPT) {
    rank_long<THREADS>(s, c, ev, l, u, len, budget, sc.lg);
    return;
  }
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
  thresholds_begin<THREADS>(range, sc.ms);
  mine = wave_reduce<WSum>(mine, 0);
  if ((tid & 63) == 0) exist_s[tid >> 6] = mine;
  __syncthreads();
  int exist = 0;
#pragma unroll
  for (int i = 0; i < THREADS / 64; ++i) exist += exist_s[i];
  int32_t *kept = l.kept + (int64_t)u * ev.max_keep;
  const int keep = kept_rows(ev, l, u, budget, exist, kept, THREADS);
  if (keep == 0) return;                                // uniform
  top_select_keys<THREADS, EPT>(key, keep, kept, nullptr, 0, sc.ms, [&](int e) { return base + e; });
}

// ------------------------------------------------------------------------------------------------
// Longer heads, a workgroup to a segment of one.  evict_count_kernel<0> writes the segment's keys one after another and counts them by their upper eleven bits.
// evict_count_kernel<1> adds up the counts of the head's segments, finds the eleven bits of the last kept key, and counts the keys that have them by the next eleven; <2> likewise by
// the last ten.  evict_list_kernel then knows that key, and how many keys above it and how many like it lie in earlier segments, and lists its own.  Each launch reads what the one
// before wrote, and nothing is added up by atomics in memory.
// Bound: latency, of four launches: 8 heads of 60 000 to 131 072 rows 5.5 + 6.8 + 6.7 + 8.2 us.  A workgroup to a head took 83 us for the same: one compute unit's loads and LDS counts.
// ------------------------------------------------------------------------------------------------
constexpr int kSegRows = 8192, kMostSegs = 32, kCopies = 4;   // kCopies: of a workgroup's counts, because keys of one head often agree in their leading bits
struct LongPlan {
  uint32_t *keys;                          // [head][stride]
  int *counts;                             // [head][2][segs][kLongBins]: the first and the third level, the second
  int4 *states;                            // [head][segs]: the last kept key's bits so far, keys to keep of those that have them, keys above them in earlier segments, keys to keep
  int64_t stride;
  int32_t segs, seg;                       // seg: rows of a segment
};
struct FoldScratch { int wsum[kMsMaxWaves], above[kMsMaxWaves], found[3]; };
struct Fold { int bin, above, above_before, in_before; };   // keys in higher bins, and in this one: of all segments, of those in front of `seg`

// The bin that the need_of(all counted keys)-th largest key is in.
template <class NeedOf>
__device__ __forceinline__ Fold fold_counts(const int *counts, int n_seg, int seg, FoldScratch &sc, NeedOf &&need_of) {
  constexpr int G = 8;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, low = kLongBins - 2 - 2 * tid;   // the thread's bins: low + 1, low
  static_assert(kLongBins == 2 * kRankThreads, "two bins a thread");
  int all[2] = {0, 0}, before[2] = {0, 0};
  for (int g = 0; g < n_seg; g += G) {
    int2 v[G];
#pragma unroll
    for (int k = 0; k < G; ++k) v[k] = *reinterpret_cast<const int2 *>(counts + min(g + k, n_seg - 1) * kLongBins + low);
#pragma unroll
    for (int k = 0; k < G; ++k) {
      const int a = g + k < n_seg ? v[k].y : 0, b = g + k < n_seg ? v[k].x : 0;
      all[0] += a; all[1] += b;
      before[0] += g + k < seg ? a : 0; before[1] += g + k < seg ? b : 0;
    }
  }
  int wtot;
  const int sum = all[0] + all[1], inc = wave_scan_incl_add(sum, &wtot);
  if (lane == 0) sc.wsum[wave] = wtot;
  __syncthreads();
  int excl = inc - sum, total = 0;
#pragma unroll
  for (int w = 0; w < kRankThreads / 64; ++w) { excl += w < wave ? sc.wsum[w] : 0; total += sc.wsum[w]; }
  const int need = need_of(total);
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    if (excl < need && need <= excl + all[b]) { sc.found[0] = low + 1 - b; sc.found[1] = excl; sc.found[2] = before[b]; }
    excl += all[b];
  }
  if (need <= 0) return Fold{0, 0, 0, 0};                     // uniform
  __syncthreads();
  Fold f{sc.found[0], sc.found[1], 0, sc.found[2]};
  const int above = wave_reduce<WSum>((low + 1 > f.bin ? before[0] : 0) + (low > f.bin ? before[1] : 0), 0);
  if (lane == 0) sc.above[wave] = above;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kRankThreads / 64; ++w) f.above_before += sc.above[w];
  return f;
}

template <int LEVEL>
__global__ __launch_bounds__(kRankThreads) void evict_count_kernel(PShape s, EvictShape ev, EvictTable tab, LongPlan p) {
  __shared__ int hist[kLongBins * kCopies];
  __shared__ FoldScratch sc;
  const int tid = threadIdx.x, copy = tid & (kCopies - 1), u = blockIdx.x, seg = blockIdx.y, layer = blockIdx.z;
  const PCache c = tab.c[layer];
  const EvictLayer l = tab.l[layer];
  const int len = head_rows(s, c, u);
  const int64_t head = layer * (int64_t)s.units_per_layer + u, r0 = (int64_t)seg * p.seg, r1 = min(r0 + p.seg, (int64_t)len);
  if (len > p.stride || (seg > 0 && r0 >= len)) return;       // (an empty head: the first segment counts nothing)
  uint32_t *keys = p.keys + head * p.stride;
  int *counts = p.counts + head * 2 * p.segs * kLongBins;
  const int n_seg = max(1, (int)(((int64_t)len + p.seg - 1) / p.seg));
  for (int i = tid; i < kLongBins * kCopies; i += kRankThreads) hist[i] = 0;
  uint32_t prefix = 0;
  if constexpr (LEVEL == 1) {
    const int budget = l.keep[u];
    int keep = 0;
    const Fold f = fold_counts(counts, n_seg, seg, sc, [&](int total) { return keep = min(min(max(budget, 0), ev.max_keep), total); });
    prefix = (uint32_t)f.bin << 21;
    if (tid == 0) p.states[head * p.segs + seg] = int4{(int)prefix, keep - f.above, f.above_before, keep};
    if (keep == 0) return;                                    // uniform
  } else if constexpr (LEVEL == 2) {
    const int4 st = p.states[head * p.segs + seg];
    if (st.w == 0) return;                                    // uniform
    const Fold f = fold_counts(counts + p.segs * kLongBins, n_seg, seg, sc, [&](int) { return st.y; });
    prefix = (uint32_t)st.x | (uint32_t)f.bin << 10;
    if (tid == 0) p.states[head * p.segs + seg] = int4{(int)prefix, st.y - f.above, st.z + f.above_before, st.w};   // (each thread has read it: fold_counts has barriers)
  }
  __syncthreads();
  for (int64_t i0 = r0 + 4 * tid; i0 < r1; i0 += 8 * kRankThreads) {
    u32x4 k[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t i = i0 + h * 4 * kRankThreads;
      k[h] = u32x4{0u, 0u, 0u, 0u};
      if (i >= r1) continue;
      if constexpr (LEVEL == 0) {
        const int id = page_at(s, c, u, (int)i >> s.lp);
        const f32x4 w = *reinterpret_cast<const f32x4 *>(l.weights + ((int64_t)max(id, 0) << s.lp) + ((int)i & (s.P - 1)));
        k[h] = four_keys(ev, len, (int)i, id, w);
        *reinterpret_cast<u32x4 *>(keys + i) = k[h];
      } else k[h] = *reinterpret_cast<const u32x4 *>(keys + i);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t x = k[h][e];
        if constexpr (LEVEL == 0) { if (x != 0) atomicAdd(&hist[(x >> 21) * kCopies + copy], 1); }
        if constexpr (LEVEL == 1) { if (x != 0 && x >> 21 == prefix >> 21) atomicAdd(&hist[((x >> 10) & 2047u) * kCopies + copy], 1); }
        if constexpr (LEVEL == 2) { if (x != 0 && x >> 10 == prefix >> 10) atomicAdd(&hist[(x & 1023u) * kCopies + copy], 1); }
      }
  }
  __syncthreads();
  for (int b = tid; b < kLongBins; b += kRankThreads) {
    int n = 0;
#pragma unroll
    for (int k = 0; k < kCopies; ++k) n += hist[b * kCopies + k];
    counts[((LEVEL & 1) * p.segs + seg) * kLongBins + b] = n;      // (the last level takes the first one's place, which nobody reads any more)
  }
}

__global__ __launch_bounds__(kRankThreads) void evict_list_kernel(PShape s, EvictShape ev, EvictTable tab, LongPlan p) {
  __shared__ union { FoldScratch fold; LongScratch lg; int wsum[kMsMaxWaves][2]; } sc;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, u = blockIdx.x, seg = blockIdx.y, layer = blockIdx.z;
  const PCache c = tab.c[layer];
  const EvictLayer l = tab.l[layer];
  const int len = head_rows(s, c, u);
  const int64_t head = layer * (int64_t)s.units_per_layer + u, r0 = (int64_t)seg * p.seg, r1 = min(r0 + p.seg, (int64_t)len);
  if (seg > 0 && r0 >= len) return;
  if (len > p.stride) {
    if (seg == 0) rank_long<kRankThreads>(s, c, ev, l, u, len, l.keep[u], sc.lg);
    return;
  }
  const uint32_t *keys = p.keys + head * p.stride;
  const int4 st = p.states[head * p.segs + seg];
  int32_t *kept = l.kept + (int64_t)u * ev.max_keep;
  if (seg == 0) kept_rows(ev, l, u, st.w, st.w, kept, kRankThreads);
  if (st.w == 0) return;                                      // uniform
  const int n_seg = (int)(((int64_t)len + p.seg - 1) / p.seg);
  const Fold f = fold_counts(p.counts + head * 2 * p.segs * kLongBins, n_seg, seg, sc.fold, [&](int) { return st.y; });
  const uint32_t last = (uint32_t)st.x | (uint32_t)f.bin;     // the last kept key; the first `need` that are it stay
  const int need = st.y - f.above, keep = st.w;
  int above = st.z + f.above_before, ties = f.in_before;      // in front of the turn's rows
  for (int64_t t0 = r0; t0 < r1; t0 += 8 * kRankThreads) {
    const int64_t i = t0 + 8 * tid;
    uint32_t k[8];
    int a = 0, t = 0, wa, wt;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const u32x4 x = i + 4 * h < r1 ? *reinterpret_cast<const u32x4 *>(keys + i + 4 * h) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        k[4 * h + e] = x[e];
        a += x[e] > last ? 1 : 0;
        t += x[e] == last ? 1 : 0;
      }
    }
    const int ia = wave_scan_incl_add(a, &wa), it = wave_scan_incl_add(t, &wt);
    __syncthreads();
    if (lane == 0) { sc.wsum[wave][0] = wa; sc.wsum[wave][1] = wt; }
    __syncthreads();
    int oa = above + ia - a, ot = ties + it - t;
#pragma unroll
    for (int w = 0; w < kRankThreads / 64; ++w) {
      const int na = sc.wsum[w][0], nt = sc.wsum[w][1];
      above += na; ties += nt;
      oa += w < wave ? na : 0; ot += w < wave ? nt : 0;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool like = k[e] == last;
      if (k[e] > last || (like && ot < need)) {
        const int o = oa + min(ot, need);
        if (o < keep) kept[o] = (int32_t)(i + e);
      }
      oa += k[e] > last ? 1 : 0;
      ot += like ? 1 : 0;
    }
  }
}

// ------------------------------------------------------------------------------------------------
// evict_move_kernel: every second workgroup of a head moves keys (with their bounds and weights), the others values, 128 rows of `into` a turn, a wave 32 of them, D/16 lanes to a row.
// The chain of loads behind a row (its place, that place's page, the row) is walked one turn ahead.
// 4-bit values: a strip of `into` holds eight rows, which come from up to eight strips.  A lane takes 16 bytes of the strip, four elements of all eight rows, out of the same 16
// bytes of theirs.
// Bound: 4 bits: neither memory nor the vector unit alone (codes to values for the bounds, codes from strip to strip): 256 heads, 2.4e6 rows, of which 1.2e6 stay, 0.55 GB with the lines that hold
// rows of both kinds in 167 us, 3.3 TB/s (a large copy 5.1), the vector unit 46 % busy, the waves waiting 65 % of their time; keys alone 83, values alone 92, and loads a further turn ahead change nothing.
// With one row of a lane under way, and the bounds by butterflies over whole workgroups, 300.  bf16: memory: 8 heads, 1.0e5 rows stay, 104 MB in 31 us.
// ------------------------------------------------------------------------------------------------
// The smallest and the largest elements of 32 rows of every wave, D/16 lanes to a row, to the bounds of their page, whose rows `waves` neighbouring waves (1, 2 or 4) have.  The lanes
// share the words of a row's two ends out by halves: with the lane 32, 16, ... away each gives the half that the other one keeps.
__device__ __forceinline__ uint32_t least_of(const RunRange<MIXKV_BF16> &, uint32_t a, uint32_t b) {
  typedef RunRange<MIXKV_BF16>::s16x2 P;
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(P, a), __builtin_bit_cast(P, b)));
}
__device__ __forceinline__ uint32_t least_of(const RunRange<MIXKV_F32> &, uint32_t a, uint32_t b) { return __float_as_uint(fminf(__uint_as_float(a), __uint_as_float(b))); }

template <int DT, int D>
__device__ __forceinline__ void store_page_bounds(char *dst, bool there, int waves, const RunRange<DT> &ra, const RunRange<DT> &rb, char (&red)[4][2 * D * (DT == MIXKV_BF16 ? 2 : 4)]) {
  constexpr int EB = DT == MIXKV_BF16 ? 2 : 4, LPR = D / 16, RB = D * EB, NW = 8 * EB;   // NW: words of a lane's two runs and two ends
  constexpr uint32_t other = DT == MIXKV_BF16 ? 0xffffffffu : 0x80000000u;               // (largest elements as smallest ones of the other sign)
  const int lane = threadIdx.x & 63;
  uint32_t w[NW];
  constexpr int Q = NW / 4;
#pragma unroll
  for (int i = 0; i < Q; ++i) {
    if constexpr (DT == MIXKV_BF16) {
      w[i] = __builtin_bit_cast(uint32_t, ra.lo[i]); w[Q + i] = __builtin_bit_cast(uint32_t, rb.lo[i]);
      w[2 * Q + i] = __builtin_bit_cast(uint32_t, ra.hi[i]) ^ other; w[3 * Q + i] = __builtin_bit_cast(uint32_t, rb.hi[i]) ^ other;
    } else {
      w[i] = __float_as_uint(ra.lo[i]); w[Q + i] = __float_as_uint(rb.lo[i]);
      w[2 * Q + i] = __float_as_uint(ra.hi[i]) ^ other; w[3 * Q + i] = __float_as_uint(rb.hi[i]) ^ other;
    }
  }
#pragma unroll
  for (int st = 0; 32 >> st >= LPR; ++st) {
    const bool up = lane & (32 >> st);
    constexpr int half = NW / 2;
#pragma unroll
    for (int i = 0; i < half >> st; ++i) {
      const uint32_t a = w[i], b = w[(half >> st) + i];
      w[i] = least_of(ra, up ? b : a, (uint32_t)__shfl_xor((int)(up ? a : b), 32 >> st));
    }
  }
  constexpr int C = NW * LPR / 64;                          // the words that are left
  struct alignas(4 * C) Words { uint32_t w[C]; };
  const bool high = lane & 32;
  const int at = (high ? RB : 0) + (lane & 16 ? RB / 2 : 0) + 8 * EB * (lane % LPR) + (lane & 15) / LPR * C * 4, wave = threadIdx.x >> 6;
  auto words = [&](char *p) -> Words & { return *reinterpret_cast<Words *>(p + at); };
  Words v;
  if (waves > 1) {                                          // uniform
#pragma unroll
    for (int i = 0; i < C; ++i) v.w[i] = w[i];
    words(red[wave]) = v;
    __syncthreads();
    for (int k = 1; k < waves; ++k) {
      v = words(red[(wave & -waves) + ((wave + k) & (waves - 1))]);
#pragma unroll
      for (int i = 0; i < C; ++i) w[i] = least_of(ra, w[i], v.w[i]);
    }
    __syncthreads();
    there = there && (wave & (waves - 1)) == 0;
  }
#pragma unroll
  for (int i = 0; i < C; ++i) {
    if (high) w[i] ^= other;
    if constexpr (DT == MIXKV_BF16) w[i] = __builtin_bit_cast(uint32_t, RunRange<DT>::turn(__builtin_bit_cast(typename RunRange<DT>::s16x2, w[i])));
    v.w[i] = w[i];
  }
  if (there) words(dst) = v;
}

// The eight elements of a word of codes.  The code's bits are the upper ones of 1 + code / 16.
__device__ __forceinline__ void word_values(uint32_t w, float step, float base, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    constexpr int top = 19;                                 // the lowest of the four
    const int sh = code_shift(e);
    x[e] = fmaf(step, __uint_as_float(((sh < top ? w << (top - sh) : w >> (sh - top)) & 0x00780000u) | 0x3f800000u), base);
  }
}

struct From { int page, row; };            // where a row comes from; page -1: there is none

template <int DT, int D, bool Q4>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(PShape s, EvictShape ev, EvictTable tab) {
  constexpr int EB = DT == MIXKV_BF16 ? 2 : 4, LPR = D / 16, RB = D * EB, NG = D / 32;
  const int tid = threadIdx.x, lane = tid & 63, j = tid % LPR, u = blockIdx.x, layer = blockIdx.z;
  const PCache c = tab.c[layer];
  const EvictLayer l = tab.l[layer];
  __shared__ __align__(16) char red[4][2 * RB];
  const PCache to{l.K, l.V, l.bounds, l.table, nullptr};
  const int32_t *kept = l.kept + (int64_t)u * ev.max_keep;
  const int n = l.n_kept[u];
  auto place_of = [&](int i) { return i < n ? kept[i] : -1; };                  // of the i-th kept row
  auto from_of = [&](int place) {                                             // (no place: none)
    From f;
    f.page = place >= 0 ? page_at(s, c, u, place >> s.lp) : -1;
    f.row = place & (s.P - 1);
    return f;
  };

  const int worker = blockIdx.y >> 1, workers = gridDim.y >> 1;
  const bool keys = (blockIdx.y & 1) == 0;
  if (keys || !Q4) {
    // A wave has the 32 rows of a turn's 128 that are its own, RS at a time, U times RS under way.
    constexpr int RS = 64 / LPR, U = D == 128 && DT == MIXKV_BF16 ? 4 : 2, PARTS = 32 / (RS * U);
    const int slot = lane / LPR, wave = tid >> 6;
    const bool bounds = keys && c.bounds && to.bounds;       // (uniform over the launch)
    const float *w_in = keys && l.into ? l.weights : nullptr;
    const char *from_pool = keys ? c.K : c.V;
    char *to_pool = keys ? to.K : to.V;
    auto row_at = [&](int q) { return (q / PARTS * workers + worker) * 128 + wave * 32 + q % PARTS * (RS * U) + slot; };    // of the wave's part q
    From f[U];
    int next[U];
#pragma unroll
    for (int k = 0; k < U; ++k) next[k] = place_of(row_at(0) + k * RS);
#pragma unroll
    for (int k = 0; k < U; ++k) f[k] = from_of(next[k]);
#pragma unroll
    for (int k = 0; k < U; ++k) next[k] = place_of(row_at(1) + k * RS);
    RunRange<DT> ra, rb;
    for (int q = 0; (q / PARTS * workers + worker) * 128 < n; ++q) {   // (uniform over the workgroup)
      const int i0 = row_at(q), id = (i0 & -32) < n ? page_at(s, to, u, i0 >> s.lp) : -1;
      Run<DT> ka[U], kb[U];
      u32x2 kw[U], sc[U];
      float w[U];
      // (a lane without a row reads the first page's, and stores nothing)
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const char *ks = from_pool + (int64_t)max(f[k].page, 0) * s.page_bytes;
        if constexpr (!Q4) {
          const char *src = ks + (int64_t)f[k].row * RB + 8 * EB * j;
          ka[k].load(src); kb[k].load(src + RB / 2);
        } else {
          const Place4<D> a(j, f[k].row, s.P);
          kw[k] = *a.key_words(const_cast<char *>(ks));
          sc[k] = *a.key_scales(const_cast<char *>(ks));
        }
        if (w_in) w[k] = w_in[((int64_t)max(f[k].page, 0) << s.lp) + f[k].row];
      }
      From f1[U];
#pragma unroll
      for (int k = 0; k < U; ++k) f1[k] = from_of(next[k]);
#pragma unroll
      for (int k = 0; k < U; ++k) next[k] = place_of(row_at(q + 2) + k * RS);
      if (PARTS == 1 || q % PARTS == 0) { ra.none(); rb.none(); }
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int r = (i0 + k * RS) & (s.P - 1);
        if (id >= 0 && f[k].page >= 0) {
          char *kp = to_pool + (int64_t)id * s.page_bytes;
          if constexpr (!Q4) {
            char *dst = kp + (int64_t)r * RB + 8 * EB * j;
            ka[k].store(dst); kb[k].store(dst + RB / 2);
          } else {
            const Place4<D> z(j, r, s.P);
            *z.key_words(kp) = kw[k];
            if ((j & 3) == 0) *z.key_scales(kp) = sc[k];
            if (bounds) {
              float x0[8], x1[8];
              word_values(kw[k][0], f16_value(sc[k][0] & 0xffffu), f16_value(sc[k][0] >> 16), x0);
              word_values(kw[k][1], f16_value(sc[k][1] & 0xffffu), f16_value(sc[k][1] >> 16), x1);
              ka[k].set(x0); kb[k].set(x1);
            }
          }
          if (bounds) { ra.add(ka[k]); rb.add(kb[k]); }
          if (w_in && j == 0) l.into[((int64_t)id << s.lp) + r] = w[k];
        }
        f[k] = f1[k];
      }
      if (bounds && (q + 1) % PARTS == 0) store_page_bounds<DT, D>(to.bounds + (int64_t)id * 2 * RB, id >= 0, s.P >> 5, ra, rb, red);
    }
  } else {
    // a wave to the strips of half a tile of 32 rows (D = 128), or of a whole one
    constexpr int LS = D / 4, SW = 64 / LS, WT = 4 / SW;     // lanes of a strip, strips of a wave, waves of a tile
    const int wave = tid >> 6, part = wave % WT, step = workers * (4 / WT), tiles = (n + 31) >> 5;
    const int l32 = lane & 31, sl = part * SW + lane / LS, at = lane % LS;
    int t = worker * (4 / WT) + wave / WT;
    From f = from_of(place_of(t < tiles ? t * 32 + l32 : INT32_MAX));           // lane i: the tile's row i
    int next = tiles - t > step ? place_of((t + step) * 32 + l32) : -1;
    while (t < tiles) {
      const int id = page_at(s, to, u, (t * 32) >> s.lp);
      const From f1 = from_of(next);
      next = tiles - t > 2 * (int64_t)step ? place_of((t + 2 * step) * 32 + l32) : -1;
      if (id >= 0) {                                         // uniform over the wave
        char *vp = to.V + (int64_t)id * s.page_bytes;
        const int r0 = (t * 32) & (s.P - 1);
        u32x4 *dst = reinterpret_cast<u32x4 *>(reinterpret_cast<uint32_t *>(vp) + ((r0 >> 5) * 4 + sl) * D + 4 * at);
        u32x4 x[8];
        int sh[8];
        bool full = true;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int from = 4 * sl + (e >> 1) + 16 * (e & 1), page = __shfl(f.page, from), row = __shfl(f.row, from);
          sh[e] = page >= 0 ? code_shift(2 * (row & 3) + ((row >> 4) & 1)) : -1;
          full = full && page >= 0;
          x[e] = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const uint32_t *>(c.V + (int64_t)max(page, 0) * s.page_bytes) + ((row >> 5) * 4 + ((row & 15) >> 2)) * D + 4 * at);
        }
        // steps and bases: a lane to a row of the wave's strips and a group
        const int row_s = lane / NG, g = lane % NG, strip_s = row_s / 8, e_s = row_s % 8;
        const int from = 4 * (part * SW + strip_s) + (e_s >> 1) + 16 * (e_s & 1), page = __shfl(f.page, from), row = __shfl(f.row, from);
        if (page >= 0) {
          const Place4<D> pa(0, row, s.P), pz(0, r0 + from, s.P);
          const uint16_t *p = pa.value_scale(c.V + (int64_t)page * s.page_bytes, g);
          uint16_t *z = pz.value_scale(vp, g);
          z[0] = p[0];
          z[8] = p[8];
        }
        u32x4 w = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int k = 0; k < 4; ++k) w[k] |= sh[e] >= 0 ? ((x[e][k] >> sh[e]) & 15u) << code_shift(e) : 0u;
        if (!full) {                                         // codes of rows that are not written stay
          const u32x4 old = *dst;
#pragma unroll
          for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] |= sh[e] >= 0 ? 0u : old[k] & (15u << code_shift(e));
        }
        *dst = w;
      }
      f = f1;
      if (tiles - t <= step) break;
      t += step;
    }
  }
}

// Heads that a workgroup holds in registers, as long as the host says; longer ones have keys and counts in the workspace.
constexpr int kRankRows = 16384;
// Layers of a launch: at a thousand threads a head, fewer than 2^32.
static int evict_layers(const PShape &s, int n_layers) { return std::min(std::min(n_layers, kEvictLayers), ((1 << 22) - 1) / s.units_per_layer); }
static int64_t most_rows(const PShape &s, int max_rows) { return std::min<int64_t>(max_rows, (int64_t)s.max_pages * s.P); }
static size_t evict_plan(const PShape &s, int n_layers, int max_rows, void *workspace, LongPlan *p) {
  const int64_t rows = most_rows(s, max_rows), heads = (int64_t)evict_layers(s, n_layers) * s.units_per_layer;
  *p = LongPlan{};
  if (rows <= kRankRows) return 0;
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(kMostSegs, ((int64_t)1 << 21) / heads));        // fewer than 2^32 threads
  p->stride = (rows + 3) / 4 * 4;
  p->seg = (int32_t)(((rows + most - 1) / most + kSegRows - 1) / kSegRows * kSegRows);
  p->segs = (int32_t)((rows + p->seg - 1) / p->seg);
  const size_t states = (size_t)heads * p->segs * sizeof(int4), counts = (size_t)heads * 2 * p->segs * kLongBins * sizeof(int);
  p->states = static_cast<int4 *>(workspace);
  if (workspace) {
    p->counts = reinterpret_cast<int *>(static_cast<char *>(workspace) + states);
    p->keys = reinterpret_cast<uint32_t *>(static_cast<char *>(workspace) + states + counts);
  }
  return states + counts + (size_t)heads * p->stride * sizeof(uint32_t);
}

}  // namespace mixkv

extern "C" mixkv_status mixkv_paged_evict_workspace_size(const mixkv_paged_params *params, int32_t n_layers, int32_t max_rows, size_t *bytes) {
  using namespace mixkv;
  PShape s;
  const mixkv_status st = make_pshape(params, &s);
  if (st != MIXKV_OK) return st;
  if (!bytes || n_layers < 1 || n_layers > MIXKV_MAX_LAYERS || max_rows < 1) return MIXKV_ERR_INVALID_ARG;
  LongPlan plan;
  *bytes = (evict_plan(s, n_layers, max_rows, nullptr, &plan) + 255) / 256 * 256;
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
  LongPlan plan;
  const size_t need = evict_plan(s, n_layers, max_rows, workspace, &plan);
  if (need > 0) {
    if (!workspace || misaligned(workspace, 256)) return MIXKV_ERR_INVALID_ARG;
    if (workspace_bytes < need) return MIXKV_ERR_WORKSPACE_TOO_SMALL;
  }
  const int64_t rows = most_rows(s, max_rows);
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  const EvictShape ev{max_keep, keep_first, keep_last};
  const int per = evict_layers(s, n_layers);
  for (int l0 = 0; l0 < n_layers; l0 += per) {
    const int nl = std::min(n_layers - l0, per);
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
    if (rows <= 1024) rank(evict_rank_kernel<256, 4>, 256);
    else if (rows <= 4096) rank(evict_rank_kernel<512, 8>, 512);
    else if (rows <= kRankRows) rank(evict_rank_kernel<1024, 16>, 1024);
    else {
      const dim3 parts((unsigned)s.units_per_layer, (unsigned)plan.segs, (unsigned)nl);
      auto part = [&](auto kern) { hipLaunchKernelGGL(kern, parts, dim3(kRankThreads), 0, stream, s, ev, t, plan); };
      part(evict_count_kernel<0>);
      part(evict_count_kernel<1>);
      part(evict_count_kernel<2>);
      part(evict_list_kernel);
    }
    // Workgroups of a head: one for 128 rows of keys and one for as many of values, as long as all of them are on the chip together.
    const int64_t work = ((int64_t)max_keep + 127) / 128, fit = std::max<int64_t>(1, 4096 / ((int64_t)s.units_per_layer * nl));
    const dim3 grid((unsigned)s.units_per_layer, (unsigned)(2 * std::min(work, std::min(fit, (most + 1) / 2))), (unsigned)nl);
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(kMoveThreads), 0, stream, s, ev, t); };
    if (s.q4) { if (s.D == 128) go(evict_move_kernel<MIXKV_BF16, 128, true>); else go(evict_move_kernel<MIXKV_BF16, 64, true>); }
    else if (params->dtype == MIXKV_BF16) { if (s.D == 128) go(evict_move_kernel<MIXKV_BF16, 128, false>); else go(evict_move_kernel<MIXKV_BF16, 64, false>); }
    else { if (s.D == 128) go(evict_move_kernel<MIXKV_F32, 128, false>); else go(evict_move_kernel<MIXKV_F32, 64, false>); }
    if (hipGetLastError() != hipSuccess) return MIXKV_ERR_HIP;
  }
  return MIXKV_OK;
}
