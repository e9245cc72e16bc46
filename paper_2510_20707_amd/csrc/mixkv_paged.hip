// The paged cache: rows into pages (mixkv_paged_append), and out of them (mixkv_paged_read).
//
// What the rows of a page share (the words of a 4-bit value strip, the key bounds) has one writer: the workgroup that has the page, or, where a
// head gets a few rows, the lanes that walk them.  D/16 lanes hold a row: lane j the elements [8 j, 8 j + 8) and
// [D/2 + 8 j, D/2 + 8 j + 8), the two halves of eight rotated pairs.
#include "mixkv_pagedrow.h"

namespace mixkv {

constexpr int kPagedLayers = 16;         // pointer-table entries of a launch: the dense rows' strides travel with them
constexpr int kPagedThreads = 256;

// Rows of a head up to which a few lanes walk them (append_step_kernel) instead of a workgroup to a page and a wave to a row of queries
// (append_many_kernel: shared memory and barriers whatever the count).  us for 1, 2, 3, 4, 6, 8 rows of 8 heads of 128 with 32 query heads, bounds
// kept, walked | by pages: bf16 rows, one sequence 3.7 5.0 6.4 7.3 10.0 12.7 | 6.1 6.3 6.3 6.5 6.6 6.6, 64 sequences 4.0 5.4 6.8 8.2 11.5 17.4 | 7.7 8.9
// 9.1 9.2 9.4 9.8; 4-bit with the rows read back, one sequence 8.9 12.1 15.8 18.8 26.1 33.1 | 10.3 10.3 10.4 10.4 10.5 10.6, 64 sequences
// 9.7 12.9 16.4 20.1 28.0 35.9 | 12.5 14.1 15.0 16.7 17.7 18.6.  The rule goes by the format alone, as one sequence has it: with 64 of them two rows in
// 4 bits and four in full precision would be a tenth faster walked.
static int step_rows(bool q4) { return q4 ? 1 : 3; }

struct PRows {
  char *K, *V;
  int64_t sn, sh;                        // strides in bytes
  const int32_t *start, *count;
  const char *Q;
  int64_t qsn, qsh;
  char *Q_out;
};
struct PTable { PCache c[kPagedLayers]; PRows r[kPagedLayers]; };

struct PRope {
  const float *cos, *sin;                // null: no rotation
  const int32_t *positions;
  int32_t n_positions, n_axes, s0, s1;   // pairs below s0 are axis 0's, below s1 axis 1's
};

// The rows of one unit that a call moves: rows [r0, r1) of the head, row r being dense row r + shift.
struct RowRange { int r0, r1; int64_t shift; };
__device__ __forceinline__ RowRange row_range(const PShape &s, const PCache &c, const PRows &d, int u, int n_rows) {
  const int len = head_rows(s, c, u);
  const int64_t count = max(d.count[u], 0), first = (int64_t)len - count, src = d.start[u];
  RowRange x;
  x.shift = src - first;
  x.r0 = (int)min((int64_t)len, max((int64_t)0, max(first, -x.shift)));
  x.r1 = (int)max((int64_t)x.r0, min((int64_t)len, n_rows - x.shift));
  return x;
}

// Cosines and sines of the N pairs from pair i0 on (elements i and D/2 + i), of dense row `row`.
template <int N> struct Angles { float c[N], s[N]; };
template <int D, int N>
__device__ __forceinline__ void load_angles(const PRope &rp, int64_t row, int n_rows, int i0, Angles<N> &t) {
  int64_t at[3];                                          // the row's place in the tables, for each axis
#pragma unroll
  for (int k = 0; k < 3; ++k) at[k] = k < rp.n_axes ? rp.positions[(int64_t)k * n_rows + row] : 0;
#pragma unroll
  for (int k = 0; k < 3; ++k) at[k] = (int64_t)min(max((int)at[k], 0), rp.n_positions - 1) * (D / 2);
#pragma unroll
  for (int h = 0; h < N; h += 4) {                        // four pairs at a time: 16 bytes of each table
    const int p0 = i0 + h;
    f32x4 c, s;
    if (p0 + 4 <= rp.s0 || (p0 >= rp.s0 && p0 + 4 <= rp.s1) || p0 >= rp.s1) {
      const int64_t p = (p0 + 4 <= rp.s0 ? at[0] : (p0 >= rp.s1 ? at[2] : at[1])) + p0;
      c = *reinterpret_cast<const f32x4 *>(rp.cos + p);
      s = *reinterpret_cast<const f32x4 *>(rp.sin + p);
    } else {                                              // an axis ends among the four
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t p = (p0 + i < rp.s0 ? at[0] : (p0 + i < rp.s1 ? at[1] : at[2])) + p0 + i;
        c[i] = rp.cos[p];
        s[i] = rp.sin[p];
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) { t.c[h + i] = c[i]; t.s[h + i] = s[i]; }
  }
}
// The pairs rotated.  In 64 bits: the products of a table entry and an element are exact there, so the result is the rounded exact rotation
// whatever the order, and a row that is then quantised gets the codes of its definition.  The operator is bound by memory; the 64-bit
// unit is idle otherwise.
template <int DT>
__device__ __forceinline__ void rotate(const Angles<8> &t, Run<DT> &a, Run<DT> &b) {
  float x[8], y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const double p = a.at(i), q = b.at(i);
    const double c = t.c[i], s = t.s[i];
    x[i] = (float)(p * c - q * s);
    y[i] = (float)(q * c + p * s);
    asm("" : "+v"(x[i]), "+v"(y[i]));                     // by way of fp32: the two roundings to bf16 are not made one
  }
  a.set(x);
  b.set(y);
}

// ------------------------------------------------------------------------------------------------
// append_step_kernel (few rows per head: a decoding step).  Every row of a (layer, sequence, KV head) that a call moves, key, value, or one of its
// queries, is a task for D/16 lanes, which walk the head's new rows one after another: no barrier, and one writer for what rows share.
// Bound: a chain of some eight memory round trips, for lanes of one wave may be of different layers: the layer's pointers, its lengths and counts, the table's entry, the row,
// the positions axis by axis, the angles, then the strip's old words or the page's bounds.  3.5 us for one sequence's row into bf16 pages, 6.5 us
// for 64 sequences into 4-bit ones.
// ------------------------------------------------------------------------------------------------
template <int DT, int D, bool Q4>
__global__ __launch_bounds__(kPagedThreads) void append_step_kernel(PShape s, PTable tab, PRope rp, int n_rows, int tasks, int groups) {
  constexpr int EB = DT == MIXKV_BF16 ? 2 : 4, LPR = D / 16, RB = D * EB;
  const int at = blockIdx.x * (kPagedThreads / LPR) + threadIdx.x / LPR, j = threadIdx.x % LPR;
  if (at >= groups) return;                                // whole groups of lanes
  const int ul = at / tasks, task = at - ul * tasks;       // 0: the keys, 1: the values, then the queries
  const int layer = ul / s.units_per_layer, u = ul - layer * s.units_per_layer, h = u % s.hkv;
  const PCache c = tab.c[layer];
  const PRows d = tab.r[layer];
  const RowRange x = row_range(s, c, d, u, n_rows);
  const bool turn = rp.cos != nullptr && task != 1;
  for (int r = x.r0; r < x.r1; ++r) {
    const int64_t row = r + x.shift;
    const int place = r >> s.lp, in_page = r & (s.P - 1);
    const int id = task < 2 ? page_at(s, c, u, place) : 0;
    const char *src = task == 0 ? d.K + row * d.sn + h * d.sh : (task == 1 ? d.V + row * d.sn + h * d.sh : d.Q + row * d.qsn + (h * s.G + task - 2) * d.qsh);
    Run<DT> a, b;
    a.load(src + 8 * EB * j);
    b.load(src + 8 * EB * (LPR + j));
    if (turn) {
      Angles<8> t;
      load_angles<D>(rp, row, n_rows, 8 * j, t);
      rotate<DT>(t, a, b);
    }
    if (task >= 2) {
      char *dst = d.Q_out + (row * s.hq + h * s.G + task - 2) * RB;
      a.store(dst + 8 * EB * j);
      b.store(dst + 8 * EB * (LPR + j));
      continue;
    }
    if (id < 0) continue;                                  // the rows of no page are dropped
    char *page = (task == 0 ? c.K : c.V) + (int64_t)id * s.page_bytes;
    if constexpr (!Q4) {
      a.store(page + (int64_t)in_page * RB + 8 * EB * j);
      b.store(page + (int64_t)in_page * RB + 8 * EB * (LPR + j));
    } else {
      const Place4<D> pl(j, in_page, s.P);
      const GroupScale sa = run_scale(a), sb = run_scale(b);
      if (task == 0) {
        pl.store_keys(page, a, b, sa, sb);
      } else {
        pl.store_value_scales(page, sa, sb);
        const uint32_t wa = run_codes(a, sa), wb = run_codes(b, sb), sh = code_shift(pl.e);
        uint32_t *words = pl.strip_words(page), old[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) old[i] = words[Place4<D>::word_of((i < 8 ? 0 : D / 2) + 8 * j + (i & 7))];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t code = ((i < 8 ? wa : wb) >> code_shift(i & 7)) & 15u;
          words[Place4<D>::word_of((i < 8 ? 0 : D / 2) + 8 * j + (i & 7))] = (old[i] & ~(15u << sh)) | (code << sh);
        }
      }
    }
    if (task == 0 && c.bounds) {
      char *lo = c.bounds + (int64_t)id * 2 * RB, *hi = lo + RB;
      Run<DT> la = a, lb = b, ha = a, hb = b;
      if (in_page > 0) {                                   // rows of before are in the page
        RunRange<DT> ra, rb;
        Run<DT> o[4];
        o[0].load(lo + 8 * EB * j); o[1].load(lo + 8 * EB * (LPR + j));
        o[2].load(hi + 8 * EB * j); o[3].load(hi + 8 * EB * (LPR + j));
        ra.none(); rb.none();
        ra.add(a); rb.add(b);
        ra.lower(o[0]); rb.lower(o[1]);
        ra.raise(o[2]); rb.raise(o[3]);
        la = ra.low(); lb = rb.low(); ha = ra.high(); hb = rb.high();
      }
      la.store(lo + 8 * EB * j); lb.store(lo + 8 * EB * (LPR + j));
      ha.store(hi + 8 * EB * j); hb.store(hi + 8 * EB * (LPR + j));
    }
  }
}

// ------------------------------------------------------------------------------------------------
// append_queries (many rows).  Workers on the rows of a (layer, sequence), a wave to a row, the sequences one after another.  A lane has 16 bytes of
// every 64 / LR-th head (neighbouring lanes neighbouring bytes: an instruction takes a kilobyte of the row), its elements' partners are in the lane
// LR / 2 away, and it keeps its angles for all heads, or, where the KV heads do not have the same rows, for those of
// one KV head at a time.
// Bound: memory; loads and stores pass the caches by (a prompt's queries are more than they keep).  us for four prompts of 84 thousand
// tokens together, 28 heads of 128, 1.20 GB, where torch's copy of the same strided rows takes 211: 208, 5.8 TB/s; with workgroups that follow each other on
// different sequences 254, for DRAM then has four places to read from and to write to; in 1024, 2048, 8192 and 16 384 workgroups instead of 4096 218, 211,
// 209, 228; with the next row's positions fetched ahead and a third of the instructions less 218.
// ------------------------------------------------------------------------------------------------
template <int OFF>
__device__ __forceinline__ uint32_t from_lane_xor(uint32_t x) {
  if constexpr (OFF == 8) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, true);      // row_ror:8
  else return (uint32_t)__shfl_xor((int)x, OFF);
}

template <int DT, int D>
__device__ __forceinline__ void append_queries(const PShape &s, const PTable &tab, const PRope &rp, int n_rows, int lb, int worker, int workers) {
  constexpr int EB = DT == MIXKV_BF16 ? 2 : 4, E = 16 / EB, RB = D * EB, LR = RB / 16, HPI = 64 / LR, U = 8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane % LR, sub = lane / LR;
  const bool upper = l >= LR / 2;
  const int layer = lb / s.batch, b = lb - layer * s.batch;
  const PRows d = tab.r[layer];
  const RowRange x0 = row_range(s, tab.c[layer], d, b * s.hkv, n_rows);
  bool same = true;
  for (int h = 1; h < s.hkv; ++h) {
    const RowRange y = row_range(s, tab.c[layer], d, b * s.hkv + h, n_rows);
    same &= y.r1 - y.r0 == x0.r1 - x0.r0 && y.r0 + y.shift == x0.r0 + x0.shift;
  }
  for (int h = 0; h < s.hkv; h += same ? s.hkv : 1) {
    const RowRange x = h == 0 ? x0 : row_range(s, tab.c[layer], d, b * s.hkv + h, n_rows);
    const int heads = same ? s.hq : s.G;
    for (int r = x.r0 + worker * 4 + wave; r < x.r1; r += workers * 4) {
      const int64_t row = r + x.shift;
      const char *src = d.Q + row * d.qsn + (int64_t)h * s.G * d.qsh + l * 16;
      char *dst = d.Q_out + (row * s.hq + h * s.G) * RB + l * 16;
      Angles<E> t;
      for (int g0 = 0; g0 < heads; g0 += U * HPI) {
        u32x4 v[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int g = g0 + i * HPI + sub;
          v[i] = u32x4{0u, 0u, 0u, 0u};
          if (g < heads) v[i] = load_vec<true>(src + g * d.qsh);
        }
        if (g0 == 0 && rp.cos) {
          load_angles<D>(rp, row, n_rows, E * (l % (LR / 2)), t);
#pragma unroll
          for (int e = 0; e < E; ++e) t.s[e] = upper ? t.s[e] : -t.s[e];
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int g = g0 + i * HPI + sub;
          if (rp.cos) {                                    // (all lanes take part in the exchange)
            u32x4 o;
#pragma unroll
            for (int k = 0; k < 4; ++k) o[k] = from_lane_xor<LR / 2>(v[i][k]);
            float y[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
              float mine, other;
              if constexpr (EB == 2) {
                mine = __uint_as_float(e & 1 ? v[i][e >> 1] & 0xffff0000u : v[i][e >> 1] << 16);
                other = __uint_as_float(e & 1 ? o[e >> 1] & 0xffff0000u : o[e >> 1] << 16);
              } else {
                mine = __uint_as_float(v[i][e]);
                other = __uint_as_float(o[e]);
              }
              y[e] = (float)((double)mine * (double)t.c[e] + (double)other * (double)t.s[e]);
              asm("" : "+v"(y[e]));                        // by way of fp32, as in rotate()
            }
            if constexpr (EB == 2) {
              Run<MIXKV_BF16> z;
              z.set(y);
              v[i] = z.v;
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) v[i][e] = __float_as_uint(y[e]);
            }
          }
          if (g < heads) __builtin_nontemporal_store(v[i], reinterpret_cast<u32x4 *>(dst + (int64_t)g * RB));
        }
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------
// append_pages (many rows).  Workers on the pages of a (layer, sequence, KV head), a workgroup to a page: D/16 lanes
// to a row, codes of values turned into the strips' words through LDS, bounds folded over the page's passes.
// Bound: in 4 bits the quantiser's and the rotation's arithmetic.  us for four prompts of 5 to 32 thousand tokens, 4 KV heads of 128, 171 MB in,
// in a launch of their own: 118 (without the units dealt to the dies in turn 158, and in at most 4096 workgroups 121).
// ------------------------------------------------------------------------------------------------
template <int DT, int D, bool Q4>
__device__ __forceinline__ void append_pages(const PShape &s, const PTable &tab, const PRope &rp, int n_rows, int ul, int worker, int workers) {
  constexpr int EB = DT == MIXKV_BF16 ? 2 : 4, LPR = D / 16, RS = kPagedThreads / LPR, RB = D * EB, RUNS = D / 8;
  __shared__ uint32_t words[Q4 ? RS * RUNS : 1];           // codes of the value rows of a pass, a word per eight elements
  __shared__ __align__(16) char red[4][2 * RB];
  const int tid = threadIdx.x, j = tid % LPR, slot = tid / LPR;
  const int layer = ul / s.units_per_layer, u = ul - layer * s.units_per_layer;
  const int h = u % s.hkv;
  const PCache c = tab.c[layer];
  const PRows d = tab.r[layer];
  const RowRange x = row_range(s, c, d, u, n_rows);
  const bool turn = rp.cos != nullptr;

  for (int pg = (x.r0 >> s.lp) + worker; pg << s.lp < x.r1; pg += workers) {
    const int id = page_at(s, c, u, pg);
    if (id < 0) continue;                                  // uniform: the rows of no page are dropped
    const int first = pg << s.lp, lo_row = max(x.r0 - first, 0), hi_row = min(x.r1 - first, s.P);   // rows of the page to be written
    if (lo_row >= hi_row) continue;
    char *kp = c.K + (int64_t)id * s.page_bytes, *vp = c.V + (int64_t)id * s.page_bytes;
    RunRange<DT> ra, rb;
    ra.none(); rb.none();
    for (int s0 = lo_row / RS * RS; s0 < hi_row; s0 += RS) {
      const int r = s0 + slot;
      const bool live = r >= lo_row && r < hi_row;
      const int64_t row = first + r + x.shift;
      const char *ks = d.K + row * d.sn + h * d.sh + 8 * EB * j, *vs = d.V + row * d.sn + h * d.sh + 8 * EB * j;
      Run<DT> ka{}, kb{}, va{}, vb{};
      if (live) {
        ka.load(ks);
        kb.load(ks + RB / 2);
        va.load(vs);
        vb.load(vs + RB / 2);
        if (turn) {
          Angles<8> t;
          load_angles<D>(rp, row, n_rows, 8 * j, t);
          rotate<DT>(t, ka, kb);
        }
        if (c.bounds) { ra.add(ka); rb.add(kb); }
      }
      if constexpr (!Q4) {
        if (live) {
          const int64_t at = (int64_t)r * RB + 8 * EB * j;
          ka.store(kp + at);
          kb.store(kp + at + RB / 2);
          va.store(vp + at);
          vb.store(vp + at + RB / 2);
        }
      } else {
        const GroupScale ska = run_scale(ka), skb = run_scale(kb), sva = run_scale(va), svb = run_scale(vb);
        if (live) {
          const Place4<D> pl(j, r, s.P);
          pl.store_keys(kp, ka, kb, ska, skb);
          pl.store_value_scales(vp, sva, svb);
          words[slot * RUNS + j] = run_codes(va, sva);
          words[slot * RUNS + LPR + j] = run_codes(vb, svb);
        }
        __syncthreads();
        store_strips<D, RS, kPagedThreads>(vp, words, s0, lo_row, hi_row);
        __syncthreads();
      }
    }
    if (c.bounds) store_bounds<DT, D>(c.bounds + (int64_t)id * 2 * RB, ra, rb, red, lo_row > 0);   // uniform
  }
}

// append_many_kernel.  The pages' workgroups, then (QUERIES) the queries' in one launch.  us against two launches: 17 rows of 33 sequences (12 query
// heads, read back) 15.3 and 19.6, a prompt of 4000 tokens 28.3 and 32.7, one of 32 768 into bf16 pages 118 and 121, four of 84 thousand together
// 374 and 369; with the queries first 15.1, 31.9, 118, 380.
template <int DT, int D, bool Q4, bool QUERIES>
__global__ __launch_bounds__(kPagedThreads) void append_many_kernel(PShape s, PTable tab, PRope rp, int n_rows, int units, int page_workers, int query_workers) {
  const int i = blockIdx.x, q = i - units * page_workers;
  if (!QUERIES || q < 0) {
    const int turn = i / units;
    append_pages<DT, D, Q4>(s, tab, rp, n_rows, dealt_unit(i - turn * units, turn, units), turn, page_workers);
  } else if constexpr (QUERIES) {
    const int lb = q / query_workers;
    append_queries<DT, D>(s, tab, rp, n_rows, lb, q - lb * query_workers, query_workers);
  }
}

// The kernels of a page's format: for a few rows, for many of keys and values, and of queries beside them.
template <int DT, int D, bool Q4, typename Go>
static void append_kernels(Go &&go) { go(append_step_kernel<DT, D, Q4>, append_many_kernel<DT, D, Q4, false>, append_many_kernel<DT, D, Q4, true>); }

// ------------------------------------------------------------------------------------------------
// read_paged_kernel.  blockIdx.x: (layer, sequence, KV head); blockIdx.y: workers on the head's passes of RS rows.
// Bound: memory, the dense rows' stores first: the same four prompts, 54 MB of 4-bit pages to 171 MB of rows, in 46 us
// (without the units dealt to the dies in turn 55).
// ------------------------------------------------------------------------------------------------
template <int DT, int D, bool Q4>
__global__ __launch_bounds__(D * 2) void read_paged_kernel(PShape s, PTable tab, int n_rows) {
  constexpr int EB = DT == MIXKV_BF16 ? 2 : 4, LPR = D / 16, RS = 32, RB = D * EB, STRIP = D + 8;   // (a strip's words, padded)
  __shared__ __align__(16) uint32_t words[Q4 ? 4 * STRIP : 4];
  const int tid = threadIdx.x, j = tid % LPR, slot = tid / LPR;
  const int ul = dealt_unit(blockIdx.x, blockIdx.y, gridDim.x), layer = ul / s.units_per_layer, u = ul - layer * s.units_per_layer;
  const int h = u % s.hkv;
  const PCache c = tab.c[layer];
  const PRows d = tab.r[layer];
  const RowRange x = row_range(s, c, d, u, n_rows);
  for (int t0 = x.r0 / RS + (int)blockIdx.y; t0 * RS < x.r1; t0 += gridDim.y) {
    const int id = page_at(s, c, u, (t0 * RS) >> s.lp);
    if (id < 0) continue;                                  // uniform
    const int r0 = (t0 * RS) & (s.P - 1), r = r0 + slot, at = t0 * RS + slot;   // the pass's first row of the page, the row of the page, of the head
    const bool live = at >= x.r0 && at < x.r1;
    char *kp = c.K + (int64_t)id * s.page_bytes, *vp = c.V + (int64_t)id * s.page_bytes;
    Run<DT> ka{}, kb{}, va{}, vb{};
    if constexpr (!Q4) {
      const int64_t from = (int64_t)r * RB + 8 * EB * j;
      if (live) {
        ka.load(kp + from);
        kb.load(kp + from + RB / 2);
        va.load(vp + from);
        vb.load(vp + from + RB / 2);
      }
    } else {
      const Place4<D> pl(j, r, s.P);
      // the pass's four strips through LDS: a word has eight rows' codes
      u32x4 strip = {};
      if (tid < D) strip = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const uint32_t *>(vp) + (r0 >> 5) * 4 * D + 4 * tid);
      const u32x2 kw = *pl.key_words(kp), ks = *pl.key_scales(kp);
      const uint16_t *sa = pl.value_scale(vp, pl.ga()), *sb = pl.value_scale(vp, pl.gb());
      const float s0 = f16_value(sa[0]), b0 = f16_value(sa[8]), s1 = f16_value(sb[0]), b1 = f16_value(sb[8]);
      __syncthreads();                                     // the pass before has read the strips
      if (tid < D) *reinterpret_cast<u32x4 *>(words + (tid / (D / 4)) * STRIP + (tid % (D / 4)) * 4) = strip;
      __syncthreads();
      const uint32_t *vw = words + (pl.strip & 3) * STRIP, sh = code_shift(pl.e);
      float x0[8], x1[8], y0[8], y1[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x0[i] = code_value((kw[0] >> code_shift(i)) & 15u, f16_value(ks[0] & 0xffffu), f16_value(ks[0] >> 16));
        x1[i] = code_value((kw[1] >> code_shift(i)) & 15u, f16_value(ks[1] & 0xffffu), f16_value(ks[1] >> 16));
        y0[i] = code_value((vw[Place4<D>::word_of(8 * j + i)] >> sh) & 15u, s0, b0);
        y1[i] = code_value((vw[Place4<D>::word_of(D / 2 + 8 * j + i)] >> sh) & 15u, s1, b1);
      }
      ka.set(x0); kb.set(x1); va.set(y0); vb.set(y1);
    }
    if (!live) continue;
    const int64_t row = at + x.shift;
    char *kd = d.K + row * d.sn + h * d.sh + 8 * EB * j, *vd = d.V + row * d.sn + h * d.sh + 8 * EB * j;
    ka.store(kd);
    kb.store(kd + RB / 2);
    va.store(vd);
    vb.store(vd + RB / 2);
  }
}

mixkv_status make_pshape(const mixkv_paged_params *p, PShape *s) {
  if (!p) return MIXKV_ERR_INVALID_ARG;
  if (p->dtype != MIXKV_F32 && p->dtype != MIXKV_BF16) return MIXKV_ERR_INVALID_ARG;
  if (p->format != MIXKV_PAGE_ROWS && p->format != MIXKV_PAGE_4BIT) return MIXKV_ERR_INVALID_ARG;
  if (p->batch < 1 || p->n_q_heads < 1 || p->n_kv_heads < 1 || p->n_q_heads % p->n_kv_heads != 0) return MIXKV_ERR_INVALID_ARG;
  if (p->max_pages < 1 || p->n_pages < 1) return MIXKV_ERR_INVALID_ARG;
  if (!(p->softmax_scale > 0.f) || p->softmax_scale > 0x1p127f) return MIXKV_ERR_INVALID_ARG;   // times log2(e) it has to be finite
  if (p->head_dim != 64 && p->head_dim != 128) return MIXKV_ERR_UNSUPPORTED;
  if (p->page_rows != 32 && p->page_rows != 64 && p->page_rows != 128) return MIXKV_ERR_UNSUPPORTED;
  if (p->format == MIXKV_PAGE_4BIT && p->dtype != MIXKV_BF16) return MIXKV_ERR_UNSUPPORTED;
  if ((int64_t)p->max_pages * p->page_rows > (1 << 30)) return MIXKV_ERR_UNSUPPORTED;
  if ((int64_t)p->batch * p->n_q_heads > (1 << 18)) return MIXKV_ERR_UNSUPPORTED;      // a launch has fewer than 2^32 threads
  s->batch = p->batch; s->hq = p->n_q_heads; s->hkv = p->n_kv_heads; s->G = p->n_q_heads / p->n_kv_heads; s->D = p->head_dim;
  s->P = p->page_rows; s->lp = p->page_rows == 32 ? 5 : p->page_rows == 64 ? 6 : 7;
  s->max_pages = p->max_pages; s->n_pages = p->n_pages;
  s->units_per_layer = p->batch * p->n_kv_heads;
  s->q4 = p->format == MIXKV_PAGE_4BIT;
  s->page_bytes = page_bytes_of(s->q4, p->dtype, s->P, s->D);
  s->scale_log2e = p->softmax_scale * 1.44269504088896340736f;
  return MIXKV_OK;
}

mixkv_status check_caches(const mixkv_paged_cache *c, int n_layers, bool pages, bool bounds) {
  if (!c || n_layers < 1 || n_layers > MIXKV_MAX_LAYERS) return MIXKV_ERR_INVALID_ARG;
  for (int l = 0; l < n_layers; ++l) {
    if (pages && (!c[l].K_pages || !c[l].V_pages || c[l].K_pages == c[l].V_pages)) return MIXKV_ERR_INVALID_ARG;
    if (misaligned(c[l].K_pages, 16) || misaligned(c[l].V_pages, 16) || misaligned(c[l].K_bounds, 16)) return MIXKV_ERR_INVALID_ARG;
    if (bounds && !c[l].K_bounds) return MIXKV_ERR_INVALID_ARG;
    if (!c[l].page_table || !c[l].lengths || misaligned(c[l].page_table, 4) || misaligned(c[l].lengths, 4)) return MIXKV_ERR_INVALID_ARG;
  }
  return MIXKV_OK;
}

static PCache cache_of(const mixkv_paged_cache &c) {
  return PCache{static_cast<char *>(c.K_pages), static_cast<char *>(c.V_pages), static_cast<char *>(c.K_bounds), c.page_table, c.lengths};
}

static mixkv_status check_rows(const PShape &s, int eb, const mixkv_paged_rows *r, int n_layers, int64_t n_rows, bool append) {
  if (!r) return MIXKV_ERR_INVALID_ARG;
  auto bad_stride = [&](int64_t n, int64_t h) { return bad_row_strides(s, eb, n_rows, n, h); };
  auto span = [&](int64_t n, int64_t h, int heads) { return row_span(s, eb, n_rows, n, h, heads); };
  auto overlap = regions_overlap;
  for (int l = 0; l < n_layers; ++l) {
    const mixkv_paged_rows &d = r[l];
    if (!d.K || !d.V || misaligned(d.K, 16) || misaligned(d.V, 16) || bad_stride(d.stride_n, d.stride_h)) return MIXKV_ERR_INVALID_ARG;
    if (!d.row_start || !d.row_count || misaligned(d.row_start, 4) || misaligned(d.row_count, 4)) return MIXKV_ERR_INVALID_ARG;
    const uint64_t kv = span(d.stride_n, d.stride_h, s.hkv);
    if (!append) {
      if (d.K == d.V) return MIXKV_ERR_INVALID_ARG;
      continue;
    }
    if (!d.Q != !d.Q_out || !d.Q != !r[0].Q) return MIXKV_ERR_INVALID_ARG;    // for all layers of a call or none
    if (!d.Q) continue;
    if (misaligned(d.Q, 16) || misaligned(d.Q_out, 16) || bad_stride(d.q_stride_n, d.q_stride_h)) return MIXKV_ERR_INVALID_ARG;
    const uint64_t out = (uint64_t)n_rows * s.hq * s.D * eb;
    if (overlap(d.Q_out, out, d.Q, span(d.q_stride_n, d.q_stride_h, s.hq)) || overlap(d.Q_out, out, d.K, kv) || overlap(d.Q_out, out, d.V, kv))
      return MIXKV_ERR_INVALID_ARG;
  }
  return MIXKV_OK;
}

static PTable table_of(const mixkv_paged_cache *c, const mixkv_paged_rows *r, int nl, int eb) {
  PTable t;
  for (int l = 0; l < kPagedLayers; ++l) {
    t.c[l] = PCache{};
    t.r[l] = PRows{};
    if (l >= nl) continue;
    t.c[l] = cache_of(c[l]);
    t.r[l] = PRows{static_cast<char *>(r[l].K), static_cast<char *>(r[l].V), r[l].stride_n * eb, r[l].stride_h * eb, r[l].row_start,
                   r[l].row_count, static_cast<const char *>(r[l].Q), r[l].q_stride_n * eb, r[l].q_stride_h * eb, static_cast<char *>(r[l].Q_out)};
  }
  return t;
}

// Workers of a unit: those that are wanted, one to a page or a few rows, as long as a launch has no more workgroups than `groups`; the workers
// then walk.
static int workers(int64_t wanted, int64_t units, int64_t groups = 16384) {
  const int64_t most = groups / units < 1 ? 1 : groups / units;
  return (int)(wanted < most ? wanted : most);
}

}  // namespace mixkv

extern "C" mixkv_status mixkv_page_bytes(const mixkv_paged_params *params, size_t *bytes) {
  using namespace mixkv;
  PShape s;
  const mixkv_status st = make_pshape(params, &s);
  if (st != MIXKV_OK) return st;
  if (!bytes) return MIXKV_ERR_INVALID_ARG;
  *bytes = (size_t)s.page_bytes;
  return MIXKV_OK;
}

extern "C" mixkv_status mixkv_paged_append(const mixkv_paged_params *params, const mixkv_paged_cache *caches, const mixkv_paged_rows *rows,
                                           int32_t n_layers, const mixkv_rope *rope, int32_t n_rows, int32_t max_count, void *hip_stream) {
  using namespace mixkv;
  PShape s;
  mixkv_status st = make_pshape(params, &s);
  if (st != MIXKV_OK) return st;
  if (n_rows < 1 || max_count < 1) return MIXKV_ERR_INVALID_ARG;
  if ((st = check_caches(caches, n_layers, true, false)) != MIXKV_OK) return st;
  const int eb = params->dtype == MIXKV_BF16 ? 2 : 4;
  if ((st = check_rows(s, eb, rows, n_layers, n_rows, true)) != MIXKV_OK) return st;
  PRope rp{};
  rp.n_axes = 1; rp.n_positions = 1;
  if (rope) {
    if (!rope->cos || !rope->sin || !rope->positions || misaligned(rope->cos, 16) || misaligned(rope->sin, 16) || misaligned(rope->positions, 4))
      return MIXKV_ERR_INVALID_ARG;
    if (rope->n_positions < 1 || (rope->n_axes != 1 && rope->n_axes != 3)) return MIXKV_ERR_INVALID_ARG;
    rp = PRope{rope->cos, rope->sin, rope->positions, rope->n_positions, rope->n_axes, s.D / 2, s.D / 2};
    if (rope->n_axes == 3) {
      const int32_t *q = rope->sections;
      if (q[0] < 0 || q[1] < 0 || q[2] < 0 || (int64_t)q[0] + q[1] + q[2] != s.D / 2) return MIXKV_ERR_INVALID_ARG;
      rp.s0 = q[0]; rp.s1 = q[0] + q[1];
    }
  }
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  if (max_count > n_rows) max_count = n_rows;
  for (int l0 = 0; l0 < n_layers; l0 += kPagedLayers) {
    const int nl = n_layers - l0 < kPagedLayers ? n_layers - l0 : kPagedLayers;
    const PTable t = table_of(caches + l0, rows + l0, nl, eb);
    const int64_t units = (int64_t)nl * s.units_per_layer;
    const bool queries = rows[0].Q != nullptr;
    auto go = [&](auto step, auto many, auto many_queries) {
      if (max_count <= step_rows(s.q4)) {
        const int tasks = 2 + (queries ? s.G : 0), per = kPagedThreads / (s.D / 16), groups = (int)units * tasks;
        hipLaunchKernelGGL(step, dim3((unsigned)((groups + per - 1) / per)), dim3(kPagedThreads), 0, stream, s, t, rp, n_rows, tasks, groups);
        return;
      }
      const int pw = workers(((int64_t)max_count + s.P - 2) / s.P + 1, units), qw = workers(((int64_t)max_count + 3) / 4, (int64_t)nl * s.batch, 4096);
      const dim3 grid((unsigned)(units * pw + (queries ? (int64_t)nl * s.batch * qw : 0)));
      if (queries) hipLaunchKernelGGL(many_queries, grid, dim3(kPagedThreads), 0, stream, s, t, rp, n_rows, (int)units, pw, qw);
      else hipLaunchKernelGGL(many, grid, dim3(kPagedThreads), 0, stream, s, t, rp, n_rows, (int)units, pw, qw);
    };
    if (s.q4) { if (s.D == 128) append_kernels<MIXKV_BF16, 128, true>(go); else append_kernels<MIXKV_BF16, 64, true>(go); }
    else if (params->dtype == MIXKV_BF16) { if (s.D == 128) append_kernels<MIXKV_BF16, 128, false>(go); else append_kernels<MIXKV_BF16, 64, false>(go); }
    else { if (s.D == 128) append_kernels<MIXKV_F32, 128, false>(go); else append_kernels<MIXKV_F32, 64, false>(go); }
    if (hipGetLastError() != hipSuccess) return MIXKV_ERR_HIP;
  }
  return MIXKV_OK;
}

extern "C" mixkv_status mixkv_paged_read(const mixkv_paged_params *params, const mixkv_paged_cache *caches, const mixkv_paged_rows *rows,
                                         int32_t n_layers, int32_t n_rows, int32_t max_count, void *hip_stream) {
  using namespace mixkv;
  PShape s;
  mixkv_status st = make_pshape(params, &s);
  if (st != MIXKV_OK) return st;
  if (n_rows < 1 || max_count < 1) return MIXKV_ERR_INVALID_ARG;
  if ((st = check_caches(caches, n_layers, true, false)) != MIXKV_OK) return st;
  const int eb = params->dtype == MIXKV_BF16 ? 2 : 4;
  if ((st = check_rows(s, eb, rows, n_layers, n_rows, false)) != MIXKV_OK) return st;
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  if (max_count > n_rows) max_count = n_rows;
  for (int l0 = 0; l0 < n_layers; l0 += kPagedLayers) {
    const int nl = n_layers - l0 < kPagedLayers ? n_layers - l0 : kPagedLayers;
    const PTable t = table_of(caches + l0, rows + l0, nl, eb);
    const int64_t units = (int64_t)nl * s.units_per_layer;
    const int w = workers(((int64_t)max_count + 30) / 32 + 1, units);
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3((unsigned)units, (unsigned)w), dim3(2 * s.D), 0, stream, s, t, n_rows); };
    if (s.q4) { if (s.D == 128) go(read_paged_kernel<MIXKV_BF16, 128, true>); else go(read_paged_kernel<MIXKV_BF16, 64, true>); }
    else if (params->dtype == MIXKV_BF16) { if (s.D == 128) go(read_paged_kernel<MIXKV_BF16, 128, false>); else go(read_paged_kernel<MIXKV_BF16, 64, false>); }
    else { if (s.D == 128) go(read_paged_kernel<MIXKV_F32, 128, false>); else go(read_paged_kernel<MIXKV_F32, 64, false>); }
    if (hipGetLastError() != hipSuccess) return MIXKV_ERR_HIP;
  }
  return MIXKV_OK;
}
