// The attention that cached rows have been given (mixkv_paged_weights): column sums of the new rows' attention weights, from their log-sum-exp.
//
// With a row's normaliser known, a key's sum needs no running softmax: exp2(x c - lse), one multiply-add and one exponential an element, and no other
// key.  A tile of 32 keys belongs to one wave, which goes through the rows that see it: no atomics, and the order of a sum is that of the rows.
#include "mixkv_pagedwin.h"

namespace mixkv {

struct WeightPtrs { float *w[kLayersPerLaunch]; };

// Steps of 16 rows whose weights are summed up on their own.  A lane adds four rows a step: 256 additions a run, and one a run behind them, each off by at most 2^-24 of the sum: 2^17 rows, 128
// runs, by at most 2^-15.4; 2^12 rows by 2^-16.
constexpr int kSumRun = 64;

// ------------------------------------------------------------------------------------------------
// weights_step_kernel (few rows): a wave to tiles of 32 keys, rows on the output rows of 16 x 16 products, keys on their columns, so that a lane has
// two keys and their sums over four rows each.  With up to 16 rows in all (a step's single tokens) every wave prepares the queries once, with up to 64 the workgroup does.
// 4-bit keys as in paged_q4_kernel: codes as fp16 subnormals, a product for each group of 32 elements, steps and bases behind it in fp32.
// Bound: memory, a tile of each wave in flight, the next one asked for before the exponentials: 32 sequences of up to 16 384 rows, 32 query heads on 8, 570 MB in 121 to 124 us, 4.6 to 4.7 TB/s.
// Five new rows of 16 sequences of 8192 rows: 4 bits 36 us, bf16 49; with the queries prepared anew for every tile 72 and 69.
// Workgroups of 16 tiles: heads of unequal length then end together (121 us; 64 tiles 133, 128 156, 4 144).  Loads past the caches: 124.
// ------------------------------------------------------------------------------------------------
template <int DT, int D, bool Q4, bool AHEAD = false>
__global__ __launch_bounds__(256) void weights_step_kernel(PShape s, PWindow win, WinTable tab, WeightPtrs ptrs, int ctiles) {
  constexpr bool F32 = DT == MIXKV_F32;
  constexpr int EB = F32 ? 4 : 2, RB = D * EB, NC = RB / 64, NG = D / 32, W = 4;
  constexpr int NK = Q4 ? NG / 2 : NC;                     // 16-byte registers of a lane for one of its two keys: codes and scales of the row
  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int u = blockIdx.x, layer = blockIdx.z, b = u / s.hkv, h = u - b * s.hkv;
  const PCache c = tab.c[layer];
  const WinLayer l = tab.l[layer];
  float *weights = ptrs.w[layer];
  const int len = head_rows(s, c, u), count = max(l.count[u], 0), start = l.start[u];
  const int place0 = len - count, served = min(count, win.max_count), all = (len + 31) >> 5;
  // the tiles of the first rows, and those from the first new row's window on
  const int ns = (min(win.first, len) + 31) >> 5, w0 = max(ns, max(0, max(place0, 0) - win.window + 1) >> 5), tiles = ns + max(0, all - w0);
  auto tile_at = [&](int t) { return t < ns ? t : w0 + (t - ns); };
  const int t0 = blockIdx.y * ctiles, t1 = blockIdx.y + 1 == gridDim.y ? tiles : min(tiles, t0 + ctiles);
  if (t0 >= t1) return;

  // Up to 64 rows that are not fp32 are prepared once, a wave 16 of them, and lie in LDS for all of the workgroup's tiles.
  constexpr bool KEPT = !F32;
  static_assert(kFewRows <= 16 * W, "a wave to 16 rows");
  constexpr int NV = (Q4 ? NG + 2 : NC) + 2;               // 16-byte words of a lane: queries; (4 bits) factors and sums; normalisers, places
  __shared__ u32x4 kept_s[4][NV][64];
  // ---- 16 rows: their queries, and of the rows 4 quad + e the normalisers and places.  AHEAD (fp32 of many rows): the next ones are asked for while one is worked on.
  constexpr int NQ = Q4 ? NG : NC;
  u32x4 qf[NQ], qn[NQ];
  f16x8 qs;
  float off[4], c2[4], lse = 0.f;
  int place[4], place_n = -1, row_t = 0, row_g = 0;          // row l16 of the next 16: its new row and query head
  const int step_t = 16 / s.G, step_g = 16 - step_t * s.G;
  auto begin_rows = [&](int i0) { row_t = (i0 + l16) / s.G; row_g = i0 + l16 - row_t * s.G; };
  auto ask_rows = [&](int i0, int i1) {                      // one after another
    const int64_t row = (int64_t)start + row_t, near = min(max(row, (int64_t)0), (int64_t)win.n_rows - 1);
    const char *q = l.Q + near * l.qsn + (int64_t)(h * s.G + row_g) * l.qsh;
#pragma unroll
    for (int k = 0; k < NQ; ++k) qn[k] = *reinterpret_cast<const u32x4 *>(q + (Q4 ? (32 * (D == 128 ? (k & 1) * 2 + (k >> 1) : k) + 8 * quad) * 2 : (4 * k + quad) * 16));
    const bool there = i0 + l16 < i1 && near == row;
    lse = l.lse[near * s.hq + h * s.G + row_g];
    place_n = there ? place0 + row_t : -1;
    row_t += step_t;
    row_g += step_g;
    if (row_g >= s.G) { row_g -= s.G; ++row_t; }
  };
  auto take_rows = [&]() {
    if constexpr (!Q4) {
#pragma unroll
      for (int k = 0; k < NQ; ++k) qf[k] = qn[k];
    } else {
        // to fp16, by a power of two that brings the row's largest element to [2^13, 2^14); their sums over each group in three parts, against a key's (S, B) pairs
        uint32_t most = 0;
#pragma unroll
        for (int pl = 0; pl < NG; ++pl)
#pragma unroll
          for (int j = 0; j < 4; ++j) most = max(most, max(qn[pl][j] & 0x7fffu, (qn[pl][j] >> 16) & 0x7fffu));
        most = max(most, (uint32_t)__shfl_xor((int)most, 16));
        most = max(most, (uint32_t)__shfl_xor((int)most, 32));
        const int up = 13 - (min(max((int)(most >> 7), 1), 254) - 127);
        const float back = fminf(fmaxf(ldexpf(s.scale_log2e, 20 - up), 0x1p-126f), 0x1p100f);   // (as in paged_q4_kernel: neither zero nor infinite)
#pragma unroll
        for (int e = 0; e < 4; ++e) c2[e] = __shfl(back, 4 * quad + e);
        float part[NG];
#pragma unroll
        for (int pl = 0; pl < NG; ++pl) {
          float sum = 0.f;
          f16x8 x;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t w = qn[pl][e >> 1];
            const float v = ldexpf(__uint_as_float(e & 1 ? w & 0xffff0000u : w << 16), up);
            sum += v;
            x[e] = (_Float16)((e >> 1) & 1 ? v * 0.0625f : v);
          }
          qf[pl] = __builtin_bit_cast(u32x4, x);
          sum += __shfl_xor(sum, 16);
          sum += __shfl_xor(sum, 32);
          sum *= 0.00390625f;
          const float hi = (float)(_Float16)sum, mid = (float)(_Float16)(sum - hi);
          part[pl] = quad == 0 ? hi : quad == 1 ? mid : quad == 2 ? sum - hi - mid : 0.f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) qs[e] = (_Float16)(e / 2 < NG ? part[e / 2 % NG] : 0.f);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      off[e] = __shfl(lse * -1.44269504088896340736f, 4 * quad + e);
      place[e] = __shfl(lse != -INFINITY ? place_n : -1, 4 * quad + e);  // -1: the row gives nothing
    }
  };
  const bool once = (int64_t)served * s.G <= 16;
  auto keep_rows = [&](int step) {
    u32x4(&to)[NV][64] = kept_s[step];
#pragma unroll
    for (int k = 0; k < NQ; ++k) to[k][lane] = qf[k];
    if constexpr (Q4) {
      to[NQ][lane] = u32x4{__float_as_uint(c2[0]), __float_as_uint(c2[1]), __float_as_uint(c2[2]), __float_as_uint(c2[3])};
      to[NQ + 1][lane] = __builtin_bit_cast(u32x4, qs);
    }
    to[NV - 2][lane] = u32x4{__float_as_uint(off[0]), __float_as_uint(off[1]), __float_as_uint(off[2]), __float_as_uint(off[3])};
    to[NV - 1][lane] = u32x4{(uint32_t)place[0], (uint32_t)place[1], (uint32_t)place[2], (uint32_t)place[3]};
  };
  auto kept_rows = [&](int step) {
    const u32x4(&from)[NV][64] = kept_s[step];
#pragma unroll
    for (int k = 0; k < NQ; ++k) qf[k] = from[k][lane];
    const u32x4 o = from[NV - 2][lane], p = from[NV - 1][lane];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      off[e] = __uint_as_float(o[e]);
      place[e] = (int)p[e];
      if constexpr (Q4) c2[e] = __uint_as_float(from[NQ][lane][e]);
    }
    if constexpr (Q4) qs = __builtin_bit_cast(f16x8, (u32x4)from[NQ + 1][lane]);
  };
  if (once && served > 0) {
    begin_rows(0);
    ask_rows(0, served * s.G);
    take_rows();
  }
  if constexpr (KEPT) {
    if (!once) {                                             // uniform
      if (wave * 16 < served * s.G) {
        begin_rows(wave * 16);
        ask_rows(wave * 16, served * s.G);
        take_rows();
        keep_rows(wave);
      }
      __syncthreads();
    }
  }

  for (int first = t0 + wave; first < t1; first += 64 * W) {
    // lane i: where the wave's i-th tile of 64 lies
    const int mine = first + lane * W;
    const int id_of = mine < t1 ? page_at(s, c, u, tile_at(mine) >> (s.lp - 5)) : -1;
    const int n = min((t1 - first + W - 1) / W, 64);
    u32x4 kr[2][NK];
    float old = 0.f;
    auto request = [&](int i) {
      const int id = max(__builtin_amdgcn_readlane(id_of, i), 0), row0 = tile_at(first + i * W) * 32 & (s.P - 1);
      const char *page = c.K + (int64_t)id * s.page_bytes;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int row = row0 + 16 * r + l16;
        if constexpr (Q4) {
          const char *codes = page + row * (D / 2) + quad * (NG * 4), *sb = page + s.P * (D / 2) + row * (NG * 4);
          if constexpr (NG == 4) {
            kr[r][0] = load_vec<false>(codes);
            kr[r][1] = load_vec<false>(sb);
          } else {
            const u32x2 x = *reinterpret_cast<const u32x2 *>(codes), z = *reinterpret_cast<const u32x2 *>(sb);
            kr[r][0] = u32x4{x[0], x[1], z[0], z[1]};
          }
        } else {
#pragma unroll
          for (int k = 0; k < NC; ++k) kr[r][k] = load_vec<false>(page + row * RB + (4 * k + quad) * 16);
        }
      }
      old = weights[((int64_t)id << s.lp) + row0 + (lane & 31)];
    };
    request(0);
    for (int i = 0; i < n; ++i) {
      const int k0 = tile_at(first + i * W) * 32, live = min(len - k0, 32), id = __builtin_amdgcn_readlane(id_of, i);
      const float was = old;
      // new rows [lo, hi) see some of the tile's keys
      const int lo = max(k0 - place0, 0), hi = k0 < win.first ? served : (int)min((int64_t)served, (int64_t)k0 + 31 + win.window - place0);
      const bool work = id >= 0 && lo < hi;
      float sum[2] = {0.f, 0.f}, run[2] = {0.f, 0.f};
      int steps = 0;
      const int i1 = work ? (once ? served : hi) * s.G : 0;
      if (!KEPT && work && !once) {
        begin_rows(lo * s.G);
        if constexpr (AHEAD) ask_rows(lo * s.G, i1);
      }
      for (int i0 = once ? 0 : KEPT ? lo * s.G & ~15 : lo * s.G; i0 < i1; i0 += 16) {
        if (!once) {
          if constexpr (KEPT) kept_rows(i0 >> 4);
          else {
            if constexpr (!AHEAD) ask_rows(i0, i1);
            take_rows();
            if (AHEAD && i0 + 16 < i1) ask_rows(i0 + 16, i1);
          }
        }
        f32x4 xs[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          f32x4 x = {0.f, 0.f, 0.f, 0.f};
          if constexpr (Q4) {
            const u32x4 kw = kr[r][0], sb = NG == 4 ? kr[r][NK - 1] : u32x4{kr[r][0][2], kr[r][0][3], 0u, 0u};
            f32x4 y = __builtin_amdgcn_mfma_f32_16x16x32_f16(qs, __builtin_bit_cast(f16x8, sb), f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = y[e] * 0x1p-12f;
#pragma unroll
            for (int pl = 0; pl < NG; ++pl) {
              const uint32_t w = kw[pl], w8 = w >> 8;
              const u32x4 k = {w & 0x000f000fu, w & 0x00f000f0u, w8 & 0x000f000fu, w8 & 0x00f000f0u};
              y = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, qf[pl]), __builtin_bit_cast(f16x8, k), f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
              const float step = (float)__builtin_bit_cast(f16x2, (uint32_t)sb[pl])[0];
#pragma unroll
              for (int e = 0; e < 4; ++e) x[e] = fmaf(step, y[e], x[e]);
            }
          } else if constexpr (!F32) {
#pragma unroll
            for (int k = 0; k < NC; ++k) x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, qf[k]), __builtin_bit_cast(bf16x8, kr[r][k]), x, 0, 0, 0);
          }
          xs[r] = x;
        }
        if constexpr (F32) {                                 // the two keys by turns: no product waits for the one before
#pragma unroll
          for (int k = 0; k < NC; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int r = 0; r < 2; ++r) xs[r] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(qf[k][e]), __uint_as_float(kr[r][k][e]), xs[r], 0, 0, 0);
        }
        if (i0 + 16 >= i1 && i + 1 < n) request(i + 1);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int j = k0 + 16 * r + l16;
#pragma unroll
          for (int e = 0; e < 4; ++e) run[r] += sees(win, place[e], j) ? fast_exp2(fmaf(xs[r][e], Q4 ? c2[e] : s.scale_log2e, off[e])) : 0.f;
        }
        if (++steps == kSumRun) {
          steps = 0;
#pragma unroll
          for (int r = 0; r < 2; ++r) { sum[r] += run[r]; run[r] = 0.f; }
        }
      }
      if (!work && i + 1 < n) request(i + 1);
      const bool fresh = k0 + live > place0;               // the tile has new rows
      if (id < 0 || !(work || fresh)) continue;
      float x[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        x[r] = sum[r] + run[r];
        x[r] += __shfl_xor(x[r], 16);
        x[r] += __shfl_xor(x[r], 32);
      }
      const int j = k0 + lane;
      if (lane < live) weights[((int64_t)id << s.lp) + (k0 & (s.P - 1)) + lane] = (j >= place0 ? 0.f : was) + (lane < 16 ? x[0] : x[1]);
    }
  }
}

// ------------------------------------------------------------------------------------------------
// weights_many_kernel (many rows, bf16 and 4-bit pages): a workgroup of eight waves to a block of keys and a chunk of the unit's rows.  A wave's keys stay in
// registers as the first operand of 32 x 32 x 16 products (4 bits: in two fp16 parts), the rows travel through LDS, 64 or 128 a turn, and are the second for all
// of them: a lane has 16 keys of one row, adds their weights up over its rows, and the lanes are folded at the end.
// A block's products stand beside the weights of the one before, two exponentials to a product, and a turn's last weights behind the barrier, while the next turn's operands come.
// Addresses of rows: a lane computes one row's, the lanes that load it ask for it; three 64-bit products a load took as long as a tenth of the turn.
// Bound: the vector unit: an exponential, a multiply-add and an addition are 16 to 20 cycles of a SIMD for 64 weights, its product 16, and they share the issue.  Prompts of 16 384 and
// 8731 rows, window 8192, 28 query heads on 4: 3.9e9 weights in 1.18 to 1.24 ms, 0.80 to 0.84 PFLOP/s (a large library product 1.19 to 1.22).  Turns of 64 rows: 1.41 ms.  A turn takes 4.8 us, a workgroup's
// beginning and end 10: the compiler waits for the next turn's rows behind the first products of a turn, and forms without that wait had no registers left for the loop (1.26 to 1.31 ms).
// ------------------------------------------------------------------------------------------------
constexpr int kManyWaves = 8, kManyRun = 16384;                     // rows whose weights a lane adds up on its own, every 32nd: they are off by 2^-15 at most
constexpr int many_rows(bool q4) { return q4 ? 64 : 128; }          // rows of a turn
constexpr int many_keys(bool q4) { return 32 * kManyWaves * (q4 ? 1 : 2); }    // keys of a workgroup

struct ManyShape {
  PWindow w;
  int32_t chunk, nchunks;                // rows that a block's chunk should have, the most chunks of a block
  int32_t block0, end;                   // the launch's blocks of keys of a unit: from block0 on, in front of `end`
  int32_t blocks;                        // those of them that have workgroups; longer heads' are walked
  int64_t stride;                        // keys of a unit among the partial sums
};

// Rows [i0, i1) that see some of the keys [k0, k1) of a unit.
struct Rows { int i0, i1; };
__device__ __forceinline__ Rows rows_that_see(const PShape &s, const PWindow &w, int len, int count, int k0, int k1) {
  const int place0 = len - count, served = min(count, w.max_count);
  const int lo = max(k0 - place0, 0), hi = k0 < w.first ? served : (int)min((int64_t)served, (int64_t)k1 - 1 + w.window - place0);
  Rows r;
  r.i0 = min(lo, served) * s.G;
  r.i1 = max(hi, 0) * s.G;
  return r;
}

// The chunks of equal size, whole turns of R, that a block's rows fall into: rows of one.
__device__ __forceinline__ int chunk_rows(const ManyShape &a, const Rows &r, int R) {
  const int n = max(r.i1 - (r.i0 & -R), 1), pieces = min(a.nchunks, (n - 1) / a.chunk + 1);
  return ((n - 1) / pieces / R + 1) * R;
}

template <int D, bool Q4>
__global__ __launch_bounds__(64 * kManyWaves, 2) void weights_many_kernel(PShape s, ManyShape a, WinTable tab, WeightPtrs ptrs, float *part, int64_t unit0) {
  constexpr int RB = D * 2, PPR = RB / 16, KS = D / 16, NG = D / 32, W = kManyWaves, KB = Q4 ? 1 : 2, KEYS = many_keys(Q4), R = many_rows(Q4), WR = R / W, NY = R / 32, IMG = R * RB;
  __shared__ __align__(256) char img[2][IMG];
  __shared__ float off_s[2][R], c2_s[2][R];
  __shared__ int place_s[2][R];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int units = s.units_per_layer, ch = blockIdx.x / units, u = dealt_unit((int)blockIdx.x - ch * units, (int)(blockIdx.y + ch), units), layer = blockIdx.z;
  const int b = u / s.hkv, h = u - b * s.hkv;
  const PCache c = tab.c[layer];
  const WinLayer l = tab.l[layer];
  float *weights = ptrs.w[layer];
  const int len = head_rows(s, c, u), count = max(l.count[u], 0), start = l.start[u], place0 = len - count;
  const uint32_t img_a = lds_base_of(img);
  const int G = s.G, step_t = R / G, step_g = R - step_t * G;
  const int64_t qsn = l.qsn, qsh = l.qsh;
  const char *const Q = l.Q + (int64_t)h * G * qsh;
  for (int block = a.block0 + blockIdx.y; block < a.end && (int64_t)block * KEYS < len; block += a.blocks) {
    const int kA = block * KEYS, kB = min(kA + KEYS, len);
    const Rows rows = rows_that_see(s, a.w, len, count, kA, kB);
    const bool direct = a.nchunks == 1 || kA >= a.stride;    // (keys that the host did not know of: all their rows in one go)
    if (direct && ch > 0) continue;                          // uniform
    const int size = chunk_rows(a, rows, R), i0 = (rows.i0 & -R) + (direct ? 0 : ch * size), i1 = direct ? rows.i1 : (int)min((int64_t)rows.i1, (int64_t)i0 + size);
    if (i0 >= i1 && !direct) continue;                       // uniform: nobody reads these sums
    // ---- the wave's keys
    int id[KB], key0[KB];
    u32x4 kf[KB][KS], lf[KB][Q4 ? KS : 1];
#pragma unroll
    for (int x = 0; x < KB; ++x) {
      key0[x] = kA + (wave * KB + x) * 32;
      id[x] = key0[x] < len ? page_at(s, c, u, key0[x] >> s.lp) : -1;
      const int row = (key0[x] & (s.P - 1)) + l32;
      const char *page = c.K + (int64_t)max(id[x], 0) * s.page_bytes;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        if constexpr (Q4) {
          const int g = k >> 1, run = 2 * (k & 1) + half, pl = D == 128 ? (g & 1) * 2 + (g >> 1) : g;
          const uint32_t w = reinterpret_cast<const uint32_t *>(page + row * (D / 2))[run * NG + pl], z = reinterpret_cast<const uint32_t *>(page + s.P * (D / 2))[row * NG + pl];
          const f16x2 sb = __builtin_bit_cast(f16x2, z), step = {sb[0], sb[0]}, base = {sb[1], sb[1]};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const f16x2 un = code_pair(w, j), y = __builtin_elementwise_fma(un, step, base);
            kf[x][k][j] = __builtin_bit_cast(uint32_t, y);
            lf[x][k][j] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)(fmaf((float)un[0], (float)sb[0], (float)sb[1]) - (float)y[0]), (_Float16)(fmaf((float)un[1], (float)sb[0], (float)sb[1]) - (float)y[1])});
          }
        } else {
          kf[x][k] = *reinterpret_cast<const u32x4 *>(page + row * RB + (2 * k + half) * 16);
        }
      }
    }
    // ---- rows, walked R a turn, a wave staging WR of them.  Lane e of WR knows where row e of the wave lies and takes its normaliser; the lanes that load a row ask it.  bf16: straight
    // to LDS; 4 bits: eight lanes to a row, to fp16 by a power of two that brings its largest element to [2^13, 2^14).  A row that is none gives nothing, whatever is staged for it.
    // Row i + r of the turn that begins with row i = T G + g0 is (T, g0) and what r is of its own, and one new row on where the query heads come to G.  Rows [first_row, last_row) exist.
    constexpr int RPL = 64 / PPR, LOADS = Q4 ? 1 : WR / RPL, PIECES = PPR / 8;   // bf16: rows of a load, loads of a wave; 4 bits: pieces of a thread
    static_assert(!Q4 || WR == 8, "eight lanes to a row");
    const int my_row = WR * wave + (lane & (WR - 1)), my_t = my_row / G, my_g = my_row - my_t * G;
    const int64_t my_q = my_t * qsn + my_g * qsh, wrap_q = qsn - G * qsh;
    const int first_row = (int)min((int64_t)max(-(int64_t)start, (int64_t)0) * G, (int64_t)i1), last_row = (int)min(max((int64_t)a.w.n_rows - start, (int64_t)0) * G, (int64_t)i1);
    const int from = Q4 ? lane >> 3 : lane / PPR, r_row = WR * wave + from;      // the row of the lane's first load
    int T = i0 / G, g0 = i0 - T * G;                         // of the next turn
    u32x4 q_raw[Q4 ? PIECES : 1];
    float n_lse = 0.f;
    int n_place = -1;
    auto request = [&](int i, int to) __attribute__((always_inline)) {           // rows i ... i + R - 1, a turn after the other
      const int64_t row0 = (int64_t)start + T;
      const bool in = (i + my_row >= first_row) & (i + my_row < last_row), wraps = my_g >= G - g0;
      const int64_t at = in ? row0 * qsn + g0 * qsh + my_q + (wraps ? wrap_q : 0) : 0;
#pragma unroll
      for (int j = 0; j < LOADS; ++j) {
        const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)at, from + j * RPL), hi = (uint32_t)__shfl((int)(uint32_t)(at >> 32), from + j * RPL);
        const char *q = Q + (int64_t)((uint64_t)hi << 32 | lo);
        if constexpr (!Q4) {
          load_to_lds<false>(q + ((lane % PPR) ^ tile_swz<MIXKV_BF16, D>(r_row + j * RPL)) * 16, img_a + to * IMG + (WR * wave + j * RPL) * RB);
        } else {
#pragma unroll
          for (int k = 0; k < PIECES; ++k) q_raw[k] = *reinterpret_cast<const u32x4 *>(q + ((lane & 7) * PIECES + k) * 16);
        }
      }
      n_lse = l.lse[in ? row0 * s.hq + h * G + g0 + (my_t * s.hq + my_g) + (wraps ? s.hq - G : 0) : 0];
      n_place = in ? place0 + T + my_t + (wraps ? 1 : 0) : -1;
      T += step_t;
      g0 += step_g;
      if (g0 >= G) { g0 -= G; ++T; }
    };
    auto settle = [&](int to) __attribute__((always_inline)) {                   // what was requested, into LDS
      if (lane < WR) {
        off_s[to][WR * wave + lane] = n_lse * -1.44269504088896340736f;
        place_s[to][WR * wave + lane] = n_lse != -INFINITY ? n_place : -1;
      }
      if constexpr (Q4) {
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < PIECES; ++j)
#pragma unroll
          for (int k = 0; k < 4; ++k) most = max(most, max(q_raw[j][k] & 0x7fffu, (q_raw[j][k] >> 16) & 0x7fffu));
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o));
        const int up = 13 - (min(max((int)(most >> 7), 1), 254) - 127);
        if ((lane & 7) == 0) c2_s[to][r_row] = fminf(fmaxf(ldexpf(s.scale_log2e, -up), 0x1p-126f), 0x1p100f);
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
          u32x4 x;
#pragma unroll
          for (int k = 0; k < 4; ++k)
            x[k] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)ldexpf(__uint_as_float(q_raw[j][k] << 16), up), (_Float16)ldexpf(__uint_as_float(q_raw[j][k] & 0xffff0000u), up)});
          store_lds(img_a + to * IMG + r_row * RB + (((lane & 7) * PIECES + j) ^ tile_swz<MIXKV_BF16, D>(r_row)) * 16, x);
        }
      }
    };
    const uint32_t q_off = img_a + l32 * RB + (half ^ tile_swz<MIXKV_BF16, D>(l32)) * 16;     // where the lane reads; piece 2 k + half of a row: 32 k ^ this one

    // A lane's sums of a key's weights; and folded over the lanes of a half, lanes 2 e and 2 e + 1 with the key 8 (e / 4) + 4 half + e % 4.  The lanes share the sums out by halves: each
    // gives the lane 16, 8, 4, 2 away those that it does not keep.
    const int kz = key0[KB - 1] + 31, window = a.w.window, first = a.w.first;
    const float scale = s.scale_log2e;
    float run[KB][16], mine[KB];
    auto clear = [&]() {
#pragma unroll
      for (int x = 0; x < KB; ++x)
#pragma unroll
        for (int e = 0; e < 16; ++e) run[x][e] = 0.f;
    };
    auto fold = [&]() {
#pragma unroll
      for (int x = 0; x < KB; ++x) {
#pragma unroll
        for (int st = 0; st < 4; ++st) {
          const bool up = lane & (16 >> st);
#pragma unroll
          for (int e = 0; e < 8 >> st; ++e) {
            const float a = run[x][e], b = run[x][(8 >> st) + e];
            run[x][e] = (up ? b : a) + __shfl_xor(up ? a : b, 16 >> st);
          }
        }
        mine[x] += run[x][0] + __shfl_xor(run[x][0], 1);
      }
    };
#pragma unroll
    for (int x = 0; x < KB; ++x) mine[x] = 0.f;
    clear();
    if (i0 < i1) {
      request(i0, 0);
      settle(0);
    }
    // A turn begins: its rows are in LDS, the lane's first operands are asked for; then the next turn's rows are, and it is seen whether every row sees every key.
    int to = 0;
    float off[NY], c2[NY];
    bool all = false;
    u32x4 qf[KS];
    uint32_t q_now;
    auto read_row = [&](int y, int k) __attribute__((always_inline)) {
      asm volatile("" : "+v"(q_now));                        // (the KS addresses are not kept)
      qf[k] = lds_vec((q_now ^ (32 * k)) + y * 32 * RB);
    };
    auto begin = [&]() __attribute__((always_inline)) {
      if constexpr (!Q4) wait_vm<0>();
      lds_barrier();
      q_now = q_off + to * IMG;
#pragma unroll
      for (int y = 0; y < NY; ++y) {
        off[y] = off_s[to][32 * y + l32];
        c2[y] = Q4 ? c2_s[to][32 * y + l32] : scale;
      }
#pragma unroll
      for (int k = 0; k < KS; ++k) read_row(0, k);
    };
    auto look = [&](int i) __attribute__((always_inline)) {
      if (i + R < i1) request(i + R, to ^ 1);
      all = true;
#pragma unroll
      for (int y = 0; y < NY; ++y) {
        const int place = place_s[to][32 * y + l32];
        all = all & (kz <= place) & ((key0[0] > place - window) | (kz < first));
      }
      all = __builtin_amdgcn_ballot_w64(all) == ~0ull;
    };
    auto score = [&](int x, int k, f32x16 &acc) __attribute__((always_inline)) {
      if (k == 0) {
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[e] = 0.f;
      }
      if constexpr (Q4) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, lf[x][k]), __builtin_bit_cast(f16x8, qf[k]), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, kf[x][k]), __builtin_bit_cast(f16x8, qf[k]), acc, 0, 0, 0);
      } else {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[x][k]), __builtin_bit_cast(bf16x8, qf[k]), acc, 0, 0, 0);
      }
    };
    for (int i = i0; i < i1;) {
      const int ib = min(i1 - i, kManyRun) + i;
      begin();
      look(i);
      while (i < ib) {
        if (__builtin_expect(all, 1)) {
          // every row sees every key: a block's products with the weights of the one before, in the program's order; the last weights while the next turn's operands are on their way
          constexpr int N = NY * KB;
          do {
            f32x16 acc[2];
            auto weigh = [&](int n, int e, float o, float c) __attribute__((always_inline)) { run[n % KB][e] += fast_exp2(fmaf(acc[n & 1][e], c, o)); };
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
              for (int k = 0; k < KS; ++k) {
                score(n % KB, k, acc[n & 1]);
                if (n % KB == KB - 1 && n + 1 < N) read_row(n / KB + 1, k);
                if (n > 0) {
                  float t[16 / KS];                          // (side by side, not one after the other in one register)
#pragma unroll
                  for (int e = 0; e < 16 / KS; ++e) t[e] = fmaf(acc[(n - 1) & 1][k * 16 / KS + e], c2[(n - 1) / KB], off[(n - 1) / KB]);
                  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                  for (int e = 0; e < 16 / KS; ++e) t[e] = fast_exp2(t[e]);
                  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                  for (int e = 0; e < 16 / KS; ++e) run[(n - 1) % KB][k * 16 / KS + e] += t[e];
                }
                __builtin_amdgcn_sched_barrier(0);
              }
#pragma unroll
            for (int x = 0; x < KB; ++x)
#pragma unroll
              for (int e = 0; e < 16; ++e) asm volatile("" : "+v"(run[x][e]));   // (the sums are made here, not behind the loop's branches)
            const float o = off[NY - 1], c = c2[NY - 1];
            if (i + R < i1) settle(to ^ 1);
            i += R;
            to ^= 1;
            if (i < ib) {
              begin();
#pragma unroll
              for (int e = 0; e < 16; ++e) weigh(N - 1, e, o, c);
              look(i);
            } else {
#pragma unroll
              for (int e = 0; e < 16; ++e) weigh(N - 1, e, o, c);
              break;                                         // (a path without the wait that leads back here would make the compiler wait for the rows under way)
            }
          } while (all);
        } else {
#pragma unroll
          for (int y = 0; y < NY; ++y) {
            if (y) {
#pragma unroll
              for (int k = 0; k < KS; ++k) read_row(y, k);
            }
            const int place = place_s[to][32 * y + l32], behind = place - window;
            int at = 4 * half;
            asm volatile("" : "+v"(at));
#pragma unroll
            for (int x = 0; x < KB; ++x) {
              if (__builtin_amdgcn_ballot_w64((key0[x] <= place) & ((key0[x] + 31 > behind) | (key0[x] < first))) == 0) continue;
              f32x16 acc;
#pragma unroll
              for (int k = 0; k < KS; ++k) score(x, k, acc);
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const int j = key0[x] + 8 * (e >> 2) + at + (e & 3);
                run[x][e] += (j <= place) & ((j > behind) | (j < first)) ? fast_exp2(fmaf(acc[e], c2[y], off[y])) : 0.f;
                __builtin_amdgcn_sched_barrier(0);
              }
            }
          }
          if (i + R < i1) settle(to ^ 1);
          i += R;
          to ^= 1;
          if (i < ib) {
            begin();
            look(i);
          }
        }
      }
      fold();
      clear();
    }
#pragma unroll
    for (int x = 0; x < KB; ++x) {
      const int j = key0[x] + 8 * (l32 >> 3) + 4 * half + (l32 >> 1 & 3);
      if ((l32 & 1) || j >= len || id[x] < 0) continue;
      if (!direct) {
        part[((unit0 + (int64_t)layer * units + u) * a.nchunks + ch) * a.stride + j] = mine[x];
      } else if (rows.i0 < rows.i1 || j >= place0) {
        float *w = weights + ((int64_t)id[x] << s.lp) + (j & (s.P - 1));
        *w = (j >= place0 ? 0.f : *w) + mine[x];
      }
    }
    __syncthreads();                                         // the images are written anew
  }
}

// Adds up the chunks' sums, in their order.
__global__ __launch_bounds__(256) void weights_fold_kernel(PShape s, ManyShape a, WinTable tab, WeightPtrs ptrs, const float *part, int64_t unit0, int keys, int R) {
  const int u = blockIdx.x, layer = blockIdx.z;
  const PCache c = tab.c[layer];
  const WinLayer l = tab.l[layer];
  const int len = head_rows(s, c, u), count = max(l.count[u], 0);
  for (int j = a.block0 * keys + blockIdx.y * 256 + threadIdx.x; j < len && j < a.stride; j += gridDim.y * 256) {
    const int id = page_at(s, c, u, j >> s.lp);
    if (id < 0) continue;
    const int kA = j / keys * keys;
    const Rows rows = rows_that_see(s, a.w, len, count, kA, min(kA + keys, len));
    const bool fresh = j >= len - count;
    if (rows.i0 >= rows.i1 && !fresh) continue;
    float *w = ptrs.w[layer] + ((int64_t)id << s.lp) + (j & (s.P - 1));
    float x = fresh ? 0.f : *w, sum = 0.f;
    if (rows.i0 < rows.i1) {
      const float *p = part + (unit0 + (int64_t)layer * s.units_per_layer + u) * a.nchunks * a.stride + j;
      const int n = (rows.i1 - 1 - (rows.i0 & -R)) / chunk_rows(a, rows, R) + 1;
      for (int k = 0; k < n; ++k) sum += p[k * a.stride];
    }
    *w = x + sum;
  }
}

// Chunks of the rows that see a block of keys: sixteen turns, fewer (of at least 512 rows) where that makes less than four workgroups to a compute unit, more where it makes over thirty-two (of
// which a causal prompt leaves half empty).  Two prompts, window 8192: 15 turns 1.18 ms, 28 turns 1.22.  Blocks of first keys, which every row sees, are a launch of their own where the other blocks' chunks would be more than twice as long with their rows (two prompts of up to
// 2970 rows in a window of 19, one first row: 64 us, in the other blocks' two chunks 335).  That launch has at most 256 chunks a block and 2^16 workgroups in all, layers together: a compute
// unit's 256 fill it whatever their lengths, and the sums of its chunks stay below 128 MiB, where many short sequences stand beside one long prompt.  Returns the number of launches.
static int many_config(const PShape &s, const PWindow &w, int n_layers, int max_rows, ManyShape (&out)[2]) {
  ManyShape a{};
  a.w = w;
  const int64_t R = many_rows(s.q4 != 0), keys = many_keys(s.q4 != 0), blocks = ((int64_t)max_rows + keys - 1) / keys, units = (int64_t)n_layers * s.units_per_layer;
  const int64_t firsts = std::min(blocks, (w.first + keys - 1) / keys), all = (int64_t)w.max_count * s.G;
  const int64_t rows = firsts == blocks ? all : std::min<int64_t>(w.max_count, (int64_t)w.window + keys) * s.G;
  a.stride = blocks * keys;
  const int64_t work = rows * std::min<int64_t>(blocks * units, 8192), chunk = std::max<int64_t>(std::max<int64_t>(std::min<int64_t>(std::max<int64_t>(work / 1024, 512), 16 * R), work / 8192), rows * units >> 20);
  a.chunk = (int)((std::min(chunk, rows) + R - 1) / R * R);
  a.nchunks = (int)((rows + a.chunk - 1) / a.chunk);
  a.end = INT32_MAX;
  a.blocks = (int)std::min<int64_t>(blocks, 65535);
  out[0] = a;
  if (firsts == 0 || firsts == blocks || (all + 2 * (int64_t)a.chunk - 1) / (2 * (int64_t)a.chunk) <= a.nchunks) return 1;
  const int first_chunks = (int)std::min<int64_t>((all + a.chunk - 1) / a.chunk, std::min<int64_t>(256, 65536 / (units * firsts)));
  if (first_chunks <= a.nchunks) return 1;
  out[0].block0 = (int)firsts;
  out[0].blocks = (int)std::min<int64_t>(blocks - firsts, 65535);
  a.nchunks = first_chunks;
  a.end = (int)firsts;
  a.blocks = (int)std::min<int64_t>(firsts, 65535);
  a.stride = firsts * keys;
  out[1] = a;
  return 2;
}
// Rows of a unit are counted in 32 bits; a chunk that a block does not have begins up to a unit's rows behind the block's first one, and a turn ends behind the last.
static mixkv_status make_weights_window(const PShape &s, int n_rows, int window, int first, int max_count, int max_rows, PWindow *w) {
  const mixkv_status st = make_window(s, n_rows, window, first, max_count, max_rows, w);
  return st == MIXKV_OK && (int64_t)n_rows * s.hq > 1 << 30 ? MIXKV_ERR_UNSUPPORTED : st;
}

static size_t many_bytes(const PShape &s, const ManyShape &a, int n_layers) {
  return a.nchunks == 1 ? 0 : (size_t)n_layers * s.units_per_layer * a.nchunks * a.stride * sizeof(float);
}
static size_t many_bytes(const PShape &s, const ManyShape (&a)[2], int n, int n_layers) { return many_bytes(s, a[0], n_layers) + (n > 1 ? many_bytes(s, a[1], n_layers) : 0); }

// Tiles of a workgroup: as many workgroups as four to a compute unit take, a tile to a wave at least; a launch has at most 65535 along a head, and fewer than
// 2^32 threads.
static int step_tiles(const PShape &s, int nl, int64_t tiles) {
  const int64_t units = (int64_t)s.units_per_layer * nl;
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(65535, ((int64_t)1 << 23) / units));
  const int64_t ct = std::max<int64_t>(std::max<int64_t>(4, std::min<int64_t>((tiles * units + 1023) / 1024, 16)), (tiles + most - 1) / most);
  return (int)((std::min(ct, tiles) + 3) / 4 * 4);
}

}  // namespace mixkv

extern "C" mixkv_status mixkv_paged_weights_workspace_size(const mixkv_paged_params *params, int32_t n_layers, int32_t n_rows, int32_t window, int32_t keep_first,
                                                           int32_t max_count, int32_t max_rows, size_t *bytes) {
  using namespace mixkv;
  PShape s;
  PWindow w;
  mixkv_status st = make_pshape(params, &s);
  if (st != MIXKV_OK) return st;
  if ((st = make_weights_window(s, n_rows, window, keep_first, max_count, max_rows, &w)) != MIXKV_OK) return st;
  if (!bytes || n_layers < 1 || n_layers > MIXKV_MAX_LAYERS) return MIXKV_ERR_INVALID_ARG;
  max_rows = std::min(max_rows, s.max_pages * s.P);
  *bytes = 0;
  if (many_rows(s, params->dtype, w)) {
    ManyShape a[2];
    const int n = many_config(s, w, n_layers, max_rows, a);
    *bytes = (many_bytes(s, a, n, n_layers) + 255) / 256 * 256;
  }
  return MIXKV_OK;
}

extern "C" mixkv_status mixkv_paged_weights(const mixkv_paged_params *params, const mixkv_paged_cache *caches, const mixkv_paged_queries *queries, float *const *weights,
                                            int32_t n_layers, int32_t n_rows, int32_t window, int32_t keep_first, int32_t max_count, int32_t max_rows,
                                            void *workspace, size_t workspace_bytes, void *hip_stream) {
  using namespace mixkv;
  PShape s;
  PWindow w;
  mixkv_status st = make_pshape(params, &s);
  if (st != MIXKV_OK) return st;
  if ((st = make_weights_window(s, n_rows, window, keep_first, max_count, max_rows, &w)) != MIXKV_OK) return st;
  if ((st = check_caches(caches, n_layers, false, false)) != MIXKV_OK) return st;
  const int eb = params->dtype == MIXKV_BF16 ? 2 : 4;
  if ((st = check_queries(s, eb, queries, n_layers, n_rows, false)) != MIXKV_OK) return st;
  if (!weights) return MIXKV_ERR_INVALID_ARG;
  for (int l = 0; l < n_layers; ++l)
    if (!caches[l].K_pages || !weights[l] || misaligned(weights[l], 16)) return MIXKV_ERR_INVALID_ARG;
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  max_rows = std::min(max_rows, s.max_pages * s.P);
  const bool many = many_rows(s, params->dtype, w);
  ManyShape many_shapes[2] = {};
  const int launches = many ? many_config(s, w, n_layers, max_rows, many_shapes) : 0;
  const size_t need = many ? many_bytes(s, many_shapes, launches, n_layers) : 0;
  if (need > 0) {
    if (!workspace || misaligned(workspace, 256)) return MIXKV_ERR_INVALID_ARG;
    if (workspace_bytes < need) return MIXKV_ERR_WORKSPACE_TOO_SMALL;
  }
  // many rows: a launch has fewer than 2^32 threads
  int per = kLayersPerLaunch;
  for (int i = 0; i < launches; ++i) {
    ManyShape &a = many_shapes[i];
    const int64_t fit = std::max<int64_t>(1, ((int64_t)1 << 22) / ((int64_t)s.units_per_layer * a.nchunks + 1));
    a.blocks = (int)std::min<int64_t>(a.blocks, fit);
    per = (int)std::min<int64_t>(per, std::max<int64_t>(1, fit / a.blocks));
  }
  for (int l0 = 0; l0 < n_layers; l0 += per) {
    const int nl = std::min(n_layers - l0, per);
    const int64_t unit0 = (int64_t)l0 * s.units_per_layer;
    const WinTable t = window_table(caches + l0, queries + l0, nl, eb);
    WeightPtrs p{};
    for (int l = 0; l < nl; ++l) p.w[l] = weights[l0 + l];
    if (many) {
      float *part = static_cast<float *>(workspace);
      for (int i = 0; i < launches; ++i) {
        const ManyShape &a = many_shapes[i];
        const dim3 grid((unsigned)(s.units_per_layer * a.nchunks), (unsigned)a.blocks, (unsigned)nl);
        auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(64 * kManyWaves), 0, stream, s, a, t, p, part, unit0); };
        if (s.q4) { if (s.D == 128) go(weights_many_kernel<128, true>); else go(weights_many_kernel<64, true>); }
        else { if (s.D == 128) go(weights_many_kernel<128, false>); else go(weights_many_kernel<64, false>); }
        if (a.nchunks > 1) {
          const int64_t y = std::min<int64_t>((a.stride + 255) / 256, std::max<int64_t>(1, std::min<int64_t>(65535, ((int64_t)1 << 23) / ((int64_t)s.units_per_layer * nl))));
          hipLaunchKernelGGL(weights_fold_kernel, dim3((unsigned)s.units_per_layer, (unsigned)y, (unsigned)nl), dim3(256), 0, stream, s, a, t, p, (const float *)part, unit0,
                             many_keys(s.q4 != 0), many_rows(s.q4 != 0));
        }
        part += many_bytes(s, a, n_layers) / sizeof(float);
      }
      if (hipGetLastError() != hipSuccess) return MIXKV_ERR_HIP;
      continue;
    }
    const int64_t tiles = most_tiles(s, w, max_rows, (int)std::min<int64_t>((int64_t)w.max_count * s.G, INT32_MAX / 2));
    const int ctiles = step_tiles(s, nl, tiles);
    const dim3 grid((unsigned)s.units_per_layer, (unsigned)((tiles + ctiles - 1) / ctiles), (unsigned)nl);
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, stream, s, w, t, p, ctiles); };
    if (s.q4) { if (s.D == 128) go(weights_step_kernel<MIXKV_BF16, 128, true>); else go(weights_step_kernel<MIXKV_BF16, 64, true>); }
    else if (params->dtype == MIXKV_BF16) { if (s.D == 128) go(weights_step_kernel<MIXKV_BF16, 128, false>); else go(weights_step_kernel<MIXKV_BF16, 64, false>); }
    else if ((int64_t)w.max_count * s.G <= 16) { if (s.D == 128) go(weights_step_kernel<MIXKV_F32, 128, false>); else go(weights_step_kernel<MIXKV_F32, 64, false>); }
    else { if (s.D == 128) go(weights_step_kernel<MIXKV_F32, 128, false, true>); else go(weights_step_kernel<MIXKV_F32, 64, false, true>); }
    if (hipGetLastError() != hipSuccess) return MIXKV_ERR_HIP;
  }
  return MIXKV_OK;
}
