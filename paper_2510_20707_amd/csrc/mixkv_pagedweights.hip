// The attention that cached rows have been given (mixkv_paged_weights): column sums of the new rows' attention weights, from their log-sum-exp.
//
// With a row's normaliser known, a key's sum needs no running softmax: exp2(x c - lse), one multiply-add and one exponential an element, and no other
// key.  A tile of 32 keys belongs to one wave, which goes through the rows that see it: no atomics, and the order of a sum is that of the rows.
#include "mixkv_pagedwin.h"

namespace mixkv {

struct WeightPtrs { float *w[kLayersPerLaunch]; };

constexpr int kSumRun = 64;              // steps of 16 rows whose weights are summed up on their own: 2^17 rows are then off by some 2^-18 at most

// bf16 bits to fp16, times 2^up.
__device__ __forceinline__ _Float16 scaled_half(uint32_t bits, int up) { return (_Float16)ldexpf(__uint_as_float(bits), up); }

// ------------------------------------------------------------------------------------------------
// weights_step_kernel (few rows): a wave to tiles of 32 keys, rows on the output rows of 16 x 16 products, keys on their columns, so that a lane has
// two keys and their sums over four rows each.  With up to 16 rows in all (a step's single tokens) the queries are prepared once.
// 4-bit keys as in paged_q4_kernel: codes as fp16 subnormals, a product for each group of 32 elements, steps and bases behind it in fp32.
// ------------------------------------------------------------------------------------------------
template <int DT, int D, bool Q4>
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
  const int t0 = blockIdx.y * ctiles, t1 = blockIdx.y + 1 == gridDim.y ? all : min(all, t0 + ctiles);
  if (t0 >= t1) return;

  // ---- 16 rows: their queries, and of the rows 4 quad + e the normalisers and places
  u32x4 qf[Q4 ? NG : NC];
  f16x8 qs;
  float off[4], c2[4];
  int place[4];
  auto rows_from = [&](int i0, int i1) {
    {
      const int i = min(i0 + l16, i1 - 1), t = i / s.G, g = i - t * s.G;
      const int64_t row = min(max((int64_t)start + t, (int64_t)0), (int64_t)win.n_rows - 1);
      const char *q = l.Q + row * l.qsn + (int64_t)(h * s.G + g) * l.qsh;
      if constexpr (!Q4) {
#pragma unroll
        for (int k = 0; k < NC; ++k) qf[k] = *reinterpret_cast<const u32x4 *>(q + (4 * k + quad) * 16);
      } else {
        // to fp16, by a power of two that brings the row's largest element to [2^13, 2^14); their sums over each group in two parts, against a key's (S, B) pairs
        u32x4 qr[NG];
        uint32_t most = 0;
#pragma unroll
        for (int pl = 0; pl < NG; ++pl) {
          qr[pl] = *reinterpret_cast<const u32x4 *>(q + (32 * (D == 128 ? (pl & 1) * 2 + (pl >> 1) : pl) + 8 * quad) * 2);
#pragma unroll
          for (int j = 0; j < 4; ++j) most = max(most, max(qr[pl][j] & 0x7fffu, (qr[pl][j] >> 16) & 0x7fffu));
        }
        most = max(most, (uint32_t)__shfl_xor((int)most, 16));
        most = max(most, (uint32_t)__shfl_xor((int)most, 32));
        const int up = 13 - (min(max((int)(most >> 7), 1), 254) - 127);
        const float back = fminf(fmaxf(ldexpf(s.scale_log2e, 20 - up), 0x1p-126f), 0x1p100f);   // (as in paged_q4_kernel: neither zero nor infinite)
#pragma unroll
        for (int e = 0; e < 4; ++e) c2[e] = __shfl(back, 4 * quad + e);
        float hi[NG], lo[NG];
#pragma unroll
        for (int pl = 0; pl < NG; ++pl) {
          float sum = 0.f;
          f16x8 x;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t w = qr[pl][e >> 1];
            const float v = ldexpf(__uint_as_float(e & 1 ? w & 0xffff0000u : w << 16), up);
            sum += v;
            x[e] = (_Float16)((e >> 1) & 1 ? v * 0.0625f : v);
          }
          qf[pl] = __builtin_bit_cast(u32x4, x);
          sum += __shfl_xor(sum, 16);
          sum += __shfl_xor(sum, 32);
          sum *= 0.00390625f;
          hi[pl] = (float)(_Float16)sum;
          lo[pl] = sum - hi[pl];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) qs[e] = (_Float16)(e / 2 < NG ? (quad == 0 ? hi[e / 2 % NG] : (quad == 1 ? lo[e / 2 % NG] : 0.f)) : 0.f);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = i0 + 4 * quad + e, t = min(i, i1 - 1) / s.G, g = min(i, i1 - 1) - t * s.G;
      const int64_t row = (int64_t)start + t;
      const bool there = i < i1 && row >= 0 && row < win.n_rows;
      const float lse = l.lse[(there ? row : 0) * s.hq + h * s.G + g];
      off[e] = lse * -1.44269504088896340736f;
      place[e] = there && lse != -INFINITY ? place0 + t : -1;           // -1: the row gives nothing
    }
  };
  const bool once = (int64_t)served * s.G <= 16;
  if (once && served > 0) rows_from(0, served * s.G);

  for (int first = t0 + wave; first < t1; first += 64 * W) {
    // lane i: where the wave's i-th tile of 64 lies
    const int mine = first + lane * W;
    const int id_of = mine < t1 ? page_at(s, c, u, mine >> (s.lp - 5)) : -1;
    const int n = min((t1 - first + W - 1) / W, 64);
    u32x4 kr[2][NK];
    float old = 0.f;
    auto request = [&](int i) {
      const int id = max(__builtin_amdgcn_readlane(id_of, i), 0), row0 = (first + i * W) * 32 & (s.P - 1);
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
      const int tile = first + i * W, k0 = tile * 32, live = min(len - k0, 32), id = __builtin_amdgcn_readlane(id_of, i);
      const float was = old;
      // new rows [lo, hi) see some of the tile's keys
      const int lo = max(k0 - place0, 0), hi = k0 < win.first ? served : (int)min((int64_t)served, (int64_t)k0 + 31 + win.window - place0);
      const bool work = id >= 0 && lo < hi;
      float sum[2] = {0.f, 0.f}, run[2] = {0.f, 0.f};
      int steps = 0;
      const int i1 = work ? (once ? served : hi) * s.G : 0;
      for (int i0 = once ? 0 : lo * s.G; i0 < i1; i0 += 16) {
        if (!once) rows_from(i0, i1);
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
          } else {
#pragma unroll
            for (int k = 0; k < NC; ++k) {
              if constexpr (F32) {
#pragma unroll
                for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(qf[k][e]), __uint_as_float(kr[r][k][e]), x, 0, 0, 0);
              } else {
                x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, qf[k]), __builtin_bit_cast(bf16x8, kr[r][k]), x, 0, 0, 0);
              }
            }
          }
          const int j = k0 + 16 * r + l16;
#pragma unroll
          for (int e = 0; e < 4; ++e) run[r] += sees(win, place[e], j) ? fast_exp2(fmaf(x[e], Q4 ? c2[e] : s.scale_log2e, off[e])) : 0.f;
        }
        if (++steps == kSumRun) {
          steps = 0;
#pragma unroll
          for (int r = 0; r < 2; ++r) { sum[r] += run[r]; run[r] = 0.f; }
        }
      }
      if (i + 1 < n) request(i + 1);
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

// Tiles of a workgroup: as many workgroups as four to a compute unit take, a tile to a wave at least; a launch has at most 65535 along a head, and fewer than
// 2^32 threads.
static int step_tiles(const PShape &s, int nl, int max_rows) {
  const int64_t tiles = ((int64_t)max_rows + 31) / 32, units = (int64_t)s.units_per_layer * nl;
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(65535, ((int64_t)1 << 23) / units));
  const int64_t ct = std::max<int64_t>(std::max<int64_t>(4, (tiles * units + 1023) / 1024), (tiles + most - 1) / most);
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
  if ((st = make_window(s, n_rows, window, keep_first, max_count, max_rows, &w)) != MIXKV_OK) return st;
  if (!bytes || n_layers < 1 || n_layers > MIXKV_MAX_LAYERS) return MIXKV_ERR_INVALID_ARG;
  *bytes = 0;
  return MIXKV_OK;
}

extern "C" mixkv_status mixkv_paged_weights(const mixkv_paged_params *params, const mixkv_paged_cache *caches, const mixkv_paged_queries *queries, float *const *weights,
                                            int32_t n_layers, int32_t n_rows, int32_t window, int32_t keep_first, int32_t max_count, int32_t max_rows,
                                            void *workspace, size_t workspace_bytes, void *hip_stream) {
  using namespace mixkv;
  (void)workspace; (void)workspace_bytes;
  PShape s;
  PWindow w;
  mixkv_status st = make_pshape(params, &s);
  if (st != MIXKV_OK) return st;
  if ((st = make_window(s, n_rows, window, keep_first, max_count, max_rows, &w)) != MIXKV_OK) return st;
  if ((st = check_caches(caches, n_layers, false, false)) != MIXKV_OK) return st;
  const int eb = params->dtype == MIXKV_BF16 ? 2 : 4;
  if ((st = check_queries(s, eb, queries, n_layers, n_rows, false)) != MIXKV_OK) return st;
  if (!weights) return MIXKV_ERR_INVALID_ARG;
  for (int l = 0; l < n_layers; ++l)
    if (!caches[l].K_pages || !weights[l] || misaligned(weights[l], 16)) return MIXKV_ERR_INVALID_ARG;
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  max_rows = std::min(max_rows, s.max_pages * s.P);
  for (int l0 = 0; l0 < n_layers; l0 += kLayersPerLaunch) {
    const int nl = std::min(n_layers - l0, kLayersPerLaunch);
    const WinTable t = window_table(caches + l0, queries + l0, nl, eb);
    WeightPtrs p{};
    for (int l = 0; l < nl; ++l) p.w[l] = weights[l0 + l];
    const int ctiles = step_tiles(s, nl, max_rows);
    const dim3 grid((unsigned)s.units_per_layer, (unsigned)(((int64_t)max_rows + 32 * ctiles - 1) / (32 * ctiles)), (unsigned)nl);
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, stream, s, w, t, p, ctiles); };
    if (s.q4) { if (s.D == 128) go(weights_step_kernel<MIXKV_BF16, 128, true>); else go(weights_step_kernel<MIXKV_BF16, 64, true>); }
    else if (params->dtype == MIXKV_BF16) { if (s.D == 128) go(weights_step_kernel<MIXKV_BF16, 128, false>); else go(weights_step_kernel<MIXKV_BF16, 64, false>); }
    else { if (s.D == 128) go(weights_step_kernel<MIXKV_F32, 128, false>); else go(weights_step_kernel<MIXKV_F32, 64, false>); }
    if (hipGetLastError() != hipSuccess) return MIXKV_ERR_HIP;
  }
  return MIXKV_OK;
}
