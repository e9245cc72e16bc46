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
__device__ __forceinline__ int head_tiles(const PShape &s, const AShape &a, const AttnLayer &l, int u, int len) {
  if (a.keep == 0) return (len + 31) >> 5;
  return min(max(l.nsel[u], 0), a.keep) << (s.lp - 5);
}
// The table entry of tile t (any number >= 0), and its place in the table.  No length is needed.  (The optional list makes a branch, before which the compiler waits for
// what was asked for earlier: in both kernels entry and length are asked for once the queries are there.)
__device__ __forceinline__ int tile_entry(const PShape &s, const AShape &a, const PCache &c, const AttnLayer &l, int u, int t, int &place) {
  place = t >> (s.lp - 5);
  if (a.keep) place = l.sel[(int64_t)u * a.keep + min(place, a.keep - 1)];
  return c.table[(int64_t)u * s.max_pages + min(max(place, 0), s.max_pages - 1)];
}
struct Tile { int page, row, live; };
__device__ __forceinline__ Tile tile_of_entry(const PShape &s, int len, int t, int place, int entry) {
  Tile x;
  x.row = (t & ((1 << (s.lp - 5)) - 1)) * 32;
  const bool on = (uint32_t)place < (uint32_t)s.max_pages && (uint32_t)entry < (uint32_t)s.n_pages;
  x.page = on ? entry : 0;
  x.live = on ? min(max(len - ((place << s.lp) + x.row), 0), 32) : 0;
  return x;
}
// The first tile of chunk `ch`, which may lie behind the head's last, and the end of the chunk.
__device__ __forceinline__ int chunk_end(const AShape &a, int tiles, int ch) { return ch == a.nchunks - 1 ? tiles : min(tiles, (ch + 1) * a.ctiles); }
__device__ __forceinline__ int chunks_used(const AShape &a, int tiles) { return min(a.nchunks, (int)(((uint32_t)tiles + a.ctiles - 1) / (uint32_t)a.ctiles)); }

// A weighted sum over its sum of weights; no rows give zeros, a NaN stays one.
__device__ __forceinline__ float row_result(float acc, float tot) { return tot == 0.f ? 0.f : acc / tot; }

// The first partial row of a chunk.
__device__ __forceinline__ int64_t slot_of(const PShape &s, const AShape &a, int64_t unit0, int layer, int u, int gc, int ch) {
  return (((unit0 + layer * s.units_per_layer + u) * a.gchunks + gc) * a.nchunks + ch) * a.gt;
}

// The workgroup's end: folds the waves' shares in order (o_s of head g holds element d at d ^ g) and writes the rows, or the chunk's partial:
// weighted values in `part`, offset and sum in `part_ml`.
template <int DT, int D>
__device__ __forceinline__ void finish_chunk(const PShape &s, const AShape &a, const AttnLayer &l, float (&o_s)[4][kAttnHeads][D], float (&m_s)[4][kAttnHeads],
                                             float (&l_s)[4][kAttnHeads], float *part, float *part_ml, int64_t slot, int64_t q0, int ng, bool whole) {
  __syncthreads();
  for (int idx = threadIdx.x; idx < ng * D; idx += 256) {
    const int g = idx / D, d = idx - g * D;
    float mn = m_s[0][g];
#pragma unroll
    for (int w = 1; w < 4; ++w) mn = fmaxf(mn, m_s[w][g]);
    const float mu = mn == -INFINITY ? 0.f : mn;
    float acc = 0.f, tot = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = fast_exp2(m_s[w][g] - mu);
      acc = fmaf(o_s[w][g][d ^ g], f, acc);
      tot = fmaf(l_s[w][g], f, tot);
    }
    if (!whole) {
      part[(slot + g) * D + d] = acc;
      if (d == 0) reinterpret_cast<float2 *>(part_ml)[slot + g] = make_float2(mn, tot);
      continue;
    }
    const float res = row_result(acc, tot);
    if constexpr (DT == MIXKV_BF16) reinterpret_cast<uint16_t *>(l.out)[(q0 + g) * D + d] = f32_to_bf16_rne(res);
    else reinterpret_cast<float *>(l.out)[(q0 + g) * D + d] = res;
  }
}

// ------------------------------------------------------------------------------------------------
// paged_q4_kernel (4-bit pages): a workgroup of four waves, every wave on 32-row tiles of its own, which travel through a ring of its
// own in LDS (direct loads, the next tiles on their way while one is worked on; no barrier before the end).
//   * Scores: query heads on the output rows, keys on the columns of a 16 x 16 x 32 fp16 product for each group of 32 elements.  A word's codes,
//     masked in place, are fp16 subnormals, code 2^-24 and, one nibble up, code 2^-20 (the queries of those elements are taken by 16 less): no
//     conversion, exact products.  Queries are brought to [2^13, 2^14) by a power of two per head, which makes bf16 exact in fp16 down to
//     2^-26 of the largest, smaller ones off by at most 2^-34 of it.  With acc_g = sum q code of group g and element = B + S + S code / 16, a score is
//     sum_g S_g acc_g / 16 + sum_g (B_g + S_g) sum(q_g): four multiply-adds, and one product of the key's raw (S, B) pairs with the sums of
//     the queries in two fp16 parts.
//   * Weights as fp16 through the wave's LDS image (head, key): a lane holds two keys 16 rows apart, a word of the image.
//   * Values: a word of a page holds eight rows' codes of one element, an operand of the second product: the code on top of the mantissa of
//     1.0 is u = 1 + code / 16, and B + S u a packed fp16 multiply-add with the strip's scales.  Fp16 rounds weights and values by 2^-11, an
//     eighth of the output's own rounding; both are averaged over the rows: 1.681e-3 off from 64 bits (2-norms, 64 sequences of up to 16 384 rows), where the
//     output's rounding alone is 1.664e-3.  That is what this costs to avoid: with the codes as exact operands and the products of weights and steps in two bf16
//     parts, the bases by a product of their own, 1.664e-3 in 177 us instead of 138 (the vector unit then bounds it).  The weights are relative to an offset that puts the
//     largest near 2^8: fp16 then resolves weights down to 2^-32 of it.
// Bound: memory for long heads: 64 sequences of 8192 rows, 8 heads of 128, 671 MB in 114 us, 5.9 TB/s, and the merge behind it; for
// few rows the workgroup's own beginning and end (4 heads of 260 rows: 7.8 us).
// ------------------------------------------------------------------------------------------------
// Images of a wave's ring and waves per SIMD, as LDS holds them; us for 64 sequences of 8192 rows, 8 heads of 128: 2 and 3 125, 3 and 2 139.
constexpr int kQ4Ring = 2, kQ4Waves = 3;
constexpr float kTopWeight = 8.f, kWeightLimit = 16384.f;     // log2 of the largest weight where an offset is chosen; where it moves

// Over the 16 lanes of a row, in every one of them: rotations in the vector ALU.
template <int CTRL>
__device__ __forceinline__ float row_turned(float x) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true)); }
__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, row_turned<0x128>(x));                         // row_ror:8, 4, 2, 1
  x = fmaxf(x, row_turned<0x124>(x));
  x = fmaxf(x, row_turned<0x122>(x));
  return fmaxf(x, row_turned<0x121>(x));
}
__device__ __forceinline__ float row_sum(float x) {
  x += row_turned<0x128>(x);
  x += row_turned<0x124>(x);
  x += row_turned<0x122>(x);
  return x + row_turned<0x121>(x);
}

template <int D, bool ONCE>
__global__ __launch_bounds__(256, kQ4Waves) void paged_q4_kernel(PShape s, AShape a, AttnTable tab, float *part, float *part_ml, int64_t unit0) {
  constexpr int NG = D / 32, NB = D / 16, H = kAttnHeads, W = 4;
  constexpr int CODES = 16 * D, SCALES = 32 * NG * 4, TILE = 2 * (CODES + SCALES);   // bytes of a tile: keys' codes, values', keys' scales, values'
  constexpr int NL = CODES / 1024, LOADS = 2 * NL + 1, RING = kQ4Ring;
  constexpr int PROW = 20;                                    // words of an image row of weights, padded
  struct Share { float o[W][H][D]; };
  struct Work { uint4 ring[W * RING * TILE / 16]; uint32_t p[W][H * PROW]; };
  __shared__ union { Share share; Work work; } sh;
  __shared__ float m_s[W][H], l_s[W][H];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int u = blockIdx.x, ch = blockIdx.y, layer = blockIdx.z / a.gchunks, gc = blockIdx.z - layer * a.gchunks;
  const int b = u / s.hkv, h = u - b * s.hkv, ng = min(H, s.G - gc * H);
  const PCache c = tab.c[layer];
  const AttnLayer l = tab.l[layer];
  const int64_t q0 = (int64_t)b * s.hq + h * s.G + gc * H;   // first query row
  // group of the words at place g' of a key row, and the queries in that order: lane (head, quad) holds elements 8 quad + e of the group
  auto group_at = [](int pl) { return D == 128 ? (pl & 1) * 2 + (pl >> 1) : pl; };
  u32x4 qr[NG];
#pragma unroll
  for (int pl = 0; pl < NG; ++pl)
    qr[pl] = *reinterpret_cast<const u32x4 *>(l.Q + ((q0 + (l16 < ng ? l16 : 0)) * D + 32 * group_at(pl) + 8 * quad) * 2);
  const int t0 = ch * a.ctiles;
  int place, entry = tile_entry(s, a, c, l, u, t0 + wave + lane * W, place);
  const int len = head_rows(s, c, u), tiles = head_tiles(s, a, l, u, len), t1 = chunk_end(a, tiles, ch);
  if (t0 >= t1 && ch > 0) return;
  const int codes = s.P * D / 2;                             // bytes of codes in front of a page's scales
  const char *ring = reinterpret_cast<const char *>(sh.work.ring) + wave * (RING * TILE);
  const uint32_t ring_a = lds_base_of(sh.work.ring) + wave * (RING * TILE);
  uint32_t *p_img = sh.work.p[wave];
  // what the lane fetches of a tile: a key row's four pieces lie rotated in the image by the row's number, so that 16 rows are read at once
  // without conflict; the scales' 16-byte pieces are the keys' in the first half of the load, the values' in the second
  constexpr int PPR = D / 32;                                 // 16-byte pieces of a key row's codes
  const int krow = lane / PPR, kpiece = D == 128 ? (lane & 3) ^ ((krow >> 2) & 3) : lane % PPR;
  const uint32_t k_off = krow * (D / 2) + kpiece * 16;
  const bool s_keys = lane < SCALES / 16;
  const uint32_t s_off = codes + (s_keys ? lane : lane - SCALES / 16) * 16;
  int x_page = 0, x_rows = 0, n = 0;                           // lane i: where the wave's i-th tile of a batch of 64 lies; tiles of the batch
  auto batch = [&](int first) {                                // from the lanes' table entries
    const Tile x = tile_of_entry(s, len, first + lane * W, place, entry);
    x_page = x.page;
    x_rows = x.row | (x.live << 8);
    n = min(max((t1 - first + W - 1) / W, 0), 64);
  };
  // tile i into its image
  auto request = [&](int i, uint32_t img) {
    const int64_t page = (int64_t)__builtin_amdgcn_readlane(x_page, i) * s.page_bytes;
    const int row = __builtin_amdgcn_readlane(x_rows, i) & 255;
    const char *kp = c.K + page, *vp = c.V + page;
#pragma unroll
    for (int j = 0; j < NL; ++j) load_to_lds<ONCE>(kp + (uint32_t)(row * (D / 2)) + (k_off + j * 1024), img + j * 1024);
#pragma unroll
    for (int j = 0; j < NL; ++j) load_to_lds<ONCE>(vp + (uint32_t)(row * (D / 2)) + (uint32_t)(lane * 16 + j * 1024), img + CODES + j * 1024);
    const char *sp = (s_keys ? kp : vp) + (uint32_t)(row * NG * 4) + s_off;
    if (2 * SCALES / 16 == 64 || lane < 2 * SCALES / 16) load_to_lds<ONCE>(sp, img + 2 * CODES);
  };
  auto begin = [&](int first) {                                // the batch's first tiles on their way
    batch(first);
    wait_vm<0>();                                              // the loop counts its own requests
#pragma unroll
    for (int i = 0; i < RING - 1; ++i)
      if (i < n) request(i, ring_a + i * TILE);
  };
  begin(t0 + wave);

  // ---- the queries: to fp16, by a power of two per head; their sums over each group, in two parts, against a key's (S, B) pairs
  f16x8 qf[NG], qs;
  float c2[4];                                                 // heads 4 quad + e: what brings a score, times 2^-24 2^k, to the exponent of 2
  {
    uint32_t most = 0;
#pragma unroll
    for (int pl = 0; pl < NG; ++pl)
#pragma unroll
      for (int j = 0; j < 4; ++j) most = max(most, max(qr[pl][j] & 0x7fffu, (qr[pl][j] >> 16) & 0x7fffu));
    most = max(most, (uint32_t)__shfl_xor((int)most, 16));
    most = max(most, (uint32_t)__shfl_xor((int)most, 32));
    const int ex = min(max((int)(most >> 7), 1), 254) - 127, sh2 = l16 < ng ? 13 - ex : 0;   // 2^ex <= the largest < 2^(ex + 1); NaN and infinities stay what they are
    // (Between 2^-126 and 2^100: a factor of zero or infinity would make NaNs of rows that do not exist or of scores of zero.  Below, the scores, under 2^18
    // here, make no difference to a weight; above, any score but zero, at least 2^-72, is a logit of 2^28 or more.)
    const float back = fminf(fmaxf(ldexpf(s.scale_log2e, 20 - sh2), 0x1p-126f), 0x1p100f);
#pragma unroll
    for (int e = 0; e < 4; ++e) c2[e] = __shfl(back, 4 * quad + e);
    float hi[NG], lo[NG];
#pragma unroll
    for (int pl = 0; pl < NG; ++pl) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t w = qr[pl][e >> 1];
        float q = ldexpf(__uint_as_float(e & 1 ? w & 0xffff0000u : w << 16), sh2);
        if (l16 >= ng) q = 0.f;                                // heads past the group are zero rows
        sum += q;
        qf[pl][e] = (_Float16)((e >> 1) & 1 ? q * 0.0625f : q);
      }
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      sum *= 0.00390625f;                                      // at most 32 2^14 2^-8
      hi[pl] = (float)(_Float16)sum;
      lo[pl] = sum - hi[pl];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) qs[e] = (_Float16)(e / 2 < NG ? (quad == 0 ? hi[e / 2 % NG] : (quad == 1 ? lo[e / 2 % NG] : 0.f)) : 0.f);
  }
  uint32_t one_f16;                                            // an and-or takes one scalar constant: the other one is kept in a register
  asm("v_mov_b32 %0, 0x3c003c00" : "=v"(one_f16));

  f32x4 o[NB];
  float nm[4] = {0.f, 0.f, 0.f, 0.f}, ls[4] = {0.f, 0.f, 0.f, 0.f};   // minus the offsets of heads 4 quad + i (0: none yet), sums of weights
  bool has[4] = {false, false, false, false};
#pragma unroll
  for (int i = 0; i < NB; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  bool fresh = true;                                           // some head has no offset yet

  for (int first = t0 + wave; first < t1; first += 64 * W) {
    if (first != t0 + wave) {
      entry = tile_entry(s, a, c, l, u, first + lane * W, place);
      begin(first);
    }
    int slot = 0;
    for (int i = 0; i < n; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      {
        const int to = slot == 0 ? RING - 1 : slot - 1;        // the image that tile i - 1 has left
        if (i + RING - 1 < n) {
          request(i + RING - 1, ring_a + to * TILE);
          wait_vm<(RING - 1) * LOADS>();
        } else {
          wait_vm<0>();
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      const char *img = ring + slot * TILE;
      const int live = __builtin_amdgcn_readlane(x_rows, i) >> 8;
      if (live < 32) {                                         // the values' scales of rows that do not exist: zeros
        u32x4 *at = reinterpret_cast<u32x4 *>(const_cast<char *>(img) + 2 * CODES + SCALES) + lane;
        if (lane < SCALES / 16) {
          const int q = lane / (2 * NG);
          u32x4 v = *at;
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] &= (4 * q + k < live ? 0xffffu : 0u) | (16 + 4 * q + k < live ? 0xffff0000u : 0u);
          *at = v;
        }
        wave_lds_fence();
      }
      slot = slot == RING - 1 ? 0 : slot + 1;
      // ---- scores of the keys l16 and 16 + l16 against the heads 4 quad + e, by 2^-24 2^k
      f32x4 acc[2][NG], x2[2];
      uint32_t ks[2][NG];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int row = 16 * r + l16;
        uint32_t kc[NG];
        u32x4 sb = {0u, 0u, 0u, 0u};
        if constexpr (NG == 4) {
          const u32x4 w = *reinterpret_cast<const u32x4 *>(img + row * 64 + (quad ^ ((row >> 2) & 3)) * 16);
          sb = *reinterpret_cast<const u32x4 *>(img + 2 * CODES + row * 16);
#pragma unroll
          for (int g = 0; g < 4; ++g) kc[g] = w[g];
        } else {
          const u32x2 w = *reinterpret_cast<const u32x2 *>(img + row * 32 + quad * 8), z = *reinterpret_cast<const u32x2 *>(img + 2 * CODES + row * 8);
#pragma unroll
          for (int g = 0; g < 2; ++g) { kc[g] = w[g]; sb[g] = z[g]; }
        }
        x2[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(qs, __builtin_bit_cast(f16x8, sb), f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
        for (int pl = 0; pl < NG; ++pl) {
          ks[r][pl] = sb[pl];
          const uint32_t w = kc[pl], w8 = w >> 8;
          const u32x4 k = {w & 0x000f000fu, w & 0x00f000f0u, w8 & 0x000f000fu, w8 & 0x00f000f0u};
          acc[r][pl] = __builtin_amdgcn_mfma_f32_16x16x32_f16(qf[pl], __builtin_bit_cast(f16x8, k), f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
        }
      }
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x = x2[r][e] * 0x1p-12f;                       // 2^8 2^-20
#pragma unroll
          for (int pl = 0; pl < NG; ++pl) x = fmaf((float)__builtin_bit_cast(f16x2, ks[r][pl])[0], acc[r][pl][e], x);
          x2[r][e] = x;
        }
      if (live < 32) {
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int e = 0; e < 4; ++e) x2[r][e] = 16 * r + l16 < live ? x2[r][e] : -INFINITY;
        asm volatile("" : "+v"(x2[0]), "+v"(x2[1]));           // a branch, not selects in every tile
      }
      // ---- weights; the offsets move where a head has none yet or a weight leaves fp16's range
      float p[2][4];
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) p[r][e] = fast_exp2(fmaf(x2[r][e], c2[e], nm[e]));
      const float top = fmaxf(fmaxf(fmaxf(p[0][0], p[0][1]), fmaxf(p[0][2], p[0][3])), fmaxf(fmaxf(p[1][0], p[1][1]), fmaxf(p[1][2], p[1][3])));
      if (fresh || __builtin_amdgcn_ballot_w64(!(top < kWeightLimit)) != 0) {
        fresh = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float t = fmaxf(x2[0][e], x2[1][e]);
          t = row_max(t);
          const float want = kTopWeight - t * c2[e];         // minus the offset that puts this tile's largest weight at 2^kTopWeight
          const bool move = t > -INFINITY && (!has[e] || want < nm[e]);
          const float f = move ? (has[e] ? fast_exp2(want - nm[e]) : 0.f) : 1.f;
          nm[e] = move ? want : nm[e];
          has[e] |= move;
          fresh |= !has[e];
          ls[e] *= f;
#pragma unroll
          for (int k = 0; k < NB; ++k) o[k][e] *= f;
#pragma unroll
          for (int r = 0; r < 2; ++r) p[r][e] = fast_exp2(fmaf(x2[r][e], c2[e], nm[e]));
        }
        fresh = __builtin_amdgcn_ballot_w64(fresh) != 0;
      }
      // ---- the image of the weights (head, key pair)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        ls[e] += p[0][e] + p[1][e];
        p_img[(4 * quad + e) * PROW + l16] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)p[0][e], (_Float16)p[1][e]});
      }
      wave_lds_fence();
      const f16x8 pw = __builtin_bit_cast(f16x8, *reinterpret_cast<const u32x4 *>(p_img + l16 * PROW + 4 * quad));
      // ---- weighted values
      const char *vimg = img + CODES + quad * (D * 4) + l16 * 16, *simg = img + 2 * CODES + SCALES + quad * (NG * 32);
      u32x4 vc = {};
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        if (g % 2 == 0) vc = *reinterpret_cast<const u32x4 *>(vimg + g / 2 * 256);
        const u32x4 st = *reinterpret_cast<const u32x4 *>(simg + g * 32), ba = *reinterpret_cast<const u32x4 *>(simg + g * 32 + 16);
#pragma unroll
        for (int hb = 0; hb < 2; ++hb) {
          const int blk = 2 * g + hb;
          const uint32_t w = vc[blk & 3];
          u32x4 v;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t un = ((j < 2 ? w << (6 - 4 * j) : w >> (4 * j - 6)) & 0x03c003c0u) | one_f16;
            const f16x2 val = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, un), __builtin_bit_cast(f16x2, (uint32_t)st[j]),
                                                        __builtin_bit_cast(f16x2, (uint32_t)ba[j]));
            v[j] = __builtin_bit_cast(uint32_t, val);
          }
          o[blk] = __builtin_amdgcn_mfma_f32_16x16x32_f16(pw, __builtin_bit_cast(f16x8, v), o[blk], 0, 0, 0);
        }
      }
      wave_lds_fence();
    }
  }

  // ---- the waves' shares: offsets, sums over the 16 keys of a lane row, weighted values of head 4 quad + e, element 16 k + l16
  __syncthreads();                                             // the shares take the rings' place
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    ls[e] = row_sum(ls[e]);
    if (l16 == 0) { m_s[wave][4 * quad + e] = has[e] ? -nm[e] : -INFINITY; l_s[wave][4 * quad + e] = ls[e]; }
#pragma unroll
    for (int k = 0; k < NB; ++k) sh.share.o[wave][4 * quad + e][(16 * k + l16) ^ (4 * quad + e)] = o[k][e];
  }
  finish_chunk<MIXKV_BF16, D>(s, a, l, sh.share.o, m_s, l_s, part, part_ml, slot_of(s, a, unit0, layer, u, gc, ch), q0, ng, chunks_used(a, tiles) <= 1);
}

// ------------------------------------------------------------------------------------------------
// paged_rows_kernel (full-precision pages): a workgroup of four waves, every wave on 32-row tiles of its own; keys come from memory into the
// operand of the first product (lane (key, quad): every fourth 16-byte piece of its row), keys on the output rows, so that a lane (head,
// quad) has its weights in the order in which they are the operand of the second.
//   bf16  weights as a bf16 head and remainder; values through the wave's LDS image, read transposed.
//   fp32  products of four elements' contraction; a lane takes four neighbouring elements of a value row at a time, which are four blocks'
//         operands, the blocks' rows then being every fourth element: no image.
// Offsets as in decode_mfma_kernel, with a limit of their own.
// Bound: memory, a tile of each wave in flight and not always whole: value loads are branches (rows that may not exist), so that a tile's values are waited for
// before its last score product, and the next tile's keys alone are on their way during the weights.  bf16, 16 sequences of 8192 rows, 8 heads of 128, 537 MB in 94 us, 5.7 TB/s.
// ------------------------------------------------------------------------------------------------
// A lane's sum of weights that reaches this moves the head's offset.  The weighted values stay below it times the largest value: values of up to 2^100
// do not overflow, whatever the logits behind them.
constexpr float kRowsSumLimit = 0x1p20f;

template <int DT, int D, bool ONCE>
__global__ __launch_bounds__(256) void paged_rows_kernel(PShape s, AShape a, AttnTable tab, float *part, float *part_ml, int64_t unit0) {
  constexpr bool F32 = DT == MIXKV_F32;
  constexpr int EB = F32 ? 4 : 2, RB = D * EB, PPR = RB / 16, NC = PPR / 4, NB = D / 16, H = kAttnHeads, W = 4;
  constexpr int NV = F32 ? 8 * (D / 64) : 32 * PPR / 64, RPL = 64 / PPR;     // 16-byte loads of a lane for a tile of values
  __shared__ float o_s[W][H][D];
  __shared__ float m_s[W][H], l_s[W][H];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int u = blockIdx.x, ch = blockIdx.y, layer = blockIdx.z / a.gchunks, gc = blockIdx.z - layer * a.gchunks;
  const int b = u / s.hkv, h = u - b * s.hkv, ng = min(H, s.G - gc * H);
  const PCache c = tab.c[layer];
  const AttnLayer l = tab.l[layer];
  const int64_t q0 = (int64_t)b * s.hq + h * s.G + gc * H;   // first query row
  u32x4 qf[NC];
#pragma unroll
  for (int k = 0; k < NC; ++k) qf[k] = *reinterpret_cast<const u32x4 *>(l.Q + (q0 + (l16 < ng ? l16 : 0)) * RB + (4 * k + quad) * 16);
  const int t0 = ch * a.ctiles;
  int place, entry = tile_entry(s, a, c, l, u, t0 + wave + lane * W, place);   // lane i: where the wave's i-th tile of 64 lies
  const int len = head_rows(s, c, u), tiles = head_tiles(s, a, l, u, len), t1 = chunk_end(a, tiles, ch);
  if (t0 >= t1 && ch > 0) return;
#pragma unroll
  for (int k = 0; k < NC; ++k)
    if (l16 >= ng) qf[k] = u32x4{0u, 0u, 0u, 0u};              // heads past the group are zero columns
  const float c2 = s.scale_log2e;
  float m = -INFINITY, sum = 0.f;                              // the head's offset, this lane's share of its sum of weights
  f32x4 o[NB];
#pragma unroll
  for (int k = 0; k < NB; ++k) o[k] = f32x4{0.f, 0.f, 0.f, 0.f};
  char *img = reinterpret_cast<char *>(o_s[wave]);             // bf16: a tile of values, 32 rows
  static_assert(F32 || 32 * RB <= H * D * 4, "the image lies in the wave's share of the output");
  const uint32_t img_a = (uint32_t)(uintptr_t)(lds_void_t *)img;

  for (int first = t0 + wave; first < t1; first += 64 * W) {
    if (first != t0 + wave) entry = tile_entry(s, a, c, l, u, first + lane * W, place);
    const Tile x = tile_of_entry(s, len, first + lane * W, place, entry);
    const int x_page = x.page, x_rows = x.row | (x.live << 8);
    const int n = min((t1 - first + W - 1) / W, 64);
    u32x4 kr[2][NC], vr[NV];
    auto tile_of = [&](const char *pool, int i) {
      return pool + (int64_t)__builtin_amdgcn_readlane(x_page, i) * s.page_bytes + (__builtin_amdgcn_readlane(x_rows, i) & 255) * RB;
    };
    auto load_keys = [&](int i) {
      const char *p = tile_of(c.K, i) + l16 * RB + quad * 16;
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int k = 0; k < NC; ++k) kr[r][k] = load_vec<ONCE>(p + r * 16 * RB + k * 64);
    };
    // value load j of a lane: bf16: piece lane % PPR of row RPL j + lane / PPR; fp32: elements 64 (j / 8) + 4 l16 + ... of row
    // 16 (j / 4 % 2) + 4 quad + j % 4
    auto value_row = [&](int j) { return F32 ? 16 * ((j >> 2) & 1) + 4 * quad + (j & 3) : RPL * j + lane / PPR; };
    auto load_values = [&](int i) {
      const char *p = tile_of(c.V, i);
      const int live = __builtin_amdgcn_readlane(x_rows, i) >> 8;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const char *at = p + value_row(j) * RB + (F32 ? (j >> 3) * 256 + l16 * 16 : (lane % PPR) * 16);
        if (live == 32) vr[j] = load_vec<ONCE>(at);
        else vr[j] = value_row(j) < live ? load_vec<ONCE>(at) : u32x4{0u, 0u, 0u, 0u};   // rows that do not exist: zeros
      }
    };
    load_keys(0);
    load_values(0);
    for (int i = 0; i < n; ++i) {
      const int live = __builtin_amdgcn_readlane(x_rows, i) >> 8;
      f32x4 acc[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        acc[r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < NC; ++k) {
          if constexpr (F32) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              acc[r] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kr[r][k][e]), __uint_as_float(qf[k][e]), acc[r], 0, 0, 0);
          } else {
            acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[r][k]), __builtin_bit_cast(bf16x8, qf[k]), acc[r], 0, 0, 0);
          }
        }
      }
      if (i + 1 < n) load_keys(i + 1);
      float x8[8], p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float v = e < 4 ? acc[0][e & 3] : acc[1][e & 3];
        x8[e] = 16 * (e >> 2) + 4 * quad + (e & 3) < live ? v : -INFINITY;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = fast_exp2(fmaf(x8[e], c2, -m));
      float next = sum + (((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7])));
      if (__builtin_amdgcn_ballot_w64(!(next < kRowsSumLimit)) != 0) {
        float t = fmaxf(fmaxf(fmaxf(x8[0], x8[1]), fmaxf(x8[2], x8[3])), fmaxf(fmaxf(x8[4], x8[5]), fmaxf(x8[6], x8[7])));
        t = fmaxf(t, __shfl_xor(t, 16));
        t = fmaxf(t, __shfl_xor(t, 32));
        const float mn = fmaxf(m, t * c2), mu = mn == -INFINITY ? 0.f : mn;
        const float f = fast_exp2(m - mu);                     // 0 while there is no offset yet
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = fast_exp2(fmaf(x8[e], c2, -mu));
        next = sum * f + (((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7])));
#pragma unroll
        for (int k = 0; k < NB; ++k) o[k] *= f;
        m = mn;
      }
      sum = next;
      if constexpr (F32) {
#pragma unroll
        for (int k = 0; k < NB; ++k)
#pragma unroll
          for (int e = 0; e < 8; ++e)                          // block k: elements 64 (k / 4) + 4 i + k % 4
            o[k] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vr[(k >> 2) * 8 + e][k & 3]), p[e], o[k], 0, 0, 0);
        if (i + 1 < n) load_values(i + 1);
      } else {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const int row = value_row(j);
          reinterpret_cast<u32x4 *>(img)[row * PPR + ((lane % PPR) ^ value_swz<D>(row))] = vr[j];
        }
        if (i + 1 < n) load_values(i + 1);
        wave_lds_fence();
        bf16x8 ph, pl;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const __bf16 hi = (__bf16)p[e];
          ph[e] = hi;
          pl[e] = (__bf16)(p[e] - (float)hi);
        }
        const uint32_t r0 = 4 * quad + (l16 >> 2);             // rows 4 quad ... and 16 + 4 quad ... of block k of 16 elements
#pragma unroll
        for (int k = 0; k < NB; ++k) {
          uint32_t at[2];
#pragma unroll
          for (int r = 0; r < 2; ++r)
            at[r] = img_a + (r0 + 16 * r) * RB + ((2 * k + ((l16 & 3) >> 1)) ^ value_swz<D>(r0 + 16 * r)) * 16 + (l16 & 1) * 8;
          const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)at[0]);
          const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)at[1]);
          const bf16x8 vv = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
          o[k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, ph, o[k], 0, 0, 0);
          o[k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, pl, o[k], 0, 0, 0);
        }
        wave_lds_fence();
      }
    }
  }

  // ---- the waves' shares: lane (head, quad) has rows 4 quad + e of every block
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  if (quad == 0) { m_s[wave][l16] = m; l_s[wave][l16] = sum; }
#pragma unroll
  for (int k = 0; k < NB; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      o_s[wave][l16][(F32 ? 64 * (k >> 2) + 4 * (4 * quad + e) + (k & 3) : 16 * k + 4 * quad + e) ^ l16] = o[k][e];
  finish_chunk<DT, D>(s, a, l, o_s, m_s, l_s, part, part_ml, slot_of(s, a, unit0, layer, u, gc, ch), q0, ng, chunks_used(a, tiles) <= 1);
}

// Folds the chunks of one query head: slices of D/4 threads take every S-th chunk, 16 bytes of its row a thread, and are summed in order.
template <int DT, int D>
__global__ __launch_bounds__(256) void paged_merge_kernel(PShape s, AShape a, AttnTable tab, const float *part, const float *part_ml, int64_t unit0) {
  constexpr int T = D / 4, S = 256 / T;
  __shared__ float red[4];
  __shared__ f32x4 acc_s[S][T];
  __shared__ float tot_s[S];
  const int tid = threadIdx.x, t = tid % T, slice = tid / T;
  const int u = blockIdx.x, g = blockIdx.y, layer = blockIdx.z / a.gchunks, gc = blockIdx.z - layer * a.gchunks;
  const int b = u / s.hkv, h = u - b * s.hkv;
  if (g >= min(kAttnHeads, s.G - gc * kAttnHeads)) return;
  const PCache c = tab.c[layer];
  const AttnLayer l = tab.l[layer];
  const int64_t slot = slot_of(s, a, unit0, layer, u, gc, 0) + g;
  const float2 *ml = reinterpret_cast<const float2 *>(part_ml) + slot;
  const float *rows = part + slot * D + 4 * t;
  // the thread's first chunks, asked for beside the head's length: in bounds, and of no use where the head has fewer
  const int64_t i0 = (int64_t)min(slice, a.nchunks - 1) * a.gt;
  const float m0 = ml[(int64_t)min(tid, a.nchunks - 1) * a.gt].x;
  const float2 x0 = ml[i0];
  const f32x4 r0 = *reinterpret_cast<const f32x4 *>(rows + i0 * D);
  const int used = chunks_used(a, head_tiles(s, a, l, u, head_rows(s, c, u)));
  if (used <= 1) return;
  float m = tid < used ? m0 : -INFINITY;
  for (int i = tid + 256; i < used; i += 256) m = fmaxf(m, ml[(int64_t)i * a.gt].x);
  m = wave_reduce<WMax>(m, -INFINITY);
  if ((tid & 63) == 0) red[tid >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const float mu = m == -INFINITY ? 0.f : m;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float tot = 0.f;
  if (slice < used) {
    const float f = fast_exp2(x0.x - mu);
    acc = r0 * f;
    tot = x0.y * f;
  }
#pragma unroll 4
  for (int i = slice + S; i < used; i += S) {
    const float2 x = ml[(int64_t)i * a.gt];
    const float f = fast_exp2(x.x - mu);
    acc += *reinterpret_cast<const f32x4 *>(rows + (int64_t)i * a.gt * D) * f;
    tot = fmaf(x.y, f, tot);
  }
  acc_s[slice][t] = acc;
  if (t == 0) tot_s[slice] = tot;
  __syncthreads();
  if (tid >= T) return;
#pragma unroll
  for (int i = 1; i < S; ++i) { acc += acc_s[i][t]; tot += tot_s[i]; }
  const int64_t at = ((int64_t)b * s.hq + h * s.G + gc * kAttnHeads + g) * D + 4 * t;
#pragma unroll
  for (int e = 0; e < 4; ++e) acc[e] = row_result(acc[e], tot);
  if constexpr (DT == MIXKV_BF16) {
    u32x2 v;
#pragma unroll
    for (int e = 0; e < 2; ++e) v[e] = (uint32_t)f32_to_bf16_rne(acc[2 * e]) | ((uint32_t)f32_to_bf16_rne(acc[2 * e + 1]) << 16);
    *reinterpret_cast<u32x2 *>(reinterpret_cast<uint16_t *>(l.out) + at) = v;
  } else {
    *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(l.out) + at) = acc;
  }
}

// Tiles of a chunk and chunks of a head, from nothing but the arguments.  A workgroup costs some 4 us before and after its tiles (its chain of
// loads, the queries, the fold of its waves), a tile some 1 us of a wave, the merge 4 us with the gap before it: as many workgroups as
// there are compute units as soon as there are tiles for them, then longer chunks, up to two workgroups for every unit (all of them at once: LDS and registers hold three in 4 bits, four at
// 64 elements), then, in 4 bits, up to 64 tiles (full-precision tiles take three times the bytes: 16).  us in chunks of 4, 8, 16, 32, 64, 128 tiles, 4-bit rows of 128: 4 heads of 2048
// rows 10 11 13 17 23 21; 4 of 32 768 22 16 15 18 25 39; 4 of 131 072 59 41 32 26 27 40; 64 of 4096 25 19 16 17 24 37; 64 of 64 pages of 64
// 28 22 17 19 25 37; 512 of up to 16 384 336 223 172 149 138 140; bf16 rows, 128 heads of up to 8192 100 79 73 78 80 87, 4 of 8192 12 12 16 23 38
// 69; fp32, 128 of up to 8192 97 86 88 85 85 138.  Heads of up to 12 tiles stay whole: 4 of 260 rows 8.4 against 9.5 in chunks of 4.
static void attn_config(const PShape &s, int n_layers, int max_rows, AShape *a) {
  a->gchunks = (s.G + kAttnHeads - 1) / kAttnHeads;
  a->gt = std::min(s.G, kAttnHeads);
  const int64_t groups = (int64_t)n_layers * s.units_per_layer * a->gchunks, tiles = ((int64_t)max_rows + 31) / 32, all = tiles * groups;
  int64_t ct = std::max<int64_t>(4, std::max(std::min<int64_t>((all + 255) / 256, 16), std::min<int64_t>((all + 511) / 512, s.q4 ? 64 : 16)));
  if (tiles <= 12) ct = tiles;
  a->ctiles = (int)((ct + 3) / 4 * 4);
  // a launch has at most 65535 chunks, and fewer than 2^32 threads; the last chunk of a head takes what is left
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(65535, ((int64_t)1 << 23) / (std::min(n_layers, kLayersPerLaunch) * s.units_per_layer * (int64_t)a->gchunks)));
  a->nchunks = (int)std::min(most, std::max<int64_t>(1, (tiles + a->ctiles - 1) / a->ctiles));
}
// Rows of partials; each has D floats, and behind them all each has two more.
static size_t attn_slots(const PShape &s, const AShape &a, int n_layers) {
  return a.nchunks == 1 ? 0 : (size_t)n_layers * s.units_per_layer * a.gchunks * a.nchunks * a.gt;
}
static size_t attn_bytes(const PShape &s, const AShape &a, int n_layers) { return attn_slots(s, a, n_layers) * (s.D + 2) * sizeof(float); }
// ONCE: the rows pass the caches by.  With more query heads to a KV head than a workgroup takes, several workgroups read the same rows, and they go
// through the caches.  us by the caches and through them, rows of 128: 4-bit, 64 sequences of 8192, 4 query heads to a KV head 125 and 138, 48 heads
// to one KV head 60 and 51; bf16, 16 of 8192, 4 to a head 94 and 107, 32 to a head 56 and 54; fp32, 32 to a head 103 and 98.
template <bool ONCE, typename Go>
static void launch_attention(const PShape &s, int dtype, Go &&go) {
  constexpr int B16 = MIXKV_BF16, F32 = MIXKV_F32;
  if (s.q4) { if (s.D == 128) go(paged_q4_kernel<128, ONCE>, paged_merge_kernel<B16, 128>); else go(paged_q4_kernel<64, ONCE>, paged_merge_kernel<B16, 64>); }
  else if (dtype == B16) { if (s.D == 128) go(paged_rows_kernel<B16, 128, ONCE>, paged_merge_kernel<B16, 128>); else go(paged_rows_kernel<B16, 64, ONCE>, paged_merge_kernel<B16, 64>); }
  else { if (s.D == 128) go(paged_rows_kernel<F32, 128, ONCE>, paged_merge_kernel<F32, 128>); else go(paged_rows_kernel<F32, 64, ONCE>, paged_merge_kernel<F32, 64>); }
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
  if ((st = check_caches(caches, n_layers, true, false)) != MIXKV_OK) return st;
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
  if ((int64_t)std::min(n_layers, kLayersPerLaunch) * a.gchunks > 65535) return MIXKV_ERR_UNSUPPORTED;
  a.keep = sparse ? max_selected : 0;
  const size_t need = attn_bytes(s, a, n_layers);
  if (need > 0) {
    if (!workspace || misaligned(workspace, 256)) return MIXKV_ERR_INVALID_ARG;
    if (workspace_bytes < need) return MIXKV_ERR_WORKSPACE_TOO_SMALL;
  }
  hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
  float *part = static_cast<float *>(workspace), *part_ml = need > 0 ? part + attn_slots(s, a, n_layers) * s.D : nullptr;
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
    const int64_t unit0 = (int64_t)l0 * s.units_per_layer;
    const unsigned z = (unsigned)(nl * a.gchunks);
    auto go = [&](auto kern, auto merge) {
      hipLaunchKernelGGL(kern, dim3((unsigned)s.units_per_layer, (unsigned)a.nchunks, z), dim3(256), 0, stream, s, a, t, part, part_ml, unit0);
      if (a.nchunks > 1)
        hipLaunchKernelGGL(merge, dim3((unsigned)s.units_per_layer, (unsigned)a.gt, z), dim3(256), 0, stream, s, a, t, (const float *)part, (const float *)part_ml, unit0);
    };
    if (a.gchunks == 1) launch_attention<true>(s, params->dtype, go);
    else launch_attention<false>(s, params->dtype, go);
    if (hipGetLastError() != hipSuccess) return MIXKV_ERR_HIP;
  }
  return MIXKV_OK;
}
