// Attention of many new rows (prompts, chunks of them) over the pages of a cache: mixkv_paged_window_attention where a unit has more rows than a few.
//
// A workgroup has kPromptRows rows of a unit (new rows times the G query heads of a KV head, row i being query head i % G of new row i / G, so that a tile of
// keys serves all of them), a wave 32 of them, and goes through the 32-row tiles that they see, two at a time, which travel through LDS.
//   * Scores: S' = K Q', keys on the output rows of 32 x 32 x 16 products: a lane has 16 keys of one row, its neighbour 32 lanes on the other 16, so that the
//     softmax stays in the lane.
//   * The second product is O' = V' P': the weights are its second operand as they lie in the lane, because the order of its contraction is free: slot 8 h + j of 16
//     keys is what the lane's registers hold.
//   * The offset of a row's exponents moves only where a sum of weights reaches a limit: no maximum is taken otherwise.
//   * The weights of bf16 rows are rounded to bf16 for the second product, the sum that divides them is not: an output is off by the root of two times what its own
//     rounding makes (2.3e-3 and 1.6e-3 of its 2-norm).  A second part of the weights, as paged_rows_kernel takes it, would be half as many products again.
//   * 4-bit keys in two fp16 parts (one is off by 2^-12: logits, lse and weights then by some 1e-4), values and weights in one, as in paged_q4_kernel.
//   * In the program's order a product stands beside what the vector unit does of the other tile meanwhile, and the reads of its operands in front; everything that a turn
//     needs to know of its pages comes by lane reads from words made for 64 tiles at once.  256 rows to a workgroup: 2467 us (two prompts), 128 rows 2645.
// Bound: the matrix unit.  bf16, prompts of 16 384 and 9349 rows, 28 query heads on 4 of 128, 2.33 to 2.52 ms, 1.01 to 1.09 PFLOP/s, 85 to 89 % of what a large library
// product reaches on the same card; the products alone took 1.63 ms.  4 bits, 32 768 rows, window 4096 and 16 first rows, 2.64 to 2.86 ms: 1.5 times the products, at the same rate.  Short windows: tiles at their edges are
// masked select by select, with a barrier more a turn: 16 384 rows, 32 query heads on 8, window 1024 383 us, 256 196, 1.8 and 3 times their products' time.
#include "mixkv_pagedwin.h"

namespace mixkv {

constexpr int kPromptWaves = 8, kPromptRows = 32 * kPromptWaves;
// bf16 weights: a lane's sum of weights that reaches this moves the row's offset (the weighted values stay below it times the largest value).  fp16 weights: a
// tile's sum of weights in a lane does, and the offset puts the largest weight at 2^8: fp16 then resolves weights down to 2^-32 of it.
constexpr int kNowhere = 1 << 30;        // no head has so many rows
constexpr float kPromptSum = 0x1p20f, kPromptSum16 = 0x1p14f;

struct PromptShape {
  PWindow w;
  int32_t qtiles;                        // groups of rows of a unit
  int32_t q0, qn;                        // those of the launch
  int32_t nchunks, ctiles;               // chunks of a group's tiles, tiles of a chunk (even)
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// Four rows' elements, transposed.  (A parameter that is said to alias nothing: otherwise the compiler waits for every load on its way to LDS first.)
__device__ __forceinline__ s16x4 read_transposed(lds_s16x4 *__restrict p) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16(p); }

// Rotation of the 16-byte pieces of a value row: half a wave reads two pieces of four neighbouring rows at two places (those of 32 bytes further).
template <int D>
__device__ __forceinline__ int read_swz(int r) { return D == 128 ? (4 * r) & 15 : (2 * r) & 4; }

template <int D, bool Q4>
__global__ __launch_bounds__(64 * kPromptWaves, 2) void paged_prompt_kernel(PShape s, PromptShape a, WinTable tab, float *part, float *part_ml, int64_t unit0) {
  constexpr int RB = D * 2, PPR = RB / 16, KS = D / 16, NB = D / 32, W = kPromptWaves, R = kPromptRows;
  constexpr int TILE = 32 * RB, IMG = 2 * TILE;              // a tile of 32 rows; two of them
  constexpr int KEYS = (Q4 ? 2 : 1) * IMG;                   // keys' tiles, and (4 bits) behind them what their elements lack in fp16
  __shared__ __align__(16) char img[2 * KEYS + 2 * IMG];
  __shared__ int odd_s[W];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int units = s.units_per_layer, turn = a.q0 + a.qn - 1 - (int)blockIdx.y, ch = blockIdx.x / units;     // the rows that see most come first
  const int u = dealt_unit((int)blockIdx.x - ch * units, blockIdx.y, units), layer = blockIdx.z, b = u / s.hkv, h = u - b * s.hkv;
  const PCache c = tab.c[layer];
  const WinLayer l = tab.l[layer];
  const View v = view_of(s, a.w, c, l, u, turn * R, R);
  if (v.ng <= 0) return;
  const int t0 = ch * a.ctiles, t1 = ch == a.nchunks - 1 ? v.tiles : min(v.tiles, t0 + a.ctiles);
  if (t0 >= t1 && ch > 0) return;

  // ---- the lane's row: its query as the second operand, and its place
  const int mine = 32 * wave + l32, i_row = min(mine, v.ng - 1), place = v.place(s, i_row);
  u32x4 qf[KS];
  float c2 = s.scale_log2e;
  {
    const char *q = v.query(s, a.w, l, h, i_row) + half * 16;
#pragma unroll
    for (int k = 0; k < KS; ++k) qf[k] = *reinterpret_cast<const u32x4 *>(q + k * 32);
    if constexpr (Q4) {                                      // to fp16, by a power of two that brings the row's largest element to [2^13, 2^14)
      uint32_t most = 0;
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) most = max(most, max(qf[k][j] & 0x7fffu, (qf[k][j] >> 16) & 0x7fffu));
      most = max(most, (uint32_t)__shfl_xor((int)most, 32));
      const int up = 13 - (min(max((int)(most >> 7), 1), 254) - 127);
      c2 = fminf(fmaxf(ldexpf(c2, -up), 0x1p-126f), 0x1p100f);
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          qf[k][j] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)ldexpf(__uint_as_float(qf[k][j] << 16), up), (_Float16)ldexpf(__uint_as_float(qf[k][j] & 0xffff0000u), up)});
    }
  }

  // ---- tiles, two at a time: lane i knows where the i-th of a batch of 64 lies, and whether all of the group's rows see all of it.  One that does not exist lies
  // behind everything that is seen.  (What a turn needs of it are a few words: scalar registers are short here.)
  struct Pair { int row0[2], row; bool part; const char *k, *v; };            // first rows; not all seen by all; of the tile that the wave fetches: its first row, the pages
  const int side = wave / (W / 2), in_page = s.P - 1;        // which of the two tiles the wave fetches
  const int behind = place - a.w.window, first = a.w.first;
  uint32_t x_word = 0, x_k[2] = {}, x_v[2] = {};
  const int n = t1 - t0;
  auto pair_at = [&](int i) __attribute__((always_inline)) {     // (asked for in order)
    if (__builtin_expect((i & 63) == 0, 0)) {
      const int t = t0 + i + lane, tile = v.tile(t), id = t < t1 ? page_at(s, c, u, tile >> (s.lp - 5)) : -1;
      const int row0 = id >= 0 ? tile * 32 : kNowhere;
      const bool all = row0 + 31 <= v.pa && (row0 > v.pb - a.w.window || row0 + 31 < a.w.first);
      const int64_t page = max(id, 0) * s.page_bytes;
      const uint64_t k = reinterpret_cast<uint64_t>(c.K + page), w = reinterpret_cast<uint64_t>(c.V + page);
      x_word = (uint32_t)row0 | (all ? 0u : 1u);
      x_k[0] = (uint32_t)k; x_k[1] = (uint32_t)(k >> 32);
      x_v[0] = (uint32_t)w; x_v[1] = (uint32_t)(w >> 32);
    }
    auto word = [&](uint32_t x, int j) { return (uint32_t)__builtin_amdgcn_readlane((int)x, (i & 63) + j); };
    Pair p;
    const uint32_t w0 = word(x_word, 0), w1 = word(x_word, 1);
    p.row0[0] = (int)(w0 & ~31u);
    p.row0[1] = (int)(w1 & ~31u);
    p.row = (side ? p.row0[1] : p.row0[0]) & in_page;
    p.part = ((w0 | w1) & 1u) != 0;
    p.k = reinterpret_cast<const char *>((uint64_t)word(x_k[1], side) << 32 | word(x_k[0], side));
    p.v = reinterpret_cast<const char *>((uint64_t)word(x_v[1], side) << 32 | word(x_v[0], side));
    return p;
  };
  const uint32_t img_a = lds_base_of(img);
  auto key_image = [&](int to) { return img_a + to * KEYS; };
  auto value_image = [&](int to) { return img_a + 2 * KEYS + to * IMG; };
  // where the lane reads: the rest of an address is a constant
  uint32_t k_at[KS], v_at[NB];
#pragma unroll
  for (int k = 0; k < KS; ++k) k_at[k] = img_a + l32 * RB + ((2 * k + half) ^ tile_swz<MIXKV_BF16, D>(l32)) * 16;
#pragma unroll
  for (int blk = 0; blk < NB; ++blk) {
    const int l16 = lane & 15, sub = (lane >> 4) & 1, r = 4 * half + (l16 >> 2);       // (the rows that are 8 and 16 further have the same rotation)
    v_at[blk] = img_a + 2 * KEYS + (Q4 ? (half * D + 32 * blk + l32) * 16 : r * RB + ((4 * blk + 2 * sub + ((l16 & 3) >> 1)) ^ read_swz<D>(r)) * 16 + (l16 & 1) * 8);
  }

  // bf16: a wave fetches 8 rows of one tile, directly: the lane's place in what each load takes
  constexpr int RPL = 64 / PPR, FROWS = 64 / W, LOADS = FROWS / RPL;         // rows of a load; rows and loads of a wave
  const int f_row = FROWS * (wave % (W / 2));
  uint32_t f_at[2][LOADS];
#pragma unroll
  for (int j = 0; j < LOADS; ++j) {
    const int r = j * RPL + lane / PPR;
    f_at[0][j] = r * RB + ((lane % PPR) ^ tile_swz<MIXKV_BF16, D>(f_row + r)) * 16;
    f_at[1][j] = r * RB + ((lane % PPR) ^ read_swz<D>(f_row + r)) * 16;
  }
  auto fetch = [&](const Pair &p, int values, uint32_t to) __attribute__((always_inline)) {
    const char *base = (values ? p.v : p.k) + (p.row + f_row) * RB;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      uint32_t at = f_at[values][j];
      asm("" : "+v"(at));                                    // 32 bits beside a scalar base
      load_to_lds<false>(base + at, to + side * TILE + f_row * RB + j * 1024);
    }
  };
  // 4 bits: a thread's words and scales of a tile, then in fp16 into the images.  The thread's key row, run and words of it; the values' strip, words
  // 64 vj + 4 vm + 2 vh + (0, 1) of it
  constexpr int NG = D / 32, VT = 2 * D;                     // groups of a row; threads with values of a tile
  const int r256 = tid & 255, krow = r256 >> 3, krun = (r256 >> 1) & 3, kpl = (r256 & 1) * (NG / 2);
  const int vq = r256 / (VT / 4), vj = r256 % (VT / 4) >> 5, vm = (r256 >> 1) & 15, vh = r256 & 1, codes = s.P * (D / 2);
  uint32_t kw[NG / 2], ksb[NG / 2];
  u32x2 vw;
  u32x4 vst, vba;
  auto ask_keys = [&](const Pair &p) __attribute__((always_inline)) {
    const char *kp = p.k;
    const int row = p.row + krow;
    const uint32_t *kc = reinterpret_cast<const uint32_t *>(kp + row * (D / 2) + krun * (NG * 4)) + kpl, *kz = reinterpret_cast<const uint32_t *>(kp + codes + row * (NG * 4)) + kpl;
#pragma unroll
    for (int g = 0; g < NG / 2; ++g) { kw[g] = kc[g]; ksb[g] = kz[g]; }
  };
  auto ask_values = [&](const Pair &p) __attribute__((always_inline)) {
    if (VT < 256 && r256 >= VT) return;
    const char *vp = p.v;
    const int strip = (p.row >> 5) * 4 + vq;
    vw = *reinterpret_cast<const u32x2 *>(vp + (strip * D + 64 * vj + 4 * vm + 2 * vh) * 4);
    const char *z = vp + codes + (strip * NG + 2 * vj + vh) * 32;
    vst = *reinterpret_cast<const u32x4 *>(z);
    vba = *reinterpret_cast<const u32x4 *>(z + 16);
  };
  auto unpack_keys = [&](uint32_t to) __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < NG / 2; ++g) {
      const int pl = kpl + g, piece = 4 * (D == 128 ? (pl & 1) * 2 + (pl >> 1) : pl) + krun;
      const f16x2 sb = __builtin_bit_cast(f16x2, ksb[g]), step = {sb[0], sb[0]}, base = {sb[1], sb[1]};
      u32x4 hi, lo;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f16x2 un = code_pair(kw[g], j), x = __builtin_elementwise_fma(un, step, base);
        hi[j] = __builtin_bit_cast(uint32_t, x);
        lo[j] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)(fmaf((float)un[0], (float)sb[0], (float)sb[1]) - (float)x[0]), (_Float16)(fmaf((float)un[1], (float)sb[0], (float)sb[1]) - (float)x[1])});
      }
      const uint32_t at = to + side * TILE + krow * RB + (piece ^ tile_swz<MIXKV_BF16, D>(krow)) * 16;
      store_lds(at, hi);
      store_lds(at + IMG, lo);
    }
  };
  auto unpack_values = [&](const Pair &p, uint32_t to) __attribute__((always_inline)) {      // rows that do not exist: zeros
    if (VT < 256 && r256 >= VT) return;
    const int live = v.len - (side ? p.row0[1] : p.row0[0]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t on = (4 * vq + j < live ? 0xffffu : 0u) | (16 + 4 * vq + j < live ? 0xffff0000u : 0u);
      vst[j] &= on;
      vba[j] &= on;
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      u32x4 x;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        x[j] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(code_pair(vw[w], j), __builtin_bit_cast(f16x2, (uint32_t)vst[j]), __builtin_bit_cast(f16x2, (uint32_t)vba[j])));
      store_lds(to + side * TILE + (vq * D + 64 * vj + 16 * (2 * vh + w) + vm) * 16, x);
    }
  };

  // ---- scores of 32 keys: register e is key 8 (e / 4) + 4 half + e % 4.  (4 bits: the keys in two parts, so that a logit is off by no more than fp32 makes it, as
  // lse and weights have to be)
  constexpr int AHEAD = Q4 ? KS / 2 : KS;                    // reads under way
  u32x4 kf[AHEAD], lf[Q4 ? AHEAD : 1];
  auto read_keys = [&](int at0, int i) __attribute__((always_inline)) {        // the i-th of a turn's 2 KS pieces
    const uint32_t at = k_at[i % KS] + at0 + i / KS * TILE;
    kf[i % AHEAD] = lds_vec(at);
    if constexpr (Q4) lf[i % AHEAD] = lds_vec(at + IMG);
  };
  auto score = [&](int i, int at0, f32x16 &acc) __attribute__((always_inline)) {
    const int k = i % KS;
    if (k == 0) {
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[e] = 0.f;
    }
    if constexpr (Q4) {
      acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, lf[i % AHEAD]), __builtin_bit_cast(f16x8, qf[k]), acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, kf[i % AHEAD]), __builtin_bit_cast(f16x8, qf[k]), acc, 0, 0, 0);
    } else {
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[i % AHEAD]), __builtin_bit_cast(bf16x8, qf[k]), acc, 0, 0, 0);
    }
    if (i + AHEAD < 2 * KS) read_keys(at0, i + AHEAD);
  };
  // ---- the values of 16 keys and 32 elements as the second product's first operand
  auto value = [&](int at0, int k, int blk) __attribute__((always_inline)) {
    if constexpr (Q4) {
      return lds_vec(v_at[blk] + at0 + 2 * k * D * 16);
    } else {
      const s16x4 v0 = read_transposed((lds_s16x4 *)(uintptr_t)(v_at[blk] + at0 + 16 * k * RB));
      const s16x4 v1 = read_transposed((lds_s16x4 *)(uintptr_t)(v_at[blk] + at0 + (16 * k + 8) * RB));
      return __builtin_bit_cast(u32x4, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  };
  auto product = [&](u32x4 vf, u32x4 pf, f32x16 acc) __attribute__((always_inline)) {
    if constexpr (Q4) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, vf), __builtin_bit_cast(f16x8, pf), acc, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf), __builtin_bit_cast(bf16x8, pf), acc, 0, 0, 0);
  };

  // ---- the weights of 32 keys against an offset as the second product's second operand: the i-th of eight pairs, and their sum
  auto weigh = [&](const f32x16 &x, int i, float off, u32x4 (&pw)[2]) __attribute__((always_inline)) {
    const int k = i / 4, j = i % 4, e0 = Q4 ? 4 * k + j : 8 * k + 2 * j, e1 = Q4 ? 8 + 4 * k + j : e0 + 1;
    const float p0 = fast_exp2(fmaf(x[e0], c2, -off)), p1 = fast_exp2(fmaf(x[e1], c2, -off));
    pw[k][j] = Q4 ? __builtin_bit_cast(uint32_t, f16x2{(_Float16)p0, (_Float16)p1}) : __builtin_bit_cast(uint32_t, bf16x2{(__bf16)p0, (__bf16)p1});
    return p0 + p1;
  };

  f32x16 o[NB];
#pragma unroll
  for (int k = 0; k < NB; ++k)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[k][e] = 0.f;
  float m = -INFINITY, sum = 0.f;                            // the row's offset, this lane's share of its sum of weights

  Pair cur = pair_at(0);
  if constexpr (Q4) {
    ask_keys(cur);
    ask_values(cur);
    unpack_keys(key_image(0));
    unpack_values(cur, value_image(0));
  } else {
    fetch(cur, 0, key_image(0));
    fetch(cur, 1, value_image(0));
  }
  // What a row does not see has no weight.
  auto hide = [&](int row0, f32x16 &acc) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int j = row0 + 8 * (e >> 2) + 4 * half + (e & 3);
      acc[e] = (j <= place) & ((j > behind) | (j < first)) ? acc[e] : -INFINITY;
      __builtin_amdgcn_sched_barrier(0);                     // (one after another: side by side they take more scalar registers than there are)
    }
  };
  // The offset moves where a sum of weights reaches its limit.
  auto settle = [&](const f32x16 &acc, float next, u32x4 (&pw)[2]) __attribute__((always_inline)) {
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(!((Q4 ? next : sum + next) < (Q4 ? kPromptSum16 : kPromptSum))) != 0, 0)) {
      float t = acc[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) t = fmaxf(t, acc[e]);
      t = fmaxf(t, __shfl_xor(t, 32));
      const float mn = fmaxf(m, t * c2 - (Q4 ? 8.f : 0.f)), mu = mn == -INFINITY ? 0.f : mn, f = fast_exp2(m - mu);
      next = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) next += weigh(acc, k, mu, pw);
      sum *= f;
#pragma unroll
      for (int k = 0; k < NB; ++k)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[k][e] *= f;
      m = mn;
    }
    sum += next;
  };
  // Two tiles, that all of the group's rows see all of, or not (part).  Then values that are no numbers are turned to zeros, and added behind the product where their
  // rows are seen: a weight of zero does not make NaN of them.
  auto tiles_of = [&](int r0, int r1, bool part, auto turn_c) __attribute__((always_inline)) {
    constexpr int to = decltype(turn_c)::value;
    bool mixed = false;
    if constexpr (!Q4) {
      if (__builtin_expect(part, 0)) {
        bool odd = false;
#pragma unroll
        for (int j = 0; j < IMG / (1024 * W); ++j) {
          const uint32_t at = value_image(to) + (j * W + wave) * 1024 + lane * 16;
          u32x4 w = lds_vec(at);
          bool bad = false;
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            bad |= no_number<MIXKV_BF16>(w[z]);
            w[z] = numbers_only<MIXKV_BF16>(w[z]);
          }
          if (bad) store_lds(at, w);
          odd |= bad;
        }
        odd = __builtin_amdgcn_ballot_w64(odd) != 0;
        if (lane == 0) odd_s[wave] = odd;
        lds_barrier();
#pragma unroll
        for (int w = 0; w < W; ++w) mixed |= odd_s[w] != 0;
      }
    }
    // The matrix unit works on one tile's product while the vector unit forms the other's weights: in the program's order, a product and what fits beside it.
    constexpr int k0 = to * KEYS, v0 = to * IMG, SPP = 8 / KS, VPP = 8 / (2 * NB);
    f32x16 acc[2];
    u32x4 pw[2][2], vf[2][NB];
    float next[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) read_keys(k0, k);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      score(k, k0, acc[0]);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (__builtin_expect(part, 0)) hide(r0, acc[0]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i % SPP == 0) score(KS + i / SPP, k0, acc[1]);
      if (!Q4 && i % VPP == 0) vf[i / VPP / NB][i / VPP % NB] = value(v0, i / VPP / NB, i / VPP % NB);
      next[0] += weigh(acc[0], i, m, pw[0]);
      __builtin_amdgcn_sched_barrier(0);
    }
    settle(acc[0], next[0], pw[0]);
    if (__builtin_expect(part, 0)) hide(r1, acc[1]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i % VPP == 0) {
        const int k = i / VPP / NB, blk = i / VPP % NB;
        o[blk] = product(Q4 ? value(v0, k, blk) : vf[k][blk], pw[0][k], o[blk]);
        if constexpr (!Q4) vf[k][blk] = value(v0 + TILE, k, blk);
      }
      next[1] += weigh(acc[1], i, m, pw[1]);
      __builtin_amdgcn_sched_barrier(0);
    }
    settle(acc[1], next[1], pw[1]);
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int blk = 0; blk < NB; ++blk) o[blk] = product(Q4 ? value(v0 + TILE, k, blk) : vf[k][blk], pw[1][k], o[blk]);
    if (__builtin_expect(mixed, 0)) {
#pragma unroll 1
      for (int r = 0; r < 64; ++r) {
        const int j = (r < 32 ? r0 : r1) + (r & 31);
        if (!sees(a.w, place, j)) continue;
        const uint16_t *from = reinterpret_cast<const uint16_t *>(c.V + page_at(s, c, u, j >> s.lp) * s.page_bytes + (j & in_page) * RB);
#pragma unroll
        for (int blk = 0; blk < NB; ++blk)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float y = __uint_as_float((uint32_t)from[32 * blk + 8 * (e >> 2) + 4 * half + (e & 3)] << 16);
            if (no_number<MIXKV_F32>(__float_as_uint(y))) o[blk][e] += y;
          }
      }
    }
  };
  auto turn_of = [&](int i, auto turn_c) __attribute__((always_inline)) {
    constexpr int to = decltype(turn_c)::value;
    if constexpr (!Q4) wait_vm<0>();
    lds_barrier();
    const int r0 = cur.row0[0], r1 = cur.row0[1];
    const bool part = cur.part;
    const Pair nxt = pair_at(i + 2);
    if (i + 2 < n) {
      if constexpr (Q4) {
        ask_keys(nxt);
        ask_values(nxt);
      } else {
        fetch(nxt, 0, key_image(to ^ 1));
        fetch(nxt, 1, value_image(to ^ 1));
      }
    }
    tiles_of(r0, r1, part, turn_c);
    if constexpr (Q4) {
      if (i + 2 < n) {
        unpack_keys(key_image(to ^ 1));
        unpack_values(nxt, value_image(to ^ 1));
      }
    }
    cur = nxt;
  };
  for (int i = 0; i < n; i += 4) {
    turn_of(i, std::integral_constant<int, 0>{});
    if (i + 2 < n) turn_of(i + 2, std::integral_constant<int, 1>{});
  }

  // ---- lane (row, half) has the elements 32 blk + 8 (e / 4) + 4 half + e % 4
  if (mine >= v.ng) return;
  sum += __shfl_xor(sum, 32);
  if (a.nchunks > 1) {
    const int64_t slot = (((unit0 + (int64_t)layer * units + u) * a.qtiles + turn) * a.nchunks + ch) * R + mine;
#pragma unroll
    for (int blk = 0; blk < NB; ++blk)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4 *>(part + slot * D + 32 * blk + 8 * q + 4 * half) = f32x4{o[blk][4 * q], o[blk][4 * q + 1], o[blk][4 * q + 2], o[blk][4 * q + 3]};
    if (half == 0) reinterpret_cast<float2 *>(part_ml)[slot] = make_float2(m, sum);
    return;
  }
  const int64_t row = v.out_row(s, a.w, h, mine);
  if (row < 0) return;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int blk = 0; blk < NB; ++blk)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      u32x2 w;
#pragma unroll
      for (int j = 0; j < 2; ++j) w[j] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)(o[blk][4 * q + 2 * j] * inv), (__bf16)(o[blk][4 * q + 2 * j + 1] * inv)});
      *reinterpret_cast<u32x2 *>(l.out + row * RB + (32 * blk + 8 * q + 4 * half) * 2) = w;
    }
  if (half == 0 && l.lse) l.lse[row] = row_lse(m == -INFINITY ? 0.f : m, sum);
}

// Folds the chunks of a group's rows: D/4 threads to a row, in the order of the chunks.
template <int D>
__global__ __launch_bounds__(256) void prompt_merge_kernel(PShape s, PromptShape a, WinTable tab, const float *part, const float *part_ml, int64_t unit0) {
  constexpr int T = D / 4, ROWS = 256 / T;
  const int R = kPromptRows, t = threadIdx.x % T, i = blockIdx.y * ROWS + threadIdx.x / T, turn = a.q0 + blockIdx.z % a.qn, layer = blockIdx.z / a.qn, u = blockIdx.x;
  const int h = u % s.hkv;
  const WinLayer l = tab.l[layer];
  const View v = view_of(s, a.w, tab.c[layer], l, u, turn * R, R);
  if (i >= v.ng) return;
  const int64_t row = v.out_row(s, a.w, h, i);
  if (row < 0) return;
  const int used = max(1, min(a.nchunks, (v.tiles + a.ctiles - 1) / a.ctiles));
  const int64_t slot = ((unit0 + (int64_t)layer * s.units_per_layer + u) * a.qtiles + turn) * a.nchunks * R + i;
  const float2 *ml = reinterpret_cast<const float2 *>(part_ml);
  float m = -INFINITY, tot = 0.f;
  for (int k = 0; k < used; ++k) m = fmaxf(m, ml[slot + (int64_t)k * R].x);
  const float mu = m == -INFINITY ? 0.f : m;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int k = 0; k < used; ++k) {
    const float2 x = ml[slot + (int64_t)k * R];
    const float f = fast_exp2(x.x - mu);
    acc += *reinterpret_cast<const f32x4 *>(part + (slot + (int64_t)k * R) * D + 4 * t) * f;
    tot = fmaf(x.y, f, tot);
  }
  u32x2 w;
#pragma unroll
  for (int j = 0; j < 2; ++j) w[j] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)row_result(acc[2 * j], tot), (__bf16)row_result(acc[2 * j + 1], tot)});
  *reinterpret_cast<u32x2 *>(l.out + (row * D + 4 * t) * 2) = w;
  if (t == 0 && l.lse) l.lse[row] = row_lse(mu, tot);
}

// Chunks of a group's tiles: one, unless the groups are fewer than the chip takes at once; then as many as fill it, of at least eight tiles.
static PromptShape prompt_config(const PShape &s, const PWindow &w, int n_layers, int max_rows) {
  PromptShape a{};
  const int rows = kPromptRows, groups_at_once = 256;
  a.w = w;
  a.qtiles = (int)(((int64_t)w.max_count * s.G + rows - 1) / rows);
  const int64_t groups = (int64_t)n_layers * s.units_per_layer * a.qtiles, tiles = most_tiles(s, w, max_rows, rows);
  int64_t chunks = std::max<int64_t>(1, std::min<int64_t>(groups_at_once / groups, (tiles + 7) / 8));
  a.ctiles = (int)(((tiles + chunks - 1) / chunks + 1) / 2 * 2);
  a.nchunks = (int)((tiles + a.ctiles - 1) / a.ctiles);
  return a;
}
static size_t prompt_slots(const PShape &s, const PromptShape &a, int n_layers) {
  return a.nchunks == 1 ? 0 : (size_t)n_layers * s.units_per_layer * a.qtiles * a.nchunks * kPromptRows;
}

size_t prompt_bytes(const PShape &s, const PWindow &w, int n_layers, int max_rows) {
  return prompt_slots(s, prompt_config(s, w, n_layers, max_rows), n_layers) * (s.D + 2) * sizeof(float);
}

mixkv_status launch_prompt(const PShape &s, const PWindow &w, const mixkv_paged_cache *caches, const mixkv_paged_queries *queries, int n_layers, int max_rows,
                           void *workspace, hipStream_t stream) {
  PromptShape a = prompt_config(s, w, n_layers, max_rows);
  const size_t slots = prompt_slots(s, a, n_layers);
  float *part = static_cast<float *>(workspace), *part_ml = slots ? part + slots * s.D : nullptr;
  // a launch has at most 65535 groups of rows, and fewer than 2^32 threads
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(65535, ((int64_t)1 << 22) / ((int64_t)s.units_per_layer * std::max(a.nchunks, kPromptRows))));
  for (int l0 = 0; l0 < n_layers;) {
    const int nl = (int)std::min<int64_t>(std::min(n_layers - l0, kLayersPerLaunch), std::max<int64_t>(1, most / a.qtiles));
    const WinTable t = window_table(caches + l0, queries + l0, nl, 2);
    const int64_t unit0 = (int64_t)l0 * s.units_per_layer;
    for (a.q0 = 0; a.q0 < a.qtiles; a.q0 += a.qn) {
      a.qn = (int)std::min<int64_t>(a.qtiles - a.q0, std::max<int64_t>(1, most / nl));
      const dim3 grid((unsigned)(s.units_per_layer * a.nchunks), (unsigned)a.qn, (unsigned)nl);
      auto go = [&](auto kern, auto merge, int rows) {
        hipLaunchKernelGGL(kern, grid, dim3(64 * kPromptWaves), 0, stream, s, a, t, part, part_ml, unit0);
        if (a.nchunks > 1)
          hipLaunchKernelGGL(merge, dim3((unsigned)s.units_per_layer, (unsigned)(kPromptRows / rows), (unsigned)(nl * a.qn)), dim3(256), 0, stream, s, a, t, (const float *)part,
                             (const float *)part_ml, unit0);
      };
      if (s.q4) { if (s.D == 128) go(paged_prompt_kernel<128, true>, prompt_merge_kernel<128>, 8); else go(paged_prompt_kernel<64, true>, prompt_merge_kernel<64>, 16); }
      else { if (s.D == 128) go(paged_prompt_kernel<128, false>, prompt_merge_kernel<128>, 8); else go(paged_prompt_kernel<64, false>, prompt_merge_kernel<64>, 16); }
      if (hipGetLastError() != hipSuccess) return MIXKV_ERR_HIP;
    }
    l0 += nl;
  }
  return MIXKV_OK;
}

}  // namespace mixkv
