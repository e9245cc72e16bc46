// Rows of the paged cache as a few lanes hold them, and their places in 4-bit pages: what append, read and evict share.  D/16 lanes hold a row: lane j the
// elements [8 j, 8 j + 8) and [D/2 + 8 j, D/2 + 8 j + 8).
#pragma once
#include "mixkv_paged.h"

namespace mixkv {

// What another lane of the row of 16 has, by a move of the vector ALU (DPP control CTRL).
template <int CTRL>
__device__ __forceinline__ int lane_moved(int x) { return __builtin_amdgcn_mov_dpp(x, CTRL, 0xf, 0xf, true); }

// Eight elements of a row as memory has them, and as floats.
template <int DT> struct Run;
template <> struct Run<MIXKV_BF16> {
  u32x4 v;
  __device__ __forceinline__ void load(const char *p) { v = *reinterpret_cast<const u32x4 *>(p); }
  __device__ __forceinline__ void store(char *p) const { *reinterpret_cast<u32x4 *>(p) = v; }
  __device__ __forceinline__ float at(int i) const { return __uint_as_float(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16); }
  __device__ __forceinline__ void set(const float (&x)[8]) {            // rounded to nearest even
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});
  }
};
template <> struct Run<MIXKV_F32> {
  f32x4 lo, hi;
  __device__ __forceinline__ void load(const char *p) { lo = reinterpret_cast<const f32x4 *>(p)[0]; hi = reinterpret_cast<const f32x4 *>(p)[1]; }
  __device__ __forceinline__ void store(char *p) const { reinterpret_cast<f32x4 *>(p)[0] = lo; reinterpret_cast<f32x4 *>(p)[1] = hi; }
  __device__ __forceinline__ float at(int i) const { return i < 4 ? lo[i & 3] : hi[i & 3]; }
  __device__ __forceinline__ void set(const float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { lo[i] = x[i]; hi[i] = x[4 + i]; }
  }
};

// Smallest and largest of each of a run's eight elements.  bf16 pairs as signed 16-bit numbers of the same order (all bits below the sign
// turned over in negative ones), two elements an instruction.
template <int DT> struct RunRange;
template <> struct RunRange<MIXKV_BF16> {
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  s16x2 lo[4], hi[4];
  __device__ __forceinline__ static s16x2 turn(s16x2 x) { return x ^ ((x >> 15) & (short)0x7fff); }
  __device__ __forceinline__ void none() {
#pragma unroll
    for (int i = 0; i < 4; ++i) { lo[i] = s16x2{0x7f80, 0x7f80}; hi[i] = turn(s16x2{(short)0xff80, (short)0xff80}); }   // the infinities
  }
  __device__ __forceinline__ void add(const Run<MIXKV_BF16> &x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const s16x2 v = turn(__builtin_bit_cast(s16x2, (uint32_t)x.v[i]));
      lo[i] = __builtin_elementwise_min(lo[i], v);
      hi[i] = __builtin_elementwise_max(hi[i], v);
    }
  }
  __device__ __forceinline__ void lower(const Run<MIXKV_BF16> &x) {        // by smallest, by largest elements of before
#pragma unroll
    for (int i = 0; i < 4; ++i) lo[i] = __builtin_elementwise_min(lo[i], turn(__builtin_bit_cast(s16x2, (uint32_t)x.v[i])));
  }
  __device__ __forceinline__ void raise(const Run<MIXKV_BF16> &x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) hi[i] = __builtin_elementwise_max(hi[i], turn(__builtin_bit_cast(s16x2, (uint32_t)x.v[i])));
  }
  __device__ __forceinline__ void join(int off) {          // with the lane `off` away
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo[i] = __builtin_elementwise_min(lo[i], __builtin_bit_cast(s16x2, __shfl_xor(__builtin_bit_cast(int, lo[i]), off)));
      hi[i] = __builtin_elementwise_max(hi[i], __builtin_bit_cast(s16x2, __shfl_xor(__builtin_bit_cast(int, hi[i]), off)));
    }
  }
  __device__ __forceinline__ Run<MIXKV_BF16> low() const { return back(lo); }
  __device__ __forceinline__ Run<MIXKV_BF16> high() const { return back(hi); }
  __device__ __forceinline__ static Run<MIXKV_BF16> back(const s16x2 (&x)[4]) {
    Run<MIXKV_BF16> r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[i] = __builtin_bit_cast(uint32_t, turn(x[i]));
    return r;
  }
};
template <> struct RunRange<MIXKV_F32> {
  float lo[8], hi[8];
  __device__ __forceinline__ void none() {
#pragma unroll
    for (int i = 0; i < 8; ++i) { lo[i] = INFINITY; hi[i] = -INFINITY; }
  }
  __device__ __forceinline__ void add(const Run<MIXKV_F32> &x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) { lo[i] = fminf(lo[i], x.at(i)); hi[i] = fmaxf(hi[i], x.at(i)); }
  }
  __device__ __forceinline__ void lower(const Run<MIXKV_F32> &x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) lo[i] = fminf(lo[i], x.at(i));
  }
  __device__ __forceinline__ void raise(const Run<MIXKV_F32> &x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) hi[i] = fmaxf(hi[i], x.at(i));
  }
  __device__ __forceinline__ void join(int off) {
#pragma unroll
    for (int i = 0; i < 8; ++i) { lo[i] = fminf(lo[i], __shfl_xor(lo[i], off)); hi[i] = fmaxf(hi[i], __shfl_xor(hi[i], off)); }
  }
  __device__ __forceinline__ Run<MIXKV_F32> low() const { Run<MIXKV_F32> r; r.set(lo); return r; }
  __device__ __forceinline__ Run<MIXKV_F32> high() const { Run<MIXKV_F32> r; r.set(hi); return r; }
};

// ---- 4 bits.  Step and base of a group from its extremes: the differences in 64 bits, rounded to fp32 and then to fp16.
struct GroupScale {
  float step, base;
  uint32_t bits;                                           // step, and base above it
  bool wide;                                               // elements beyond the format's range
};
__device__ __forceinline__ float clip(float x) { return fminf(fmaxf(x, -16384.f), 16384.f); }
__device__ __forceinline__ GroupScale group_scale(float least, float most) {
  GroupScale g;
  const float lo = clip(least), hi = clip(most);
  g.wide = lo != least || hi != most;
  const uint32_t sb = f16_bits((float)(((double)hi - (double)lo) * (16.0 / 15.0)));
  g.step = f16_value(sb);
  const uint32_t bb = f16_bits((float)((double)lo - (double)g.step) + 0.f);       // no negative zero
  g.base = f16_value(bb);
  g.bits = sb | (bb << 16);
  return g;
}
// Step and base of a run's group, whose other runs lie in the neighbouring three lanes.
__device__ __forceinline__ GroupScale run_scale(const Run<MIXKV_BF16> &x) {
  typedef RunRange<MIXKV_BF16> R;
  R::s16x2 v[4], lo, hi;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = R::turn(__builtin_bit_cast(R::s16x2, (uint32_t)x.v[i]));
  lo = __builtin_elementwise_min(__builtin_elementwise_min(v[0], v[1]), __builtin_elementwise_min(v[2], v[3]));
  hi = __builtin_elementwise_max(__builtin_elementwise_max(v[0], v[1]), __builtin_elementwise_max(v[2], v[3]));
  lo = __builtin_elementwise_min(lo, __builtin_bit_cast(R::s16x2, lane_moved<0xb1>(__builtin_bit_cast(int, lo))));   // lane ^ 1
  hi = __builtin_elementwise_max(hi, __builtin_bit_cast(R::s16x2, lane_moved<0xb1>(__builtin_bit_cast(int, hi))));
  lo = __builtin_elementwise_min(lo, __builtin_bit_cast(R::s16x2, lane_moved<0x4e>(__builtin_bit_cast(int, lo))));   // lane ^ 2
  hi = __builtin_elementwise_max(hi, __builtin_bit_cast(R::s16x2, lane_moved<0x4e>(__builtin_bit_cast(int, hi))));
  const R::s16x2 ends = R::turn(R::s16x2{lo[0] < lo[1] ? lo[0] : lo[1], hi[0] > hi[1] ? hi[0] : hi[1]});
  const uint32_t w = __builtin_bit_cast(uint32_t, ends);
  return group_scale(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

// The codes of eight elements in a word.  16 (x - base - step) / step as one multiply-add with 16 / step is off by less than 2^-21 of what its
// product and its constant are together (the reciprocal by 2^-23, the constant and the sum by another 2^-24 each, and the constant holds the
// reciprocal).  An element for which that could decide the rounding, and in bf16 rows exact ties between two codes are frequent (a run in some
// hundred), is taken again in 64 bits, one after another, as are those of a group with elements to be clipped.
__device__ __forceinline__ uint32_t run_codes(const Run<MIXKV_BF16> &x, const GroupScale &g) {
  const float r = g.step > 0.f ? 16.f * __builtin_amdgcn_rcpf(g.step) : 0.f, k = -(g.base + g.step) * r;
  uint32_t w = 0;
  float off = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float t = fmaf(x.at(e), r, k), n = __builtin_rintf(t);
    off = __builtin_fmaxf(off, __builtin_fabsf(t - n));
    w |= (uint32_t)__builtin_amdgcn_fmed3f(n, 0.f, 15.f) << code_shift(e);
  }
  const float far = 0.5f - 0x1p-21f * (40.f + 2.f * fabsf(k));
  if ((g.wide || off > far) && g.step > 0.f) {
    uint32_t again = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float t = fmaf(x.at(e), r, k);
      again |= g.wide || __builtin_fabsf(t - __builtin_rintf(t)) > far ? 1u << e : 0u;
    }
#pragma unroll 1
    while (again != 0) {
      const int e = __builtin_ctz(again);
      again &= again - 1;
      const uint32_t q = e < 4 ? (e < 2 ? x.v[0] : x.v[1]) : (e < 6 ? x.v[2] : x.v[3]), sh = code_shift(e);
      const double v = clip(__uint_as_float(e & 1 ? q & 0xffff0000u : q << 16));
      const double n = __builtin_rint((v - (double)g.base - (double)g.step) * 16.0 / (double)g.step);
      w = (w & ~(15u << sh)) | ((uint32_t)(n < 0. ? 0. : (n > 15. ? 15. : n)) << sh);
    }
  }
  return w;
}

// Where things lie in a 4-bit page, for lane j of a row's D/16: the words of the lane's two runs in a key row and their groups' scales are
// neighbours; a value row's element e of its strip.
template <int D>
struct Place4 {
  static constexpr int NG = D / 32;
  int j, r, e, strip;
  int64_t codes;                                          // bytes of codes in front of the scales
  __device__ __forceinline__ Place4(int j, int r, int P) : j(j), r(r), e(2 * (r & 3) + ((r >> 4) & 1)), strip((r >> 5) * 4 + ((r & 15) >> 2)), codes((int64_t)P * D / 2) {}
  __device__ __forceinline__ int ga() const { return j >> 2; }              // groups of the first and the second run
  __device__ __forceinline__ int gb() const { return (j >> 2) + NG / 2; }
  __device__ __forceinline__ u32x2 *key_words(char *page) const { return reinterpret_cast<u32x2 *>(page + r * (D / 2) + (j & 3) * (NG * 4) + 8 * ga()); }
  __device__ __forceinline__ u32x2 *key_scales(char *page) const { return reinterpret_cast<u32x2 *>(page + codes + (r * NG + 2 * ga()) * 4); }
  __device__ __forceinline__ uint16_t *value_scale(char *page, int g) const { return reinterpret_cast<uint16_t *>(page + codes) + (strip * NG + g) * 16 + e; }
  __device__ __forceinline__ uint32_t *strip_words(char *page) const { return reinterpret_cast<uint32_t *>(page) + strip * D; }
  // the word of a strip that holds element d
  __device__ __forceinline__ static int word_of(int d) { return (d >> 6) * 64 + (d & 15) * 4 + ((d >> 4) & 3); }
  __device__ __forceinline__ void store_keys(char *page, const Run<MIXKV_BF16> &a, const Run<MIXKV_BF16> &b, const GroupScale &sa, const GroupScale &sb) const {
    *key_words(page) = u32x2{run_codes(a, sa), run_codes(b, sb)};
    if ((j & 3) == 0) *key_scales(page) = u32x2{sa.bits, sb.bits};
  }
  __device__ __forceinline__ void store_value_scales(char *page, const GroupScale &sa, const GroupScale &sb) const {
    if ((j & 3) != 0) return;
    uint16_t *a = value_scale(page, ga()), *b = value_scale(page, gb());
    a[0] = (uint16_t)sa.bits; a[8] = (uint16_t)(sa.bits >> 16);
    b[0] = (uint16_t)sb.bits; b[8] = (uint16_t)(sb.bits >> 16);
  }
};

// The strips' words of the RS rows of a page from row s0 on, of which [lo_row, hi_row) are written, by a workgroup: eight rows' codes of an element each, out
// of words[row - s0][run] in LDS, a word for a run's eight codes.
template <int D, int RS, int THREADS>
__device__ __forceinline__ void store_strips(char *vp, const uint32_t *words, int s0, int lo_row, int hi_row) {
  constexpr int RUNS = D / 8;
  const bool full = s0 >= lo_row && s0 + RS <= hi_row;
  for (int i = threadIdx.x; i < RS / 8 * D; i += THREADS) {
    const int sl = i / D, wi = i - sl * D, el = (wi >> 6) * 64 + (wi & 3) * 16 + ((wi >> 2) & 15);   // strip of the pass, word, element
    const int t0 = s0 + (sl >> 2) * 32 + (sl & 3) * 4;   // the strip's first row in the page
    const uint32_t *from = words + (t0 - s0) * RUNS + (el >> 3);
    uint32_t *dst = reinterpret_cast<uint32_t *>(vp) + (t0 >> 5) * 4 * D + ((t0 & 15) >> 2) * D + wi;
    const uint32_t sh = code_shift(el & 7);
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) w |= ((from[((e >> 1) + 16 * (e & 1)) * RUNS] >> sh) & 15u) << code_shift(e);
    if (!full) {                                     // rows of the pass that are not written keep their codes
      uint32_t mask = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int rr = t0 + (e >> 1) + 16 * (e & 1);
        mask |= rr >= lo_row && rr < hi_row ? 15u << code_shift(e) : 0u;
      }
      if (mask == 0) continue;
      if (mask != 0xffffffffu) w = (w & mask) | (*dst & ~mask);
    }
    *dst = w;
  }
}

// Over a page's rows, of which every lane holds the range of its own: a workgroup's lanes with the same elements, then its waves, then (`add`) what the page's bounds hold.
// Barriers: one before the waves' parts are read, and one behind it.
template <int DT, int D>
__device__ __forceinline__ void store_bounds(char *dst, RunRange<DT> &ra, RunRange<DT> &rb, char (&red)[4][2 * D * (DT == MIXKV_BF16 ? 2 : 4)], bool add) {
  constexpr int EB = DT == MIXKV_BF16 ? 2 : 4, LPR = D / 16, RB = D * EB, RUNS = D / 8;
  const int tid = threadIdx.x, j = tid % LPR, lane = tid & 63, wave = tid >> 6;
#pragma unroll
  for (int off = LPR; off < 64; off <<= 1) { ra.join(off); rb.join(off); }
  if (lane < LPR) {
    char *at = red[wave] + 8 * EB * j;
    ra.low().store(at); rb.low().store(at + RB / 2);
    ra.high().store(at + RB); rb.high().store(at + RB + RB / 2);
  }
  __syncthreads();
  if (tid < 2 * RUNS) {                                // a run of the smallest, or of the largest elements
    const int side = tid / RUNS, run = tid - side * RUNS;
    RunRange<DT> m;
    m.none();
    Run<DT> v;
#pragma unroll
    for (int w = 0; w < 4; ++w) { v.load(red[w] + side * RB + 8 * EB * run); m.add(v); }
    dst += side * RB + 8 * EB * run;
    if (add) { v.load(dst); m.add(v); }                // rows of an earlier call are in the page
    (side ? m.high() : m.low()).store(dst);
  }
  __syncthreads();
}

}  // namespace mixkv
