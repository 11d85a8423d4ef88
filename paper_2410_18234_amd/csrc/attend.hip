// Attention over the paged 8-bit cache (gfx950).
//
//   s_j = scale q . k_j,  out = sum_j softmax(s)_j v_j  over the cached tokens j <= the query's own position,
// with k_j = code 2^ke and v_j = code 2^ve, the exponents of the token's page and head.
//
// A wave takes 64 tokens at a time against MT tiles of 16 query rows (a row = one new token of one of the query
// heads that share a cache head).  It computes S^T = K Q^T and then O^T = V^T P^T, so that the accumulators of the
// first product are, lane by lane, the second's operand: lane (m, g) = (lane & 15, lane >> 4) holds row m's scores of
// the 16 tokens of unit g in both.  Codes go from memory to registers (16 bytes of a key chunk or of a value's
// 16 tokens), are widened (exactly: bf16 or f16 keys, f16 values) and feed the matrix cores: straight from the registers
// for few rows, through LDS for many (the two kernels below).  One pass with a running maximum: with t = s log2(e) + ve, in the
// frame M = max t so far,
//   p = 2^(t - M + kLift) <= 2^15 carries the value's scale,
//   l = sum p 2^-ve the softmax's sum in the same frame (fp32), out = sum p code / l.
// (c_g = scale log2(e) 2^ke is the lane's, so t is one fused multiply-add.)
// The matrix cores take p in f16, which holds 11 bits of it down to 2^-14: 2^-29 of the largest.  Smaller ones matter where the
// tokens that lead hold values near zero, or a page has a much larger scale: where what f16 drops could reach 2^-16 of a row's
// largest element (`lacks`) a wave goes over its tokens again (PRECISE), and it goes through a product of its own in a frame of its
// own (left_of_low).  That costs such a wave more than its first pass; doing it in the one pass, in every tile that has smaller
// weights, took peaked scores (twice the usual spread, 4 x up to 1024 new of up to 5000 tokens) from 256 to 580 us.  Exponents lie in
// [-40, 40]: a term that l loses (below 2^-126) has less than 2^-61 of the largest weight.
#include "cache.h"

#include <math.h>

namespace mdss {

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

struct AttendArgs {
  const void* q;
  const uint8_t *k, *v;
  const int8_t *k_exp, *v_exp;
  const int32_t *starts, *table, *lengths;
  void* out;
  float* lse;
  float *part, *part_ml;  // partial rows of a split call: [T * heads_q][splits][D], [..][splits][2]
  int64_t q_st, q_sh, width, T, pages;
  int S, heads, group, page_shift;
  int per_seq;   // row tiles of a sequence (uniform), 0: found from starts
  int slot0;     // first row tile of the launch
  int splits, split_tiles;
  float scale_log2;  // |scale| log2(e)
  bool negative;
};

template <bool BF>
struct Elem;
template <>
struct Elem<true> {
  typedef bf16x8 vec;
  typedef __bf16 one;
  static __device__ __forceinline__ f32x4 mfma(vec a, vec b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ vec widen(uint32_t lo, uint32_t hi) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    return vec{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  }
};
template <>
struct Elem<false> {
  typedef f16x8 vec;
  typedef _Float16 one;
  static __device__ __forceinline__ f32x4 mfma(vec a, vec b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ vec widen(uint32_t lo, uint32_t hi) {
    const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false);
    const f16x2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
    const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false);
    const f16x2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
    return vec{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  }
};

constexpr float kLift = 15.0f;  // p <= 2^kLift

template <bool V>
struct Flag {
  static constexpr bool value = V;
};

// Maximum / sum over the four lanes (m, 0..3) of a row.
__device__ __forceinline__ float row_max4(float x) {
  uint32_t u = __builtin_bit_cast(uint32_t, x);
  auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  x = fmaxf(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
  u = __builtin_bit_cast(uint32_t, x);
  a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
}
__device__ __forceinline__ float row_sum4(float x) {
  uint32_t u = __builtin_bit_cast(uint32_t, x);
  auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  x = __builtin_bit_cast(float, (uint32_t)a[0]) + __builtin_bit_cast(float, (uint32_t)a[1]);
  u = __builtin_bit_cast(uint32_t, x);
  a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __builtin_bit_cast(float, (uint32_t)a[0]) + __builtin_bit_cast(float, (uint32_t)a[1]);
}

// 2^e for a whole number e in [-126, 127]
__device__ __forceinline__ float pow2i(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }

// Bytes that are a NaN code (0x7f, 0xff): 0x80 in their place
__device__ __forceinline__ uint32_t nan_bytes(uint32_t x) { return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// `keep` (0 .. 16) lowest bytes of 16
__device__ __forceinline__ u32x4 low_bytes(u32x4 x, int keep) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int n = min(max(keep - 4 * w, 0), 4);
    x[w] = n == 4 ? x[w] : x[w] & ((1u << (8 * n)) - 1u);
  }
  return x;
}

// The natural log of a row's sum of exp(scale q . k), from its frame and its sum l there.  (l's octave goes to the frame first:
// the logarithm left is of 0.5 .. 1, where its rounding is small.)
__device__ __forceinline__ float log_sum(float M, float l) {
  if (l == 0.0f) return -INFINITY;
  int octave;
  const float part = frexpf(l, &octave);
  return ((M + ((float)octave - kLift)) + log2f(part)) * 0.693147180559945f;
}

// The frame of two partial sums: their weights, given (M, l) of each; rows without a visible token have M = -inf.
__device__ __forceinline__ float frame_weight(float M, float top) { return M == -INFINITY ? 0.0f : exp2f(M - top); }

// The pages of a sequence's units, never out of the table or the pool.
struct PageWalk {
  const int32_t* row;
  int64_t pages;
  int heads, h, unit_shift, last_page;  // (a page has 1 << unit_shift units)
  __device__ __forceinline__ PageWalk(const AttendArgs& a, const struct Place& p);
  __device__ __forceinline__ int page(int unit) const { return row[min(unit >> unit_shift, last_page)]; }
  __device__ __forceinline__ int valid(int page, bool& ok) const {  // page 0 in place of none
    ok = (uint32_t)page < (uint64_t)pages;
    return ok ? page : 0;
  }
  __device__ __forceinline__ const uint8_t* unit(const uint8_t* base, int page, int unit, int bytes) const {
    return base + ((((int64_t)page * heads + h) << unit_shift) + (unit & ((1 << unit_shift) - 1))) * bytes;
  }
};

// Where a workgroup stands: its row tile of a sequence, and what that sequence holds.
struct Place {
  int s, tile, h;
  int n, rows;      // new tokens, and rows (tokens x query heads of this cache head)
  int64_t start;    // its first token of T
  int len, before;  // cached tokens (as far as the table goes); those before the new ones (negative: the first rows see nothing)
};
// The head is the fastest index of the grid: the row tiles that read one head's pages run on the same XCD where heads
// are a multiple of 8 (workgroups go round the XCDs in order), and find them in its L2.  A sequence's last rows, which see the
// most tokens, start first (a prompt of 3000 tokens, 64 query heads: 205 us, 246 the other way round).
__device__ __forceinline__ bool attend_place(const AttendArgs& a, int tile_rows, int lane, Place& p) {
  const int part = blockIdx.x / a.heads, slot = a.slot0 + part;
  p.h = blockIdx.x - part * a.heads;
  if (a.per_seq > 0) {
    p.s = slot / a.per_seq;
    p.tile = slot - p.s * a.per_seq;
  } else {
    p.s = slot_sequence(a.starts, a.S, slot, a.group, tile_rows, 1, lane);
    p.tile = slot - (int)slot_first(a.starts, p.s, a.group, tile_rows, 1);
  }
  if (a.starts) {
    p.start = a.starts[p.s];
    p.n = (int)(a.starts[p.s + 1] - p.start);
  } else {
    p.n = (int)(a.T / a.S);
    p.start = (int64_t)p.s * p.n;
  }
  if (p.start < 0 || p.n <= 0 || p.start + p.n > a.T) return false;  // no rows, or starts that do not ascend within T
  p.rows = p.n * a.group;
  const int tiles = (p.rows + tile_rows - 1) / tile_rows;
  if (p.tile < 0 || p.tile >= tiles) return false;  // (below 0: starts[0] is not 0)
  p.tile = tiles - 1 - p.tile;
  const int length = a.lengths[p.s];
  p.len = max(0, min(length, (int)min(a.width << a.page_shift, (int64_t)INT32_MAX)));
  p.before = length - p.n;
  return true;
}
// Tokens that the rows up to `last` see at most.
__device__ __forceinline__ int seen_by(const AttendArgs& a, const Place& p, int last) {
  return min(p.len, p.before + min(p.rows - 1, last) / a.group + 1);
}

__device__ __forceinline__ PageWalk::PageWalk(const AttendArgs& a, const Place& p)
    : row(a.table + (int64_t)p.s * a.width), pages(a.pages), heads(a.heads), h(p.h), unit_shift(a.page_shift - 4),
      last_page(p.len > 0 ? (p.len - 1) >> a.page_shift : 0) {}

// Row r's queries: lane (m, g) holds elements 64 i + 16 g + 0 .. 15 (the last 32 of a D that is no multiple of 64: 8 g ..),
// negated where the scale is negative, so that a larger product is a larger score.
template <int D, bool BF, int MT>
__device__ __forceinline__ void load_queries(const AttendArgs& a, const Place& p, int row0, int m, int g,
                                             typename Elem<BF>::vec (&qf)[MT][D / 32], int (&lim)[MT]) {
  typedef typename Elem<BF>::vec vec;
  typedef typename Elem<BF>::one one;
#pragma unroll
  for (int r = 0; r < MT; ++r) {
    const int row = row0 + 16 * r + m;
    const bool in = row < p.rows;
    const int i = in ? row / a.group : 0, hg = in ? row - i * a.group : 0;
    lim[r] = in ? min(p.len, p.before + i + 1) : 0;
    const one* qr = static_cast<const one*>(a.q) + (p.start + i) * a.q_st + (int64_t)(p.h * a.group + hg) * a.q_sh;
#pragma unroll
    for (int st = 0; st < D / 32; ++st) {
      const int at = (D % 64 != 0 && st == D / 32 - 1) ? D - 32 + 8 * g : 64 * (st >> 1) + 16 * g + 8 * (st & 1);
      vec x;
      if ((reinterpret_cast<uintptr_t>(qr) & 15) == 0) {
        x = *reinterpret_cast<const vec*>(qr + at);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = qr[at + j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = !in ? (one)0.0f : a.negative ? -x[j] : x[j];
      qf[r][st] = x;
    }
  }
}

// The weights of 64 tokens from their scores: raise_frame sets the frame M, weigh takes the weights in it.  All of a lane's
// scores are of one unit, so its page's scales are one factor and one addend (c_g >= 0, ve_g), and the extremes can be taken of
// the products themselves.  upto[r]: the unit's tokens that row r sees.
//
// The frame follows the maximum whenever some row of the wave finds a larger one, a few times in a sequence: by alpha, what was
// summed before shrinks (returns whether it does).  A frame that lags would leave f16 less range below.
//
// t - M + kLift is one fused multiply-add with ve - M + kLift, whose rounding grows with M.  From kFar on (`far`) the precise frame is
// one of scores without ve, max s log2(e), and weights are 2^((s log2(e) - M) + (ve + kLift)): the largest score is exact, and equal
// scores weigh the same whatever their pages.  M is a reference that sums carry, so rows may change from one to the other.
constexpr float kFar = 65536.0f;
__device__ __forceinline__ bool is_far(float M) { return fabsf(M) > kFar && M > -INFINITY; }
template <int MT, bool MASKED, bool PRECISE>
__device__ __forceinline__ bool raise_frame(const f32x4 (&sc)[4][MT], float c_g, float ve_g, const int (&upto)[MT], float (&M)[MT],
                                            float (&l)[MT], float (&alpha)[MT], bool& far) {
  float top[MT], score[MT];
  bool grown = false;
#pragma unroll
  for (int r = 0; r < MT; ++r) {
    float mx = -INFINITY;
#pragma unroll
    for (int tt = 0; tt < 4; ++tt)
#pragma unroll
      for (int i = 0; i < 4; ++i) mx = fmaxf(mx, !MASKED || 4 * tt + i < upto[r] ? sc[tt][r][i] : -INFINITY);
    score[r] = mx;
    top[r] = row_max4(mx == -INFINITY ? mx : fmaf(mx, c_g, ve_g));
    grown |= top[r] > M[r];
  }
  grown = __ballot(grown) != 0;
  if (grown) {
    far = false;
    if (PRECISE) {
#pragma unroll
      for (int r = 0; r < MT; ++r) far |= is_far(fmaxf(M[r], top[r]));
      far = __ballot(far) != 0;
    }
#pragma unroll
    for (int r = 0; r < MT; ++r) {
      if (PRECISE && far) top[r] = row_max4(score[r] == -INFINITY ? score[r] : score[r] * c_g);
      const float to = fmaxf(M[r], top[r]);
      alpha[r] = M[r] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(M[r] - to);
      l[r] *= alpha[r];
      M[r] = to;
    }
  }
  return grown;
}
__device__ __forceinline__ float weight_offset(float ve_g, float M) { return ve_g + kLift - (M == -INFINITY ? 0.0f : M); }

// The weight of a far tile's score (fp32: up to 2^55, before the sum takes the value's scale out)
__device__ __forceinline__ float far_weight(float sc, float c_g, float ve_g, float M) {
  return __builtin_amdgcn_exp2f((sc * c_g - (M == -INFINITY ? 0.0f : M)) + (ve_g + kLift));
}

// The sums of a far tile's weights, which leave f16's range: left_of_low takes all of them.
template <int MT>
__device__ __forceinline__ void weigh_far(const f32x4 (&sc)[4][MT], float c_g, float ve_g, float inv_v, const int (&upto)[MT],
                                          const float (&M)[MT], float (&l)[MT], f16x8 (&pf)[MT][2]) {
#pragma unroll
  for (int r = 0; r < MT; ++r) {
    float sum = 0.0f;
#pragma unroll
    for (int tt = 0; tt < 4; ++tt)
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += 4 * tt + i < upto[r] ? far_weight(sc[tt][r][i], c_g, ve_g, M[r]) : 0.0f;
    l[r] = fmaf(sum, inv_v, l[r]);
    pf[r][0] = pf[r][1] = f16x8{0, 0, 0, 0, 0, 0, 0, 0};
  }
}

// least: the smallest visible weight so far, by its bits (weights are not negative).
template <int MT, bool MASKED>
__device__ __forceinline__ void weigh(const f32x4 (&sc)[4][MT], float c_g, float ve_g, float inv_v, const int (&upto)[MT],
                                      const float (&M)[MT], float (&l)[MT], f16x8 (&pf)[MT][2], u16x2& least) {
#pragma unroll
  for (int r = 0; r < MT; ++r) {
    const float off = weight_offset(ve_g, M[r]);
    float sum = 0.0f;
#pragma unroll
    for (int tt = 0; tt < 4; ++tt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float p = __builtin_amdgcn_exp2f(fmaf(sc[tt][r][i], c_g, off));
        if (MASKED) p = 4 * tt + i < upto[r] ? p : 0.0f;
        sum += p;
        pf[r][tt >> 1][4 * (tt & 1) + i] = (_Float16)p;
      }
    l[r] = fmaf(sum, inv_v, l[r]);
#pragma unroll
    for (int j = 0; j < 16; j += 2) {
      const f16x2 two = {pf[r][j >> 3][j & 7], pf[r][j >> 3][(j & 7) + 1]};
      u16x2 bits = __builtin_bit_cast(u16x2, two);
      if (MASKED) bits = u16x2{j < upto[r] ? bits[0] : (uint16_t)0x3c00, j + 1 < upto[r] ? bits[1] : (uint16_t)0x3c00};
      least = __builtin_elementwise_min(least, bits);
    }
  }
}

// Whether a wave's sums may lack too much: its scores are far; or f16 dropped something of its weights (some lay below its normal
// range), and pages' scales are 2^kSpread and more apart (what one page has large in some elements may hide another's in the rest), or
// some row's sums are all small.  `tokens` weights that f16 rounded below 2^-14 are off by tokens 2^-25 448 in all, 2^-16 of a sum
// that reaches `tokens`.
constexpr float kSpread = 12.0f;
template <int MT, int TILES>
__device__ __forceinline__ bool lacks(const f32x4 (&acc)[TILES][MT], const float (&M)[MT], const int (&lim)[MT], u16x2 least,
                                      float ve_least, float ve_most, float tokens) {
  bool far = false;
#pragma unroll
  for (int r = 0; r < MT; ++r) far |= is_far(M[r]);
  if (__ballot(far) != 0) return true;
  if (__ballot(min(least[0], least[1]) < 0x0400) == 0) return false;
  if (wave_max(ve_most) + wave_max(-ve_least) >= kSpread) return true;
  bool small = false;
#pragma unroll
  for (int r = 0; r < MT; ++r) {
    float most = 0.0f;
#pragma unroll
    for (int dt = 0; dt < TILES; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) most = fmaxf(most, fabsf(acc[dt][r][i]));
    small |= row_max4(most) < tokens && lim[r] > 0 && M[r] > -INFINITY;
  }
  return __ballot(small) != 0;
}

// What f16 does not hold of a row tile's weights below its normal range, p - f16(p), as f16 in a frame of its own: times a power
// of two that brings the row's largest to 2^14 .. 2^15; back: what brings a sum of them into the frame M again.  Of a far
// tile all of p.
template <int MT>
__device__ __forceinline__ void left_of_low(const f32x4 (&sc)[4][MT], int r, float c_g, float ve_g, int upto, float M, bool far,
                                            f16x8 (&left)[2], float& back) {
  __builtin_amdgcn_sched_barrier(0);
  float off = weight_offset(ve_g, M);
  asm volatile("" : "+v"(off));  // (weights computed again, not held from weigh)
  const auto weight = [&](int tt, int i) {  // (as in weigh)
    const float p = far ? far_weight(sc[tt][r][i], c_g, ve_g, M) : __builtin_amdgcn_exp2f(fmaf(sc[tt][r][i], c_g, off));
    return 4 * tt + i < upto && (far || p < 0x1p-14f) ? p : 0.0f;
  };
  float most = 0.0f;
#pragma unroll
  for (int tt = 0; tt < 4; ++tt)
#pragma unroll
    for (int i = 0; i < 4; ++i) most = fmaxf(most, weight(tt, i));
  // (what is left of a weight of 2^-24 or more is at most 2^-25)
  most = fmaxf(row_max4(most), 0x1p-110f);
  if (!far) most = fminf(most, 0x1p-25f);
  const uint32_t octave = __builtin_bit_cast(uint32_t, most) & 0x7f800000u;
  const float up = __builtin_bit_cast(float, 0x7f000000u - octave) * 0x1p14f;
  back = __builtin_bit_cast(float, octave) * 0x1p-14f;
#pragma unroll
  for (int tt = 0; tt < 4; ++tt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p = weight(tt, i);
      left[tt >> 1][4 * (tt & 1) + i] = (_Float16)((far ? p : p - (float)(_Float16)p) * up);
    }
}

// Adds what is left of a row tile's low weights to its sums: v(dt, half) are the tile's values as operands (one accumulator after
// the other, in few registers).
template <int MT, int TILES, typename Values>
__device__ __forceinline__ void add_left(const f16x8 (&left)[2], float back, int r, f32x4 (&acc)[TILES][MT], Values values) {
#pragma unroll
  for (int dt = 0; dt < TILES; ++dt) {
    __builtin_amdgcn_sched_barrier(0);
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int hs = 0; hs < 2; ++hs) sum = Elem<false>::mfma(values(dt, hs), left[hs], sum);
    acc[dt][r] = __builtin_elementwise_fma(sum, f32x4{back, back, back, back}, acc[dt][r]);
  }
  __builtin_amdgcn_sched_barrier(0);
}

// A NaN code among tokens that only some rows see must reach those rows alone: it is taken out of the values (a lane's 16
// tokens of one d) and counted in a product of its own.
__device__ __forceinline__ uint32_t nan_any(const u32x4& v) {
  return nan_bytes(v[0]) | nan_bytes(v[1]) | nan_bytes(v[2]) | nan_bytes(v[3]);
}
__device__ __forceinline__ u32x4 nan_out(u32x4 v) {
#pragma unroll
  for (int w = 0; w < 4; ++w) v[w] &= ~((nan_bytes(v[w]) >> 7) * 0xffu);
  return v;
}
template <int MT>
__device__ __forceinline__ void mark_nan(const u32x4& v, const int (&upto)[MT], f32x4 (&acc)[MT]) {
  u32x4 flag;
#pragma unroll
  for (int w = 0; w < 4; ++w) flag[w] = (nan_bytes(v[w]) >> 7) * 0x38u;  // the code of 1.0
#pragma unroll
  for (int r = 0; r < MT; ++r) {
    f32x4 hit = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int hs = 0; hs < 2; ++hs) {
      f16x8 see;
#pragma unroll
      for (int j = 0; j < 8; ++j) see[j] = 8 * hs + j < upto[r] ? (_Float16)1.0f : (_Float16)0.0f;
      hit = Elem<false>::mfma(Elem<false>::widen(flag[2 * hs], flag[2 * hs + 1]), see, hit);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[r][i] = hit[i] > 0.0f ? NAN : acc[r][i];
  }
}

template <int MT>
__device__ __forceinline__ void add_values(const f16x8 (&v)[2], const f16x8 (&pf)[MT][2], f32x4 (&acc)[MT]) {
#pragma unroll
  for (int hs = 0; hs < 2; ++hs)
#pragma unroll
    for (int r = 0; r < MT; ++r) acc[r] = Elem<false>::mfma(v[hs], pf[r][hs], acc[r]);
}

// Few rows: the four waves of a workgroup take the same rows against tiles of 64 tokens in turn, straight from memory
// to registers, and join at the end.  Bound by memory: a tile's keys are loaded while the one before is
// weighed, its values while its keys are multiplied.  4 x 131072 tokens, 8 heads of 128: 194 us, 5.5 TB/s; 64 sequences of 1024 to
// 4096 tokens with up to 5 new ones: 66 us, 4.3 TB/s.
constexpr int joined_part(int D) { return 16 * (D + 4); }  // floats of a wave
template <int D, bool BF, int MT>
__device__ __forceinline__ void attend_rows(const AttendArgs& a, const Place& p, float* joined, float* joined_ml,
                                            typename Elem<BF>::vec* queries) {
  using E = Elem<BF>;
  using vec = typename E::vec;
  using one = typename E::one;
  constexpr int kSteps = D / 32;       // matrix steps over d
  constexpr int kWhole = D / 64;       // 16-byte loads of a key's quarter
  constexpr bool kHalf = D % 64 != 0;  // and one of 8 bytes
  constexpr int kTiles = D / 16;       // accumulator tiles over d
  constexpr int kPad = D + 4;
  constexpr int NW = 4;  // waves

  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int split = blockIdx.y;
  const int row0 = p.tile * 16 * MT, h = p.h;
  const int lim_lo = seen_by(a, p, row0), lim_hi = seen_by(a, p, row0 + 16 * MT - 1);
  const int tiles = lim_hi > 0 ? (lim_hi + 63) >> 6 : 0;
  const int t_begin = split * a.split_tiles;
  const int t_end = split == a.splits - 1 ? tiles : min(tiles, t_begin + a.split_tiles);
  // a split without tokens for any of the rows has nothing to say (the first one always speaks)
  if (split > 0 && t_begin >= tiles) return;

  int lim[MT];
  {
    vec qf[MT][kSteps];
    load_queries<D, BF, MT>(a, p, row0, m, g, qf, lim);
    if (wave == 0) {
#pragma unroll
      for (int r = 0; r < MT; ++r)
#pragma unroll
        for (int st = 0; st < kSteps; ++st) queries[(r * kSteps + st) * 64 + lane] = qf[r][st];
    }
    __syncthreads();
  }
  f32x4 acc[kTiles][MT];
  float M[MT], l[MT];
  u16x2 least = {0x3c00, 0x3c00};
  float ve_least = INFINITY, ve_most = -INFINITY;  // of the units' value exponents

  float* const part = joined + wave * joined_part(D);  // the wave's sums, after the tokens

  const int t0 = t_begin + wave;
  const PageWalk walk(a, p);
  u32x4 kc[4][kWhole];
  u32x2 kh[4];
  const auto load_k = [&](int page, int t) __attribute__((always_inline)) {
    const uint8_t* at = walk.unit(a.k, page, 4 * t + (m >> 2), 16 * D) + (m & 3) * 16;
#pragma unroll
    for (int tt = 0; tt < 4; ++tt) {
#pragma unroll
      for (int i = 0; i < kWhole; ++i) kc[tt][i] = *reinterpret_cast<const u32x4*>(at + tt * 64 + i * 1024 + g * 256);
      if (kHalf) kh[tt] = *reinterpret_cast<const u32x2*>(at + tt * 64 + (4 * kWhole + (g >> 1)) * 256 + (g & 1) * 8);
    }
  };

  const auto pass = [&](auto flag) __attribute__((always_inline)) {
    constexpr bool PRECISE = decltype(flag)::value;
#pragma unroll
    for (int r = 0; r < MT; ++r) {
      M[r] = -INFINITY;
      l[r] = 0.0f;
#pragma unroll
      for (int dt = 0; dt < kTiles; ++dt) acc[dt][r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    if (t0 >= t_end) return;
    bool far = false;
    bool ok, ok_k;
    int pk, pv, ke, ve;
    const auto load_tile = [&](int page_k, int page_v, int t) __attribute__((always_inline)) {
      pk = walk.valid(page_k, ok_k);
      load_k(pk, t);
      pv = walk.valid(page_v, ok);
      ke = a.k_exp[(int64_t)pv * a.heads + h];
      ve = a.v_exp[(int64_t)pv * a.heads + h];
    };
    int pk_next = walk.page(4 * t0 + (m >> 2)), pv_next = walk.page(4 * t0 + g);
    if (!PRECISE) {
      load_tile(pk_next, pv_next, t0);
      pk_next = walk.page(4 * (t0 + NW) + (m >> 2));
      pv_next = walk.page(4 * (t0 + NW) + g);
    }
    for (int t = t0; t < t_end; t += NW) {
      if (PRECISE) load_tile(walk.page(4 * t + (m >> 2)), walk.page(4 * t + g), t);  // (nothing ahead: few registers)
      u32x4 vc[kTiles];
      {
        const uint8_t* at = walk.unit(a.v, pv, 4 * t + g, 16 * D) + m * 16;
#pragma unroll
        for (int dt = 0; dt < kTiles; ++dt) vc[dt] = *reinterpret_cast<const u32x4*>(at + dt * 256);
      }
      f32x4 sc[4][MT];
#pragma unroll
      for (int st = 0; st < kSteps; ++st) {
        vec qf[MT];
#pragma unroll
        for (int r = 0; r < MT; ++r) qf[r] = queries[(r * kSteps + st) * 64 + lane];
#pragma unroll
        for (int tt = 0; tt < 4; ++tt) {
          const vec kf = (kHalf && st == kSteps - 1) ? E::widen(kh[tt][0], kh[tt][1])
                                                      : E::widen(kc[tt][st >> 1][2 * (st & 1)], kc[tt][st >> 1][2 * (st & 1) + 1]);
#pragma unroll
          for (int r = 0; r < MT; ++r)
            sc[tt][r] = E::mfma(kf, qf[r], st == 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : sc[tt][r]);
        }
      }
      if (!ok) ke = ve = 0;  // (no page: page 0 was read in its place, whose exponents may be any byte)
      float c_g = a.scale_log2 * pow2i(ke), ve_g = (float)ve, inv_v = pow2i(-ve);
      asm volatile("" : "+v"(c_g), "+v"(ve_g), "+v"(inv_v));  // (before the next tile's exponents are loaded, into the same registers)
      const bool ok_now = ok;
      // the next tile's keys, exponents, and the page ids after it
      __builtin_amdgcn_sched_barrier(0);  // (into the registers of this one's)
      if (!PRECISE) {
        load_tile(pk_next, pv_next, t + NW);
        pk_next = walk.page(4 * (t + 2 * NW) + (m >> 2));
        pv_next = walk.page(4 * (t + 2 * NW) + g);
      }

      const bool masked = 64 * (t + 1) > lim_lo || __ballot(ok_now) != ~0ull;
      const int first = 64 * t + 16 * g;  // the lane's first token
      int upto[MT];
#pragma unroll
      for (int r = 0; r < MT; ++r) upto[r] = ok_now ? lim[r] - first : 0;
      float alpha[MT];
      f16x8 pf[MT][2];
      bool grown;
      if constexpr (PRECISE) {
        grown = raise_frame<MT, true, true>(sc, c_g, ve_g, upto, M, l, alpha, far);
        if (far)
          weigh_far<MT>(sc, c_g, ve_g, inv_v, upto, M, l, pf);
        else
          weigh<MT, true>(sc, c_g, ve_g, inv_v, upto, M, l, pf, least);
      } else {
        ve_least = fminf(ve_least, ve_g);
        ve_most = fmaxf(ve_most, ve_g);
        grown = masked ? raise_frame<MT, true, false>(sc, c_g, ve_g, upto, M, l, alpha, far)
                       : raise_frame<MT, false, false>(sc, c_g, ve_g, upto, M, l, alpha, far);
        if (masked)
          weigh<MT, true>(sc, c_g, ve_g, inv_v, upto, M, l, pf, least);
        else
          weigh<MT, false>(sc, c_g, ve_g, inv_v, upto, M, l, pf, least);
      }
      if (grown) {
#pragma unroll
        for (int r = 0; r < MT; ++r)
#pragma unroll
          for (int dt = 0; dt < kTiles; ++dt) acc[dt][r] *= alpha[r];
      }
      if (masked) {
        // what lies past the sequence's end is not the cache's: any bytes
        const int keep = ok_now ? min(max(p.len - first, 0), 16) : 0;
        uint32_t any = 0;
#pragma unroll
        for (int dt = 0; dt < kTiles; ++dt) {
          vc[dt] = low_bytes(vc[dt], keep);
          any |= nan_any(vc[dt]);
        }
        if (__ballot(any != 0) != 0) {
#pragma unroll
          for (int dt = 0; dt < kTiles; ++dt) {
            mark_nan<MT>(vc[dt], upto, acc[dt]);
            vc[dt] = nan_out(vc[dt]);
          }
        }
      }
#pragma unroll
      for (int dt = 0; dt < kTiles; ++dt) {
        const f16x8 v[2] = {Elem<false>::widen(vc[dt][0], vc[dt][1]), Elem<false>::widen(vc[dt][2], vc[dt][3])};
        add_values<MT>(v, pf, acc[dt]);
      }
      if constexpr (PRECISE) {
#pragma unroll
        for (int r = 0; r < MT; ++r) {
          f16x8 left[2];
          float back;
          left_of_low<MT>(sc, r, c_g, ve_g, upto[r], M[r], far, left, back);
          add_left<MT, kTiles>(left, back, r, acc, [&](int dt, int hs) {
            uint32_t lo = vc[dt][2 * hs], hi = vc[dt][2 * hs + 1];
            asm volatile("" : "+v"(lo), "+v"(hi));  // (widened again, not held from above)
            return Elem<false>::widen(lo, hi);
          });
        }
      }
    }
  };
  pass(Flag<false>{});
  if (t0 < t_end && lacks<MT, kTiles>(acc, M, lim, least, ve_least, ve_most, 64.0f * ((t_end - t0 + NW - 1) / NW))) pass(Flag<true>{});

  // join the four waves, 16 rows at a time: thread -> a row and a share of its elements
#pragma unroll
  for (int r = 0; r < MT; ++r) l[r] = row_sum4(l[r]);
  const int64_t heads_q = (int64_t)a.heads * a.group;
  constexpr int kShare = D / (4 * NW);  // elements of a thread
  const int jr = threadIdx.x / (4 * NW), jd = threadIdx.x % (4 * NW) * kShare;
#pragma unroll
  for (int r = 0; r < MT; ++r) {
    if (r > 0) __syncthreads();
    float* w = part + m * kPad + 4 * g;
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt) *reinterpret_cast<f32x4*>(w + 16 * dt) = acc[dt][r];
    if (g == 0) {
      joined_ml[(wave * 16 + m) * 2] = M[r];
      joined_ml[(wave * 16 + m) * 2 + 1] = l[r];
    }
    __syncthreads();
    float top = -INFINITY, lsum = 0.0f, wgt[NW];
#pragma unroll
    for (int i = 0; i < NW; ++i) top = fmaxf(top, joined_ml[(i * 16 + jr) * 2]);
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      wgt[i] = frame_weight(joined_ml[(i * 16 + jr) * 2], top);
      lsum = fmaf(wgt[i], joined_ml[(i * 16 + jr) * 2 + 1], lsum);
    }
    const int row = row0 + 16 * r + jr;
    if (row < p.rows) {
      const int i = row / a.group;
      const int64_t id = (p.start + i) * heads_q + h * a.group + (row - i * a.group);  // row of [T][heads_q]
      const float inv = lsum == 0.0f ? 0.0f : 1.0f / lsum;
#pragma unroll
      for (int e = 0; e < kShare; e += 2) {
        f32x2 o = {0.0f, 0.0f};
#pragma unroll
        for (int w4 = 0; w4 < NW; ++w4) {
          const f32x2 x = *reinterpret_cast<const f32x2*>(joined + w4 * joined_part(D) + jr * kPad + jd + e);
          o[0] = fmaf(wgt[w4], x[0], o[0]);
          o[1] = fmaf(wgt[w4], x[1], o[1]);
        }
        if (a.splits == 1) {
          typedef one one2 __attribute__((ext_vector_type(2)));
          const one2 w2 = {(one)(lsum == 0.0f ? 0.0f : o[0] * inv), (one)(lsum == 0.0f ? 0.0f : o[1] * inv)};
          *reinterpret_cast<one2*>(static_cast<one*>(a.out) + id * D + jd + e) = w2;
        } else {
          *reinterpret_cast<f32x2*>(a.part + (id * a.splits + split) * D + jd + e) = o;
        }
      }
      if (jd == 0) {
        if (a.splits == 1) {
          if (a.lse) a.lse[id] = log_sum(top, lsum);
        } else {
          a.part_ml[2 * (id * a.splits + split)] = top;
          a.part_ml[2 * (id * a.splits + split) + 1] = lsum;
        }
      }
    }
  }
}

// A sequence that fills fewer of the row tiles than the batch's most multiplies as many as it fills (64 sequences of 2000 tokens with
// up to 6 new ones, 8 query heads a cache head: 64 us, 77 with all tiles; 64 x up to 4096 with up to 5: 66 and 71).
// (The bounds are the workgroups a CU that attend_plan counts on: what does not fit the registers then is the precise pass's.)
template <int D, bool BF, int MT>
__global__ __launch_bounds__(256, D > 128 || MT > 2 ? 1 : MT == 2 || D > 96 ? 2 : D == 96 ? 3 : 4) void attend_kernel(const AttendArgs a) {
  __shared__ __align__(16) float joined[4 * joined_part(D)];
  __shared__ float joined_ml[4 * 16 * 2];
  __shared__ __align__(16) typename Elem<BF>::vec queries[MT * D / 32 * 64];  // the same for all four waves: LDS spares their registers
  Place p;
  if (!attend_place(a, 16 * MT, threadIdx.x & 63, p)) return;
  if (MT > 1 && p.rows <= 16)
    attend_rows<D, BF, 1>(a, p, joined, joined_ml, queries);
  else if (MT > 2 && p.rows <= 32)
    attend_rows<D, BF, 2>(a, p, joined, joined_ml, queries);
  else
    attend_rows<D, BF, MT>(a, p, joined, joined_ml, queries);
}

// Many rows: the four waves take different rows (MT tiles of 16 each) against the same tiles of 64 tokens, which go through
// LDS: the next tile's codes are loaded while this one is multiplied, widened once for all four waves, and written for
// the step after.  A piece of LDS is what one lane multiplies at a time (16 bytes), in the order of the lanes.  Bound by what a wave
// does one after the other (two products, the softmax between them, widening): vector instructions take 56 % of a SIMD's
// cycles, matrix instructions 31 %, and its two waves hardly overlap; LDS is busy for 23 %.  4 x up to 1024 new of up to 5000 tokens,
// 32 query heads of 128: 252 us, 744 TFLOP/s.  (64 rows a wave leave one wave a SIMD: an earlier form took 382 us so, 283 with 32.)
template <int D, bool BF, int MT>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void attend_wide_kernel(const AttendArgs a) {
  using E = Elem<BF>;
  using vec = typename E::vec;
  using one = typename E::one;
  constexpr int kSteps = D / 32, kWhole = D / 64, kTiles = D / 16;
  constexpr bool kHalf = D % 64 != 0;
  constexpr int kKeys = 4 * kWhole, kGroups = kKeys + kTiles;  // a lane's 16 codes: of keys (tt, i), then of values (dt)
  constexpr int kEach = (kGroups + 3) / 4;                     // a wave loads these
  constexpr int kKeyVecs = 4 * kSteps;                         // widened: keys (tt, step), then values (dt, half)
  constexpr int kBuffers = D <= 128 ? 2 : 1;                   // (two workgroups a CU fit its 160 KB)
  __shared__ __align__(16) vec key_tile[kBuffers][kKeyVecs * 64];
  __shared__ __align__(16) f16x8 value_tile[kBuffers][2 * kTiles * 64];
  __shared__ int nan_tile[2][4];  // whether a wave took NaN codes out of the values it wrote
  __shared__ int again_any[4];    // whether a wave's sums lack too much

  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int split = blockIdx.y;
  Place p;
  if (!attend_place(a, 64 * MT, lane, p)) return;
  const int tile0 = p.tile * 64 * MT, row0 = tile0 + wave * 16 * MT, h = p.h;
  const int lim_first = seen_by(a, p, tile0), lim_lo = seen_by(a, p, row0), lim_wave = row0 < p.rows ? seen_by(a, p, row0 + 16 * MT - 1) : 0;
  const int lim_hi = seen_by(a, p, tile0 + 64 * MT - 1);
  const int tiles = lim_hi > 0 ? (lim_hi + 63) >> 6 : 0;
  const int t_begin = split * a.split_tiles;
  const int t_end = split == a.splits - 1 ? tiles : min(tiles, t_begin + a.split_tiles);
  if (split > 0 && t_begin >= tiles) return;

  vec qf[MT][kSteps];
  int lim[MT];
  load_queries<D, BF, MT>(a, p, row0, m, g, qf, lim);
  f32x4 acc[kTiles][MT];
  float M[MT], l[MT];
  u16x2 least = {0x3c00, 0x3c00};
  float ve_least = INFINITY, ve_most = -INFINITY;  // of the units' value exponents

  const PageWalk walk(a, p);
  u32x4 stage[kEach];
  u32x2 stage_half;
  // the wave's groups of tile t, from its lanes' pages (all keys or all values, but for a D with an odd share)
  constexpr bool kMixed = kKeys % kEach != 0;
  const bool keys = wave * kEach < kKeys;
  const int64_t lane_k = (m & 3) * 16 + g * 256, lane_v = m * 16;
  const auto load = [&](int pk, int pv, int t) __attribute__((always_inline)) {
    const uint8_t* ka = walk.unit(a.k, pk, 4 * t + (m >> 2), 16 * D) + lane_k;
    const uint8_t* va = walk.unit(a.v, pv, 4 * t + g, 16 * D) + lane_v;
    const uint8_t* at = keys ? ka : va;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int q = wave * kEach + j;
      if (kGroups % 4 != 0 && q >= kGroups) break;
      if (kMixed) at = q < kKeys ? ka : va;
      const int off = q < kKeys ? (q / kWhole) * 64 + (q % kWhole) * 1024 : (q - kKeys) * 256;
      stage[j] = *reinterpret_cast<const u32x4*>(at + off);
    }
    if (kHalf)
      stage_half = *reinterpret_cast<const u32x2*>(ka - g * 256 + wave * 64 + (4 * kWhole + (g >> 1)) * 256 + (g & 1) * 8);
  };
  const auto put = [&](int t, bool ok) __attribute__((always_inline)) {
    const int b = t & (kBuffers - 1);
    if (64 * (t + 1) > p.len || __ballot(ok) != ~0ull) {  // values past the sequence's end are not the cache's: any bytes
      const int keep = ok ? max(p.len - (64 * t + 16 * g), 0) : 0;
#pragma unroll
      for (int j = 0; j < kEach; ++j)
        if (wave * kEach + j >= kKeys) stage[j] = low_bytes(stage[j], keep);
    }
    if (64 * (t + 1) > lim_first) {  // some rows do not see all of the tile
      uint32_t any = 0;
#pragma unroll
      for (int j = 0; j < kEach; ++j)
        if (wave * kEach + j >= kKeys && wave * kEach + j < kGroups) any |= nan_any(stage[j]);
      const bool bad = __ballot(any != 0) != 0;
      if (bad) {
#pragma unroll
        for (int j = 0; j < kEach; ++j)
          if (wave * kEach + j >= kKeys) stage[j] = nan_out(stage[j]);
      }
      if (lane == 0) nan_tile[t & 1][wave] = bad;
    }
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int q = wave * kEach + j;
      if (kGroups % 4 != 0 && q >= kGroups) break;
      if (kMixed ? q < kKeys : keys) {
        vec* to = key_tile[b] + (q / kWhole * kSteps + 2 * (q % kWhole)) * 64 + lane;
        to[0] = E::widen(stage[j][0], stage[j][1]);
        to[64] = E::widen(stage[j][2], stage[j][3]);
      } else {
        f16x8* to = value_tile[b] + 2 * (q - kKeys) * 64 + lane;
        to[0] = Elem<false>::widen(stage[j][0], stage[j][1]);
        to[64] = Elem<false>::widen(stage[j][2], stage[j][3]);
      }
    }
    if (kHalf) key_tile[b][(wave * kSteps + kSteps - 1) * 64 + lane] = E::widen(stage_half[0], stage_half[1]);
  };

  // (the precise pass: waves that are content help with the tiles)
  const auto pass = [&](auto flag, bool mine) __attribute__((always_inline)) {
    constexpr bool PRECISE = decltype(flag)::value;
    if (mine) {
#pragma unroll
      for (int r = 0; r < MT; ++r) {
        M[r] = -INFINITY;
        l[r] = 0.0f;
#pragma unroll
        for (int dt = 0; dt < kTiles; ++dt) acc[dt][r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      }
    }
    if (t_begin >= t_end) return;
    bool far = false;
    bool ok, ok_k;
    int pk = walk.valid(walk.page(4 * t_begin + (m >> 2)), ok_k), pv = walk.valid(walk.page(4 * t_begin + g), ok);
    load(pk, pv, t_begin);
    int ke = a.k_exp[(int64_t)pv * a.heads + h], ve = a.v_exp[(int64_t)pv * a.heads + h];
    int pk_next = walk.page(4 * (t_begin + 1) + (m >> 2)), pv_next = walk.page(4 * (t_begin + 1) + g);
    put(t_begin, ok);
    __syncthreads();
    for (int t = t_begin; t < t_end; ++t) {
      if (!ok) ke = ve = 0;  // (no page: page 0 was read in its place, whose exponents may be any byte)
      float c_g = a.scale_log2 * pow2i(ke), ve_g = (float)ve, inv_v = pow2i(-ve);
      asm volatile("" : "+v"(c_g), "+v"(ve_g), "+v"(inv_v));  // (before the next tile's exponents are loaded, into the same registers)
      const bool ok_now = ok;
      const bool more = t + 1 < t_end;
      if (more) {
        pk = walk.valid(pk_next, ok_k);
        pv = walk.valid(pv_next, ok);
        load(pk, pv, t + 1);
        ke = a.k_exp[(int64_t)pv * a.heads + h];
        ve = a.v_exp[(int64_t)pv * a.heads + h];
        pk_next = walk.page(4 * (t + 2) + (m >> 2));
        pv_next = walk.page(4 * (t + 2) + g);
      }
      if (64 * t < lim_wave && mine) {
        const vec* kt = key_tile[t & (kBuffers - 1)] + lane;
        const f16x8* vt = value_tile[t & (kBuffers - 1)] + lane;
        f32x4 sc[4][MT];
#pragma unroll
        for (int tt = 0; tt < 4; ++tt) {
#pragma unroll
          for (int r = 0; r < MT; ++r) sc[tt][r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int st = 0; st < kSteps; ++st) {
            const vec kf = kt[(tt * kSteps + st) * 64];
#pragma unroll
            for (int r = 0; r < MT; ++r) sc[tt][r] = E::mfma(kf, qf[r][st], sc[tt][r]);
          }
        }
        const bool masked = 64 * (t + 1) > lim_lo || __ballot(ok_now) != ~0ull;
        const int first = 64 * t + 16 * g;
        int upto[MT];
#pragma unroll
        for (int r = 0; r < MT; ++r) upto[r] = ok_now ? lim[r] - first : 0;
        float alpha[MT];
        f16x8 pf[MT][2];
        bool grown;
        if constexpr (PRECISE) {
          grown = raise_frame<MT, true, true>(sc, c_g, ve_g, upto, M, l, alpha, far);
          if (far)
            weigh_far<MT>(sc, c_g, ve_g, inv_v, upto, M, l, pf);
          else
            weigh<MT, true>(sc, c_g, ve_g, inv_v, upto, M, l, pf, least);
        } else {
          ve_least = fminf(ve_least, ve_g);
          ve_most = fmaxf(ve_most, ve_g);
          grown = masked ? raise_frame<MT, true, false>(sc, c_g, ve_g, upto, M, l, alpha, far)
                         : raise_frame<MT, false, false>(sc, c_g, ve_g, upto, M, l, alpha, far);
          if (masked)
            weigh<MT, true>(sc, c_g, ve_g, inv_v, upto, M, l, pf, least);
          else
            weigh<MT, false>(sc, c_g, ve_g, inv_v, upto, M, l, pf, least);
        }
        if (grown) {
#pragma unroll
          for (int r = 0; r < MT; ++r)
#pragma unroll
            for (int dt = 0; dt < kTiles; ++dt) acc[dt][r] *= alpha[r];
        }
        if (64 * (t + 1) > lim_first && (nan_tile[t & 1][0] | nan_tile[t & 1][1] | nan_tile[t & 1][2] | nan_tile[t & 1][3])) {
          // (rare: the tile was written without its NaN codes, which are read from the cache again)
          const uint8_t* va = walk.unit(a.v, walk.valid(walk.page(4 * t + g), ok_k), 4 * t + g, 16 * D) + lane_v;
          const int keep = ok_now ? max(p.len - first, 0) : 0;
#pragma unroll
          for (int dt = 0; dt < kTiles; ++dt)
            mark_nan<MT>(low_bytes(*reinterpret_cast<const u32x4*>(va + dt * 256), keep), upto, acc[dt]);
        }
#pragma unroll
        for (int dt = 0; dt < kTiles; ++dt) {
          const f16x8 v[2] = {vt[2 * dt * 64], vt[(2 * dt + 1) * 64]};
          add_values<MT>(v, pf, acc[dt]);
        }
        if constexpr (PRECISE) {
#pragma unroll
          for (int r = 0; r < MT; ++r) {
            f16x8 left[2];
            float back;
            left_of_low<MT>(sc, r, c_g, ve_g, upto[r], M[r], far, left, back);
            add_left<MT, kTiles>(left, back, r, acc, [&](int dt, int hs) {
              f16x8 v = vt[(2 * dt + hs) * 64];
              asm volatile("" : "+v"(v));  // (read again, not held from above)
              return v;
            });
          }
        }
      }
      if (kBuffers == 1) __syncthreads();  // every wave is done with the tile
      if (more) {
        put(t + 1, ok);
        __syncthreads();
      }
    }
  };
  pass(Flag<false>{}, true);
  const bool again = 64 * t_begin < lim_wave && t_begin < t_end &&
                     lacks<MT, kTiles>(acc, M, lim, least, ve_least, ve_most, 64.0f * (t_end - t_begin));
  if (lane == 0) again_any[wave] = again;
  __syncthreads();
  if (again_any[0] | again_any[1] | again_any[2] | again_any[3]) pass(Flag<true>{}, again);

  const int64_t heads_q = (int64_t)a.heads * a.group;
#pragma unroll
  for (int r = 0; r < MT; ++r) {
    const float ls = row_sum4(l[r]);
    const int row = row0 + 16 * r + m;
    if (row >= p.rows) continue;
    const int i = row / a.group;
    const int64_t id = (p.start + i) * heads_q + h * a.group + (row - i * a.group);
    if (a.splits == 1) {
      const float inv = ls == 0.0f ? 0.0f : 1.0f / ls;
      one* o = static_cast<one*>(a.out) + id * D + 4 * g;
#pragma unroll
      for (int dt = 0; dt < kTiles; ++dt) {
        typedef one one4 __attribute__((ext_vector_type(4)));
        one4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (one)(ls == 0.0f ? 0.0f : acc[dt][r][e] * inv);
        *reinterpret_cast<one4*>(o + 16 * dt) = w;
      }
      if (a.lse && g == 0) a.lse[id] = log_sum(M[r], ls);
    } else {
      float* o = a.part + (id * a.splits + split) * D + 4 * g;
#pragma unroll
      for (int dt = 0; dt < kTiles; ++dt) *reinterpret_cast<f32x4*>(o + 16 * dt) = acc[dt][r];
      if (g == 0) {
        a.part_ml[2 * (id * a.splits + split)] = M[r];
        a.part_ml[2 * (id * a.splits + split) + 1] = ls;
      }
    }
  }
}

// Joins the splits of a row: one wave a row.
template <int D, bool BF>
__global__ __launch_bounds__(256) void attend_join_kernel(const AttendArgs a, int rows_tile, int64_t total) {
  using one = typename Elem<BF>::one;
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (id >= total) return;
  const int heads_q = a.heads * a.group;
  const int64_t t = id / heads_q;
  const int hg = (int)(id - t * heads_q) % a.group;
  int s, n;
  int64_t start;
  if (a.starts) {
    s = slot_sequence(a.starts, a.S, t, 1, 1, 0, lane);
    start = a.starts[s];
    n = (int)(a.starts[s + 1] - start);
  } else {
    n = (int)(a.T / a.S);
    s = (int)(t / n);
    start = (int64_t)s * n;
  }
  if (start < 0 || t < start || t >= start + n || start + n > a.T) return;  // a token of no sequence
  const int rows = n * a.group;
  const int row = (int)(t - start) * a.group + hg;
  const int row0 = row / rows_tile * rows_tile;
  const int len = max(0, min(a.lengths[s], (int)min(a.width << a.page_shift, (int64_t)INT32_MAX)));
  const int before = a.lengths[s] - n;
  const int lim_hi = min(len, before + min(rows - 1, row0 + rows_tile - 1) / a.group + 1);
  const int tiles = lim_hi > 0 ? (lim_hi + 63) >> 6 : 0;
  // the splits that had tokens for the row's tile
  const int splits = max(1, min(a.splits, (tiles + a.split_tiles - 1) / a.split_tiles));
  const float* ml = a.part_ml + 2 * id * a.splits;
  float M = -INFINITY, l = 0.0f;
  for (int i = lane; i < splits; i += 64) M = fmaxf(M, ml[2 * i]);
  const float top = wave_max(M);
  for (int i = lane; i < splits; i += 64) l = fmaf(frame_weight(ml[2 * i], top), ml[2 * i + 1], l);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) l += __shfl_xor(l, off, 64);
  // D / 64 elements a lane where that is whole, the lanes past D idle otherwise
  constexpr int kPer = (D + 63) / 64;
  float o[kPer];
#pragma unroll
  for (int e = 0; e < kPer; ++e) o[e] = 0.0f;
  const float* part = a.part + id * a.splits * D;
#pragma unroll 4
  for (int i = 0; i < splits; ++i) {
    const float w = frame_weight(ml[2 * i], top);
#pragma unroll
    for (int e = 0; e < kPer; ++e)
      if (kPer * lane + e < D) o[e] = fmaf(w, part[(int64_t)i * D + kPer * lane + e], o[e]);
  }
#pragma unroll
  for (int e = 0; e < kPer; ++e)
    if (kPer * lane + e < D)
      static_cast<one*>(a.out)[id * D + kPer * lane + e] = (one)(l == 0.0f ? 0.0f : o[e] / l);
  if (a.lse && lane == 0) a.lse[id] = log_sum(top, l);
}

// How a call is cut: rows a wave holds, whether the waves take different rows, splits of the tokens.
struct AttendPlan {
  int mt, per_seq, splits, split_tiles;
  bool wide;
  int64_t slots;
};

AttendPlan attend_plan(const CacheView& c, int64_t T, int64_t S, int64_t width, int group, bool uniform,
                       int64_t max_new, int64_t max_length) {
  AttendPlan p;
  const int64_t n = uniform || max_new <= 0 ? (T + S - 1) / S : (max_new < T ? max_new : T);
  const int64_t rows = n * group;
  const int most = c.d > 128 ? 2 : 4;
  p.wide = rows > 16 * most;
  p.mt = p.wide ? (c.d > 128 ? 1 : 2) : rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  const int tile_rows = (p.wide ? 64 : 16) * p.mt;
  p.per_seq = uniform ? (int)((rows + tile_rows - 1) / tile_rows) : 0;
  p.slots = uniform ? S * p.per_seq : T * group / tile_rows + S;
  int64_t tokens = width << c.page_shift;
  if (max_length > 0 && max_length < tokens) tokens = max_length;
  const int64_t tiles = (tokens + 63) >> 6;
  // (ragged slots are an upper bound: rows that hardly fill their tiles take one a sequence)
  const int64_t full = (T * group + tile_rows - 1) / tile_rows, base = (p.per_seq ? p.slots : full > S ? full : S) * c.heads;
  // Few rows: each split has at least 8 tiles; none below 2048 tokens, where the second launch costs more than the tiles'
  // latency (one sequence, the call: 1024 tokens 15 us whole, 19 split; 4096 20.6 and 18.7).  As many workgroups as the 256 CUs
  // hold at a time by the kernels' registers, but where those are of one row tile and d = 96 (three a CU) or 128 (two):
  //   up to 32 (sequence, head) pairs take a little less than two a CU (4 x 131072 tokens, 8 heads: 480 workgroups 195 us, 512 224,
  //   768 214, 1536 212; 2 x 131072: 496 106 us, 512 120), and
  //   few of them fewer splits, which are joined one after the other (1 x 100000: 32 splits 47 us, 40 55);
  //   more pairs take twice what is resident, so that unlike lengths even out (d = 128, 16 x up to 30000, a quarter up: 1024
  //   workgroups 73 us, 512 97, 1536 78; 8 x up to 60000: 1024 79, 1536 87; 32 x up to 8192: 1024 45, 1536 49; all of 30000: 192,
  //   203, 190; d = 96, 32 x up to 8192: 1024 44, 1536 39; 16 x up to 30000: 73 and 65).
  // Where the one passes into the other is a choice between equal lengths and unlike ones, which the host does not know: at 32 pairs
  // 15 splits take 98 us (60000 tokens each) and 96 (up to 100000), 31 splits 102 and 80; at 40 pairs 12 take 118 and 123, 25 124 and 110.
  // Many rows: two workgroups a CU, and only where that leaves half of them idle.
  const int resident = p.mt == 1 ? (c.d <= 64 ? 4 : c.d <= 96 ? 3 : c.d <= 128 ? 2 : 1) : c.d <= 128 && p.mt == 2 ? 2 : 1;
  int64_t splits;
  if (p.wide) {
    splits = 512 / base;
  } else if (tiles < 32) {
    splits = 1;
  } else if (p.mt > 1 || c.d <= 64 || c.d > 128) {
    splits = (256 * resident + base / 2) / base;
  } else if (base > 32) {
    splits = 512 * resident / base;
  } else {
    const int64_t most = base > 8 ? 32 : 256 / base;
    splits = 511 / base < most ? 511 / base : most;
  }
  if (splits > (tiles + 7) / 8) splits = (tiles + 7) / 8;
  if (splits > 128) splits = 128;
  if (splits < 1) splits = 1;
  p.split_tiles = (int)((tiles + splits - 1) / splits);
  if (p.split_tiles < 1) p.split_tiles = 1;
  p.splits = (int)((tiles + p.split_tiles - 1) / p.split_tiles);
  if (p.splits < 1) p.splits = 1;
  return p;
}

// The launches of a call: a dimension of one holds less than 2^32 threads.
template <typename Kernel>
void attend_slots(Kernel kernel, AttendArgs a, int64_t slots, hipStream_t st) {
  const int64_t most = ((1 << 24) - 1) / a.heads;
  for (int64_t at = 0; at < slots; at += most) {
    a.slot0 = (int)at;
    const int64_t n = slots - at < most ? slots - at : most;
    kernel<<<dim3((unsigned)(n * a.heads), (unsigned)a.splits), 256, 0, st>>>(a);
  }
}

template <int D, bool BF>
hipError_t attend_launch(const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
  if (p.wide) {
    attend_slots(attend_wide_kernel<D, BF, D == 256 ? 1 : 2>, a, p.slots, st);
  } else if (p.mt == 1) {
    attend_slots(attend_kernel<D, BF, 1>, a, p.slots, st);
  } else if (p.mt == 2) {
    attend_slots(attend_kernel<D, BF, 2>, a, p.slots, st);
  } else if constexpr (D <= 128) {
    attend_slots(attend_kernel<D, BF, 4>, a, p.slots, st);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t total = a.T * a.heads * a.group;  // (at most 2^16: calls of more rows are not split)
  attend_join_kernel<D, BF><<<(unsigned)((total + 3) / 4), 256, 0, st>>>(a, 16 * p.mt, total);
  return hipGetLastError();
}

}  // namespace

size_t workspace_bytes_attention(const CacheView& c, int64_t T, int64_t S, int64_t width, int64_t heads_q,
                                 int64_t max_new, int64_t max_length, bool uniform) {
  const AttendPlan p = attend_plan(c, T, S, width, (int)(heads_q / c.heads), uniform, max_new, max_length);
  return p.splits == 1 ? 0 : (size_t)T * heads_q * p.splits * (c.d + 2) * sizeof(float);
}

hipError_t launch_cache_attention(const CacheView& c, int layer, const void* q, int dtype, int64_t heads_q,
                                  int64_t q_st, int64_t q_sh, const CacheRows& rows, float scale, int64_t max_new,
                                  int64_t max_length, void* out, float* lse, void* workspace, hipStream_t st) {
  const AttendPlan p = attend_plan(c, rows.T, rows.S, rows.width, (int)(heads_q / c.heads), rows.starts == nullptr,
                                   max_new, max_length);
  AttendArgs a;
  a.q = q;
  a.k = c.k + layer * c.pages * c.region();
  a.v = c.v + layer * c.pages * c.region();
  a.k_exp = c.k_exp + layer * c.pages * c.heads;
  a.v_exp = c.v_exp + layer * c.pages * c.heads;
  a.starts = rows.starts;
  a.table = rows.table;
  a.lengths = rows.lengths;
  a.out = out;
  a.lse = lse;
  a.part = static_cast<float*>(workspace);
  a.part_ml = a.part + (p.splits == 1 ? 0 : rows.T * heads_q * p.splits * c.d);
  a.q_st = q_st;
  a.q_sh = q_sh;
  a.width = rows.width;
  a.T = rows.T;
  a.pages = c.pages;
  a.S = rows.S;
  a.heads = c.heads;
  a.group = (int)(heads_q / c.heads);
  a.page_shift = c.page_shift;
  a.per_seq = p.per_seq;
  a.splits = p.splits;
  a.split_tiles = p.split_tiles;
  a.scale_log2 = fabsf(scale) * 1.4426950408889634f;
  a.negative = scale < 0.0f;
  const bool bf = dtype == MDSS_BF16;
  switch (c.d) {
    case 64: return bf ? attend_launch<64, true>(a, p, st) : attend_launch<64, false>(a, p, st);
    case 96: return bf ? attend_launch<96, true>(a, p, st) : attend_launch<96, false>(a, p, st);
    case 128: return bf ? attend_launch<128, true>(a, p, st) : attend_launch<128, false>(a, p, st);
    default: return bf ? attend_launch<256, true>(a, p, st) : attend_launch<256, false>(a, p, st);
  }
}

}  // namespace mdss
