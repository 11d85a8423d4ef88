// Attention over the paged 8-bit cache (gfx950).
//
//   s_j = scale q . k_j,  out = sum_j softmax(s)_j v_j  over the cached tokens j <= the query's own position,
// with k_j = code 2^ke and v_j = code 2^ve, the exponents of the token's page and head.
//
// A wave takes 64 tokens at a time against MT tiles of 16 query rows (a row = one new token of one of the query
// heads that share a cache head).  It computes S^T = K Q^T and then O^T = V^T P^T, so that the accumulators of the
// first product are, lane by lane, the second's operand: lane (m, g) = (lane & 15, lane >> 4) holds row m's scores of
// the 16 tokens of unit g in both.  Codes go from memory to registers (16 bytes of a key chunk or of a value's
// 16 tokens), are widened there (exactly: bf16 or f16 keys, f16 values) and feed the matrix cores; LDS only joins the
// waves of a workgroup at the end.  One pass with a running maximum: with t = s log2(e) + ve, in the frame M = max t,
//   p = 2^(t - M) <= 1 carries the value's scale (so f16 holds the terms that matter, whatever the pages' scales),
//   l = sum p 2^-ve the softmax's sum in the same frame, out = sum p code / l.
// Exponents lie in [-40, 40]: a term that the frame loses (below 2^-126) has less than 2^-46 of the largest weight.
#include "cache.h"

#include <math.h>

namespace mdss {

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
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
  int splits, split_tiles;
  float scale_log2;
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

// The frame of two partial sums: their weights, given (M, l) of each; rows without a visible token have M = -inf.
__device__ __forceinline__ float frame_weight(float M, float top) { return M == -INFINITY ? 0.0f : exp2f(M - top); }

// WIDE: the four waves of a workgroup take different rows of the same tokens (many rows); else the same rows of
// different tokens, joined at the end.
template <int D, bool BF, int MT, bool WIDE>
__global__ __launch_bounds__(256) void attend_kernel(const AttendArgs a) {
  using E = Elem<BF>;
  using vec = typename E::vec;
  using one = typename E::one;
  constexpr int kSteps = D / 32;             // matrix steps over d
  constexpr int kWhole = D / 64;             // 16-byte loads of a key row's quarter
  constexpr bool kHalf = D % 64 != 0;        // and one of 8 bytes
  constexpr int kTiles = D / 16;             // accumulator tiles over d
  constexpr int kRows = (WIDE ? 64 : 16) * MT;
  constexpr int kPad = D + 4;
  __shared__ __align__(16) float joined[WIDE ? 1 : 4 * 16 * kPad];
  __shared__ float joined_ml[WIDE ? 1 : 4 * 16 * 2];

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
  // the head is the fastest index: the row tiles that read one head's pages run on the same XCD where heads are a
  // multiple of 8 (workgroups go round the XCDs in order), and find them in its L2
  const int slot = blockIdx.x / a.heads, h = blockIdx.x - slot * a.heads, split = blockIdx.y;
  int s, tile;
  int64_t start;
  int n;
  if (a.per_seq > 0) {
    s = slot / a.per_seq;
    tile = slot - s * a.per_seq;
  } else {
    s = slot_sequence(a.starts, a.S, slot, a.group, kRows, 1, lane);
    tile = slot - (int)slot_first(a.starts, s, a.group, kRows, 1);
  }
  if (a.starts) {
    start = a.starts[s];
    n = (int)(a.starts[s + 1] - start);
  } else {
    n = (int)(a.T / a.S);
    start = (int64_t)s * n;
  }
  if (start < 0 || n <= 0 || start + n > a.T) return;  // no rows, or starts that are not ascending within T
  const int rows = n * a.group;
  if (tile * kRows >= rows) return;
  const int row0 = tile * kRows + (WIDE ? wave * 16 * MT : 0);
  if (row0 >= rows) return;  // (WIDE only: the wave has no row, and there is no barrier below)
  const int len = max(0, min(a.lengths[s], (int)min(a.width << a.page_shift, (int64_t)INT32_MAX)));
  const int before = a.lengths[s] - n;  // tokens cached before the new ones (negative: the first rows see nothing)
  const int lim_lo = min(len, before + row0 / a.group + 1);
  const int lim_hi = min(len, before + min(rows - 1, row0 + 16 * MT - 1) / a.group + 1);
  const int tiles = lim_hi > 0 ? (lim_hi + 63) >> 6 : 0;
  const int t_begin = split * a.split_tiles;
  const int t_end = split == a.splits - 1 ? tiles : min(tiles, t_begin + a.split_tiles);
  // a split without tokens for any row of the workgroup has nothing to say (the first one always speaks)
  if (split > 0 && t_begin >= tiles) return;

  // queries: lane (m, g) holds row m's elements 64 i + 16 g + 0..15 (8 g' of the last 32 where D is no multiple of 64)
  vec qf[MT][kSteps];
  int lim[MT];
#pragma unroll
  for (int r = 0; r < MT; ++r) {
    const int row = row0 + 16 * r + m;
    const bool in = row < rows;
    const int i = in ? row / a.group : 0, hg = in ? row - i * a.group : 0;
    lim[r] = in ? min(len, before + i + 1) : 0;
    const one* qr = static_cast<const one*>(a.q) + (start + i) * a.q_st + (int64_t)(h * a.group + hg) * a.q_sh;
#pragma unroll
    for (int st = 0; st < kSteps; ++st) {
      const int at = (kHalf && st == kSteps - 1) ? 64 * kWhole + 8 * g : 64 * (st >> 1) + 16 * g + 8 * (st & 1);
      vec x;
      if (((reinterpret_cast<uintptr_t>(qr) & 15) == 0)) {
        x = *reinterpret_cast<const vec*>(qr + at);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = qr[at + j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = in ? x[j] : (one)0.0f;
      qf[r][st] = x;
    }
  }

  f32x4 acc[kTiles][MT];
  float M[MT], l[MT];
#pragma unroll
  for (int r = 0; r < MT; ++r) {
    M[r] = -INFINITY;
    l[r] = 0.0f;
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt) acc[dt][r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  const int step = WIDE ? 1 : 4;
  const int t0 = t_begin + (WIDE ? 0 : wave);
  const int32_t* trow = a.table + (int64_t)s * a.width;
  const int unit_shift = a.page_shift - 4;
  const int last_page = len > 0 ? (len - 1) >> a.page_shift : 0;
  const int per_page = 1 << unit_shift;
  const auto page_at = [&](int unit) {  // page id of a unit, clamped into the row: never out of the table
    return trow[min(unit >> unit_shift, last_page)];
  };
  const auto unit_base = [&](const uint8_t* base, int page, int unit) {
    return base + ((((int64_t)page * a.heads + h) << unit_shift) + (unit & (per_page - 1))) * (16 * D);
  };

  u32x4 kc[4][kWhole > 0 ? kWhole : 1];
  u32x2 kh[4];
  const auto load_k = [&](int page, int t) {
    const int unit = 4 * t + (m >> 2);
    const uint8_t* p = unit_base(a.k, page, unit) + g * 256 + (m & 3) * 16;
#pragma unroll
    for (int tt = 0; tt < 4; ++tt) {
#pragma unroll
      for (int i = 0; i < kWhole; ++i) kc[tt][i] = *reinterpret_cast<const u32x4*>(p + tt * 64 + i * 1024);
      if (kHalf)
        kh[tt] = *reinterpret_cast<const u32x2*>(p - g * 256 + (4 * kWhole + (g >> 1)) * 256 + (g & 1) * 8 + tt * 64);
    }
  };

  if (t0 < t_end) {
    int pk = page_at(4 * t0 + (m >> 2)), pv = page_at(4 * t0 + g);
    bool ok_k = (uint32_t)pk < (uint32_t)a.pages;
    load_k(ok_k ? pk : 0, t0);
    bool ok = (uint32_t)pv < (uint32_t)a.pages;
    pv = ok ? pv : 0;
    int ke = a.k_exp[(int64_t)pv * a.heads + h], ve = a.v_exp[(int64_t)pv * a.heads + h];
    int pk_next = page_at(4 * (t0 + step) + (m >> 2)), pv_next = page_at(4 * (t0 + step) + g);
    for (int t = t0; t < t_end; t += step) {
      u32x4 vc[kTiles];
      {
        const uint8_t* p = unit_base(a.v, pv, 4 * t + g) + m * 16;
#pragma unroll
        for (int dt = 0; dt < kTiles; ++dt) vc[dt] = *reinterpret_cast<const u32x4*>(p + dt * 256);
      }
      f32x4 sc[4][MT];
#pragma unroll
      for (int tt = 0; tt < 4; ++tt) {
#pragma unroll
        for (int r = 0; r < MT; ++r) sc[tt][r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
          const vec kf = (kHalf && st == kSteps - 1) ? E::widen(kh[tt][0], kh[tt][1])
                                                      : E::widen(kc[tt][st >> 1][2 * (st & 1)], kc[tt][st >> 1][2 * (st & 1) + 1]);
#pragma unroll
          for (int r = 0; r < MT; ++r) sc[tt][r] = E::mfma(kf, qf[r][st], sc[tt][r]);
        }
      }
      const float c_g = a.scale_log2 * pow2i(ke), ve_g = (float)ve, inv_v = pow2i(-ve);
      const bool ok_now = ok;
      // the next tile's keys, exponents, and the page ids after it
      {
        const bool nk = (uint32_t)pk_next < (uint32_t)a.pages;
        load_k(nk ? pk_next : 0, t + step);
        ok = (uint32_t)pv_next < (uint32_t)a.pages;
        pv = ok ? pv_next : 0;
        ke = a.k_exp[(int64_t)pv * a.heads + h];
        ve = a.v_exp[(int64_t)pv * a.heads + h];
        pk_next = page_at(4 * (t + 2 * step) + (m >> 2));
        pv_next = page_at(4 * (t + 2 * step) + g);
      }
      const bool masked = 64 * (t + 1) > lim_lo || __ballot(ok_now) != ~0ull;
      const int first = 64 * t + 16 * g;  // the lane's first token
      f16x8 pf[MT][2];
      bool grown = false;
      float alpha[MT];
#pragma unroll
      for (int r = 0; r < MT; ++r) {
        float x[4][4], mx = -INFINITY;
        if (masked) {
          const int upto = ok_now ? lim[r] - first : 0;  // visible tokens of the unit
#pragma unroll
          for (int tt = 0; tt < 4; ++tt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              x[tt][i] = 4 * tt + i < upto ? fmaf(sc[tt][r][i], c_g, ve_g) : -INFINITY;
              mx = fmaxf(mx, x[tt][i]);
            }
        } else {
#pragma unroll
          for (int tt = 0; tt < 4; ++tt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              x[tt][i] = fmaf(sc[tt][r][i], c_g, ve_g);
              mx = fmaxf(mx, x[tt][i]);
            }
        }
        const float top = fmaxf(M[r], row_max4(mx));
        const float ref = top == -INFINITY ? 0.0f : top;
        alpha[r] = __builtin_amdgcn_exp2f(M[r] - ref);
        grown |= top > M[r];
        M[r] = top;
        float sum = 0.0f;
#pragma unroll
        for (int tt = 0; tt < 4; ++tt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p = __builtin_amdgcn_exp2f(x[tt][i] - ref);
            sum += p;
            pf[r][tt >> 1][4 * (tt & 1) + i] = (_Float16)p;
          }
        l[r] = fmaf(l[r], alpha[r], sum * inv_v);
      }
      if (__ballot(grown) != 0) {
#pragma unroll
        for (int r = 0; r < MT; ++r)
#pragma unroll
          for (int dt = 0; dt < kTiles; ++dt) acc[dt][r] *= alpha[r];
      }
      if (masked) {
        // what lies past the sequence's end is not the cache's (any bytes), and a NaN code among the tokens that
        // only some rows see must reach those rows alone: it is taken out here and counted in its own product
        const int keep = ok_now ? min(max(len - first, 0), 16) : 0;
        uint32_t bad = 0;
#pragma unroll
        for (int dt = 0; dt < kTiles; ++dt) {
          vc[dt] = low_bytes(vc[dt], keep);
#pragma unroll
          for (int w = 0; w < 4; ++w) bad |= nan_bytes(vc[dt][w]);
        }
        if (__ballot(bad != 0) != 0) {
#pragma unroll
          for (int dt = 0; dt < kTiles; ++dt) {
            u32x4 flag;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const uint32_t b = nan_bytes(vc[dt][w]) >> 7;  // 0x01 in the bytes of NaN codes
              flag[w] = b * 0x38u;                           // the code of 1.0
              vc[dt][w] &= ~(b * 0xffu);
            }
#pragma unroll
            for (int r = 0; r < MT; ++r) {
              const int upto = ok_now ? lim[r] - first : 0;
              f32x4 hit = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
              for (int hs = 0; hs < 2; ++hs) {
                f16x8 see;
#pragma unroll
                for (int j = 0; j < 8; ++j) see[j] = 8 * hs + j < upto ? (_Float16)1.0f : (_Float16)0.0f;
                hit = Elem<false>::mfma(Elem<false>::widen(flag[2 * hs], flag[2 * hs + 1]), see, hit);
              }
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[dt][r][i] = hit[i] > 0.0f ? NAN : acc[dt][r][i];
            }
          }
        }
      }
#pragma unroll
      for (int dt = 0; dt < kTiles; ++dt)
#pragma unroll
        for (int hs = 0; hs < 2; ++hs) {
          const f16x8 vf = Elem<false>::widen(vc[dt][2 * hs], vc[dt][2 * hs + 1]);
#pragma unroll
          for (int r = 0; r < MT; ++r) acc[dt][r] = Elem<false>::mfma(vf, pf[r][hs], acc[dt][r]);
        }
    }
  }

  const int64_t heads_q = (int64_t)a.heads * a.group;
  const auto row_id = [&](int row) {  // row of [T][heads_q]
    const int i = row / a.group;
    return (start + i) * heads_q + h * a.group + (row - i * a.group);
  };
#pragma unroll
  for (int r = 0; r < MT; ++r) l[r] = row_sum4(l[r]);

  if (WIDE) {
#pragma unroll
    for (int r = 0; r < MT; ++r) {
      const int row = row0 + 16 * r + m;
      if (row >= rows) continue;
      const int64_t id = row_id(row);
      if (a.splits == 1) {
        const float inv = l[r] == 0.0f ? 0.0f : 1.0f / l[r];
        one* o = static_cast<one*>(a.out) + id * D + 4 * g;
#pragma unroll
        for (int dt = 0; dt < kTiles; ++dt) {
          typedef one one4 __attribute__((ext_vector_type(4)));
          one4 w;
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = (one)(l[r] == 0.0f ? 0.0f : acc[dt][r][i] * inv);
          *reinterpret_cast<one4*>(o + 16 * dt) = w;
        }
        if (a.lse && g == 0) a.lse[id] = l[r] == 0.0f ? -INFINITY : (M[r] + log2f(l[r])) * 0.693147180559945f;
      } else {
        float* o = a.part + (id * a.splits + split) * D + 4 * g;
#pragma unroll
        for (int dt = 0; dt < kTiles; ++dt) *reinterpret_cast<f32x4*>(o + 16 * dt) = acc[dt][r];
        if (g == 0) {
          a.part_ml[2 * (id * a.splits + split)] = M[r];
          a.part_ml[2 * (id * a.splits + split) + 1] = l[r];
        }
      }
    }
    return;
  }
  // join the four waves, 16 rows at a time: thread -> a row and D / 16 of its elements
  const int jr = threadIdx.x >> 4, jd = (threadIdx.x & 15) * (D / 16);
#pragma unroll
  for (int r = 0; r < MT; ++r) {
    if (r > 0) __syncthreads();
    float* w = joined + (wave * 16 + m) * kPad + 4 * g;
#pragma unroll
    for (int dt = 0; dt < kTiles; ++dt) *reinterpret_cast<f32x4*>(w + 16 * dt) = acc[dt][r];
    if (g == 0) {
      joined_ml[(wave * 16 + m) * 2] = M[r];
      joined_ml[(wave * 16 + m) * 2 + 1] = l[r];
    }
    __syncthreads();
    float top = -INFINITY, lsum = 0.0f, wgt[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) top = fmaxf(top, joined_ml[(i * 16 + jr) * 2]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      wgt[i] = frame_weight(joined_ml[(i * 16 + jr) * 2], top);
      lsum = fmaf(wgt[i], joined_ml[(i * 16 + jr) * 2 + 1], lsum);
    }
    const int row = row0 + 16 * r + jr;
    if (row < rows) {
      const int64_t id = row_id(row);
      const float inv = lsum == 0.0f ? 0.0f : 1.0f / lsum;
#pragma unroll
      for (int e = 0; e < D / 16; e += 2) {
        f32x2 o = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x2 x = *reinterpret_cast<const f32x2*>(joined + (i * 16 + jr) * kPad + jd + e);
          o[0] = fmaf(wgt[i], x[0], o[0]);
          o[1] = fmaf(wgt[i], x[1], o[1]);
        }
        if (a.splits == 1) {
          typedef one one2 __attribute__((ext_vector_type(2)));
          one2 w2 = {(one)(lsum == 0.0f ? 0.0f : o[0] * inv), (one)(lsum == 0.0f ? 0.0f : o[1] * inv)};
          *reinterpret_cast<one2*>(static_cast<one*>(a.out) + id * D + jd + e) = w2;
        } else {
          *reinterpret_cast<f32x2*>(a.part + (id * a.splits + split) * D + jd + e) = o;
        }
      }
      if ((threadIdx.x & 15) == 0) {
        if (a.splits == 1) {
          if (a.lse) a.lse[id] = lsum == 0.0f ? -INFINITY : (top + log2f(lsum)) * 0.693147180559945f;
        } else {
          a.part_ml[2 * (id * a.splits + split)] = top;
          a.part_ml[2 * (id * a.splits + split) + 1] = lsum;
        }
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
  if (a.lse && lane == 0) a.lse[id] = l == 0.0f ? -INFINITY : (top + log2f(l)) * 0.693147180559945f;
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
  const int64_t base = p.slots * c.heads;
  // enough workgroups for four on each CU, each with at least 8 tiles (2 a wave)
  int64_t splits = (1024 + base - 1) / base;
  if (splits > (tiles + 7) / 8) splits = (tiles + 7) / 8;
  if (splits > 128) splits = 128;
  if (splits < 1) splits = 1;
  p.split_tiles = (int)((tiles + splits - 1) / splits);
  if (p.split_tiles < 1) p.split_tiles = 1;
  p.splits = (int)((tiles + p.split_tiles - 1) / p.split_tiles);
  if (p.splits < 1) p.splits = 1;
  return p;
}

template <int D, bool BF, int MT, bool WIDE>
void attend_one(const AttendArgs& a, int64_t slots, hipStream_t st) {
  attend_kernel<D, BF, MT, WIDE><<<dim3((unsigned)(slots * a.heads), (unsigned)a.splits), 256, 0, st>>>(a);
}

template <int D, bool BF>
hipError_t attend_launch(const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
  if (p.wide) {
    attend_one<D, BF, D == 256 ? 1 : 2, true>(a, p.slots, st);
  } else if (p.mt == 1) {
    attend_one<D, BF, 1, false>(a, p.slots, st);
  } else if (p.mt == 2) {
    attend_one<D, BF, 2, false>(a, p.slots, st);
  } else if constexpr (D <= 128) {
    attend_one<D, BF, 4, false>(a, p.slots, st);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t total = a.T * a.heads * a.group;
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
  a.scale_log2 = scale * 1.4426950408889634f;
  const bool bf = dtype == MDSS_BF16;
  switch (c.d) {
    case 64: return bf ? attend_launch<64, true>(a, p, st) : attend_launch<64, false>(a, p, st);
    case 96: return bf ? attend_launch<96, true>(a, p, st) : attend_launch<96, false>(a, p, st);
    case 128: return bf ? attend_launch<128, true>(a, p, st) : attend_launch<128, false>(a, p, st);
    default: return bf ? attend_launch<256, true>(a, p, st) : attend_launch<256, false>(a, p, st);
  }
}

}  // namespace mdss
