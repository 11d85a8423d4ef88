// Pages of the 8-bit cache (gfx950): appending tokens, forking sequences (with growth and copy on write),
// compacting the pool, copying pages.
//
// Page ids come from the caller's tables: an id outside [0, pages) is never followed.
#include "cache.h"

namespace mdss {

namespace {

constexpr int kThreads = 256;

// ---------------------------------------------------------------- append
// The least e with amax <= 448 2^e, clamped into the exponents' range (448 = 0.875 2^9 is e4m3's largest value).
__device__ __forceinline__ int exponent_of(float amax) {
  if (!(amax > 0.0f)) return kCacheMinExp;
  int x;
  const float m = frexpf(amax, &x);
  return min(max(m <= 0.875f ? x - 9 : x - 8, kCacheMinExp), kCacheMaxExp);
}
__device__ __forceinline__ float pow2f(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.0f;  // NaN and infinities set no scale
}
// Codes of two values: round to nearest even, beyond 448 (a clamped exponent) the largest code, non-finite NaN.
__device__ __forceinline__ uint32_t code_of(float x) {
  if (!(fabsf(x) < INFINITY)) return 0x7fu | (__builtin_bit_cast(uint32_t, x) >> 31 << 7);
  return __builtin_amdgcn_cvt_pk_fp8_f32(fminf(fmaxf(x, -448.0f), 448.0f), 0.0f, 0, false) & 0xffu;
}
__device__ __forceinline__ uint32_t codes_of(float a, float b) {
  if (fabsf(a) < INFINITY && fabsf(b) < INFINITY)
    return __builtin_amdgcn_cvt_pk_fp8_f32(fminf(fmaxf(a, -448.0f), 448.0f), fminf(fmaxf(b, -448.0f), 448.0f), 0, false) & 0xffffu;
  return code_of(a) | code_of(b) << 8;
}
// Four codes at another exponent (values times f = 2^(old - new) <= 1); NaN codes stay.
__device__ __forceinline__ uint32_t recode(uint32_t c, float f) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
  uint32_t r = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0] * f, lo[1] * f, 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(hi[0] * f, hi[1] * f, r, true);
  const uint32_t nan = ((((c & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7) * 0xffu;
  return (r & ~nan) | (c & nan);
}

template <bool BF>
__device__ __forceinline__ float widen16(uint16_t x) {
  if (BF) return __builtin_bit_cast(float, (uint32_t)x << 16);
  return (float)__builtin_bit_cast(_Float16, x);
}
__device__ __forceinline__ u32x4 load8(const uint16_t* p, bool aligned) {
  if (aligned) return *reinterpret_cast<const u32x4*>(p);
  u32x4 r;
#pragma unroll
  for (int w = 0; w < 4; ++w) r[w] = (uint32_t)p[2 * w] | (uint32_t)p[2 * w + 1] << 16;
  return r;
}

struct AppendArgs {
  CacheRows rows;
  const uint16_t *key, *val;
  int64_t key_st, key_sh, val_st, val_sh;
  uint8_t *k, *v;
  int8_t *k_exp, *v_exp;
  int64_t pages;
  int heads, page_shift, per_seq;
  bool key_al, val_al;
  int32_t* row_status;
};

// A workgroup of NT threads writes the new tokens of one page and head, of the keys or of the values.  The new values
// are read once (kHeld pieces of 8 a thread stay in registers between the maximum and the rounding; longer pages
// are read again).  Values go through LDS to become 16 tokens a row of d.
template <int D, bool BF, int NT>
__global__ __launch_bounds__(NT) void append_kernel(const AppendArgs a) {
  constexpr int kHeld = 4;
  constexpr int kLine = D / 8;  // pieces of a token
  constexpr int kSlab = 64;     // tokens turned at a time
  __shared__ __align__(16) uint8_t slab[kSlab * (D + 4)];
  __shared__ float red[NT / 64];
  const int tid = threadIdx.x, lane = tid & 63;
  const bool is_v = blockIdx.y & 1;
  const int h = blockIdx.y >> 1, ps = 1 << a.page_shift;
  const int64_t slot = blockIdx.x;
  int s, i;
  if (a.per_seq > 0) {
    s = (int)(slot / a.per_seq);
    i = (int)(slot - (int64_t)s * a.per_seq);
  } else {
    s = slot_sequence(a.rows.starts, a.rows.S, slot, 1, ps, 2, lane);
    i = (int)(slot - slot_first(a.rows.starts, s, 1, ps, 2));
  }
  int64_t start;
  int n;
  if (a.rows.starts) {
    start = a.rows.starts[s];
    n = (int)(a.rows.starts[s + 1] - start);
  } else {
    n = (int)(a.rows.T / a.rows.S);
    start = (int64_t)s * n;
  }
  if (start < 0 || n <= 0 || start + n > a.rows.T) return;
  const int len = a.rows.lengths[s], before = len - n;
  const bool fits = before >= 0 && (int64_t)len <= a.rows.width << a.page_shift;
  if (!fits) {
    if (i == 0 && blockIdx.y == 0 && tid == 0 && a.row_status) atomicOr(a.row_status + s, kRowNoPage);
    return;
  }
  const int pi = (before >> a.page_shift) + i;
  if (pi > (len - 1) >> a.page_shift) return;
  const int page = a.rows.table[(int64_t)s * a.rows.width + pi];
  if ((uint32_t)page >= (uint64_t)a.pages) {
    if (blockIdx.y == 0 && tid == 0 && a.row_status) atomicOr(a.row_status + s, kRowNoPage);
    return;
  }
  const int base = pi << a.page_shift;
  const int o = max(before - base, 0), cnt = min(len - base, ps) - o;
  const int64_t tok = start + (base + o - before);
  const int64_t st = is_v ? a.val_st : a.key_st;
  const uint16_t* x = (is_v ? a.val + (int64_t)h * a.val_sh : a.key + (int64_t)h * a.key_sh) + tok * st;
  const bool al = is_v ? a.val_al : a.key_al;
  const int64_t ph = (int64_t)page * a.heads + h;
  uint8_t* dst = (is_v ? a.v : a.k) + (ph << a.page_shift) * D;
  int8_t* ep = (is_v ? a.v_exp : a.k_exp) + ph;

  // the largest magnitude
  const int total = cnt * kLine;
  u32x4 held[kHeld];
  float amax = 0.0f;
  const auto fetch = [&](int e) { return load8(x + (int64_t)(e / kLine) * st + (e % kLine) * 8, al); };
  const auto largest = [&](u32x4 r) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      amax = fmaxf(amax, finite_abs(widen16<BF>((uint16_t)r[w])));
      amax = fmaxf(amax, finite_abs(widen16<BF>((uint16_t)(r[w] >> 16))));
    }
  };
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (tid + NT * j < total) held[j] = fetch(tid + NT * j);
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (tid + NT * j < total) largest(held[j]);
  for (int e = tid + NT * kHeld; e < total; e += NT) largest(fetch(e));
  amax = wave_max(amax);
  if (NT > 64) {
    if (lane == 0) red[tid >> 6] = amax;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) amax = fmaxf(amax, red[w]);
  }
  int e_new = exponent_of(amax);
  if (o > 0) {
    const int e_old = *ep;
    e_new = max(e_new, e_old);
    if (e_new > e_old) {
      // the page's earlier tokens go to the larger exponent
      const float f = pow2f(max(e_old - e_new, -126));
      const int units = (o + 15) >> 4;
      for (int e = tid; e < units * D; e += NT) {  // 16 bytes each: keys (unit, chunk, token), values (unit, d)
        u32x4* w = reinterpret_cast<u32x4*>(dst + (int64_t)e * 16);
        const int unit = e / D, have = min(o - unit * 16, 16);
        if (!is_v && (e & 15) >= have) continue;
        u32x4 c = *w;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t r = recode(c[q], f);
          const int keep = is_v ? min(max(have - 4 * q, 0), 4) : 4;
          const uint32_t mask = keep == 4 ? ~0u : (1u << (8 * keep)) - 1u;
          c[q] = (r & mask) | (c[q] & ~mask);
        }
        *w = c;
      }
    }
  }
  __syncthreads();  // every thread has read the old exponent, and old codes are written before new ones
  if (tid == 0) *ep = (int8_t)e_new;
  const float f = pow2f(-e_new);
  const auto encode = [&](u32x4 r) {
    u32x2 c;
#pragma unroll
    for (int w = 0; w < 2; ++w)
      c[w] = codes_of(widen16<BF>((uint16_t)r[2 * w]) * f, widen16<BF>((uint16_t)(r[2 * w] >> 16)) * f) |
             codes_of(widen16<BF>((uint16_t)r[2 * w + 1]) * f, widen16<BF>((uint16_t)(r[2 * w + 1] >> 16)) * f) << 16;
    return c;
  };
  if (!is_v) {
    const auto put = [&](int e, u32x4 r) {
      const int t = o + e / kLine, d8 = e % kLine;
      *reinterpret_cast<u32x2*>(dst + (int64_t)(t >> 4) * (16 * D) + (d8 >> 1) * 256 + (t & 15) * 16 + (d8 & 1) * 8) = encode(r);
    };
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
      if (tid + NT * j < total) put(tid + NT * j, held[j]);
    for (int e = tid + NT * kHeld; e < total; e += NT) put(e, fetch(e));
    return;
  }
  // values: kSlab tokens (from a unit's start) at a time through LDS, [token][D + 4]
  const int first = o & ~15, last = o + cnt;
  for (int c0 = first; c0 < last; c0 += kSlab) {
    if (c0 > first) __syncthreads();
    const int from = max(c0, o), to = min(c0 + kSlab, last);
    const auto put = [&](int e, u32x4 r) {
      const int t = o + e / kLine;
      if (t < from || t >= to) return;
      const u32x2 c = encode(r);
      uint32_t* w = reinterpret_cast<uint32_t*>(slab + (t - c0) * (D + 4) + (e % kLine) * 8);
      w[0] = c[0];
      w[1] = c[1];
    };
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
      if (tid + NT * j < total) put(tid + NT * j, held[j]);
    {  // pieces past the held ones that lie in this slab
      const int e0 = max(NT * kHeld, (from - o) * kLine), e1 = min(total, (to - o) * kLine);
      for (int e = e0 + tid; e < e1; e += NT) put(e, fetch(e));
    }
    __syncthreads();
    const int units = (to - c0 + 15) >> 4;
    for (int e = tid; e < units * D; e += NT) {
      const int u = e / D, d = e % D, t0 = c0 + 16 * u;
      uint8_t* w = dst + (int64_t)(t0 >> 4) * (16 * D) + d * 16;
      const int b = max(from - t0, 0), z = min(to - t0, 16);
      const uint8_t* col = slab + 16 * u * (D + 4) + d;
      if (b == 0 && z == 16) {
        u32x4 r;
#pragma unroll
        for (int q = 0; q < 4; ++q)
          r[q] = (uint32_t)col[(4 * q) * (D + 4)] | (uint32_t)col[(4 * q + 1) * (D + 4)] << 8 |
                 (uint32_t)col[(4 * q + 2) * (D + 4)] << 16 | (uint32_t)col[(4 * q + 3) * (D + 4)] << 24;
        *reinterpret_cast<u32x4*>(w) = r;
      } else {
        for (int t = b; t < z; ++t) w[t] = col[t * (D + 4)];
      }
    }
  }
}

template <int D, bool BF>
void append_launch(const AppendArgs& a, dim3 grid, bool small, hipStream_t st) {
  if (small)
    append_kernel<D, BF, 64><<<grid, 64, 0, st>>>(a);
  else
    append_kernel<D, BF, 256><<<grid, 256, 0, st>>>(a);
}

// ---------------------------------------------------------------- fork and compact: shared pieces
constexpr int kChunk = 1024;  // pages a workgroup counts

// Copies the listed pages in every layer; workgroups take (page, layer, keys or values, 16 KB piece) in turn.
__device__ __forceinline__ void copy_listed(const CacheView& c, const int32_t* src, const int32_t* dst, int64_t count,
                                            int64_t first, int64_t stride) {
  const int64_t region = c.region();
  const int pieces = (int)((region + kPiece - 1) / kPiece);
  const int64_t per = (int64_t)c.layers * 2 * pieces, total = count * per;
  for (int64_t i = first; i < total; i += stride) {
    const int64_t e = i / per;
    const int r = (int)(i - e * per), layer = r / (2 * pieces), rest = r - layer * 2 * pieces;
    const int kv = rest / pieces, piece = rest - kv * pieces;
    const int from = src[e], to = dst[e];
    if ((uint32_t)from >= (uint64_t)c.pages || (uint32_t)to >= (uint64_t)c.pages) continue;
    uint8_t* base = (kv ? c.v : c.k) + (int64_t)layer * c.pages * region + (int64_t)piece * kPiece;
    const int bytes = (int)min((int64_t)kPiece, region - (int64_t)piece * kPiece);
    copy_piece(base + from * region, base + to * region, bytes);
    if (piece == 0) {
      int8_t* ex = (kv ? c.v_exp : c.k_exp) + (int64_t)layer * c.pages * c.heads;
      for (int h = threadIdx.x; h < c.heads; h += kThreads) ex[(int64_t)to * c.heads + h] = ex[(int64_t)from * c.heads + h];
    }
  }
}

__global__ __launch_bounds__(kThreads) void copy_kernel(CacheView c, const int32_t* src, const int32_t* dst, int64_t n) {
  copy_listed(c, src, dst, n, blockIdx.x, gridDim.x);
}

int64_t copy_grid(const CacheView& c, int64_t most) {
  const int64_t units = most * c.layers * 2 * ((c.region() + kPiece - 1) / kPiece);
  return units < 1 ? 1 : units > 2048 ? 2048 : units;
}

// Exclusive prefix of v over the workgroup's threads (a multiple of 64) and its total; `red` has one slot a wave.
__device__ __forceinline__ int block_prefix(int v, int* red, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int incl = wave_inclusive_scan_int(v, lane);
  if (lane == 63) red[wave] = incl;
  __syncthreads();
  int before = 0, all = 0;
  for (int w = 0; w < waves; ++w) {
    if (w < wave) before += red[w];
    all += red[w];
  }
  __syncthreads();
  *total = all;
  return before + incl - v;
}

// Four of the refs from p on (0 in place of what lies past the pool).
__device__ __forceinline__ void refs4(const int32_t* refs, int64_t p, int64_t pages, int (&r)[4], int past) {
#pragma unroll
  for (int j = 0; j < 4; ++j) r[j] = p + j < pages ? refs[p + j] : past;
}

// ---------------------------------------------------------------- fork
// Workspace (int32): writers [pages], keeper [pages], free bits [chunks * 32], chunk counts [chunks + 1],
// per row: offset, flags; copy list src, dst [rows]; totals.
struct ForkWork {
  int32_t *writers, *keeper, *free_bits, *chunk, *offset, *flags, *src, *dst, *totals;
};
constexpr int kTotals = 64;  // need, copies

int64_t chunks_of(int64_t pages) { return (pages + kChunk - 1) / kChunk; }

ForkWork fork_work(void* ws, int64_t pages, int64_t rows) {
  ForkWork w;
  const int64_t n = chunks_of(pages);
  int32_t* p = static_cast<int32_t*>(ws);
  w.totals = p;
  p += kTotals;
  w.free_bits = p;
  p += n * 32;
  w.chunk = p;
  p += (n + 64) / 64 * 64;
  w.writers = p;
  p += n * kChunk;
  w.keeper = p;
  p += n * kChunk;
  w.offset = p;
  p += rows;
  w.flags = p;
  p += rows;
  w.src = p;
  p += rows;
  w.dst = p;
  return w;
}

struct ForkArgs {
  CacheView c;
  const int32_t *table, *lengths, *refs, *parent, *keep, *grow;
  int32_t *table_out, *lengths_out, *refs_out, *row_status;
  int64_t S, S_out, width;
  ForkWork w;
};

// Counts and marks the free pages, copies the reference counts, clears the per-page scratch.
__global__ __launch_bounds__(kThreads) void fork_free_kernel(ForkArgs a) {
  __shared__ int red[kThreads / 64];
  const int64_t p = (int64_t)blockIdx.x * kChunk + 4 * threadIdx.x;
  int r[4];
  refs4(a.refs, p, a.c.pages, r, 1);
  uint32_t bits = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    bits |= (r[j] == 0 ? 1u : 0u) << j;
    if (p + j < a.c.pages) a.refs_out[p + j] = r[j];
  }
  *reinterpret_cast<u32x4*>(a.w.writers + p) = u32x4{0, 0, 0, 0};
  *reinterpret_cast<u32x4*>(a.w.keeper + p) = u32x4{0, 0, 0, 0};
  uint32_t word = bits << (4 * (threadIdx.x & 7));  // eight threads make a word
#pragma unroll
  for (int off = 1; off < 8; off <<= 1) word |= __shfl_xor(word, off, 64);
  if ((threadIdx.x & 7) == 0) a.w.free_bits[(int64_t)blockIdx.x * 32 + (threadIdx.x >> 3)] = (int32_t)word;
  int total;
  block_prefix(__popc(bits), red, &total);
  if (threadIdx.x == 0) a.w.chunk[blockIdx.x] = total;
}

struct ForkRow {
  int parent, len, pages, more;  // source row (-1: none), tokens kept, their pages, pages that the growth adds
  bool over;                     // the growth passes the table's width
};
__device__ __forceinline__ int clamp_len(const ForkArgs& a, int64_t s) {
  return (int)min((int64_t)max(a.lengths[s], 0), min(a.width << a.c.page_shift, (int64_t)INT32_MAX));
}
__device__ __forceinline__ ForkRow fork_row(const ForkArgs& a, int64_t i) {
  ForkRow r;
  const int ps1 = a.c.page_size() - 1;
  r.parent = a.parent ? a.parent[i] : (int)i;
  if (r.parent < 0 || r.parent >= a.S) r.parent = -1;
  r.len = r.parent >= 0 ? clamp_len(a, r.parent) : 0;
  if (a.keep && r.parent >= 0) r.len = min(r.len, max(a.keep[i], 0));
  r.pages = (r.len + ps1) >> a.c.page_shift;
  const int64_t grow = a.grow && r.parent >= 0 ? max(a.grow[i], 0) : 0;
  const int64_t upto = r.len + grow;
  r.over = upto > min(a.width << a.c.page_shift, (int64_t)INT32_MAX);
  r.more = r.over ? 0 : (int)((upto + ps1) >> a.c.page_shift) - r.pages;
  return r;
}
__device__ __forceinline__ int fork_grow(const ForkArgs& a, int64_t i, const ForkRow& r) {
  return a.grow && r.parent >= 0 && !r.over ? max(a.grow[i], 0) : 0;
}

// Gathers the rows and counts references: one workgroup a row, first those that come in (what they held is given
// back), then those that go out.  A row that stays its own parent touches only the pages it drops.
__global__ __launch_bounds__(kThreads) void fork_rows_kernel(ForkArgs a) {
  const int64_t b = blockIdx.x;
  if (b < a.S) {
    const int64_t s = b;
    const int pages = (int)(((int64_t)clamp_len(a, s) + a.c.page_size() - 1) >> a.c.page_shift);
    int from = 0;
    if (s < a.S_out) {
      const ForkRow own = fork_row(a, s);
      if (own.parent == s) from = own.pages;
    }
    for (int j = from + threadIdx.x; j < pages; j += kThreads) {
      const int page = a.table[s * a.width + j];
      if ((uint32_t)page < (uint64_t)a.c.pages) atomicSub(a.refs_out + page, 1);
    }
    return;
  }
  const int64_t i = b - a.S;
  const ForkRow r = fork_row(a, i);
  const bool counted = r.parent == i && i < a.S;
  for (int64_t j = threadIdx.x; j < a.width; j += kThreads) {
    int page = -1;
    if (j < r.pages) {
      page = a.table[(int64_t)r.parent * a.width + j];
      if ((uint32_t)page >= (uint64_t)a.c.pages)
        page = -1;
      else if (!counted)
        atomicAdd(a.refs_out + page, 1);
    }
    a.table_out[i * a.width + j] = page;
  }
  if (threadIdx.x == 0 && fork_grow(a, i, r) > 0 && (r.len & (a.c.page_size() - 1)) != 0) {
    const int page = a.table[(int64_t)r.parent * a.width + r.pages - 1];
    if ((uint32_t)page < (uint64_t)a.c.pages) {
      atomicAdd(a.w.writers + page, 1);
      atomicMax(a.w.keeper + page, (int32_t)i + 1);
    }
  }
}

// The page of free rank g: its chunk from the exclusive prefix, then its bit.
__device__ __forceinline__ int free_page(const int32_t* chunk, const int32_t* bits, int chunks, int g) {
  int lo = 0, hi = chunks;  // last chunk with prefix <= g
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (chunk[mid] <= g) lo = mid; else hi = mid;
  }
  int left = g - chunk[lo];
  for (int w = 0; w < 32; ++w) {
    uint32_t x = (uint32_t)bits[lo * 32 + w];
    const int c = __popc(x);
    if (left < c) {
      while (left-- > 0) x &= x - 1;
      return lo * kChunk + 32 * w + __ffs((int)x) - 1;
    }
    left -= c;
  }
  return -1;
}

// One workgroup: the rows' needs, their places among the free pages, the list of copies, the new lengths.
constexpr int kPlanThreads = 1024;
__global__ __launch_bounds__(kPlanThreads) void fork_plan_kernel(ForkArgs a, int chunks) {
  __shared__ int red[kPlanThreads / 64];
  const int tid = threadIdx.x;
  int have = 0, need = 0, copies = 0, total;
  for (int c0 = 0; c0 < chunks; c0 += kPlanThreads) {
    const int c = c0 + tid, v = c < chunks ? a.w.chunk[c] : 0;
    const int at = block_prefix(v, red, &total);
    if (c < chunks) a.w.chunk[c] = have + at;
    have += total;
  }
  const int ps1 = a.c.page_size() - 1;
  for (int64_t i0 = 0; i0 < a.S_out; i0 += kPlanThreads) {
    const int64_t i = i0 + tid;
    int n = 0, cow = 0;
    if (i < a.S_out) {
      const ForkRow r = fork_row(a, i);
      n = r.more;
      if (fork_grow(a, i, r) > 0 && (r.len & ps1) != 0) {
        const int page = a.table[(int64_t)r.parent * a.width + r.pages - 1];
        if ((uint32_t)page < (uint64_t)a.c.pages) {
          const int refs = a.refs_out[page];
          cow = refs > 1 && !(a.w.writers[page] == refs && a.w.keeper[page] == (int)i + 1);
          if (cow) a.w.src[i] = page;  // (by row here; the list is made below)
        }
      }
      n += cow;
    }
    const int at = block_prefix(n, red, &total);
    if (i < a.S_out) {
      a.w.offset[i] = need + at;
      a.w.flags[i] = cow;
    }
    need += total;
    block_prefix(cow, red, &total);
    copies += total;
  }
  const bool enough = need <= have;
  __syncthreads();  // chunk prefixes, offsets and decisions are read by other threads from here on
  int listed = 0;
  for (int64_t i0 = 0; i0 < a.S_out; i0 += kPlanThreads) {
    const int64_t i = i0 + tid;
    int cow = 0, page = 0;
    if (i < a.S_out) {
      const ForkRow r = fork_row(a, i);
      const int grow = fork_grow(a, i, r);
      a.lengths_out[i] = r.len + (enough ? grow : 0);
      if (a.row_status && (r.over || (!enough && grow > 0))) atomicOr(a.row_status + i, kRowNoPage);
      cow = enough ? a.w.flags[i] : 0;
      page = cow ? a.w.src[i] : 0;
    }
    const int at = block_prefix(cow, red, &total);  // (its barriers part the reads of src above from the writes below)
    if (cow) {
      const int to = free_page(a.w.chunk, a.w.free_bits, chunks, a.w.offset[i]);
      a.w.src[listed + at] = page;
      a.w.dst[listed + at] = to;
      const ForkRow r = fork_row(a, i);
      a.table_out[i * a.width + r.pages - 1] = to;
      atomicSub(a.refs_out + page, 1);
      a.refs_out[to] = 1;
    }
    listed += total;
  }
  if (tid == 0) {
    a.w.totals[0] = enough ? need : 0;
    a.w.totals[1] = enough ? copies : 0;
  }
}

// Hands out the pages of the growth and copies what the plan listed.
__global__ __launch_bounds__(kThreads) void fork_take_kernel(ForkArgs a, int chunks) {
  const int need = a.w.totals[0];
  for (int64_t g = (int64_t)blockIdx.x * kThreads + threadIdx.x; g < need; g += (int64_t)gridDim.x * kThreads) {
    int64_t lo = 0, hi = a.S_out;  // last row with offset <= g
    while (hi - lo > 1) {
      const int64_t mid = (lo + hi) >> 1;
      if (a.w.offset[mid] <= g) lo = mid; else hi = mid;
    }
    const int k = (int)(g - a.w.offset[lo]) - a.w.flags[lo];
    if (k < 0) continue;  // the copied page, in place already
    const ForkRow r = fork_row(a, lo);
    const int page = free_page(a.w.chunk, a.w.free_bits, chunks, (int)g);
    a.table_out[lo * a.width + r.pages + k] = page;
    a.refs_out[page] = 1;
  }
  copy_listed(a.c, a.w.src, a.w.dst, a.w.totals[1], blockIdx.x, gridDim.x);
}

// ---------------------------------------------------------------- compact
struct CompactArgs {
  CacheView c;
  const int32_t *table, *lengths, *refs;
  int32_t *table_out, *refs_out, *used;
  int64_t S, width;
  int32_t *chunk, *map, *src, *dst, *totals;
};

__global__ __launch_bounds__(kThreads) void compact_count_kernel(CompactArgs a) {
  __shared__ int red[kThreads / 64];
  int r[4], total;
  refs4(a.refs, (int64_t)blockIdx.x * kChunk + 4 * threadIdx.x, a.c.pages, r, 0);
  block_prefix((r[0] > 0) + (r[1] > 0) + (r[2] > 0) + (r[3] > 0), red, &total);
  if (threadIdx.x == 0) a.chunk[blockIdx.x] = total;
}

// With U used pages, the r-th highest used page >= U goes to the r-th lowest hole below U.  map[p]: where a used page
// goes (~r for the r-th that moves), or for a hole below U its rank.
__global__ __launch_bounds__(kThreads) void compact_rank_kernel(CompactArgs a, int chunks) {
  __shared__ int red[kThreads / 64];
  int mine = 0, all = 0;
  for (int c = threadIdx.x; c < chunks; c += kThreads) {
    const int v = a.chunk[c];
    all += v;
    if (c < (int)blockIdx.x) mine += v;
  }
  int before, U;
  block_prefix(mine, red, &before);
  block_prefix(all, red, &U);
  const int64_t p0 = (int64_t)blockIdx.x * kChunk + 4 * threadIdx.x;
  int r[4], total;
  refs4(a.refs, p0, a.c.pages, r, 0);
  int up = before + block_prefix((r[0] > 0) + (r[1] > 0) + (r[2] > 0) + (r[3] > 0), red, &total);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t p = p0 + j;
    if (p >= a.c.pages) break;
    if (p == U) a.totals[0] = U - up;  // holes below U = pages that move
    if (r[j] > 0) {
      if (p >= U) a.src[U - 1 - up] = (int32_t)p;
      a.map[p] = p < U ? (int32_t)p : ~(U - 1 - up);
    } else if (p < U) {
      a.dst[p - up] = (int32_t)p;
      a.map[p] = (int32_t)(p - up);
    }
    up += r[j] > 0;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (U == a.c.pages) a.totals[0] = 0;
    *a.used = U;
    a.totals[1] = U;
  }
}

__global__ __launch_bounds__(kThreads) void compact_move_kernel(CompactArgs a) {
  const int count = a.totals[0], U = a.totals[1];
  const int64_t stride = (int64_t)gridDim.x * kThreads, first = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  for (int64_t i = first; i < a.S * a.width; i += stride) {
    const int64_t s = i / a.width;
    int page = a.table[i], to = -1;
    if ((i - s * a.width) << a.c.page_shift >= a.lengths[s]) page = -1;  // past the row's tokens
    if ((uint32_t)page < (uint64_t)a.c.pages && a.refs[page] > 0) {
      to = a.map[page];
      if (to < 0) to = a.dst[~to];
    }
    a.table_out[i] = to;
  }
  for (int64_t p = first; p < a.c.pages; p += stride) {
    int n = 0;
    if (p < U) {
      n = a.refs[p];
      if (n <= 0) n = a.refs[a.src[a.map[p]]];
    }
    a.refs_out[p] = n;
  }
  copy_listed(a.c, a.src, a.dst, count, blockIdx.x, gridDim.x);
}

}  // namespace

hipError_t launch_cache_append(const CacheView& c, int layer, const void* key, const void* value, int dtype,
                               int64_t key_st, int64_t key_sh, int64_t val_st, int64_t val_sh, const CacheRows& rows,
                               int32_t* row_status, hipStream_t st) {
  AppendArgs a;
  a.rows = rows;
  a.key = static_cast<const uint16_t*>(key);
  a.val = static_cast<const uint16_t*>(value);
  a.key_st = key_st;
  a.key_sh = key_sh;
  a.val_st = val_st;
  a.val_sh = val_sh;
  a.k = c.k + layer * c.pages * c.region();
  a.v = c.v + layer * c.pages * c.region();
  a.k_exp = c.k_exp + layer * c.pages * c.heads;
  a.v_exp = c.v_exp + layer * c.pages * c.heads;
  a.pages = c.pages;
  a.heads = c.heads;
  a.page_shift = c.page_shift;
  a.row_status = row_status;
  a.key_al = (reinterpret_cast<uintptr_t>(key) & 15) == 0 && key_st % 8 == 0 && key_sh % 8 == 0;
  a.val_al = (reinterpret_cast<uintptr_t>(value) & 15) == 0 && val_st % 8 == 0 && val_sh % 8 == 0;
  // pages that n new tokens touch: one for n = 1, at most (n - 1) / page_size + 2
  const int64_t n = rows.T / rows.S;
  a.per_seq = rows.starts ? 0 : n == 1 ? 1 : (int)(((n - 1) >> c.page_shift) + 2);
  const int64_t slots = rows.starts ? (rows.T >> c.page_shift) + 2 * (int64_t)rows.S : (int64_t)rows.S * a.per_seq;
  const dim3 grid((unsigned)slots, (unsigned)(2 * c.heads));
  // few tokens a page: a wave is enough
  const bool small = rows.T <= 2 * (int64_t)rows.S, bf = dtype == MDSS_BF16;
  switch (c.d) {
    case 64: bf ? append_launch<64, true>(a, grid, small, st) : append_launch<64, false>(a, grid, small, st); break;
    case 96: bf ? append_launch<96, true>(a, grid, small, st) : append_launch<96, false>(a, grid, small, st); break;
    case 128: bf ? append_launch<128, true>(a, grid, small, st) : append_launch<128, false>(a, grid, small, st); break;
    default: bf ? append_launch<256, true>(a, grid, small, st) : append_launch<256, false>(a, grid, small, st); break;
  }
  return hipGetLastError();
}

size_t workspace_bytes_cache_fork(int64_t pages, int64_t rows) {
  const int64_t n = chunks_of(pages);
  return sizeof(int32_t) * (size_t)(kTotals + n * 32 + (n + 64) / 64 * 64 + 2 * n * kChunk + 4 * rows);
}

hipError_t launch_cache_fork(const CacheView& c, const int32_t* table, const int32_t* lengths, int64_t S,
                             int64_t width, const int32_t* refs, const int32_t* parent, const int32_t* keep,
                             const int32_t* grow, int64_t S_out, int32_t* table_out, int32_t* lengths_out,
                             int32_t* refs_out, int32_t* row_status, void* workspace, hipStream_t st) {
  ForkArgs a;
  a.c = c;
  a.table = table;
  a.lengths = lengths;
  a.refs = refs;
  a.parent = parent;
  a.keep = keep;
  a.grow = grow;
  a.table_out = table_out;
  a.lengths_out = lengths_out;
  a.refs_out = refs_out;
  a.row_status = row_status;
  a.S = S;
  a.S_out = S_out;
  a.width = width;
  a.w = fork_work(workspace, c.pages, S_out);
  const int chunks = (int)chunks_of(c.pages);
  fork_free_kernel<<<chunks, kThreads, 0, st>>>(a);
  if (S + S_out > 0) fork_rows_kernel<<<(unsigned)(S + S_out), kThreads, 0, st>>>(a);
  if (S_out > 0) {
    fork_plan_kernel<<<1, kPlanThreads, 0, st>>>(a, chunks);
    if (grow) fork_take_kernel<<<(unsigned)copy_grid(c, S_out), kThreads, 0, st>>>(a, chunks);
  }
  return hipGetLastError();
}

size_t workspace_bytes_cache_compact(int64_t pages) {
  const int64_t n = chunks_of(pages);
  return sizeof(int32_t) * (size_t)(kTotals + (n + 63) / 64 * 64 + 3 * n * kChunk);
}

hipError_t launch_cache_compact(const CacheView& c, const int32_t* table, const int32_t* lengths, int64_t S,
                                int64_t width, const int32_t* refs, int32_t* table_out, int32_t* refs_out,
                                int32_t* used, void* workspace, hipStream_t st) {
  CompactArgs a;
  a.c = c;
  a.table = table;
  a.lengths = lengths;
  a.refs = refs;
  a.table_out = table_out;
  a.refs_out = refs_out;
  a.used = used;
  a.S = S;
  a.width = width;
  const int64_t n = chunks_of(c.pages);
  int32_t* p = static_cast<int32_t*>(workspace);
  a.totals = p;
  p += kTotals;
  a.chunk = p;
  p += (n + 63) / 64 * 64;
  a.map = p;
  p += n * kChunk;
  a.src = p;
  p += n * kChunk;
  a.dst = p;
  compact_count_kernel<<<(unsigned)n, kThreads, 0, st>>>(a);
  compact_rank_kernel<<<(unsigned)n, kThreads, 0, st>>>(a, (int)n);
  compact_move_kernel<<<(unsigned)copy_grid(c, c.pages), kThreads, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_cache_copy(const CacheView& c, const int32_t* src, const int32_t* dst, int64_t n, hipStream_t st) {
  copy_kernel<<<(unsigned)copy_grid(c, n), kThreads, 0, st>>>(c, src, dst, n);
  return hipGetLastError();
}

}  // namespace mdss
