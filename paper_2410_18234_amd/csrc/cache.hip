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

// A workgroup of NT threads writes the new tokens of one page and head, keys and values.  They are read once (kHeld pieces of
// 8 a thread of each stay in registers between the maximum and the rounding; longer pages are read again), keys and
// values together, since what a workgroup waits for is the chain starts - lengths - table - tokens.  Values go
// through LDS to become 16 tokens a row of d.  Bound by memory on prompts (16 x up to 2048 tokens, 8 heads of 128, 174 MB: 44 us,
// 3.9 TB/s), by the launch on single tokens (256 of them: 12 us a call).
template <int D, bool BF, int NT>
__global__ __launch_bounds__(NT, 4) void append_kernel(const AppendArgs a) {
  constexpr int kHeld = NT == 64 ? 2 : 4;
  constexpr int kLine = D / 8;           // pieces of a token
  constexpr int kSlab = NT == 64 ? 16 : 64;  // tokens turned at a time
  __shared__ __align__(16) uint8_t slab[kSlab * (D + 4)];
  __shared__ float red[2][NT / 64];
  const int tid = threadIdx.x, lane = tid & 63;
  const int h = blockIdx.y, ps = 1 << a.page_shift;
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
    if (i == 0 && h == 0 && tid == 0 && a.row_status) atomicOr(a.row_status + s, kRowNoPage);
    return;
  }
  const int pi = (before >> a.page_shift) + i;
  if (i < 0 || pi > (len - 1) >> a.page_shift) return;  // (i < 0: starts[0] is not 0)
  const int page = a.rows.table[(int64_t)s * a.rows.width + pi];
  if ((uint32_t)page >= (uint64_t)a.pages) {
    if (h == 0 && tid == 0 && a.row_status) atomicOr(a.row_status + s, kRowNoPage);
    return;
  }
  const int base = pi << a.page_shift;
  const int o = max(before - base, 0), cnt = min(len - base, ps) - o, total = cnt * kLine;
  const int64_t tok = start + (base + o - before);
  const uint16_t* kx = a.key + (int64_t)h * a.key_sh + tok * a.key_st;
  const uint16_t* vx = a.val + (int64_t)h * a.val_sh + tok * a.val_st;
  const int64_t ph = (int64_t)page * a.heads + h;
  uint8_t *kd = a.k + (ph << a.page_shift) * D, *vd = a.v + (ph << a.page_shift) * D;
  const auto fetch_k = [&](int e) { return load8(kx + (int64_t)(e / kLine) * a.key_st + (e % kLine) * 8, a.key_al); };
  const auto fetch_v = [&](int e) { return load8(vx + (int64_t)(e / kLine) * a.val_st + (e % kLine) * 8, a.val_al); };

  // the largest magnitudes
  u32x4 kh[kHeld], vh[kHeld];
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (tid + NT * j < total) {
      kh[j] = fetch_k(tid + NT * j);
      vh[j] = fetch_v(tid + NT * j);
    }
  int ke = kCacheMinExp, ve = kCacheMinExp;  // of the page's earlier tokens
  if (o > 0) {
    ke = a.k_exp[ph];
    ve = a.v_exp[ph];
  }
  const auto largest = [&](u32x4 r, float m) {
#pragma unroll
    for (int w = 0; w < 4; ++w)
      m = fmaxf(m, fmaxf(finite_abs(widen16<BF>((uint16_t)r[w])), finite_abs(widen16<BF>((uint16_t)(r[w] >> 16)))));
    return m;
  };
  float km = 0.0f, vm = 0.0f;
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (tid + NT * j < total) {
      km = largest(kh[j], km);
      vm = largest(vh[j], vm);
    }
  for (int e = tid + NT * kHeld; e < total; e += NT) {
    km = largest(fetch_k(e), km);
    vm = largest(fetch_v(e), vm);
  }
  km = wave_max(km);
  vm = wave_max(vm);
  if (NT > 64) {
    if (lane == 0) {
      red[0][tid >> 6] = km;
      red[1][tid >> 6] = vm;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
      km = fmaxf(km, red[0][w]);
      vm = fmaxf(vm, red[1][w]);
    }
  }
  const int ke_new = max(exponent_of(km), ke), ve_new = max(exponent_of(vm), ve);
  if (o > 0) {
    // the page's earlier tokens go to the larger exponent: 16 bytes a step, of keys (unit, chunk, token), of values (unit, d)
    if (ke_new > ke) {
      const float f = pow2f(max(ke - ke_new, -126));
      for (int e = tid; e < ((o + 15) >> 4) * D; e += NT) {
        if ((e & 15) >= o - e / D * 16) continue;
        u32x4* w = reinterpret_cast<u32x4*>(kd + (int64_t)e * 16);
        u32x4 c = *w;
#pragma unroll
        for (int q = 0; q < 4; ++q) c[q] = recode(c[q], f);
        *w = c;
      }
    }
    if (ve_new > ve) {
      const float f = pow2f(max(ve - ve_new, -126));
      for (int e = tid; e < ((o + 15) >> 4) * D; e += NT) {
        u32x4* w = reinterpret_cast<u32x4*>(vd + (int64_t)e * 16);
        u32x4 c = *w;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int keep = min(max(o - e / D * 16 - 4 * q, 0), 4);
          const uint32_t mask = keep == 4 ? ~0u : (1u << (8 * keep)) - 1u;
          c[q] = (recode(c[q], f) & mask) | (c[q] & ~mask);
        }
        *w = c;
      }
    }
  }
  __syncthreads();  // every thread has the old exponents, and old codes are written before new ones
  if (tid == 0) {
    a.k_exp[ph] = (int8_t)ke_new;
    a.v_exp[ph] = (int8_t)ve_new;
  }
  const auto encode = [&](u32x4 r, float f) {
    u32x2 c;
#pragma unroll
    for (int w = 0; w < 2; ++w)
      c[w] = codes_of(widen16<BF>((uint16_t)r[2 * w]) * f, widen16<BF>((uint16_t)(r[2 * w] >> 16)) * f) |
             codes_of(widen16<BF>((uint16_t)r[2 * w + 1]) * f, widen16<BF>((uint16_t)(r[2 * w + 1] >> 16)) * f) << 16;
    return c;
  };
  const float kf = pow2f(-ke_new), vf = pow2f(-ve_new);
  const auto put_k = [&](int e, u32x4 r) {
    const int t = o + e / kLine, d8 = e % kLine;
    *reinterpret_cast<u32x2*>(kd + (t >> 4) * (16 * D) + (d8 >> 1) * 256 + (t & 15) * 16 + (d8 & 1) * 8) = encode(r, kf);
  };
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (tid + NT * j < total) put_k(tid + NT * j, kh[j]);
  for (int e = tid + NT * kHeld; e < total; e += NT) put_k(e, fetch_k(e));
  // values: kSlab tokens (from a unit's start) at a time through LDS, [token][D + 4]
  const int last = o + cnt;
  for (int c0 = o & ~15; c0 < last; c0 += kSlab) {
    if (c0 > (o & ~15)) __syncthreads();
    const int from = max(c0, o), to = min(c0 + kSlab, last);
    const auto put_v = [&](int e, u32x4 r) {
      const int t = o + e / kLine;
      if (t < from || t >= to) return;
      const u32x2 c = encode(r, vf);
      uint32_t* w = reinterpret_cast<uint32_t*>(slab + (t - c0) * (D + 4) + (e % kLine) * 8);
      w[0] = c[0];
      w[1] = c[1];
    };
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
      if (tid + NT * j < total) put_v(tid + NT * j, vh[j]);
    {  // pieces past the held ones that lie in this slab
      const int e0 = max(NT * kHeld, (from - o) * kLine), e1 = min(total, (to - o) * kLine);
      for (int e = e0 + tid; e < e1; e += NT) put_v(e, fetch_v(e));
    }
    __syncthreads();
    const int units = (to - c0 + 15) >> 4;
    for (int e = tid; e < units * D; e += NT) {
      const int u = e / D, d = e % D, t0 = c0 + 16 * u;
      uint8_t* w = vd + (t0 >> 4) * (16 * D) + d * 16;
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

// Copies the listed pages in every layer: workgroups take (page, layer, keys or values, 16 KB piece) in turn, the next
// piece on its way while one is written.  Nothing is read twice, so the caches are passed by.  0.96 GB moved by a compaction:
// 198 us, 4.9 TB/s.
constexpr int kPiece = 16384;
struct Piece {
  const uint8_t* src;
  uint8_t* dst;
  int bytes;
};
__device__ __forceinline__ void copy_listed(const CacheView& c, const int32_t* src, const int32_t* dst, int64_t count,
                                            int64_t first, int64_t stride) {
  const int64_t region = c.region();
  const int pieces = (int)((region + kPiece - 1) / kPiece);
  const int per = c.layers * 2 * pieces;
  const int64_t total = count * per;
  const auto load = [&](int64_t i, u32x4 (&r)[4]) {
    const int64_t e = total <= UINT32_MAX ? (uint32_t)i / (uint32_t)per : i / per;
    const int x = (int)(i - e * per), layer = x / (2 * pieces), rest = x - layer * 2 * pieces;
    const int kv = rest / pieces, piece = rest - kv * pieces;
    const int from = src[e], to = dst[e];
    Piece p = {nullptr, nullptr, 0};
    if ((uint32_t)from >= (uint64_t)c.pages || (uint32_t)to >= (uint64_t)c.pages) return p;
    uint8_t* base = (kv ? c.v : c.k) + (int64_t)layer * c.pages * region + (int64_t)piece * kPiece;
    p.src = base + from * region;
    p.dst = base + to * region;
    p.bytes = (int)min((int64_t)kPiece, region - (int64_t)piece * kPiece);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int at = ((int)threadIdx.x + kThreads * j) * 16;
      if (at < p.bytes) r[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p.src + at));
    }
    if (piece == 0) {
      int8_t* ex = (kv ? c.v_exp : c.k_exp) + (int64_t)layer * c.pages * c.heads;
      for (int h = threadIdx.x; h < c.heads; h += kThreads) ex[(int64_t)to * c.heads + h] = ex[(int64_t)from * c.heads + h];
    }
    return p;
  };
  const auto store = [&](const Piece& p, const u32x4 (&r)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int at = ((int)threadIdx.x + kThreads * j) * 16;
      if (at < p.bytes) __builtin_nontemporal_store(r[j], reinterpret_cast<u32x4*>(p.dst + at));
    }
  };
  if (first >= total) return;
  u32x4 ra[4], rb[4];
  Piece pa = load(first, ra);
  for (int64_t i = first + stride;; i += 2 * stride) {
    if (i >= total) return store(pa, ra);
    const Piece pb = load(i, rb);
    store(pa, ra);
    if (i + stride >= total) return store(pb, rb);
    pa = load(i + stride, ra);
    store(pb, rb);
  }
}

__global__ __launch_bounds__(kThreads) void copy_kernel(CacheView c, const int32_t* src, const int32_t* dst, int64_t n) {
  copy_listed(c, src, dst, n, blockIdx.x, gridDim.x);
}

__global__ __launch_bounds__(kThreads) void copy_counted_kernel(CacheView c, const int32_t* src, const int32_t* dst,
                                                                const int32_t* count) {
  copy_listed(c, src, dst, *count, blockIdx.x, gridDim.x);
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
// Workspace (int32): totals, free bits [chunks * 32], chunk counts, writers [pages], keeper [pages], per row: what the
// gather found (4 words) and offset, the list of copies src, dst [rows].
struct ForkWork {
  int32_t *writers, *keeper, *free_bits, *chunk, *offset, *src, *dst, *totals;
  int4* row;
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
  w.row = reinterpret_cast<int4*>(p);
  p += 4 * rows;
  w.offset = p;
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

// What the plan wants to know of a row: the page that it grows on (-1: none), tokens kept, pages added (-1: the table is too
// narrow), growth.  Counts the row among the page's writers.
__device__ __forceinline__ int4 fork_found(const ForkArgs& a, int64_t i, const ForkRow& r, int32_t* writers, int32_t* keeper) {
  const int grow = fork_grow(a, i, r);
  int page = -1;
  if (grow > 0 && (r.len & (a.c.page_size() - 1)) != 0) {
    page = a.table[(int64_t)r.parent * a.width + r.pages - 1];
    if ((uint32_t)page < (uint64_t)a.c.pages) {
      atomicAdd(writers + page, 1);
      atomicMax(keeper + page, (int32_t)i + 1);
    } else {
      page = -1;
    }
  }
  return make_int4(page, r.len, r.over ? -1 : r.more, grow);
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
  if (threadIdx.x == 0) a.w.row[i] = fork_found(a, i, r, a.w.writers, a.w.keeper);
}

// The page of free rank g: its chunk from the exclusive prefix, then its bit among the chunk's 1024.
__device__ __forceinline__ int free_page(const int32_t* chunk, const int32_t* bits, int chunks, int g) {
  int lo = 0, hi = chunks;  // last chunk with prefix <= g
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (chunk[mid] <= g) lo = mid; else hi = mid;
  }
  u32x4 w[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) w[j] = *reinterpret_cast<const u32x4*>(bits + lo * 32 + 4 * j);
  int left = g - chunk[lo], word = 0;
  uint32_t x = 0;
  bool found = false;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    const uint32_t v = w[j >> 2][j & 3];
    const int c = __popc(v);
    if (!found) {
      if (left < c) {
        found = true;
        x = v;
        word = j;
      } else {
        left -= c;
      }
    }
  }
  while (left-- > 0) x &= x - 1;
  return lo * kChunk + 32 * word + __ffs((int)x) - 1;
}

// The decisions of a fork, by one workgroup of 1024 threads: the rows' needs, their places among the free pages, the list
// of copies, the new lengths.  row(i): what the gather found of row i, count(page): the page's references, writers and
// keeper; chunk and bits: the free pages (chunk becomes its exclusive prefix), anywhere.
constexpr int kPlanThreads = 1024;
template <typename Row, typename Count, typename Take>
__device__ __forceinline__ void fork_plan(const ForkArgs& a, int chunks, int32_t* chunk, const int32_t* bits, int32_t* offset,
                                          int* red, Row row, Count count, Take take) {
  const int tid = threadIdx.x;
  int have = 0, need = 0, copies = 0, total;
  // (rows of the last tile stay in registers: all of them, mostly)
  int64_t i = tid;
  int4 r = i < a.S_out ? row(i) : make_int4(-1, 0, 0, 0);
  int cow = 0, first = 0;
  for (int c0 = 0; c0 < chunks; c0 += kPlanThreads) {
    const int c = c0 + tid, v = c < chunks ? chunk[c] : 0;
    const int at = block_prefix(v, red, &total);
    if (c < chunks) chunk[c] = have + at;
    have += total;
  }
  for (int64_t i0 = 0; i0 < a.S_out; i0 += kPlanThreads) {
    if (i0 > 0) {
      i = i0 + tid;
      r = i < a.S_out ? row(i) : make_int4(-1, 0, 0, 0);
    }
    cow = 0;
    if (r.x >= 0) {
      const int3 n = count(r.x);
      cow = n.x > 1 && !(n.y == n.x && n.z == (int)i + 1);
    }
    first = need + block_prefix(max(r.z, 0) + cow, red, &total);
    need += total;
    if (i < a.S_out) {
      offset[i] = first;
      row(i).w = cow ? r.w : -1 - r.w;  // a row without a copy: the growth's complement
    }
  }
  const bool enough = need <= have;
  __syncthreads();  // chunk prefixes and decisions are read by other threads, and counts change, from here on
  const bool kept = a.S_out <= kPlanThreads;
  for (int64_t i0 = 0; i0 < a.S_out; i0 += kPlanThreads) {
    if (!kept) {
      i = i0 + tid;
      r = make_int4(-1, 0, 0, 0);
      cow = 0;
      if (i < a.S_out) {
        r = row(i);
        cow = r.w >= 0 && r.x >= 0;
        r.w = r.w >= 0 ? r.w : -1 - r.w;
        first = offset[i];
      }
    }
    if (i < a.S_out) {
      a.lengths_out[i] = r.y + (enough ? r.w : 0);
      if (a.row_status && (r.z < 0 || (!enough && r.w > 0))) atomicOr(a.row_status + i, kRowNoPage);
    }
    const int at = copies + block_prefix(cow && enough, red, &total);
    copies += total;
    if (cow && enough) {
      const int to = free_page(chunk, bits, chunks, first);
      a.w.src[at] = r.x;
      a.w.dst[at] = to;
      a.table_out[i * a.width + (r.y >> a.c.page_shift)] = to;
      take(r.x, to);
    }
  }
  if (tid == 0) {
    a.w.totals[0] = enough ? need : 0;
    a.w.totals[1] = copies;
  }
}

// The g-th page that the rows' growth takes, put into its table; -1 for a row's copied page, which is in place already.
__device__ __forceinline__ int fork_take(const ForkArgs& a, int chunks, const int32_t* chunk, const int32_t* bits,
                                         const int32_t* offset, const int4* rows, int g) {
  int64_t lo = 0, hi = a.S_out;  // last row with offset <= g
  while (hi - lo > 1) {
    const int64_t mid = (lo + hi) >> 1;
    if (offset[mid] <= g) lo = mid; else hi = mid;
  }
  const int4 r = rows[lo];
  const int k = g - offset[lo] - (r.w >= 0 && r.x >= 0);
  if (k < 0) return -1;
  const int page = free_page(chunk, bits, chunks, g);
  a.table_out[lo * a.width + ((r.y + a.c.page_size() - 1) >> a.c.page_shift) + k] = page;
  return page;
}

// The free pages' counts and bits come into LDS (pools of up to 2^18 pages): what is looked up after the decisions is near.
constexpr int kNearChunks = 256;
__global__ __launch_bounds__(kPlanThreads) void fork_plan_kernel(ForkArgs a, int chunks) {
  __shared__ int red[kPlanThreads / 64];
  __shared__ int32_t near_chunk[kNearChunks];
  __shared__ __align__(16) int32_t near_bits[kNearChunks * 32];
  const auto row = [&](int64_t i) -> int4& { return a.w.row[i]; };
  const auto count = [&](int page) { return make_int3(a.refs_out[page], a.w.writers[page], a.w.keeper[page]); };
  const auto take = [&](int from, int to) {
    atomicSub(a.refs_out + from, 1);
    a.refs_out[to] = 1;
  };
  if (chunks <= kNearChunks) {
    for (int i = threadIdx.x; i < chunks * 8; i += kPlanThreads)
      reinterpret_cast<u32x4*>(near_bits)[i] = reinterpret_cast<const u32x4*>(a.w.free_bits)[i];
    for (int i = threadIdx.x; i < chunks; i += kPlanThreads) near_chunk[i] = a.w.chunk[i];
    __syncthreads();
    fork_plan(a, chunks, near_chunk, near_bits, a.w.offset, red, row, count, take);
    for (int i = threadIdx.x; i < chunks; i += kPlanThreads) a.w.chunk[i] = near_chunk[i];
  } else {
    fork_plan(a, chunks, a.w.chunk, a.w.free_bits, a.w.offset, red, row, count, take);
  }
}

// Hands out the pages of the growth and copies what the plan listed.
__global__ __launch_bounds__(kThreads) void fork_take_kernel(ForkArgs a, int chunks) {
  const int need = a.w.totals[0], copies = a.w.totals[1];
  for (int64_t g = (int64_t)blockIdx.x * kThreads + threadIdx.x; g < need; g += (int64_t)gridDim.x * kThreads) {
    const int page = fork_take(a, chunks, a.w.chunk, a.w.free_bits, a.w.offset, a.w.row, (int)g);
    if (page >= 0) a.refs_out[page] = 1;
  }
  copy_listed(a.c, a.w.src, a.w.dst, copies, blockIdx.x, gridDim.x);
}

// Small pools and tables: all but the copies in one workgroup, the counts in LDS (4 x 4 beams of 300 tokens: a call takes
// 20.1 us against 25.7 with the launches of the large form).
constexpr int kSmallPages = 8192, kSmallRows = 1024, kSmallEntries = 16384;
__global__ __launch_bounds__(kPlanThreads) void fork_small_kernel(ForkArgs a, int chunks) {
  __shared__ int red[kPlanThreads / 64];
  __shared__ int32_t refs[kSmallPages], writers[kSmallPages], keeper[kSmallPages];
  __shared__ int32_t chunk[kSmallPages / kChunk];
  __shared__ __align__(16) int32_t bits[kSmallPages / 32];
  __shared__ __align__(16) int4 rows[kSmallRows];
  __shared__ int32_t offset[kSmallRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), ps1 = a.c.page_size() - 1;
  if (tid < kSmallPages / kChunk) chunk[tid] = 0;
  __syncthreads();
  for (int p0 = 0; p0 < chunks * kChunk; p0 += kPlanThreads) {  // a wave makes two words of bits
    const int p = p0 + tid;
    const int r = p < a.c.pages ? a.refs[p] : 1;
    refs[p] = r;
    writers[p] = keeper[p] = 0;
    const uint64_t free = __ballot(r == 0);
    if (lane < 2) bits[(p0 + wave * 64) / 32 + lane] = (int32_t)(free >> (32 * lane));
    if (lane == 0) atomicAdd(chunk + p0 / kChunk, __popcll(free));
  }
  __syncthreads();
  for (int64_t s = wave; s < a.S; s += kPlanThreads / 64) {
    const int pages = (int)(((int64_t)clamp_len(a, s) + ps1) >> a.c.page_shift);
    for (int j = lane; j < pages; j += 64) {
      const int page = a.table[s * a.width + j];
      if ((uint32_t)page < (uint64_t)a.c.pages) atomicSub(refs + page, 1);
    }
  }
  for (int64_t i = wave; i < a.S_out; i += kPlanThreads / 64) {
    const ForkRow r = fork_row(a, i);
    for (int64_t j = lane; j < a.width; j += 64) {
      int page = -1;
      if (j < r.pages) {
        page = a.table[(int64_t)r.parent * a.width + j];
        if ((uint32_t)page >= (uint64_t)a.c.pages)
          page = -1;
        else
          atomicAdd(refs + page, 1);
      }
      a.table_out[i * a.width + j] = page;
    }
    if (lane == 0) rows[i] = fork_found(a, i, r, writers, keeper);
  }
  __syncthreads();
  fork_plan(
      a, chunks, chunk, bits, offset, red, [&](int64_t i) -> int4& { return rows[i]; },
      [&](int page) { return make_int3(refs[page], writers[page], keeper[page]); },
      [&](int from, int to) {
        atomicSub(refs + from, 1);
        refs[to] = 1;
      });
  __syncthreads();
  const int need = a.w.totals[0];
  for (int g = tid; g < need; g += kPlanThreads) {
    const int page = fork_take(a, chunks, chunk, bits, offset, rows, g);
    if (page >= 0) refs[page] = 1;
  }
  __syncthreads();
  for (int p = tid; p < a.c.pages; p += kPlanThreads) a.refs_out[p] = refs[p];
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

// Where the table's entry i points after the move (map and dst as above), -1 past the row's tokens.
template <typename Map>
__device__ __forceinline__ int compact_entry(const CompactArgs& a, int64_t i, Map to) {
  const int64_t s = i / a.width;
  const int page = a.table[i];
  if ((i - s * a.width) << a.c.page_shift >= a.lengths[s] || (uint32_t)page >= (uint64_t)a.c.pages) return -1;
  return to(page);
}

// Small pools and tables: all but the copies in one workgroup, the counts in LDS (8 rows of 200 tokens: a call takes 18.3 us
// against 21.4 with the launches of the large form).
__global__ __launch_bounds__(kPlanThreads) void compact_small_kernel(CompactArgs a) {
  __shared__ int red[kPlanThreads / 64];
  __shared__ int32_t refs[kSmallPages], map[kSmallPages], src[kSmallPages / 2], dst[kSmallPages / 2];
  constexpr int kMine = kSmallPages / kPlanThreads;  // consecutive pages of a thread
  const int p0 = threadIdx.x * kMine, pages = (int)a.c.pages;
  for (int p = threadIdx.x; p < kSmallPages; p += kPlanThreads) refs[p] = p < pages ? a.refs[p] : 0;
  __syncthreads();
  int mine = 0, U;
#pragma unroll
  for (int j = 0; j < kMine; ++j) mine += refs[p0 + j] > 0;
  int up = block_prefix(mine, red, &U);
  int moved = U;  // less the used pages below U
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    const int p = p0 + j;
    if (p >= pages) break;
    if (refs[p] > 0) {
      if (p >= U) src[U - 1 - up] = p;
      map[p] = p < U ? p : ~(U - 1 - up);
    } else if (p < U) {
      dst[p - up] = p;
      map[p] = p - up;
    }
    up += refs[p] > 0;
  }
  int below = 0;
#pragma unroll
  for (int j = 0; j < kMine; ++j) below += p0 + j < U && refs[p0 + j] > 0;
  int kept;
  block_prefix(below, red, &kept);
  moved -= kept;
  for (int64_t i = threadIdx.x; i < a.S * a.width; i += kPlanThreads)
    a.table_out[i] = compact_entry(a, i, [&](int page) { return refs[page] <= 0 ? -1 : map[page] >= 0 ? map[page] : dst[~map[page]]; });
  for (int p = threadIdx.x; p < pages; p += kPlanThreads) a.refs_out[p] = p >= U ? 0 : refs[p] > 0 ? refs[p] : refs[src[map[p]]];
  for (int r = threadIdx.x; r < moved; r += kPlanThreads) {
    a.src[r] = src[r];
    a.dst[r] = dst[r];
  }
  if (threadIdx.x == 0) {
    a.totals[0] = moved;
    *a.used = U;
  }
}

__global__ __launch_bounds__(kThreads) void compact_move_kernel(CompactArgs a) {
  const int count = a.totals[0], U = a.totals[1];
  const int64_t stride = (int64_t)gridDim.x * kThreads, first = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  for (int64_t i = first; i < a.S * a.width; i += stride) {
    a.table_out[i] = compact_entry(a, i, [&](int page) {
      if (a.refs[page] <= 0) return -1;
      const int to = a.map[page];
      return to >= 0 ? to : a.dst[~to];
    });
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
  const dim3 grid((unsigned)slots, (unsigned)c.heads);
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
  return sizeof(int32_t) * (size_t)(kTotals + n * 32 + (n + 64) / 64 * 64 + 2 * n * kChunk + 7 * rows);
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
  if (c.pages <= kSmallPages && S <= kSmallRows && S_out <= kSmallRows && (S + S_out) * width <= kSmallEntries) {
    fork_small_kernel<<<1, kPlanThreads, 0, st>>>(a, chunks);
    if (grow && S_out > 0)
      copy_counted_kernel<<<(unsigned)copy_grid(c, S_out), kThreads, 0, st>>>(c, a.w.src, a.w.dst, a.w.totals + 1);
    return hipGetLastError();
  }
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
  if (c.pages <= kSmallPages && S * width <= kSmallEntries) {
    compact_small_kernel<<<1, kPlanThreads, 0, st>>>(a);
    copy_counted_kernel<<<(unsigned)copy_grid(c, c.pages / 2), kThreads, 0, st>>>(c, a.src, a.dst, a.totals);
    return hipGetLastError();
  }
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
