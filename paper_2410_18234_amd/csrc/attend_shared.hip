// Attention for sequences that share a prefix: which tokens they share, how a call is cut, and its launches.
//
// A group's new tokens are the rows of one product over the tokens it shares, so those are read once for all of its
// sequences; each sequence's own tokens follow, with the kernels of attend.h for both.  Each part of a row is its
// maximum, sum and weighted values in the same frame, which the last launch joins.
#include "attend.h"

namespace mdss {

namespace {

// ---------------------------------------------------------------- what rows share
struct SharedArgs {
  const int32_t *starts, *table, *lengths, *groups;
  int32_t *tokens, *rows;
  int64_t T, width, pages;
  int S, G, page_shift, least;
};

// A workgroup a group.  It finds who takes part (the first one, the fewest tokens before the new ones), then compares the others' pages
// with the first one's, a wave a row at a time, up to the first difference that any wave has met.  Bound by the chain groups -
// lengths - table on few rows.
template <int NT>
__global__ __launch_bounds__(NT) void shared_kernel(const SharedArgs a) {
  __shared__ int first_row, fewest, count, common;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int g = blockIdx.x;
  if (g == 0) {  // rows of no group
    const int end = a.G > 0 ? min(max(a.groups[0], 0), a.S) : a.S;
    for (int s = threadIdx.x; s < end; s += NT) a.tokens[s] = 0;
  }
  if (a.G == 0) return;
  if (g == a.G - 1)
    for (int s = min(max(a.groups[a.G], 0), a.S) + threadIdx.x; s < a.S; s += NT) a.tokens[s] = 0;
  const int begin = a.groups[g], end = a.groups[g + 1];
  const bool fine = begin >= 0 && begin <= end && end <= a.S;
  if (threadIdx.x == 0) {
    first_row = fewest = INT32_MAX;
    count = 0;
  }
  __syncthreads();
  const int64_t most = a.width << a.page_shift, each = a.S > 0 ? a.T / a.S : 0;
  // tokens before the new ones; -1 for who takes no part
  const auto before = [&](int s) {
    const int64_t n = a.starts ? max((int64_t)a.starts[s + 1] - a.starts[s], (int64_t)0) : each;
    const int64_t b = min((int64_t)a.lengths[s], most) - n;
    return b >= max(a.least, 1) ? (int)min(b, (int64_t)INT32_MAX) : -1;
  };
  if (fine) {
    int r = INT32_MAX, few = INT32_MAX, some = 0;
    for (int s = begin + (int)threadIdx.x; s < end; s += NT) {
      const int b = before(s);
      if (b < 0) continue;
      r = min(r, s);
      few = min(few, b);
      ++some;
    }
    if (some > 0) {
      atomicMin(&first_row, r);
      atomicMin(&fewest, few);
      atomicAdd(&count, some);
    }
  }
  __syncthreads();
  const int lead = first_row;
  if (threadIdx.x == 0) common = count > 1 ? (fewest + (1 << a.page_shift) - 1) >> a.page_shift : 0;
  __syncthreads();
  if (count > 1) {
    const int32_t* mine = a.table + (int64_t)lead * a.width;
    for (int s = begin + wave; s < end; s += NT / 64) {
      if (before(s) < 0) continue;
      const int32_t* row = a.table + (int64_t)s * a.width;
      // (the shared bound only sinks: a wave that reads an old one compares more than it has to)
      for (int j0 = 0; j0 < *(volatile int*)&common; j0 += 256) {
        bool differ[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int64_t j = min((int64_t)(j0 + 64 * i + lane), a.width - 1);
          differ[i] = row[j] != mine[j] || (uint32_t)mine[j] >= (uint64_t)a.pages;
        }
        int at = -1;
#pragma unroll
        for (int i = 3; i >= 0; --i) {
          const uint64_t hit = __ballot(differ[i]);
          if (hit) at = j0 + 64 * i + __ffsll((unsigned long long)hit) - 1;
        }
        if (at >= 0) {
          if (lane == 0) atomicMin(&common, at);
          break;
        }
      }
    }
  }
  __syncthreads();
  const int unit = max(64, 1 << a.page_shift);
  int shared = 0;
  if (count > 1) {
    shared = (int)(min((int64_t)common << a.page_shift, (int64_t)fewest) / unit * unit);
    if (shared < a.least) shared = 0;
  }
  if (fine)
    for (int s = begin + (int)threadIdx.x; s < end; s += NT) a.tokens[s] = before(s) >= 0 ? shared : 0;
  if (threadIdx.x < 4) {
    const int64_t from = !fine ? 0 : a.starts ? a.starts[begin] : begin * each;
    const int64_t to = !fine ? 0 : a.starts ? a.starts[end] : end * each;
    const int word = threadIdx.x;
    a.rows[4 * (int64_t)g + word] = word == 0 ? (int)from : word == 1 ? (int)(to - from) : word == 2 ? (lead < INT32_MAX ? lead : -1) : shared;
  }
}

// ---------------------------------------------------------------- attention
struct SharedPlan {
  int mt, pre_mt;          // row tiles of a wave, for the sequences' own tokens and for the prefixes
  bool wide, pre_wide;     // whether the waves take different rows
  int per_seq;
  int64_t slots, pre_slots;
  int splits, split_tiles, pre_splits, pre_split_tiles;
  bool one_launch() const { return wide == pre_wide && mt == pre_mt; }
};

int64_t at_most(int64_t hint, int64_t most) { return hint > 0 && hint < most ? hint : most; }

// `tiles` of 64 tokens in at most `splits` pieces
void cut(int64_t tiles, int64_t splits, int* out_splits, int* out_tiles) {
  if (splits > 64) splits = 64;
  if (splits < 1) splits = 1;
  int64_t each = (tiles + splits - 1) / splits;
  if (each < 1) each = 1;
  *out_tiles = (int)each;
  *out_splits = (int)((tiles + each - 1) / each);
  if (*out_splits < 1) *out_splits = 1;
}

SharedPlan shared_plan(const CacheView& c, int64_t T, int64_t S, int64_t G, int64_t width, int group, bool uniform, int64_t max_new,
                       int64_t max_group, int64_t max_shared, int64_t max_own) {
  SharedPlan p;
  const int most = c.d > 128 ? 2 : 4;
  const int64_t n = uniform ? T / S : at_most(max_new, T), all = at_most(max_group, T);
  const auto kind = [&](int64_t rows, int& mt, bool& wide) {
    wide = rows > 16 * most;
    mt = wide ? (c.d > 128 ? 1 : 2) : rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  };
  kind(n * group, p.mt, p.wide);
  kind(all * group, p.pre_mt, p.pre_wide);
  if (p.wide == p.pre_wide) p.mt = p.pre_mt = p.mt > p.pre_mt ? p.mt : p.pre_mt;
  const int tile = (p.wide ? 64 : 16) * p.mt, pre_tile = (p.pre_wide ? 64 : 16) * p.pre_mt;
  p.per_seq = uniform ? (int)((n * group + tile - 1) / tile) : 0;
  p.slots = uniform ? S * p.per_seq : T * group / tile + S;
  p.pre_slots = G > 0 ? T * group / pre_tile + G : 0;
  const int64_t tokens = width << c.page_shift;
  const int64_t tiles = (at_most(max_own, tokens) + 63) >> 6, pre_tiles = (at_most(max_shared, tokens) + 63) >> 6;
  const auto full = [&](int64_t sets, int64_t rows) { return (sets > (T * group + rows - 1) / rows ? sets : (T * group + rows - 1) / rows) * c.heads; };
  const int64_t own = full(S, tile), pre = full(G > 0 ? G : 1, pre_tile);
  // A prefix: as many workgroups as the CUs hold, of at least four tiles (one a wave) or, where the waves take different rows, eight.
  int64_t pre_splits = 512 / pre;
  const int64_t least = p.pre_wide ? 8 : 4;
  if (pre_splits > pre_tiles / least) pre_splits = pre_tiles / least;
  cut(pre_tiles, pre_splits, &p.pre_splits, &p.pre_split_tiles);
  int64_t splits = 512 / own;
  if (splits > tiles / 8) splits = tiles / 8;
  cut(tiles, splits, &p.splits, &p.split_tiles);
  return p;
}

template <typename Kernel>
hipError_t shared_blocks(Kernel kernel, AttendArgs a, int64_t from, int64_t to, hipStream_t st) {
  constexpr int64_t most = (1 << 24) - 1;  // (a dimension of a launch holds less than 2^32 threads)
  for (; from < to; from += most) {
    a.block0 = from;
    kernel<<<(unsigned)(to - from < most ? to - from : most), 256, 0, st>>>(a);
  }
  return hipGetLastError();
}

template <int D, bool BF>
hipError_t shared_part(const AttendArgs& a, bool wide, int mt, int64_t from, int64_t to, hipStream_t st) {
  if (wide) return shared_blocks(attend_wide_kernel<D, BF, D == 256 ? 1 : 2, true>, a, from, to, st);
  if (mt == 1) return shared_blocks(attend_kernel<D, BF, 1, true>, a, from, to, st);
  if constexpr (D <= 128) {
    if (mt == 4) return shared_blocks(attend_kernel<D, BF, 4, true>, a, from, to, st);
  }
  return shared_blocks(attend_kernel<D, BF, 2, true>, a, from, to, st);
}

template <int D, bool BF>
hipError_t shared_launch(const AttendArgs& a, const SharedPlan& p, hipStream_t st) {
  const int64_t blocks = a.pre_blocks + p.slots * a.heads * p.splits;
  hipError_t e;
  if (p.one_launch()) {
    e = shared_part<D, BF>(a, p.wide, p.mt, 0, blocks, st);
  } else {
    e = shared_part<D, BF>(a, p.pre_wide, p.pre_mt, 0, a.pre_blocks, st);
    if (e == hipSuccess) e = shared_part<D, BF>(a, p.wide, p.mt, a.pre_blocks, blocks, st);
  }
  const int64_t total = a.T * a.heads * a.group, most = 1LL << 25;
  for (int64_t row = 0; e == hipSuccess && row < total; row += most) {
    const int64_t rows = total - row < most ? total - row : most;
    attend_join_kernel<D, BF, true><<<(unsigned)((rows + 3) / 4), 256, 0, st>>>(a, (p.wide ? 64 : 16) * p.mt, row + rows, row);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

hipError_t launch_cache_shared(const CacheView& c, const CacheRows& rows, const int32_t* groups, int64_t G, int32_t least,
                               int32_t* tokens, int32_t* group_rows, hipStream_t st) {
  const SharedArgs a = {rows.starts, rows.table, rows.lengths, groups,  tokens, group_rows, rows.T,
                        rows.width,  c.pages,    rows.S,       (int)G, c.page_shift, least};
  const unsigned grid = G > 0 ? (unsigned)G : 1u;
  if (rows.S > 16 * (G > 0 ? G : 1))
    shared_kernel<1024><<<grid, 1024, 0, st>>>(a);
  else
    shared_kernel<256><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

size_t workspace_bytes_attention_shared(const CacheView& c, int64_t T, int64_t S, int64_t G, int64_t width, int64_t heads_q,
                                        bool uniform, int64_t max_new, int64_t max_group, int64_t max_shared, int64_t max_own) {
  const SharedPlan p = shared_plan(c, T, S, G, width, (int)(heads_q / c.heads), uniform, max_new, max_group, max_shared, max_own);
  return (size_t)T * heads_q * (p.pre_splits + p.splits) * (c.d + 2) * sizeof(float);
}

hipError_t launch_cache_attention_shared(const CacheView& c, int layer, const void* q, int dtype, int64_t heads_q, int64_t q_st,
                                         int64_t q_sh, const CacheRows& rows, const int32_t* tokens, const int32_t* groups, int64_t G,
                                         float scale, int64_t max_new, int64_t max_group, int64_t max_shared, int64_t max_own,
                                         void* out, float* lse, void* workspace, hipStream_t st) {
  const SharedPlan p = shared_plan(c, rows.T, rows.S, G, rows.width, (int)(heads_q / c.heads), rows.starts == nullptr, max_new,
                                   max_group, max_shared, max_own);
  AttendArgs a = attend_args(c, layer, q, heads_q, q_st, q_sh, rows, scale, out, lse, workspace, p.pre_splits + p.splits);
  a.per_seq = p.per_seq;
  a.splits = p.splits;
  a.split_tiles = p.split_tiles;
  a.tokens = tokens;
  a.groups = groups;
  a.G = (int)G;
  a.slots = (int)p.slots;
  a.pre_slots = (int)p.pre_slots;
  a.pre_splits = p.pre_splits;
  a.pre_split_tiles = p.pre_split_tiles;
  a.pre_blocks = p.pre_slots * c.heads * p.pre_splits;
  const bool bf = dtype == MDSS_BF16;
  switch (c.d) {
    case 64: return bf ? shared_launch<64, true>(a, p, st) : shared_launch<64, false>(a, p, st);
    case 96: return bf ? shared_launch<96, true>(a, p, st) : shared_launch<96, false>(a, p, st);
    case 128: return bf ? shared_launch<128, true>(a, p, st) : shared_launch<128, false>(a, p, st);
    default: return bf ? shared_launch<256, true>(a, p, st) : shared_launch<256, false>(a, p, st);
  }
}

}  // namespace mdss
