// Attention over the paged 8-bit cache: how a call is cut, and its launches.  The kernels are in attend.h.
#include "attend.h"

namespace mdss {

namespace {

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
  AttendArgs a = attend_args(c, layer, q, heads_q, q_st, q_sh, rows, scale, out, lse, workspace, p.splits == 1 ? 0 : p.splits);
  a.per_seq = p.per_seq;
  a.splits = p.splits;
  a.split_tiles = p.split_tiles;
  const bool bf = dtype == MDSS_BF16;
  switch (c.d) {
    case 64: return bf ? attend_launch<64, true>(a, p, st) : attend_launch<64, false>(a, p, st);
    case 96: return bf ? attend_launch<96, true>(a, p, st) : attend_launch<96, false>(a, p, st);
    case 128: return bf ? attend_launch<128, true>(a, p, st) : attend_launch<128, false>(a, p, st);
    default: return bf ? attend_launch<256, true>(a, p, st) : attend_launch<256, false>(a, p, st);
  }
}

}  // namespace mdss
