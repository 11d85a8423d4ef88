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
  int each;  // groups of a workgroup
};

// A workgroup a group (beyond 4096 of them, several in turn).  It finds who takes part (the first one, the fewest tokens before the new ones),
// then compares the others' pages with the first one's, a wave a row at a time, up to the first difference that any wave has met.  Bound by
// the chain groups - lengths - table (4 rows: 4.6 us; 128 groups of 8 rows: 7.6 us).
//
// Bounds are the caller's, and may not ascend.  What ascends is `reach`, the largest end of the groups before (a group: bounds that ascend
// within the rows); one that begins before it would take rows of an earlier one, and is none.  Group g writes the tokens of the rows
// reach(g) .. reach(g + 1) - 1, so each row has one writer, and its first token is that of a row from reach(g) on, so these ascend
// whatever the bounds: attention's search for the group of a row tile counts on it.
template <int NT>
__global__ __launch_bounds__(NT) void shared_kernel(const SharedArgs a) {
  __shared__ int first_row, fewest, count, common, reach_before;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int g0 = blockIdx.x * a.each, g1 = min(a.G, g0 + a.each);
  const auto is_group = [&](int begin, int end) { return begin >= 0 && begin <= end && end <= a.S; };
  if (threadIdx.x == 0) {
    first_row = fewest = INT32_MAX;
    count = reach_before = 0;
  }
  __syncthreads();
  // (a bound of the groups before this one for each thread: on its way until it is asked for at the end)
  int bound0 = 0, bound1 = 0;
  if (a.G > 0) {
    bound0 = a.groups[min((int)threadIdx.x, g0)];
    bound1 = a.groups[min((int)threadIdx.x, g0) + 1];
  }
  const int64_t most = a.width << a.page_shift, each = a.S > 0 ? a.T / a.S : 0;
  // tokens before the new ones; -1 for who takes no part
  const auto before = [&](int s) {
    const int64_t n = a.starts ? max((int64_t)a.starts[s + 1] - a.starts[s], (int64_t)0) : each;
    const int64_t b = min((int64_t)a.lengths[s], most) - n;
    return b >= max(a.least, 1) ? (int)min(b, (int64_t)INT32_MAX) : -1;
  };
  int reach = 0;
  for (int g = g0; g < g1; ++g) {
    const int begin = a.groups[g], end = a.groups[g + 1];
    if (g > g0) {
      __syncthreads();  // (the last group's words are read)
      if (threadIdx.x == 0) {
        first_row = fewest = INT32_MAX;
        count = 0;
      }
      __syncthreads();
    }
    const bool ordered = is_group(begin, end);
    if (ordered) {
      int r = INT32_MAX, few = INT32_MAX, n = 0;
      for (int s = begin + (int)threadIdx.x; s < end; s += NT) {
        const int b = before(s);
        if (b < 0) continue;
        r = min(r, s);
        few = min(few, b);
        ++n;
      }
      if (n > 0) {
        atomicMin(&first_row, r);
        atomicMin(&fewest, few);
        atomicAdd(&count, n);
      }
    }
    __syncthreads();
    const int lead = first_row;
    const bool some = count > 1;
    if (threadIdx.x == 0) common = some ? (fewest + (1 << a.page_shift) - 1) >> a.page_shift : 0;
    __syncthreads();
    if (some) {
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
    if (g == g0 && g0 > 0) {
      int most_before = (int)threadIdx.x < g0 && is_group(bound0, bound1) ? bound1 : 0;
#pragma unroll 4
      for (int i = threadIdx.x + NT; i < g0; i += NT) {
        bound0 = a.groups[i];
        bound1 = a.groups[i + 1];
        most_before = is_group(bound0, bound1) ? max(most_before, bound1) : most_before;
      }
      most_before = (int)wave_max((float)most_before);  // (rows are fewer than 2^24)
      if (lane == 0) atomicMax(&reach_before, most_before);
    }
    __syncthreads();
    if (g == g0) reach = reach_before;
    const bool fine = ordered && begin >= reach;
    const int unit = max(64, 1 << a.page_shift);
    int shared = 0;
    if (fine && some) {
      shared = (int)(min((int64_t)common << a.page_shift, (int64_t)fewest) / unit * unit);
      if (shared < a.least) shared = 0;
    }
    const int next = ordered ? max(reach, end) : reach;
    for (int s = reach + (int)threadIdx.x; s < next; s += NT) a.tokens[s] = fine && s >= begin && before(s) >= 0 ? shared : 0;
    if (threadIdx.x < 4) {
      const int at = fine ? begin : reach, upto = fine ? end : reach;
      const int64_t from = a.starts ? a.starts[at] : at * each;
      const int64_t to = a.starts ? a.starts[upto] : upto * each;
      const int word = threadIdx.x;
      a.rows[4 * (int64_t)g + word] = word == 0 ? (int)from : word == 1 ? (int)(to - from) : word == 2 ? (fine && lead < INT32_MAX ? lead : -1) : shared;
    }
    reach = next;
  }
  if (g1 == a.G)  // rows past the last group
    for (int s = reach + (int)threadIdx.x; s < a.S; s += NT) a.tokens[s] = 0;
}

// ---------------------------------------------------------------- attention
// Few rows: four waves that take the same rows against tiles in turn (a prefix; own tokens of few sequences), or a wave for each
// (sequence, head), which has no partners to wait for and to join: 2048 sequences of one token of their own past the prefix.  Bound by memory,
// at two thirds of the copy's rate (heads of 128, 8 of them, four query heads each: 16 groups of 8 rows, up to 6000 shared tokens, 46 to 48 us,
// vector instructions 38 % of the cycles, matrix instructions 12 %; 256 sequences' own tokens behind 8192 shared ones
// 70 us, 4.1 TB/s).
template <int D, bool BF, int MT, int NW>
__device__ __forceinline__ void shared_rows(const AttendArgs& a, const Place& p, float* joined, float* joined_ml,
                                            typename Elem<BF>::vec* queries) {
  if (MT > 1 && p.rows <= 16)
    attend_rows<D, BF, 1, NW>(a, p, joined, joined_ml, queries);
  else
    attend_rows<D, BF, MT, NW>(a, p, joined, joined_ml, queries);
}
template <int D, bool BF, int MT>
__global__ __launch_bounds__(256, D > 128 ? 1 : MT == 2 || D > 96 ? 2 : D == 96 ? 3 : 4) void attend_shared_kernel(const AttendArgs a) {
  using vec = typename Elem<BF>::vec;
  constexpr int kQueries = MT * D / 32 * 64, kJoined = 4 * joined_part(D) + 4 * 16 * 2;
  constexpr int kTogether = kJoined * 4 + kQueries * 16, kApart = 4 * kQueries * 16;
  __shared__ __align__(16) char lds[kTogether > kApart ? kTogether : kApart];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t block = a.block0 + blockIdx.x;
  Place p;
  if (block >= a.pre_blocks && a.own_waves == 1) {
    if (attend_place<true>(a, 16 * MT, lane, p, a.pre_blocks + (block - a.pre_blocks) * 4 + wave))
      shared_rows<D, BF, MT, 1>(a, p, nullptr, nullptr, reinterpret_cast<vec*>(lds) + wave * kQueries);
  } else if (attend_place<true>(a, 16 * MT, lane, p, block)) {
    float* joined = reinterpret_cast<float*>(lds);
    shared_rows<D, BF, MT, 4>(a, p, joined, joined + 4 * joined_part(D), reinterpret_cast<vec*>(lds + kJoined * 4));
  }
}

// A prefix under many rows: four waves take different rows (MT tiles of 16 each) against the same tiles of 64 tokens, widened into LDS once for
// all of them.  The rows see all of the prefix, in whole tiles: nothing is masked but missing pages.  A tile is two steps: softmax and
// staging, then the products of its values and of the next one's keys, with their operands read ahead; the two waves of a SIMD,
// of two workgroups, fill each other's steps.  Bound by vector instructions between the matrix instructions: 2048 rows a cache head (256 sequences, eight
// query heads each) over 8192 tokens, 8 heads of 128: 92 to 100 us, 690 to 750 TFLOP/s (the kernel of whole sequences: 105); vector
// instructions 59 % of the cycles, matrix instructions 35 %, LDS 26 %.
template <int D, bool BF, int MT>
__global__ __launch_bounds__(256, 2) void attend_prefix_kernel(const AttendArgs a) {
  using E = Elem<BF>;
  using vec = typename E::vec;
  constexpr int kSteps = D / 32, kWhole = D / 64, kTiles = D / 16;
  constexpr bool kHalf = D % 64 != 0;
  constexpr int kValue = (kTiles + 3) / 4;  // a wave's 16-byte loads: keys of its quarter tt = wave, and these of the values
  constexpr int kTile = 4 * kSteps * 64;  // keys (tt, step); values (dt, half)
  __shared__ __align__(16) vec key_tile[kTile];
  __shared__ __align__(16) f16x8 value_tile[kTile];  // (2 kTiles = 4 kSteps)
  __shared__ int again_any[4];

  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Place p;
  if (!attend_place<true>(a, 64 * MT, lane, p, a.block0 + blockIdx.x)) return;
  const int row0 = p.tile * 64 * MT + wave * 16 * MT, h = p.h;
  const int t_begin = p.begin(), tiles = p.end(p.len >> 6) - t_begin;
  if (tiles <= 0) return;  // (another split than the first, which has them all)

  vec qf[MT][kSteps];
  int lim[MT];
  load_queries<D, BF, MT>(a, p, row0, m, g, qf, lim);
  const bool idle = row0 >= p.rows;
  f32x4 acc[kTiles][MT];
  float M[MT], l[MT];
  u16x2 least = {0x3c00, 0x3c00};
  float ve_least = INFINITY, ve_most = -INFINITY;

  const PageWalk walk(a, p);
  const int64_t lane_v = m * 16;
  const auto key_page = [&](int t) { return walk.page(4 * (t_begin + t) + (m >> 2)); };
  const auto value_page = [&](int t) { return walk.page(4 * (t_begin + t) + g); };
  u32x4 key_stage[kWhole], value_stage[kValue];
  u32x2 key_half;
  // (tiles past the last one: the last page again)
  const auto load_keys = [&](int page, int t) __attribute__((always_inline)) {
    bool ok;
    const uint8_t* at = walk.unit(a.k, walk.valid(page, ok), 4 * (t_begin + t) + (m >> 2), 16 * D) + (m & 3) * 16 + wave * 64;
#pragma unroll
    for (int i = 0; i < kWhole; ++i) key_stage[i] = *reinterpret_cast<const u32x4*>(at + i * 1024 + g * 256);
    if (kHalf) key_half = *reinterpret_cast<const u32x2*>(at + (4 * kWhole + (g >> 1)) * 256 + (g & 1) * 8);
  };
  const auto load_values = [&](int page, int t) __attribute__((always_inline)) {
    const uint8_t* at = walk.unit(a.v, page, 4 * (t_begin + t) + g, 16 * D) + lane_v;
#pragma unroll
    for (int j = 0; j < kValue; ++j)
      if (kTiles % 4 == 0 || wave * kValue + j < kTiles) value_stage[j] = *reinterpret_cast<const u32x4*>(at + (wave * kValue + j) * 256);
  };
  const auto put_keys = [&]() __attribute__((always_inline)) {
    vec* to = key_tile + wave * kSteps * 64 + lane;
#pragma unroll
    for (int i = 0; i < kWhole; ++i) {
      to[2 * i * 64] = E::widen(key_stage[i][0], key_stage[i][1]);
      to[(2 * i + 1) * 64] = E::widen(key_stage[i][2], key_stage[i][3]);
    }
    if (kHalf) to[(kSteps - 1) * 64] = E::widen(key_half[0], key_half[1]);
  };
  const auto put_values = [&](bool ok) __attribute__((always_inline)) {
    if (__ballot(ok) != ~0ull) {  // (any bytes in place of a page that is not there)
#pragma unroll
      for (int j = 0; j < kValue; ++j) value_stage[j] = low_bytes(value_stage[j], ok ? 16 : 0);
    }
    f16x8* to = value_tile + wave * kValue * 128 + lane;
#pragma unroll
    for (int j = 0; j < kValue; ++j)
      if (kTiles % 4 == 0 || wave * kValue + j < kTiles) {
        to[2 * j * 64] = Elem<false>::widen(value_stage[j][0], value_stage[j][1]);
        to[(2 * j + 1) * 64] = Elem<false>::widen(value_stage[j][2], value_stage[j][3]);
      }
  };

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
    bool far = false;
    f32x4 sc[4][MT];
    f16x8 pf[MT][2];
    f16x8 left[PRECISE ? MT : 1][2];
    float back[PRECISE ? MT : 1];
    int ke, ve, pv;
    bool ok;
    const auto load_exponents = [&](int page) __attribute__((always_inline)) {
      pv = walk.valid(page, ok);
      ke = a.k_exp[(int64_t)pv * a.heads + h];
      ve = a.v_exp[(int64_t)pv * a.heads + h];
    };
    // Products by chunks of kSteps operands, the next chunk's on their way from LDS meanwhile (the compiler would wait for each pair).
    // Four sums are taken in turn: chunks 0 .. 3 are the values' (two d tiles, both halves), 4 .. 7 the keys' (two token tiles, the steps).
    u32x4 operand[2][kSteps];
    const auto fetch = [&](int c) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const int f = (c & 3) * kSteps + i;
        const int at = c < 4 ? 2 * (f / 4 * 2 + (f & 1)) + f % 4 / 2 : (f / (2 * kSteps) * 2 + (f & 1)) * kSteps + f % (2 * kSteps) / 2;
        operand[c & 1][i] = c < 4 ? __builtin_bit_cast(u32x4, value_tile[at * 64 + lane]) : __builtin_bit_cast(u32x4, key_tile[at * 64 + lane]);
      }
    };
    const auto multiply = [&](int c) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const int f = (c & 3) * kSteps + i;
#pragma unroll
        for (int r = 0; r < MT; ++r) {
          if (c < 4) {
            f32x4& sum = acc[f / 4 * 2 + (f & 1)][r];
            sum = Elem<false>::mfma(__builtin_bit_cast(f16x8, operand[c & 1][i]), pf[r][f % 4 / 2], sum);
          } else {
            f32x4& sum = sc[f / (2 * kSteps) * 2 + (f & 1)][r];
            const int st = f % (2 * kSteps) / 2;
            sum = E::mfma(__builtin_bit_cast(vec, operand[c & 1][i]), qf[r][st], st == 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : sum);
          }
        }
      }
    };
    const auto multiply_chunks = [&](int from, int to) __attribute__((always_inline)) {
      fetch(from);
#pragma unroll
      for (int c = from; c < to; ++c) {
        if (c + 1 < to) fetch(c + 1);
        __builtin_amdgcn_sched_barrier(0);
        multiply(c);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    load_keys(key_page(0), 0);
    put_keys();
    load_exponents(value_page(0));
    load_keys(key_page(1), 1);
    load_values(pv, 0);
    int next_key = key_page(2), next_value = value_page(1);
    __syncthreads();
    if (mine) multiply_chunks(4, 8);
    __syncthreads();
    for (int t = 0; t < tiles; ++t) {
      const bool ok_now = ok;
      float c_g = a.scale_log2 * pow2i(ok_now ? ke : 0), ve_g = ok_now ? (float)ve : 0.0f, inv_v = pow2i(ok_now ? -ve : 0);
      asm volatile("" : "+v"(c_g), "+v"(ve_g), "+v"(inv_v));  // (before the next tile's exponents are loaded, into the same registers)
      if (mine) {
        const bool masked = __ballot(ok_now) != ~0ull;
        int upto[MT];
#pragma unroll
        for (int r = 0; r < MT; ++r) upto[r] = ok_now ? 16 : 0;
        float alpha[MT];
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
        if constexpr (PRECISE) {
#pragma unroll
          for (int r = 0; r < MT; ++r) left_of_low<MT>(sc, r, c_g, ve_g, upto[r], M[r], far, left[r], back[r]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      put_keys();
      put_values(ok_now);
      load_exponents(next_value);
      load_keys(next_key, t + 2);
      load_values(pv, t + 1);
      next_key = key_page(t + 3);
      next_value = value_page(t + 2);
      __syncthreads();
      if (mine) {
        __builtin_amdgcn_s_setprio(1);
if constexpr (PRECISE) {
          multiply_chunks(0, 4);
#pragma unroll
          for (int r = 0; r < MT; ++r)
            add_left<MT, kTiles>(left[r], back[r], r, acc, [&](int dt, int hs) {
              f16x8 v = value_tile[(2 * dt + hs) * 64 + lane];
              asm volatile("" : "+v"(v));  // (read again, not held from above)
              return v;
            });
          multiply_chunks(4, 8);
        } else {
          multiply_chunks(0, 8);
        }
        __builtin_amdgcn_s_setprio(0);
      }
      __syncthreads();
    }
  };
  pass(Flag<false>{}, !idle);
  const bool again = !idle && lacks<MT, kTiles>(acc, M, lim, least, ve_least, ve_most, 64.0f * tiles);
  if (lane == 0) again_any[wave] = again;
  __syncthreads();
  if (again_any[0] | again_any[1] | again_any[2] | again_any[3]) pass(Flag<true>{}, again);
  if (idle) return;
#pragma unroll
  for (int r = 0; r < MT; ++r) l[r] = row_sum4(l[r]);
  write_rows<D, BF, MT>(a, p, row0, m, g, acc, M, l);
}

// Joins a row's parts: those of the tokens it shares, then those of its sequence's own.  A wave has one token and as many of its heads as
// fit, eight elements a lane, so what the rows of a token have in common is found once.  Bound by the parts' bytes (256 tokens of 64 heads,
// behind 8192 shared ones: 10.9 us) and by the launch (128 tokens: 5.5 us).
template <int D, bool BF>
__global__ __launch_bounds__(256) void shared_join_kernel(const AttendArgs a, int rows_tile, int chunks, int64_t first_token) {
  using vec = typename Elem<BF>::vec;
  using one = typename Elem<BF>::one;
  constexpr int kLanes = D <= 64 ? 8 : D <= 128 ? 16 : 32;  // of a row (96: the last four idle)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t item = blockIdx.x * 4 + wave, token = item / (uint32_t)chunks;
  const int64_t t = first_token + token;
  if (t >= a.T) return;
  const int heads_q = a.heads * a.group;
  const int hq = (int)(item - token * chunks) * (64 / kLanes) + lane / kLanes, at = lane % kLanes * 8;
  int s, n;
  int64_t start;
  if (a.starts) {
    s = slot_sequence(a.starts, a.S, t, 1, 1, 0, lane);
    start = a.starts[s];
    n = (int)(a.starts[s + 1] - start);
  } else {
    n = (int)(a.T / a.S);
    s = (int)((uint32_t)t / (uint32_t)n);
    start = (int64_t)s * n;
  }
  if (start < 0 || t < start || t >= start + n || start + n > a.T) return;  // a token of no sequence
  if (hq >= heads_q || at >= D) return;
  const int length = a.lengths[s], before = length - n;
  const int first = shared_tokens(a, s, before) >> 6;
  const int prefix = min(a.pre_splits, (first + a.pre_split_tiles - 1) / a.pre_split_tiles);
  int parts = prefix + 1;
  if (a.splits > 1) {  // the splits that had tokens for the row's tile
    const int rows = n * a.group, row = (int)(t - start) * a.group + hq % a.group, row0 = row / rows_tile * rows_tile;
    const int len = max(0, min(length, (int)min(a.width << a.page_shift, (int64_t)INT32_MAX)));
    const int lim_hi = min(len, before + min(rows - 1, row0 + rows_tile - 1) / a.group + 1);
    const int tiles = (lim_hi > 0 ? (lim_hi + 63) >> 6 : 0) - first;
    parts = prefix + max(1, min(a.splits, (tiles + a.split_tiles - 1) / a.split_tiles));
  }
  const int64_t id = t * heads_q + hq, base = id * (a.pre_splits + a.splits);
  const auto part_at = [&](int i) { return base + (i < prefix ? i : i - prefix + a.pre_splits); };
  float top = -INFINITY, l = 0.0f;
#pragma unroll 4
  for (int i = 0; i < parts; ++i) top = fmaxf(top, a.part_ml[2 * part_at(i)]);
  f32x4 lo = {0.0f, 0.0f, 0.0f, 0.0f}, hi = lo;
#pragma unroll 4
  for (int i = 0; i < parts; ++i) {
    const int64_t k = part_at(i);
    const float w = frame_weight(a.part_ml[2 * k], top);
    l = fmaf(w, a.part_ml[2 * k + 1], l);
    const f32x4* x = reinterpret_cast<const f32x4*>(a.part + k * D + at);
    lo = __builtin_elementwise_fma(f32x4{w, w, w, w}, x[0], lo);
    hi = __builtin_elementwise_fma(f32x4{w, w, w, w}, x[1], hi);
  }
  vec o;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    o[e] = (one)(l == 0.0f ? 0.0f : lo[e] / l);
    o[4 + e] = (one)(l == 0.0f ? 0.0f : hi[e] / l);
  }
  *reinterpret_cast<vec*>(static_cast<one*>(a.out) + id * D + at) = o;
  if (a.lse && at == 0) a.lse[id] = log_sum(top, l);
}

struct SharedPlan {
  int mt, pre_mt;          // row tiles of a wave, for the sequences' own tokens and for the prefixes
  bool wide, pre_wide;     // whether the waves take different rows
  int per_seq;
  int64_t slots, pre_slots;
  int splits, split_tiles, pre_splits, pre_split_tiles;
  int own_waves;  // waves that share a sequence's rows (few rows)
  bool one_launch() const { return !wide && !pre_wide; }
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
  const int64_t n = uniform ? T / S : at_most(max_new, T), all = at_most(max_group, T);
  const int64_t tokens = width << c.page_shift;
  const int64_t tiles = (at_most(max_own, tokens) + 63) >> 6, pre_tiles = (at_most(max_shared, tokens) + 63) >> 6;
  p.wide = n * group > 64;
  p.mt = p.wide ? (c.d > 128 ? 1 : 2) : n * group <= 16 ? 1 : 2;
  // Which kernel a prefix takes.  Up to 32 rows: the one bound by memory.  More than 64: the many-row one.  Between them the many-row kernel
  // is the faster one by itself, but a launch of its own, behind which the sequences' own tokens wait: it is taken for long or many prefixes
  // (64 rows of 128, 8 cache heads; few and many rows' kernel: 64 groups of 6016 tokens 387 and 226 us; 32 of up to 4000, 20 rows of
  // each sequence's own: 64 and 71; 8 of 4000: 32 and 36; 64 of up to 1000: 52 and 53).
  const int64_t rows = all * group;
  p.pre_wide = rows > 64 || (rows > 32 && G * c.heads * pre_tiles >= 24576);
  p.pre_mt = p.pre_wide ? (c.d > 128 || rows <= 64 ? 1 : 2) : rows <= 16 ? 1 : 2;
  if (p.one_launch()) p.mt = p.pre_mt = p.mt > p.pre_mt ? p.mt : p.pre_mt;
  const int tile = (p.wide ? 64 : 16) * p.mt, pre_tile = (p.pre_wide ? 64 : 16) * p.pre_mt;
  p.per_seq = uniform ? (int)((n * group + tile - 1) / tile) : 0;
  p.slots = uniform ? S * p.per_seq : T * group / tile + S;
  p.pre_slots = G > 0 ? T * group / pre_tile + G : 0;
  const auto full = [&](int64_t sets, int64_t rows) { return (sets > (T * group + rows - 1) / rows ? sets : (T * group + rows - 1) / rows) * c.heads; };
  const int64_t own = full(S, tile), pre = full(G > 0 ? G : 1, pre_tile);
  // A prefix: as many workgroups as the CUs hold (the many-row kernel's with 16 rows a wave: half again, twice evens out unlike lengths: 64
  // groups of 12 rows of 4 heads, up to 6016 tokens: 162 us, 173 with 512), of at least four tiles (one a wave) or, where the waves take
  // different rows, eight.  (16 groups of 32 rows, up to 6000 tokens: 512 workgroups 52 us, 1024 60, 256 69; 2048 rows over 8192 tokens: 512
  // 167 us, 1024 181.)
  int64_t pre_splits = (p.pre_wide && p.pre_mt == 1 && c.d <= 128 ? 1024 : 512) / pre;
  const int64_t least = p.pre_wide ? 8 : 4;
  if (pre_splits > pre_tiles / least) pre_splits = pre_tiles / least;
  cut(pre_tiles, pre_splits, &p.pre_splits, &p.pre_split_tiles);
  // Own tokens: a wave for each (sequence, head) where there are enough of them (128 sequences of up to 150 tokens, 8 heads: 21.7 us, 24.1 with
  // four waves each; of 600: 44 and 47.5; 32 sequences of 600: 22.5 and 20.4) or where they are too few tiles for four (96 sequences of up to 45 tokens
  // behind prefixes: 62 us, 64 with four), else four waves, split as long as CUs are left.
  p.own_waves = !p.wide && (own >= 1024 || tiles <= 2) ? 1 : 4;
  int64_t splits = p.own_waves == 1 ? 1 : 512 / own;
  if (splits > tiles / 8) splits = tiles / 8;
  cut(tiles, splits, &p.splits, &p.split_tiles);
  return p;
}

// Whether the rows had better go over their tokens one sequence at a time, in one launch without a join: where the caller knows that what is
// shared is short, or the rows that share it are few.  8 cache heads of 128 and 32 query heads, apart and together: 4 rows over 1000 tokens
// 13.7 and 19.5 us, 4 over 16000 22 and 32, 4 x 8 over 1000 14.7 and 18.7, over 4000 28.9 and 27.2, 16 x 4 over 4000 53 and 38, 64 x 4 over
// 1000 64 and 49.  A prefix of more than 64 rows is a launch of its own: 8 x 4 rows of 5 new tokens over 2000 36 and 47, 64 rows of one over
// 1000 62 and 69, 32 x 8 of 5 over 2000 116 and 111.
bool apart(const CacheView& c, int64_t T, int64_t S, int64_t width, int group, int64_t max_group, int64_t max_shared) {
  if (max_shared <= 0) return false;
  if (max_shared < 64) return true;  // (what is shared comes in whole tiles: nothing is)
  const int64_t tiles = (at_most(max_shared, width << c.page_shift) + 63) >> 6;
  return S * c.heads * tiles < (at_most(max_group, T) * group > 64 ? 49152 : 12288);
}
int64_t longest(int64_t max_shared, int64_t max_own) { return max_shared > 0 && max_own > 0 ? max_shared + max_own : 0; }

template <typename Kernel>
hipError_t shared_blocks(Kernel kernel, AttendArgs a, int64_t from, int64_t to, hipStream_t st) {
  constexpr int64_t most = (1 << 24) - 1;  // (a dimension of a launch holds less than 2^32 threads)
  for (; from < to; from += most) {
    a.block0 = from;
    kernel<<<(unsigned)(to - from < most ? to - from : most), 256, 0, st>>>(a);
  }
  return hipGetLastError();
}

// Few rows: prefixes and own tokens in one launch, or one of them alone.
template <int D, bool BF>
hipError_t shared_few(const AttendArgs& a, int mt, int64_t from, int64_t to, hipStream_t st) {
  return mt == 1 ? shared_blocks(attend_shared_kernel<D, BF, 1>, a, from, to, st)
                 : shared_blocks(attend_shared_kernel<D, BF, 2>, a, from, to, st);
}
template <int D, bool BF>
hipError_t shared_prefix(const AttendArgs& a, int mt, hipStream_t st) {
  if constexpr (D <= 128) {
    if (mt == 2) return shared_blocks(attend_prefix_kernel<D, BF, 2>, a, 0, a.pre_blocks, st);
  }
  return shared_blocks(attend_prefix_kernel<D, BF, 1>, a, 0, a.pre_blocks, st);
}

template <int D, bool BF>
hipError_t shared_launch(const AttendArgs& a, const SharedPlan& p, hipStream_t st) {
  const int64_t tasks = p.slots * a.heads * p.splits, blocks = a.pre_blocks + (p.own_waves == 1 ? (tasks + 3) / 4 : tasks);
  hipError_t e;
  if (p.one_launch()) {
    e = shared_few<D, BF>(a, p.mt, 0, blocks, st);
  } else {
    e = p.pre_wide ? shared_prefix<D, BF>(a, p.pre_mt, st) : shared_few<D, BF>(a, p.pre_mt, 0, a.pre_blocks, st);
    if (e == hipSuccess)
      e = p.wide ? shared_blocks(attend_wide_kernel<D, BF, D == 256 ? 1 : 2, true>, a, a.pre_blocks, blocks, st)
                 : shared_few<D, BF>(a, p.mt, a.pre_blocks, blocks, st);
  }
  constexpr int kRows = D <= 64 ? 8 : D <= 128 ? 4 : 2;  // of a wave
  const int chunks = (a.heads * a.group + kRows - 1) / kRows;
  const int64_t most = ((1LL << 24) - 1) * 4 / chunks;  // tokens of a launch
  for (int64_t t = 0; e == hipSuccess && t < a.T; t += most) {
    const int64_t n = a.T - t < most ? a.T - t : most;
    shared_join_kernel<D, BF><<<(unsigned)((n * chunks + 3) / 4), 256, 0, st>>>(a, (p.wide ? 64 : 16) * p.mt, chunks, t);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

hipError_t launch_cache_shared(const CacheView& c, const CacheRows& rows, const int32_t* groups, int64_t G, int32_t least,
                               int32_t* tokens, int32_t* group_rows, hipStream_t st) {
  // (each workgroup reads the bounds before its own: as many workgroups as groups would read G^2 / 2 of them)
  const int64_t each = (G + 4095) / 4096;
  const SharedArgs a = {rows.starts, rows.table, rows.lengths, groups,       tokens, group_rows, rows.T,
                        rows.width,  c.pages,    rows.S,       (int)G,       c.page_shift, least, (int)(each > 0 ? each : 1)};
  const unsigned grid = G > 0 ? (unsigned)((G + each - 1) / each) : 1u;
  if (rows.S > 16 * (G > 0 ? G : 1))
    shared_kernel<1024><<<grid, 1024, 0, st>>>(a);
  else
    shared_kernel<256><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

size_t workspace_bytes_attention_shared(const CacheView& c, int64_t T, int64_t S, int64_t G, int64_t width, int64_t heads_q,
                                        bool uniform, int64_t max_new, int64_t max_group, int64_t max_shared, int64_t max_own) {
  if (apart(c, T, S, width, (int)(heads_q / c.heads), max_group, max_shared))
    return workspace_bytes_attention(c, T, S, width, heads_q, max_new, longest(max_shared, max_own), uniform);
  const SharedPlan p = shared_plan(c, T, S, G, width, (int)(heads_q / c.heads), uniform, max_new, max_group, max_shared, max_own);
  return (size_t)T * heads_q * (p.pre_splits + p.splits) * (c.d + 2) * sizeof(float);
}

hipError_t launch_cache_attention_shared(const CacheView& c, int layer, const void* q, int dtype, int64_t heads_q, int64_t q_st,
                                         int64_t q_sh, const CacheRows& rows, const int32_t* tokens, const int32_t* groups, int64_t G,
                                         float scale, int64_t max_new, int64_t max_group, int64_t max_shared, int64_t max_own,
                                         void* out, float* lse, void* workspace, hipStream_t st) {
  if (apart(c, rows.T, rows.S, rows.width, (int)(heads_q / c.heads), max_group, max_shared))
    return launch_cache_attention(c, layer, q, dtype, heads_q, q_st, q_sh, rows, scale, max_new, longest(max_shared, max_own), out, lse,
                                  workspace, st);
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
  a.own_waves = p.own_waves;
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
