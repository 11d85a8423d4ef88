// Beam search: the best continuations over beams and vocabulary, and the reordering of states (gfx950).
//
//   total(w, v) = ((x_v - m) - log sum_j exp(x_j - m)) + score_w,  m = max x,
// ordered by the total, then the lower beam, then the larger logit, then the lower token.  Within a beam the order
// is the logits' own, so the sum is not needed to select: the logits are read once.  A wave streams a chunk of a row
// and keeps its maximum, its sum of exponentials and a list of the tokens that may be among its n best; one
// workgroup a group of beams then joins the chunks.  What may be among the n best is what reaches the n-th largest of
// the wave's 64 running lane maxima (n of its tokens do), so that all but a few tokens are dropped by one
// comparison of their lane's maximum.
// Bound by memory on large batches, by latency on small ones.
#include "cache.h"

#include <math.h>

namespace mdss {

namespace {

constexpr int kThreads = 256;
constexpr int kList = 256;      // tokens a wave keeps before it sorts out the n best
constexpr int kPieces = 128;    // 16-byte pieces a wave keeps before it looks at their logits
constexpr int kMaxChunks = 64;  // of a row: one a lane where they are joined
constexpr int kMaxBeams = 64;

// Floats in an order of unsigned numbers (both zeros alike), and back.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t k) {
  return __builtin_bit_cast(float, k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
constexpr uint32_t kLowest = 0x007fffffu;  // ordered(-inf)
__device__ __forceinline__ uint64_t token_key(float x, int64_t token) {
  return (uint64_t)ordered(x) << 32 | (uint32_t)~(uint32_t)token;
}

struct BeamArgs {
  const void* logits;
  int64_t stride, V;
  const float* score;
  const uint8_t* done;
  uint64_t* keys;   // [rows][chunks][n], descending, 0: none
  float* stats;     // [rows][chunks][2]: maximum, sum of exponentials
  int W, n, chunks, steps;  // steps of a chunk
  int64_t rows;
  int eos;
  int32_t *parent, *token;
  float* score_out;
  uint8_t* done_out;
  int32_t* row_status;
};

__device__ __forceinline__ bool beam_open(const BeamArgs& a, int64_t row) {  // a beam that reads its logits
  return !(a.done && a.done[row]) && fabsf(a.score[row]) < INFINITY;
}

template <int TYPE>  // 0: fp32, 1: bf16, 2: f16
struct Logit;
template <>
struct Logit<0> {
  static constexpr int kVec = 4;
  typedef float one;
  static __device__ __forceinline__ float get(const u32x4& r, int i) {
    const uint32_t u = r[i];  // (a bit cast of the element itself would read the vector's first)
    return __builtin_bit_cast(float, u);
  }
  static __device__ __forceinline__ void set(u32x4& r, int i, one x) { r[i] = __builtin_bit_cast(uint32_t, x); }
  static __device__ __forceinline__ one none() { return -INFINITY; }
};
template <>
struct Logit<1> {
  static constexpr int kVec = 8;
  typedef uint16_t one;
  static __device__ __forceinline__ float get(const u32x4& r, int i) {
    return __builtin_bit_cast(float, i & 1 ? r[i >> 1] & 0xffff0000u : r[i >> 1] << 16);
  }
  static __device__ __forceinline__ void set(u32x4& r, int i, one x) {
    r[i >> 1] = i & 1 ? (r[i >> 1] & 0xffffu) | (uint32_t)x << 16 : x;
  }
  static __device__ __forceinline__ one none() { return 0xff80; }
};
template <>
struct Logit<2> {
  static constexpr int kVec = 8;
  typedef uint16_t one;
  static __device__ __forceinline__ float get(const u32x4& r, int i) {
    return (float)__builtin_bit_cast(_Float16, (uint16_t)(r[i >> 1] >> (16 * (i & 1))));
  }
  static __device__ __forceinline__ void set(u32x4& r, int i, one x) {
    r[i >> 1] = i & 1 ? (r[i >> 1] & 0xffffu) | (uint32_t)x << 16 : x;
  }
  static __device__ __forceinline__ one none() { return 0xfc00; }
};

// Largest of 64 lanes, in every lane.
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, false));   // quad_perm [1,0,3,2]
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, false));   // quad_perm [2,3,0,1]
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xF, 0xF, false));  // row_ror:4
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xF, 0xF, false));  // row_ror:8
  auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = max((uint32_t)a[0], (uint32_t)a[1]);
  a = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return max((uint32_t)a[0], (uint32_t)a[1]);
}
// Largest key over the wave, in every lane: by its upper half, then among the lanes that have it (mostly one).
__device__ __forceinline__ uint64_t wave_max64(uint64_t k) {
  const uint32_t hi = wave_max_u32((uint32_t)(k >> 32));
  const bool mine = (uint32_t)(k >> 32) == hi;
  const uint64_t who = __ballot(mine);
  const uint32_t lo = __popcll(who) == 1 ? __builtin_amdgcn_readlane((uint32_t)k, __ffsll((unsigned long long)who) - 1)
                                         : wave_max_u32(mine ? (uint32_t)k : 0u);
  return (uint64_t)hi << 32 | lo;
}
// The n-th largest of the lanes' values (n <= 64) to its BITS upper bits, the lower ones 0: bisection.
template <int BITS>
__device__ __forceinline__ uint32_t wave_nth(uint32_t x, int n) {
  uint32_t t = 0;
#pragma unroll
  for (int b = 31; b >= 32 - BITS; --b) {
    const uint32_t c = t | 1u << b;
    if (__popcll(__ballot(x >= c)) >= n) t = c;
  }
  return t;
}

// The n largest of a wave's list of c keys (in no order, each one once) in descending order at its front; returns how
// many there are.  A key's place is the number of larger ones.
__device__ __forceinline__ void sort_list(uint64_t* list, int c, int n, int lane) {
  constexpr int MINE = kList / 64;
  uint64_t key[MINE];
  int above[MINE];
#pragma unroll
  for (int q = 0; q < MINE; ++q) {
    key[q] = lane + 64 * q < c ? list[lane + 64 * q] : 0;
    above[q] = 0;
  }
  for (int j = 0; j < c; ++j) {
    const uint64_t other = list[j];
#pragma unroll
    for (int q = 0; q < MINE; ++q) above[q] += other > key[q];
  }
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int q = 0; q < MINE; ++q)
    if (lane + 64 * q < c && above[q] < n) list[above[q]] = key[q];
  __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ int sort_out(uint64_t* list, int c, int n, int lane) {
  if (c <= 64) {  // a key a lane: the others' by lane reads, without LDS
    const uint64_t key = lane < c ? list[lane] : 0;
    int above = 0;
    for (int j = 0; j < c; ++j) {
      const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)(key >> 32), j), lo = __builtin_amdgcn_readlane((uint32_t)key, j);
      const uint64_t other = (uint64_t)hi << 32 | lo;
      above += other > key;
    }
    __builtin_amdgcn_wave_barrier();
    if (lane < c && above < n) list[above] = key;
    __builtin_amdgcn_wave_barrier();
  } else {
    sort_list(list, c, n, lane);
  }
  return min(c, n);
}

// One wave a chunk of a row (the four of a workgroup have nothing in common), E logits of a lane in a step.  Pieces whose
// largest logit reaches the bound are put aside, and their logits looked at when there are many or at the end.
// 64 x 8 x 128256 bf16, 32 of the beams finished (123 MB read): 4096 logits a step, 32 us (3.8 TB/s; its vector instructions take
// 77 % of that).
template <int TYPE, int E>
__global__ __launch_bounds__(kThreads, E == 16 ? 8 : TYPE == 0 ? 4 : 5) void beam_chunk_kernel(const BeamArgs a) {
  using L = Logit<TYPE>;
  using one = typename L::one;
  constexpr int kVec = L::kVec, kLoads = E / kVec;
  // (a 16-bit logit's order is in its upper half; of 32 bits, a bound a little low lets few more pass)
  constexpr int kBits = TYPE == 1 ? 16 : TYPE == 2 ? 20 : 22;
  __shared__ uint64_t lists[kThreads / 64][kList];
  __shared__ __align__(16) one pieces[kThreads / 64][kPieces][kVec];
  __shared__ int32_t piece_ids[kThreads / 64][kPieces];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t job = (int64_t)blockIdx.x * (kThreads / 64) + wave;
  const int64_t row = job / a.chunks;
  const int chunk = (int)(job - row * a.chunks);
  if (row >= a.rows || !beam_open(a, row)) return;
  uint64_t* list = lists[wave];
  one (*piece)[kVec] = pieces[wave];
  int32_t* piece_id = piece_ids[wave];
  const one* x = static_cast<const one*>(a.logits) + row * a.stride;
  // 16-byte pieces from the address below the row's first logit on; those that cross an end go one by one
  const int shift = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(one));
  const int n = a.n, V = (int)a.V;
  float m = -INFINITY, s = 0.0f;  // the lane's; s is NaN where a logit is NaN or +inf: the row is refused where chunks are joined
  int count = 0, aside = 0;       // of list, of piece
  float bound = -INFINITY;        // no logit below it is among the n best, and of those equal to it only tokens below `tie`
  int tie = -1;
  const auto look = [&]() {
    for (int e0 = 0; e0 < aside * kVec; e0 += 64) {
      const int e = e0 + lane, at = e / kVec;
      const bool have = e < aside * kVec;
      u32x4 w = {0, 0, 0, 0};
      L::set(w, 0, have ? piece[at][e % kVec] : L::none());
      const float v = L::get(w, 0);
      const int tok = have ? piece_id[at] * kVec - shift + e % kVec : 0;
      const bool in = v > bound || (v == bound && tok < tie && v > -INFINITY);
      const uint64_t who = __ballot(in);
      if (who == 0) continue;
      if (in) list[count + __popcll(who & ((1ull << lane) - 1))] = token_key(v, tok);
      count += __popcll(who);
      __builtin_amdgcn_wave_barrier();
      if (count > kList - 64) {
        count = sort_out(list, count, n, lane);
        if (count == n) {  // from here on only what comes before the n-th
          const uint64_t least = list[n - 1];
          bound = unordered((uint32_t)(least >> 32));
          tie = (int)~(uint32_t)least;
        }
      }
    }
    aside = 0;
    __builtin_amdgcn_wave_barrier();
  };
  for (int st = 0; st < a.steps; ++st) {
    const int first = ((chunk * a.steps + st) * kLoads) * 64 + lane;  // the lane's first piece of the step
    u32x4 r[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int i0 = (first + 64 * j) * kVec - shift;
      if (i0 >= 0 && i0 + kVec <= V) {
        r[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(x + i0));
      } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) L::set(r[j], i, i0 + i >= 0 && i0 + i < V ? x[i0 + i] : L::none());
      }
    }
    float pm[kLoads], mx = -INFINITY;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      pm[j] = L::get(r[j], 0);
#pragma unroll
      for (int i = 1; i < kVec; ++i) pm[j] = fmaxf(pm[j], L::get(r[j], i));
      mx = fmaxf(mx, pm[j]);
    }
    const float top = fmaxf(m, mx), ref = top == -INFINITY ? 0.0f : top;
    s *= m == -INFINITY ? (s != s ? s : 0.0f) : __builtin_amdgcn_exp2f((m - ref) * 1.44269504f);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) asm volatile("" : "+v"(r[j]));  // widened again below, not held in fp32 from above
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
#pragma unroll
      for (int i = 0; i < kVec; ++i) s += __builtin_amdgcn_exp2f((L::get(r[j], i) - ref) * 1.44269504f);
    m = top;
    // n tokens of the chunk reach the n-th largest lane maximum
    const float reach = fmaxf(unordered(wave_nth<kBits>(ordered(m), n)), -INFINITY);
    if (reach > bound) {
      bound = reach;
      tie = INT32_MAX;
    }
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const bool in = pm[j] > bound || (pm[j] == bound && tie >= 0);
      const uint64_t who = __ballot(in);
      if (who == 0) continue;
      if (in) {
        const int to = aside + __popcll(who & ((1ull << lane) - 1));
        *reinterpret_cast<u32x4*>(piece[to]) = r[j];
        piece_id[to] = first + 64 * j;
      }
      aside += __popcll(who);
      __builtin_amdgcn_wave_barrier();
      if (aside > kPieces - 64) look();
    }
  }
  look();
  count = sort_out(list, count, n, lane);
  // the wave's maximum and sum
  const float top = wave_max(m), ref = top == -INFINITY ? 0.0f : top;
  s *= m == -INFINITY ? (s != s ? s : 0.0f) : __builtin_amdgcn_exp2f((m - ref) * 1.44269504f);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
  if (lane < n) a.keys[job * n + lane] = lane < count ? list[lane] : 0;
  if (lane == 0) {
    a.stats[2 * job] = top;
    a.stats[2 * job + 1] = s;
  }
}

// One workgroup a group of beams.  A wave joins a beam's chunks, a sorted list a lane: with r = ceil(n / chunks), the
// ceil(n / r)-th largest of the lists' r-th keys is reached by n keys, and what reaches it is ranked.  The first wave
// then joins the beams by their totals: n rounds of the largest head.
constexpr int kJoinThreads = 512;
__global__ __launch_bounds__(kJoinThreads) void beam_join_kernel(const BeamArgs a) {
  __shared__ uint64_t lists[kJoinThreads / 64][kList];
  __shared__ float total[kMaxBeams][kMaxBeams];
  __shared__ int32_t token[kMaxBeams][kMaxBeams];
  __shared__ int have[kMaxBeams], ended[kMaxBeams];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = a.n;
  const int64_t b = blockIdx.x;
  uint64_t* list = lists[wave];
  const int deep = (n + a.chunks - 1) / a.chunks, wide = (n + deep - 1) / deep;
  for (int w = wave; w < a.W; w += kJoinThreads / 64) {
    const int64_t row = b * a.W + w, at = row * a.chunks + lane;
    const bool in = lane < a.chunks;
    // everything is asked for at once (what a beam without candidates has there is not used)
    const float score = a.score[row];
    const bool done = a.done && a.done[row];
    const float m = in ? a.stats[2 * at] : -INFINITY, s = in ? a.stats[2 * at + 1] : 0.0f;
    const uint64_t* keys = a.keys + at * n;
    uint64_t head[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) head[k] = in && k < n ? keys[k] : 0;
    int got = 0;
    if (lane == 0) ended[w] = done;
    if (done) {
      if (fabsf(score) < INFINITY) {
        got = 1;
        if (lane == 0) {
          total[w][0] = score;
          token[w][0] = a.eos;
        }
      }
    } else if (fabsf(score) < INFINITY) {
      const uint64_t deepest = deep == 1 ? head[0] : deep == 2 ? head[1] : deep == 3 ? head[2] : deep == 4 ? head[3] : in ? keys[deep - 1] : 0;
      uint64_t least = (uint64_t)max(wave_nth<32>((uint32_t)(deepest >> 32), wide), kLowest + 1) << 32;
      const float top = wave_max(m), ref = top == -INFINITY ? 0.0f : top;
      const double sum = wave_sum_dpp(m == -INFINITY ? (double)(s != s ? s : 0.0f) : (double)s * (double)expf(m - ref));
      if (sum != sum) {
        if (lane == 0 && a.row_status) atomicOr(a.row_status + row, kRowBadProb);
      } else {
        for (int k = 0; k < n; ++k) {
          const uint64_t key = k == 0 ? head[0] : k == 1 ? head[1] : k == 2 ? head[2] : k == 3 ? head[3] : in ? keys[k] : 0;
          const uint64_t who = __ballot(key >= least);
          if (who == 0) break;
          if (key >= least) list[got + __popcll(who & ((1ull << lane) - 1))] = key;
          got += __popcll(who);
          __builtin_amdgcn_wave_barrier();
          if (got > kList - 64) {
            got = sort_out(list, got, n, lane);
            if (got == n) least = list[n - 1] + 1;
          }
        }
        got = sort_out(list, got, n, lane);
        if (lane < got) {
          const uint64_t key = list[lane];
          total[w][lane] = ((unordered((uint32_t)(key >> 32)) - ref) - logf((float)sum)) + score;
          token[w][lane] = (int32_t)~(uint32_t)key;
        }
      }
    }
    if (lane == 0) have[w] = got;
  }
  __syncthreads();
  if (wave != 0) return;
  const int mine = lane < a.W ? have[lane] : 0;
  int at = 0, beam = -1, place = 0;  // lane k: the beam and place of the k-th
  float head = mine > 0 ? total[lane][0] : -INFINITY;
  for (int k = 0; k < n; ++k) {
    const float next = at + 1 < mine ? total[lane][at + 1] : -INFINITY;
    const uint64_t key = head > -INFINITY ? (uint64_t)ordered(head) << 32 | (uint32_t)~lane : 0;
    const uint64_t big = wave_max64(key);
    if (big == 0) break;
    const int who = (int)~(uint32_t)big, which = __builtin_amdgcn_readlane(at, who);
    if (lane == k) {
      beam = who;
      place = which;
    }
    if (lane == who) {
      head = next;
      ++at;
    }
  }
  if (lane < n) {
    const int64_t to = b * n + lane;
    const int tok = beam >= 0 ? token[beam][place] : -1;
    a.parent[to] = beam;
    a.token[to] = tok;
    a.score_out[to] = beam >= 0 ? total[beam][place] : -INFINITY;
    a.done_out[to] = beam >= 0 && (ended[beam] || tok == a.eos);
  }
}

// Rows of bytes: out[b][j] = state[b][parent[b][j]], zeros where the parent is none of the W.
template <typename T>
__global__ __launch_bounds__(kThreads) void reorder_kernel(const T* state, const int32_t* parent, int W, int n,
                                                           int64_t words, T* out) {
  const int64_t row = blockIdx.y;
  const int p = parent[row];
  const bool in = p >= 0 && p < W;
  const T* from = state + ((row / n) * W + (in ? p : 0)) * words;
  T* to = out + row * words;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < words; i += (int64_t)gridDim.x * kThreads)
    to[i] = in ? from[i] : T{};
}

template <typename T>
void reorder_launch(const void* state, const int32_t* parent, int64_t B, int64_t W, int64_t n, int64_t words,
                    void* out, hipStream_t st) {
  int64_t x = (words + 4 * kThreads - 1) / (4 * kThreads);
  if (x > 1024) x = 1024;
  reorder_kernel<T><<<dim3((unsigned)x, (unsigned)(B * n)), kThreads, 0, st>>>(
      static_cast<const T*>(state), parent, (int)W, (int)n, words, static_cast<T*>(out));
}

struct BeamPlan {
  int each, chunks, steps;  // logits of a lane in a step, chunks of a row, steps of a chunk
};
// A step holds 64 logits of a lane; 16 where that makes fewer than 4096 waves (four on each SIMD).  At most 64 chunks of a
// row: one a lane where they are joined.  (So a chunk is one step in rows of up to 2^18 tokens, 2^16 in small batches.)
BeamPlan beam_plan(int64_t rows, int64_t V) {
  BeamPlan p;
  p.each = rows * ((V + 1023) / 1024) <= 4096 ? 16 : 64;
  const int64_t steps = (V + 7 + 64 * p.each - 1) / (64 * p.each);  // (a row that starts inside a 16-byte piece may take one more)
  p.steps = (int)((steps + kMaxChunks - 1) / kMaxChunks);
  p.chunks = (int)((steps + p.steps - 1) / p.steps);
  return p;
}

template <int TYPE>
void chunk_launch(const BeamArgs& a, int each, unsigned grid, hipStream_t st) {
  if (each == 16)
    beam_chunk_kernel<TYPE, 16><<<grid, kThreads, 0, st>>>(a);
  else
    beam_chunk_kernel<TYPE, 64><<<grid, kThreads, 0, st>>>(a);
}

}  // namespace

size_t workspace_bytes_beam(int64_t B, int64_t W, int64_t V, int64_t n) {
  return (size_t)B * W * beam_plan(B * W, V).chunks * (n + 1) * sizeof(uint64_t);
}

hipError_t launch_beam_select(const void* logits, int dtype, int64_t row_stride, const float* scores,
                              const uint8_t* done, int64_t B, int64_t W, int64_t V, int64_t n, int32_t eos,
                              int32_t* parent, int32_t* token, float* score, uint8_t* done_out, int32_t* row_status,
                              void* workspace, hipStream_t st) {
  const BeamPlan p = beam_plan(B * W, V);
  BeamArgs a;
  a.logits = logits;
  a.stride = row_stride;
  a.V = V;
  a.score = scores;
  a.done = done;
  a.keys = static_cast<uint64_t*>(workspace);
  a.stats = reinterpret_cast<float*>(a.keys + B * W * p.chunks * n);
  a.W = (int)W;
  a.n = (int)n;
  a.chunks = p.chunks;
  a.steps = p.steps;
  a.rows = B * W;
  a.eos = eos;
  a.parent = parent;
  a.token = token;
  a.score_out = score;
  a.done_out = done_out;
  a.row_status = row_status;
  const unsigned grid = (unsigned)((B * W * p.chunks + kThreads / 64 - 1) / (kThreads / 64));
  if (dtype == MDSS_F32)
    chunk_launch<0>(a, p.each, grid, st);
  else if (dtype == MDSS_BF16)
    chunk_launch<1>(a, p.each, grid, st);
  else
    chunk_launch<2>(a, p.each, grid, st);
  beam_join_kernel<<<(unsigned)B, kJoinThreads, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_beam_reorder(const void* state, const int32_t* parent, int64_t B, int64_t W, int64_t n,
                               int64_t row_bytes, void* out, hipStream_t st) {
  const uintptr_t low = (reinterpret_cast<uintptr_t>(state) | reinterpret_cast<uintptr_t>(out) | (uintptr_t)row_bytes);
  if ((low & 15) == 0)
    reorder_launch<u32x4>(state, parent, B, W, n, row_bytes / 16, out, st);
  else if ((low & 3) == 0)
    reorder_launch<uint32_t>(state, parent, B, W, n, row_bytes / 4, out, st);
  else
    reorder_launch<uint8_t>(state, parent, B, W, n, row_bytes, out, st);
  return hipGetLastError();
}

}  // namespace mdss
