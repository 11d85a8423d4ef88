// Beam search: the best continuations over beams and vocabulary, and the reordering of states (gfx950).
//
//   total(w, v) = ((x_v - m) - log sum_j exp(x_j - m)) + score_w,  m = max x,
// ordered by the total, then the lower beam, then the larger logit, then the lower token.  Within a beam the order
// is the logits' own, so the sum is not needed to select: the logits are read once.  A workgroup holds a chunk of a
// row in registers, takes its maximum, its sum of exponentials and its n best tokens; one workgroup a group of
// beams then joins the chunks.  A chunk's n best: the n-th largest of a wave's 64 per-lane maxima is a bound
// that at least n of the chunk's tokens reach and, but for ties, few more do; those are ranked against each other.
// Bound by memory on large batches: 64 x 8 x 128256 bf16 reads 115 MB.
#include "cache.h"

#include <math.h>

namespace mdss {

namespace {

constexpr int kThreads = 256;
constexpr int kList = 512;       // tokens of a chunk ranked against each other
constexpr int kMaxChunks = 64;   // of a row: one a lane where they are joined
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
  int W, n, chunks, sub;
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

template <int TYPE, int R>
__global__ __launch_bounds__(kThreads) void beam_chunk_kernel(const BeamArgs a) {
  using L = Logit<TYPE>;
  using one = typename L::one;
  constexpr int kVec = L::kVec;
  __shared__ uint64_t list[kList + kMaxBeams];
  __shared__ uint64_t best[kMaxBeams];
  __shared__ float red_m[4], red_s[4];
  __shared__ uint32_t red_t[4];
  __shared__ int red_c[4];
  __shared__ int count;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.y;
  if (!beam_open(a, row)) return;
  const one* x = static_cast<const one*>(a.logits) + row * a.stride;
  // 16-byte pieces from the address below the row's first logit on; those that cross an end go one by one
  const int shift = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(one));
  const int n = a.n;
  float M = -INFINITY, S = 0.0f;
  int kept = 0;  // of `best`, from the pieces before
  for (int sub = 0; sub < a.sub; ++sub) {
    const int64_t k0 = ((int64_t)blockIdx.x * a.sub + sub) * (kThreads * R);
    const auto at = [&](int j) { return (k0 + j * kThreads + tid) * kVec - shift; };
    if (k0 * kVec - shift >= a.V) break;
    u32x4 r[R];
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int64_t i0 = at(j);
      if (i0 >= 0 && i0 + kVec <= a.V) {
        r[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(x + i0));
      } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) L::set(r[j], i, i0 + i >= 0 && i0 + i < a.V ? x[i0 + i] : L::none());
      }
    }
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
      for (int i = 0; i < kVec; ++i) m = fmaxf(m, L::get(r[j], i));
    const float ref = m == -INFINITY ? 0.0f : m;
    float s = 0.0f;  // NaN where a logit is NaN or +inf: the row is refused where the chunks are joined
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
      for (int i = 0; i < kVec; ++i) s += __builtin_amdgcn_exp2f((L::get(r[j], i) - ref) * 1.44269504f);
    // the wave's n-th largest lane maximum, by bisection of its bits
    const uint32_t mine = ordered(m);
    uint32_t bound = 0;
#pragma unroll 4
    for (int b = 31; b >= 0; --b) {
      const uint32_t c = bound | 1u << b;
      if (__popcll(__ballot(mine >= c)) >= n) bound = c;
    }
    // the workgroup's maximum and sum
    const float wm = wave_max(m), wref = wm == -INFINITY ? 0.0f : wm;
    s *= m == -INFINITY ? (s != s ? s : 0.0f) : __builtin_amdgcn_exp2f((m - wref) * 1.44269504f);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
    if (lane == 0) {
      red_m[wave] = wm;
      red_s[wave] = s;
      red_t[wave] = bound;
    }
    if (tid == 0) count = kept;
    if (tid < kept) list[tid] = best[tid];
    __syncthreads();
    float top = M;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      top = fmaxf(top, red_m[w]);
      bound = max(bound, red_t[w]);
    }
    const float tref = top == -INFINITY ? 0.0f : top;
    S *= M == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((M - tref) * 1.44269504f);
#pragma unroll
    for (int w = 0; w < 4; ++w)
      S += red_m[w] == -INFINITY ? (red_s[w] != red_s[w] ? red_s[w] : 0.0f)
                                 : red_s[w] * __builtin_amdgcn_exp2f((red_m[w] - tref) * 1.44269504f);
    M = top;
    uint64_t least = (uint64_t)max(bound, kLowest + 1) << 32;
    const auto push = [&]() {
      if (mine < (uint32_t)(least >> 32)) return;
#pragma unroll
      for (int j = 0; j < R; ++j)
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          const uint64_t key = token_key(L::get(r[j], i), at(j) + i);
          if (key >= least) {
            const int to = atomicAdd(&count, 1);
            if (to < kList + kMaxBeams) list[to] = key;
          }
        }
    };
    push();
    __syncthreads();
    int c = count;
    if (c > kList) {
      // many tokens share the bound (or few lanes hold any): the exact key of the n-th, by bisection
      uint64_t t = 0;
      for (int b = 63; b >= 0; --b) {
        const uint64_t cand = t | 1ull << b;
        int here = 0;
#pragma unroll
        for (int j = 0; j < R; ++j)
#pragma unroll
          for (int i = 0; i < kVec; ++i) here += token_key(L::get(r[j], i), at(j) + i) >= cand;
        here = wave_sum_int(here);
        __syncthreads();
        if (lane == 0) red_c[wave] = here;
        __syncthreads();
        if (red_c[0] + red_c[1] + red_c[2] + red_c[3] >= n) t = cand;
      }
      least = max(t, (uint64_t)(kLowest + 1) << 32);
      __syncthreads();
      if (tid == 0) count = kept;
      __syncthreads();
      push();
      __syncthreads();
      c = min(count, kList + kMaxBeams);
    }
    for (int i = tid; i < c; i += kThreads) {
      const uint64_t key = list[i];
      int above = 0;
      for (int j = 0; j < c; ++j) above += list[j] > key;
      if (above < n) best[above] = key;
    }
    kept = min(c, n);
    __syncthreads();
  }
  const int64_t to = row * a.chunks + blockIdx.x;
  if (tid < n) a.keys[to * n + tid] = tid < kept ? best[tid] : 0;
  if (tid == 0) {
    a.stats[2 * to] = M;
    a.stats[2 * to + 1] = S;
  }
}

// Largest key over the wave.
__device__ __forceinline__ uint64_t wave_max64(uint64_t k) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    const uint64_t o = __shfl_xor((unsigned long long)k, off, 64);
    k = o > k ? o : k;
  }
  return k;
}

// One workgroup a group of beams: a wave joins a beam's chunks (n rounds of the largest head of the sorted lists,
// one a lane), then the first wave joins the beams in the same way by their totals.
constexpr int kJoinThreads = 512;
__global__ __launch_bounds__(kJoinThreads) void beam_join_kernel(const BeamArgs a) {
  __shared__ float total[kMaxBeams][kMaxBeams];
  __shared__ int32_t token[kMaxBeams][kMaxBeams];
  __shared__ int have[kMaxBeams];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = a.n;
  const int64_t b = blockIdx.x;
  for (int w = wave; w < a.W; w += kJoinThreads / 64) {
    const int64_t row = b * a.W + w;
    const float score = a.score[row];
    int got = 0;
    if (a.done && a.done[row]) {
      if (fabsf(score) < INFINITY) {
        got = 1;
        if (lane == 0) {
          total[w][0] = score;
          token[w][0] = a.eos;
        }
      }
    } else if (fabsf(score) < INFINITY) {
      const int64_t at = row * a.chunks + lane;
      const bool in = lane < a.chunks;
      const float m = in ? a.stats[2 * at] : -INFINITY, s = in ? a.stats[2 * at + 1] : 0.0f;
      const uint64_t* keys = a.keys + at * n;
      uint64_t head = in ? keys[0] : 0, next = in && n > 1 ? keys[1] : 0;
      int used = 1;
      const float top = wave_max(m), ref = top == -INFINITY ? 0.0f : top;
      const double sum = wave_sum(m == -INFINITY ? (double)(s != s ? s : 0.0f) : (double)s * (double)expf(m - ref));
      if (sum != sum) {
        if (lane == 0 && a.row_status) atomicOr(a.row_status + row, kRowBadProb);
      } else {
        const float logs = logf((float)sum);
        for (int k = 0; k < n; ++k) {
          const uint64_t big = wave_max64(head);
          if ((uint32_t)(big >> 32) <= kLowest) break;
          if (lane == 0) {
            const float t = ((unordered((uint32_t)(big >> 32)) - ref) - logs) + score;
            total[w][k] = t;
            token[w][k] = (int32_t)~(uint32_t)big;
          }
          got = k + 1;
          if (head == big) {
            head = next;
            ++used;
            next = used < n ? keys[used] : 0;
          }
        }
      }
    }
    if (lane == 0) have[w] = got;
  }
  __syncthreads();
  if (wave != 0) return;
  int at = 0;
  const int mine = lane < a.W ? have[lane] : 0;
  for (int k = 0; k < n; ++k) {
    const float t = at < mine ? total[lane][at] : -INFINITY;
    const uint64_t key = t > -INFINITY ? (uint64_t)ordered(t) << 32 | (uint32_t)~lane : 0;
    const uint64_t big = wave_max64(key);
    const int64_t to = b * n + k;
    if (big == 0) {
      if (lane == 0) {
        a.parent[to] = -1;
        a.token[to] = -1;
        a.score_out[to] = -INFINITY;
        a.done_out[to] = 0;
      }
      continue;
    }
    if (key == big) {
      const int tok = token[lane][at];
      a.parent[to] = lane;
      a.token[to] = tok;
      a.score_out[to] = t;
      a.done_out[to] = (a.done && a.done[b * a.W + lane]) || tok == a.eos;
      ++at;
    }
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
  bool wide;  // 64 logits a thread, else 16
  int chunks, sub;
};
BeamPlan beam_plan(int64_t rows, int64_t V) {
  BeamPlan p;
  p.wide = rows * ((V + 16383) / 16384) >= 512;
  // (a row that starts inside a 16-byte piece may take one piece more)
  const int64_t each = p.wide ? 16384 : 4096, pieces = (V + 7 + each - 1) / each;
  p.sub = (int)((pieces + kMaxChunks - 1) / kMaxChunks);
  p.chunks = (int)((pieces + p.sub - 1) / p.sub);
  return p;
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
  a.sub = p.sub;
  a.eos = eos;
  a.parent = parent;
  a.token = token;
  a.score_out = score;
  a.done_out = done_out;
  a.row_status = row_status;
  const dim3 grid((unsigned)p.chunks, (unsigned)(B * W));
  if (dtype == MDSS_F32)
    p.wide ? beam_chunk_kernel<0, 16><<<grid, kThreads, 0, st>>>(a) : beam_chunk_kernel<0, 4><<<grid, kThreads, 0, st>>>(a);
  else if (dtype == MDSS_BF16)
    p.wide ? beam_chunk_kernel<1, 8><<<grid, kThreads, 0, st>>>(a) : beam_chunk_kernel<1, 2><<<grid, kThreads, 0, st>>>(a);
  else
    p.wide ? beam_chunk_kernel<2, 8><<<grid, kThreads, 0, st>>>(a) : beam_chunk_kernel<2, 2><<<grid, kThreads, 0, st>>>(a);
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
