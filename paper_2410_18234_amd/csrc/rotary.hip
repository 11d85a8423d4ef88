// Rotary positions of queries and keys (gfx950).
#include "rotary.h"

#include "cache.h"
#include "mdss.h"

namespace mdss {

namespace {

struct RotaryArgs {
  const void* x;
  void* out;
  const int32_t* positions;
  int64_t x_st, x_sh, o_st, o_sh;
  Rope rope;
  int64_t items;
  int H, D, units, turned, slices;  // a token's units, those of them that are turned, and the threads that its heads go round
  bool copy;                        // the rest of the head is written too
};

// A thread has one unit of a token and goes over some of its heads, so an angle is formed once for them; four heads at a time are
// in flight.  WIDE: a unit is 16 bytes of both halves (or of a row of side by side pairs), else one pair or one element.
// Bound by memory on prompts (8192 tokens of 40 heads of 128, f16, 168 MB: 30.4 to 32.5 us, 5.2 to 5.5 TB/s; the angles keep vector
// instructions at 32 % of the cycles), by the launch on a step (64 tokens of 40 heads: 3.8 us, a call 9.2 us).
template <int KIND, bool WIDE, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryArgs a) {
  using P = Pack<KIND>;
  using one = typename P::one;
  constexpr int V = P::V;
  constexpr int kAngles = WIDE ? (INTERLEAVED ? V / 2 : V) : 1;
  constexpr int kPieces = INTERLEAVED && WIDE ? 1 : 2;
  const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (item >= a.items) return;
  const int64_t rest = item / a.units;
  const int unit = (int)(item - rest * a.units);
  const int64_t t = rest / a.slices;
  const int slice = (int)(rest - t * a.slices);
  const bool turned = unit < a.turned;
  if (!turned && !a.copy) return;
  // the elements of the unit's pieces, and its first angle
  const int pairs = a.rope.pairs, width = WIDE ? V : 1;
  int at0, at1;
  if (!turned) {
    at0 = at1 = 2 * pairs + (unit - a.turned) * width;
  } else if (INTERLEAVED) {
    at0 = WIDE ? unit * V : 2 * unit;
    at1 = at0 + 1;
  } else {
    at0 = unit * width;
    at1 = at0 + pairs;
  }
  float c[kAngles], s[kAngles];
  if (turned) {
    const double pos = (double)a.positions[t];
    const double* f = a.rope.freq + (INTERLEAVED ? at0 / 2 : at0);
#pragma unroll
    for (int i = 0; i < kAngles; ++i) turn(a.rope, pos, f[i], c[i], s[i]);
  }
  const one* x = static_cast<const one*>(a.x) + t * a.x_st;
  one* o = static_cast<one*>(a.out) + t * a.o_st;
  constexpr int kFlight = 4;
  for (int h0 = slice; h0 < a.H; h0 += kFlight * a.slices) {
    if constexpr (WIDE) {
      u32x4 r[kFlight][kPieces];
#pragma unroll
      for (int j = 0; j < kFlight; ++j) {
        const int h = h0 + j * a.slices;
        if (h >= a.H) continue;
        const one* p = x + h * a.x_sh;
        r[j][0] = *reinterpret_cast<const u32x4*>(p + at0);
        if (kPieces == 2 && turned) r[j][kPieces - 1] = *reinterpret_cast<const u32x4*>(p + at1);
      }
#pragma unroll
      for (int j = 0; j < kFlight; ++j) {
        const int h = h0 + j * a.slices;
        if (h >= a.H) continue;
        one* p = o + h * a.o_sh;
        if (!turned) {
          *reinterpret_cast<u32x4*>(p + at0) = r[j][0];
          continue;
        }
        float u[V];
        P::open(r[j][0], u);
        if constexpr (INTERLEAVED) {
#pragma unroll
          for (int i = 0; i < V / 2; ++i) {
            const float first = u[2 * i], second = u[2 * i + 1];
            u[2 * i] = turned_first(first, second, c[i], s[i]);
            u[2 * i + 1] = turned_second(first, second, c[i], s[i]);
          }
        } else {
          float v[V];
          P::open(r[j][1], v);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float first = u[i], second = v[i];
            u[i] = turned_first(first, second, c[i], s[i]);
            v[i] = turned_second(first, second, c[i], s[i]);
          }
          *reinterpret_cast<u32x4*>(p + at1) = P::close(v);
        }
        *reinterpret_cast<u32x4*>(p + at0) = P::close(u);
      }
    } else {
      one u[kFlight], v[kFlight];
#pragma unroll
      for (int j = 0; j < kFlight; ++j) {
        const int h = h0 + j * a.slices;
        if (h >= a.H) continue;
        const one* p = x + h * a.x_sh;
        u[j] = p[at0];
        v[j] = p[at1];
      }
#pragma unroll
      for (int j = 0; j < kFlight; ++j) {
        const int h = h0 + j * a.slices;
        if (h >= a.H) continue;
        one* p = o + h * a.o_sh;
        const float first = P::widen(u[j]), second = P::widen(v[j]);
        if (turned) {
          p[at0] = (one)turned_first(first, second, c[0], s[0]);
          p[at1] = (one)turned_second(first, second, c[0], s[0]);
        } else {
          p[at0] = u[j];
        }
      }
    }
  }
}

template <int KIND>
hipError_t rotary_launch(RotaryArgs a, int64_t T, bool wide, hipStream_t st) {
  constexpr int V = Pack<KIND>::V;
  const int width = wide ? V : 1, pairs = a.rope.pairs;
  a.turned = a.rope.interleaved && wide ? 2 * pairs / V : pairs / width;
  a.units = a.turned + (a.D - 2 * pairs) / width;
  // heads of a thread: as few as fill the GPU (256 CUs of 16 waves)
  int64_t slices = (262144 + T * a.units - 1) / (T * a.units);
  a.slices = (int)(slices < a.H ? slices : a.H);
  const int64_t most = (((1LL << 24) - 1) * 256) / ((int64_t)a.units * a.slices);  // tokens of a launch
  for (int64_t t = 0; t < T; t += most) {
    const int64_t n = T - t < most ? T - t : most;
    a.items = n * a.units * a.slices;
    const unsigned grid = (unsigned)((a.items + 255) / 256);
    if (wide)
      a.rope.interleaved ? rotary_kernel<KIND, true, true><<<grid, 256, 0, st>>>(a) : rotary_kernel<KIND, true, false><<<grid, 256, 0, st>>>(a);
    else
      a.rope.interleaved ? rotary_kernel<KIND, false, true><<<grid, 256, 0, st>>>(a) : rotary_kernel<KIND, false, false><<<grid, 256, 0, st>>>(a);
    a.positions += n;
    a.x = static_cast<const typename Pack<KIND>::one*>(a.x) + n * a.x_st;
    a.out = static_cast<typename Pack<KIND>::one*>(a.out) + n * a.o_st;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const void* x, int64_t x_st, int64_t x_sh, int dtype, int64_t T, int64_t H, int64_t D, const int32_t* positions,
                         const Rope& rope, void* out, int64_t o_st, int64_t o_sh, hipStream_t st) {
  RotaryArgs a = {};
  a.x = x;
  a.out = out;
  a.positions = positions;
  a.x_st = x_st;
  a.x_sh = x_sh;
  a.o_st = o_st;
  a.o_sh = o_sh;
  a.rope = rope;
  a.H = (int)H;
  a.D = (int)D;
  a.copy = out != x;
  const int V = dtype == MDSS_F32 ? 4 : 8, dim = 2 * rope.pairs;
  const auto fits = [&](int64_t v) { return v % V == 0; };
  const bool wide = fits(x_st) && fits(x_sh) && fits(o_st) && fits(o_sh) && fits(D) && fits(rope.interleaved ? dim : rope.pairs) &&
                    ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(out)) & 15) == 0;
  switch (dtype) {
    case MDSS_F32: return rotary_launch<0>(a, T, wide, st);
    case MDSS_BF16: return rotary_launch<1>(a, T, wide, st);
    default: return rotary_launch<2>(a, T, wide, st);
  }
}

}  // namespace mdss
