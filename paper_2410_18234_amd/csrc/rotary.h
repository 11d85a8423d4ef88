// Rotary positions: a pair (u, v) of a head's elements at position t becomes m (u cos a - v sin a, u sin a + v cos a), a = t f.
//
// The angle is formed in fp64 (fp32 loses 2^-24 of t f, whole turns at far positions): t f in quarter turns, whose whole part picks
// the quadrant and whose rest, within half a quarter turn, goes to two fp32 and two Taylor series (to r^9 and r^10: below 2^-25 there),
// whose last step is one rounding: cosine and sine are off by little more than that.
#pragma once

#include <stdint.h>

#include <hip/hip_runtime.h>

namespace mdss {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Rope {
  const double* freq;  // [pairs], radians per position
  int pairs;
  bool interleaved;
  float magnitude, sign;  // sign: -1 turns back
  float bound;            // sqrt(2) magnitude: what an element of a turned pair is at most, in the larger of the two
};

// cos and sin of position * freq, times the magnitude.
__device__ __forceinline__ void turn(const Rope& r, double position, double freq, float& c, float& s) {
  const double t = position * (freq * 0.63661977236758134308);  // quarter turns
  const double n = t + 6755399441055744.0;                      // 1.5 2^52: the nearest whole number in the low bits
  const double rest = t - (n - 6755399441055744.0);
  const float x = (float)rest, low = (float)(rest - (double)x), z = x * x;
  const uint32_t k = (uint32_t)__builtin_bit_cast(uint64_t, n);
  // pi / 2 = 1.57079637 (in fp32) - 4.37113883e-8
  const float higher = fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.6044118478735982e-4f, -4.681754135318687e-3f), 7.969262624616704e-2f), -0.6459640975062463f),
                            -4.3711388e-8f);
  const float sx = fmaf(x, 1.5707964f, fmaf(low, 1.5707964f, x * higher));
  const float cx = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -2.5202042373060605e-5f, 9.192602748394264e-4f), -2.0863480763352960e-2f),
                                        0.2536695079010480f), -1.2337005501361697f), 1.0f);
  const float co = k & 1 ? sx : cx, si = k & 1 ? cx : sx;
  c = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, co * r.magnitude) ^ (((k + 1) & 2) << 30));
  s = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, si * (r.sign * r.magnitude)) ^ ((k & 2) << 30));
}
__device__ __forceinline__ float turned_first(float u, float v, float c, float s) { return fmaf(u, c, -(v * s)); }
__device__ __forceinline__ float turned_second(float u, float v, float c, float s) { return fmaf(u, s, v * c); }

// 16 bytes of a type as floats and back (rounded to nearest, ties to even).
template <int KIND>
struct Pack;
template <>
struct Pack<0> {
  typedef float one;
  static constexpr int V = 4;
  static __device__ __forceinline__ void open(const u32x4& r, float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __builtin_bit_cast(float, (uint32_t)r[i]);
  }
  static __device__ __forceinline__ u32x4 close(const float (&x)[4]) { return __builtin_bit_cast(u32x4, f32x4{x[0], x[1], x[2], x[3]}); }
  static __device__ __forceinline__ float widen(one x) { return x; }
};
template <>
struct Pack<1> {
  typedef __bf16 one;
  typedef one vec __attribute__((ext_vector_type(8)));
  static constexpr int V = 8;
  static __device__ __forceinline__ void open(const u32x4& r, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __builtin_bit_cast(float, (uint32_t)r[i] << 16);
      x[2 * i + 1] = __builtin_bit_cast(float, (uint32_t)r[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ u32x4 close(const float (&x)[8]) {
    vec v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (one)x[i];
    return __builtin_bit_cast(u32x4, v);
  }
  static __device__ __forceinline__ float widen(one x) { return (float)x; }
};
template <>
struct Pack<2> {
  typedef _Float16 one;
  typedef one vec __attribute__((ext_vector_type(8)));
  static constexpr int V = 8;
  static __device__ __forceinline__ void open(const u32x4& r, float (&x)[8]) {
    const vec v = __builtin_bit_cast(vec, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
  }
  static __device__ __forceinline__ u32x4 close(const float (&x)[8]) {
    vec v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (one)x[i];
    return __builtin_bit_cast(u32x4, v);
  }
  static __device__ __forceinline__ float widen(one x) { return (float)x; }
};

}  // namespace mdss
