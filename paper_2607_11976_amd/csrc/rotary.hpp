// Rotary positions. Pair i of a head's values [start, start + 2 n) is turned by
// the angle position * f_i:
//   y1 = x1 cos - x2 sin,  y2 = x2 cos + x1 sin,
// the pair being values (i, i + n) of that part, or (2 i, 2 i + 1) interleaved.
//
// A position times a frequency passes float32's 24 bits long before a context of
// 2^20 tokens ends (its error would be 0.06 rad there), so the angle is taken in
// 64 bits, in quarter turns (four roundings of 2^-53 at most, together less than
// 2^-51 of the angle), and its sine and cosine are 64-bit Taylor sums over
// |x| <= pi / 4 (remainder below 2^-41): about 20 fused multiply-adds a pair, which
// a thread shares over the heads that it turns. They are rounded to float32 once,
// after the amplitude; products and sums are float32, each rounded by itself, so
// that a plain float32 program gets the same bits (but where a sine lies within 2^-41
// of a border between two float32 numbers).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lt {

constexpr double kHalfPi = 1.57079632679489661923;
// (pi / 2)^n / n!
constexpr double turn_term(int n) {
  double v = 1.0;
  for (int i = 1; i <= n; ++i) v *= kHalfPi / i;
  return v;
}

struct Turn {
  float c, s;
};
// `turns` of 2 pi: cosine and sine, times the amplitude.
__device__ __forceinline__ Turn turn_of(double turns, double amplitude) {
  const double t = (turns - rint(turns)) * 4.0, q = rint(t), f = t - q, z = f * f;
  double s = turn_term(13), c = turn_term(12);
  s = fma(-z, s, turn_term(11));
  s = fma(-z, s, turn_term(9));
  s = fma(-z, s, turn_term(7));
  s = fma(-z, s, turn_term(5));
  s = fma(-z, s, turn_term(3));
  s = fma(-z, s, turn_term(1)) * f;
  c = fma(-z, c, turn_term(10));
  c = fma(-z, c, turn_term(8));
  c = fma(-z, c, turn_term(6));
  c = fma(-z, c, turn_term(4));
  c = fma(-z, c, turn_term(2));
  c = fma(-z, c, turn_term(0));
  const int k = (int)q;  // -2..2
  const float fc = (float)(c * amplitude), fs = (float)(s * amplitude);
  const float a = k & 1 ? fs : fc, b = k & 1 ? fc : fs;
  // quarter k: cos = c, -s, -c, s; sin = s, c, -s, -c
  return Turn{(k + 1) & 2 ? -a : a, k & 2 ? -b : b};
}

// Turns per position of a frequency in radians.
__device__ __forceinline__ double turns_per(float f) { return (double)f * (0.25 / kHalfPi); }

// x c + p s, each step rounded (never fused).
__device__ __forceinline__ float turned(float x, float c, float p, float s) {
#pragma clang fp contract(off)
  const float a = x * c, b = p * s;
  return a + b;
}

__device__ __forceinline__ float bf16_float(uint32_t h) { return __uint_as_float(h << 16); }
// Nearest bfloat16, ties to even.
__device__ __forceinline__ uint16_t float_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// N values as they lie in memory, at their own alignment (the hardware takes wide loads
// and stores at any), and as float32.
template <class T, int N>
struct Raw {
  static constexpr int kBytes = N * (int)sizeof(T);
  uint32_t w[(kBytes + 3) / 4];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (kBytes >= 16) {
#pragma unroll
      for (int i = 0; i < kBytes / 16; ++i) {
        uint4 a;
        __builtin_memcpy(&a, p + i * (16 / sizeof(T)), 16);
        w[4 * i] = a.x, w[4 * i + 1] = a.y, w[4 * i + 2] = a.z, w[4 * i + 3] = a.w;
      }
    } else if constexpr (kBytes == 8) {
      uint2 a;
      __builtin_memcpy(&a, p, 8);
      w[0] = a.x, w[1] = a.y;
    } else if constexpr (kBytes == 4) {
      __builtin_memcpy(&w[0], p, 4);
    } else {
      w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
  }
  __device__ __forceinline__ void unpack(float (&x)[N]) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = __uint_as_float(w[i]);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = i & 1 ? __uint_as_float(w[i / 2] & 0xFFFF0000u) : bf16_float(w[i / 2]);
    }
  }
};
template <int N, class T>
__device__ __forceinline__ void load_values(const T* p, float (&x)[N]) {
  Raw<T, N> r;
  r.load(p);
  r.unpack(x);
}
template <int N>
__device__ __forceinline__ void store_values(float* p, const float (&x)[N]) {
  if constexpr (N >= 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 a = {x[i], x[i + 1], x[i + 2], x[i + 3]};
      __builtin_memcpy(p + i, &a, 16);
    }
  } else {
    __builtin_memcpy(p, x, 4 * N);
  }
}
template <int N>
__device__ __forceinline__ void store_values(uint16_t* p, const float (&x)[N]) {
  if constexpr (N == 1) {
    *p = float_bf16(x[0]);
  } else {
    uint32_t w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) w[i] = (uint32_t)float_bf16(x[2 * i]) | (uint32_t)float_bf16(x[2 * i + 1]) << 16;
    if constexpr (N == 8) {
      const uint4 a = {w[0], w[1], w[2], w[3]};
      __builtin_memcpy(p, &a, 16);
    } else if constexpr (N == 4) {
      const uint2 a = {w[0], w[1]};
      __builtin_memcpy(p, &a, 8);
    } else {
      __builtin_memcpy(p, &w[0], 4);
    }
  }
}

}  // namespace lt
