// Turning of channel pairs shared by the rotation kernel and the append kernel.
//
// A head's D channels are handled in units of two 16-byte pieces of P channels (8 bf16, 4 floats), so that neighbouring
// lanes have neighbouring pieces: of the n turned channels unit u holds P u.. and n/2 + P u.., of the others, which are passed
// on as they are, likewise.  In the half layout (pairs i, i + n/2) those are the two sides of the pairs P u..; in the
// interleaved one each piece holds P/2 pairs of its own.  (Two pieces side by side, fp32 gradients with half of the
// head interleaved, 3 times 5003 tokens of 16 + 4 heads: 78 us instead of 50.)  Rows are read once and written once, so both are marked as not worth keeping:
// 32K tokens of 32 + 8 heads of 128 118 -> 109 us, prompts into an 8-bit cache 90 -> 82.
#pragma once
#include "segattn_paged.h"

namespace segattn {

// Sine and cosine of `turns` whole turns, times magnitude.  The turns are formed and reduced to [-1/2, 1/2] in
// double precision: at position 10^5 a float product is off by 0.01 rad.  Sine and cosine themselves are formed in 32 bits, which
// costs fp32 results 3.8e-8 of their size in the mean against 3.6e-8 with ones rounded from 64.
__device__ inline float2 turn_of(double position, double turns, int back, float magnitude) {
  const double t = position * turns, half = 2.0 * (t - rint(t));
  const float near = (float)half;
  float sn, cs;
  sincospif(near, &sn, &cs);
  const float rest = 3.14159265f * (float)(half - near);  // what the rounding left, to first order
  const float s = sn + cs * rest, c = cs - sn * rest;
  return float2{(back ? -s : s) * magnitude, c * magnitude};
}

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// First channels of a unit's pieces; the unit is turned if P u < pairs.
template <int P>
__device__ inline void unit_channels(int u, int pairs, int D, int &lo, int &hi) {
  const bool turned = P * u < pairs;
  lo = turned ? P * u : pairs + P * u;  // 2 pairs + P (u - pairs / P)
  hi = lo + (turned ? pairs : (D - 2 * pairs) / 2);
}

// x: the unit's channels, lo piece first; sn, cs: sines and cosines of the token's pairs.
template <int P, bool kInterleaved>
__device__ inline void turn_unit(float (&x)[2 * P], int u, int pairs, const float *sn, const float *cs) {
  float s[P], c[P];
  if constexpr (kInterleaved) {
#pragma unroll
    for (int e = 0; e < P; ++e) {
      const int i = P / 2 * u + (e < P / 2 ? e : pairs / 2 + e - P / 2);
      s[e] = sn[i];
      c[e] = cs[i];
    }
#pragma unroll
    for (int e = 0; e < P; ++e) {
      const float a = x[2 * e], b = x[2 * e + 1];
      x[2 * e] = a * c[e] - b * s[e];
      x[2 * e + 1] = a * s[e] + b * c[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < P; ++e) {
      s[e] = sn[P * u + e];
      c[e] = cs[P * u + e];
    }
#pragma unroll
    for (int e = 0; e < P; ++e) {
      const float a = x[e], b = x[P + e];
      x[e] = a * c[e] - b * s[e];
      x[P + e] = a * s[e] + b * c[e];
    }
  }
}

template <typename T>
__device__ inline u32x4 load_piece(const T *at) { return __builtin_nontemporal_load((const u32x4 *)at); }
template <typename T>
__device__ inline void store_piece(T *at, u32x4 x) { __builtin_nontemporal_store(x, (u32x4 *)at); }
__device__ inline void numbers_of(u32x4 w, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ inline void numbers_of(u32x4 w, float (&x)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
}
__device__ inline u32x4 piece_of(const float (&x)[8]) {  // bf16, to nearest even
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = (unsigned)__builtin_bit_cast(unsigned short, (__bf16)x[2 * i]) |
           (unsigned)__builtin_bit_cast(unsigned short, (__bf16)x[2 * i + 1]) << 16;
  return w;
}
__device__ inline u32x4 piece_of(const float (&x)[4]) {
  return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
}
// A unit turned from and to its two pieces.
template <int P, bool kInterleaved>
__device__ inline void turn_pieces(u32x4 &lo, u32x4 &hi, int u, int pairs, const float *sn, const float *cs) {
  float a[P], b[P], x[2 * P];
  numbers_of(lo, a);
  numbers_of(hi, b);
#pragma unroll
  for (int e = 0; e < P; ++e) {
    x[e] = a[e];
    x[P + e] = b[e];
  }
  turn_unit<P, kInterleaved>(x, u, pairs, sn, cs);
#pragma unroll
  for (int e = 0; e < P; ++e) {
    a[e] = x[e];
    b[e] = x[P + e];
  }
  lo = piece_of(a);
  hi = piece_of(b);
}

}  // namespace segattn
