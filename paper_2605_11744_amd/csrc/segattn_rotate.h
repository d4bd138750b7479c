// Turning of channel pairs shared by the rotation kernel and the append kernel.
//
// A head's D channels are handled in units of 16, two pieces of 8: in the half layout (pairs i, i + n/2 of the
// first n channels) unit u holds channels 8u.. and n/2 + 8u.., otherwise channels 16u .. 16u + 15.  Either way a
// turned unit u holds the pairs 8u .. 8u + 7, so both layouts read their sines the same way, and a unit at or
// behind channel n is passed on as it is.
#pragma once
#include "segattn_paged.h"

namespace segattn {

// Sine and cosine of `turns` whole turns, times magnitude.  The turns are formed and reduced to [-1/2, 1/2] in
// double precision: at position 10^5 a float product is off by 0.01 rad.  What is left is rounded to a float
// once (2^-25 turns at most, 2e-7 rad).
__device__ inline float2 turn_of(double position, double turns, int back, float magnitude) {
  const double t = position * turns;
  float sn, cs;
  sincospif(2.f * (float)(t - rint(t)), &sn, &cs);
  return float2{(back ? -sn : sn) * magnitude, cs * magnitude};
}

__device__ inline void unit_channels(int u, int pairs, int interleaved, int &lo, int &hi) {
  const bool halves = !interleaved && 8 * u < pairs;
  lo = halves ? 8 * u : 16 * u;
  hi = halves ? pairs + 8 * u : 16 * u + 8;
}

// x: the unit's channels, lo piece first; sn, cs: of the pairs 8u .. 8u + 7.
__device__ inline void turn_unit(float (&x)[16], const float *sn, const float *cs, int interleaved) {
  float s[8], c[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    s[e] = sn[e];
    c[e] = cs[e];
  }
  if (interleaved) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float a = x[2 * e], b = x[2 * e + 1];
      x[2 * e] = a * c[e] - b * s[e];
      x[2 * e + 1] = a * s[e] + b * c[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float a = x[e], b = x[8 + e];
      x[e] = a * c[e] - b * s[e];
      x[8 + e] = a * s[e] + b * c[e];
    }
  }
}

__device__ inline void load8(const unsigned short *at, float *x) {
  const uint4 u = *(const uint4 *)at;
  const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ inline void load8(const float *at, float *x) {
  const float4 a = ((const float4 *)at)[0], b = ((const float4 *)at)[1];
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
  x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ inline void store8(unsigned short *at, const float *x) {  // bf16, to nearest even
  unsigned w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = (unsigned)__builtin_bit_cast(unsigned short, (__bf16)x[2 * i]) |
           (unsigned)__builtin_bit_cast(unsigned short, (__bf16)x[2 * i + 1]) << 16;
  *(uint4 *)at = uint4{w[0], w[1], w[2], w[3]};
}
__device__ inline void store8(float *at, const float *x) {
  ((float4 *)at)[0] = float4{x[0], x[1], x[2], x[3]};
  ((float4 *)at)[1] = float4{x[4], x[5], x[6], x[7]};
}

}  // namespace segattn
