// What the two kernels of seg_attn_paged_chosen share (not part of the ABI).
#pragma once
#include "segattn_sparse.h"

namespace segattn {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
#define LDS_AS __attribute__((address_space(3)))

constexpr int kColumns = 16;
constexpr int kChosenWaves = 4;

// Over the four lanes of a column, by exchanges between vector registers.
__device__ inline float over_quads(float x, bool sum) {
  const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = sum ? __uint_as_float(y[0]) + __uint_as_float(y[1]) : fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
  const auto z = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return sum ? __uint_as_float(z[0]) + __uint_as_float(z[1]) : fmaxf(__uint_as_float(z[0]), __uint_as_float(z[1]));
}

// Four channels of a head's output, and with the first ones its sum; ref: what it is relative to, as an exponent of two.  No row seen: zeros,
// and the logarithm of nothing.
template <int D>
__device__ inline void store_out(const PagedChosenArgs &a, long long head, int d, f32x4 o, float l, float ref) {
  const f32x4 r = o * (l == 0.f ? 0.f : 1.f / l);
  if (a.out_fp32) {
    float *dst = (float *)a.out + head * D + d;
#pragma unroll
    for (int e = 0; e < 4; ++e) dst[e] = r[e];
  } else {
    __bf16 *dst = (__bf16 *)a.out + head * D + d;
#pragma unroll
    for (int e = 0; e < 4; ++e) dst[e] = (__bf16)r[e];
  }
  if (d == 0) a.lse[head] = l == 0.f ? -INFINITY : (ref + log2f(l)) * 0.69314718055994531f;
}

// The partial (acc[D], maximum as an exponent of two, sum) of part `part` of (token, the x-th head of its set), of query head 0 of the group.
template <int D>
__device__ inline float *partial_of(const PagedChosenArgs &a, bool past, long long token, int x, int part) {
  const long long before = past ? 0 : a.parts_past > 1 ? a.total * a.n_past * a.parts_past : 0;
  const long long unit = past ? (token * a.n_past + x) * a.parts_past : (token * a.n_other + x) * a.parts_other;
  return a.slots + (before + unit + part) * a.g * ws_slot_floats(D);
}

// Where a row's 16-byte chunk lies in a tile in LDS, so that neither the transposed nor the plain reads nor the writes meet on a bank.
template <int D>
__device__ inline int chunk_k(int row, int chunk) {
  return D == 128 ? chunk ^ (chunk >> 3) ^ (row & 15) : chunk ^ ((row >> 1) & 7) ^ (row & 1);
}
template <int D>
__device__ inline int chunk_v(int row, int chunk) {
  return D == 128 ? chunk ^ (chunk >> 3) ^ (2 * (row & 7)) : chunk ^ (2 * ((row >> 1) & 3)) ^ (row & 1);
}
// Eight e4m3 elements times a power of two, as bf16 (exact below 2^128, infinite from there on: four significant bits).
__device__ inline u32x4 bf16_of_e4m3(unsigned lo, unsigned hi, float scale) {
  bf16x2 y[4];
  y[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  y[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  y[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  y[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return __builtin_bit_cast(u32x4, y);
}
// Of eight bf16 those that are not finite become zeros; whether there were some.
__device__ inline bool without_odd(u32x4 &y) {
  bool any = false;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const bool lo = (y[e] & 0x7f80u) == 0x7f80u, hi = (y[e] & 0x7f800000u) == 0x7f800000u;
    y[e] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
    any |= lo || hi;
  }
  return any;
}
__device__ inline long long of_lane(long long v, int l) {
  const unsigned lo = __builtin_amdgcn_readlane((int)v, l), hi = __builtin_amdgcn_readlane((int)(v >> 32), l);
  return (long long)(((unsigned long long)hi << 32) | lo);
}
// Rows row .. row + 15 that lie in [from, to), as bits; none for row < 0.
__device__ inline unsigned half_bits(int row, int from, int to) {
  if (row < 0 || row >= to || row + 16 <= from) return 0u;
  unsigned bits = 0xffffu;
  if (row < from) bits &= 0xffffu << (from - row);
  if (row + 16 > to) bits &= (1u << (to - row)) - 1u;
  return bits & 0xffffu;
}
// Rows [from, to) that token i of a sequence's n sees in window w of the hx-th head of the sets.
__device__ inline void token_window(const PagedChosenArgs &a, long long w, int hx, int i, int n, int &from, int &to) {
  to = rows_seen(a.rows, w, i, n, a.max_rows);
  from = 0;
  if (hx >= a.n_past) {
    const int start = fast_div(to > 0 ? to - 1 : 0, a.seg) * (int)a.seg.d;
    from = a.tail_of[hx] ? (start > a.tail ? start - a.tail : 0) : start;
  }
}
// The sequence and the first token of tile `place` of `tokens` tokens each: sequence b's tiles have the numbers from
// cu[b] / tokens + b on.  -1: no such tile.
__device__ inline int tile_of(const PagedChosenArgs &a, long long place, int tokens, int &i, int &n) {
  if (!a.cu) {
    i = 0;
    n = 1;
    return place < a.B ? (int)place : -1;
  }
  int lo = 0, hi = a.B;
  while (hi - lo > 1) {
    const int mid = lo + (hi - lo) / 2;
    if ((long long)a.cu[mid] / tokens + mid <= place) lo = mid;
    else hi = mid;
  }
  n = a.cu[lo + 1] - a.cu[lo];
  const long long first = (place - (a.cu[lo] / tokens + lo)) * tokens;
  if (first < 0 || first >= n || a.cu[lo] < 0 || a.cu[lo + 1] > a.total) return -1;
  i = (int)first;
  return lo;
}

}  // namespace segattn
