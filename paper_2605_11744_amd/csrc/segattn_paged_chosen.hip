// seg_attn_paged_chosen: attention of new tokens over a paged cache, long-range heads over the blocks that a list names for each token.
//
// A unit of work is a set of up to 16 query columns with the key rows that they see: of a PAST head one token's g query heads
// with the rows of its listed blocks, of another head the g query heads of as many neighbouring tokens of a sequence as
// fit, with the rows of all their windows.  (A group of more than 16 heads takes a pass per 16.)  Per tile of 32 rows -- two
// halves of 16, each somewhere in the pool -- a wave forms
//   S^T[key][column] = K . Q^T            v_mfma_f32_16x16x32_bf16, A = K rows, B = Q^T (registers)
//   P = exp2((S^T - m) c)                 running maximum m and sum l per column, in fp32
//   O^T[d][column] += V^T . P^T           A = V^T via ds_read_b64_tr_b16, B = P from the S^T registers
// P enters as two bf16 (what that leaves is below 2^-16 of a weight), for fp32 outputs as three.
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

__device__ inline float over_quads(float x, bool sum) {  // over the four lanes of a column
  const float y = __shfl_xor(x, 16);
  x = sum ? x + y : fmaxf(x, y);
  const float z = __shfl_xor(x, 32);
  return sum ? x + z : fmaxf(x, z);
}

// Four channels of a head's output, and with the first ones its sum.  No row seen: zeros, and the logarithm of nothing.
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
  if (d == 0) a.lse[head] = l == 0.f ? -INFINITY : ref * a.scale + logf(l);
}

// The partial of part `part` of (token, the x-th head of its set), of query head 0 of the group.
template <int D>
__device__ inline float *partial_of(const PagedChosenArgs &a, bool past, long long token, int x, int part) {
  const long long before = past ? 0 : a.parts_past > 1 ? a.total * a.n_past * a.parts_past : 0;
  const long long unit = past ? (token * a.n_past + x) * a.parts_past : (token * a.n_other + x) * a.parts_other;
  return a.slots + (before + unit + part) * a.g * ws_slot_floats(D);
}

// kMany: the columns belong to several tokens (a window's tile).
template <int D, bool kE4m3>
__global__ __launch_bounds__(64 * kChosenWaves, 2) void paged_chosen_kernel(const PagedChosenArgs a, const long long first_wg) {
  constexpr int NK = D / 32, NB = D / 16;
  constexpr int kRow = 2 * D, kTileBytes = kChosenTile * kRow;  // of a tile in LDS, bf16
  constexpr int kPieces = (kE4m3 ? D : 2 * D) / 16;             // 16-byte pieces of a row in memory
  constexpr int RPL = 64 / kPieces, NL = kChosenTile / RPL;     // rows per wave load, loads per tile and tensor
  // Where a row's 16-byte chunk lies, so that neither the transposed nor the plain reads nor the writes meet on a bank.
  auto chunk_k = [](int row, int chunk) { return D == 128 ? chunk ^ (chunk >> 3) ^ (row & 15) : chunk ^ ((row >> 1) & 7) ^ (row & 1); };
  auto chunk_v = [](int row, int chunk) { return D == 128 ? chunk ^ (chunk >> 3) ^ (2 * (row & 7)) : chunk ^ (2 * ((row >> 1) & 3)) ^ (row & 1); };

  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int quad = lane >> 4, col = lane & 15;
  const float c = a.scale_log2e;
  __shared__ __attribute__((aligned(1024))) unsigned char tiles[kChosenWaves][2 * kTileBytes];
  constexpr int MS = D + 4;  // floats per column of the merge area
  static_assert(kChosenWaves * 2 * kTileBytes >= (int)sizeof(float) * kChosenWaves * kColumns * MS, "merge area fits the tiles");

  // ---- which columns, which rows
  long long u = first_wg + blockIdx.x;
  const bool past = u < a.wgs_past;
  if (!past) u -= a.wgs_past;
  const int heads = past ? a.n_past : a.n_other, parts = past ? a.parts_past : a.parts_other;
  const int x = (int)(u % heads);
  u /= heads;
  const int pass = (int)(u % a.passes);
  u /= a.passes;
  const int part = (int)(u % parts);
  const long long place = u / parts;  // token, or number of a tile
  const int hx = past ? x : a.n_past + x, h = a.head_of[hx];
  int b, i, n, tokens = 1;
  if (past) {
    b = sequence_of(a.cu, a.B, place, i, n);
    if (b < 0) return;
  } else if (!a.cu) {
    b = (int)place;
    i = 0;
    n = 1;
    if (b >= a.B) return;
  } else {
    // Sequence b's tiles have the numbers from cu[b] / tokens + b on.
    int lo = 0, hi = a.B;
    while (hi - lo > 1) {
      const int mid = lo + (hi - lo) / 2;
      if ((long long)a.cu[mid] / a.tokens + mid <= place) lo = mid;
      else hi = mid;
    }
    b = lo;
    n = a.cu[b + 1] - a.cu[b];
    const long long first = (place - (a.cu[b] / a.tokens + b)) * a.tokens;
    if (first < 0 || first >= n || a.cu[b] < 0 || a.cu[b + 1] > a.total) return;
    i = (int)first;
    tokens = n - i < a.tokens ? n - i : a.tokens;
  }
  const long long token0 = past ? place : a.cu ? a.cu[b] + i : b;
  const long long w = (long long)b * a.Hkv + h;
  // query head of a column: of the pass's heads of one token, or of all heads of several
  const int per = a.tokens > 1 ? a.g : min(kColumns, a.g - pass * kColumns);  // columns of a token
  const int live = tokens * per;
  const int my_token = col < live ? col / per : 0, my_head = pass * kColumns + (col < live ? col % per : 0);
  auto bounds_of = [&](int token, int &from, int &to) {
    to = rows_seen(a.rows, w, i + token, n, a.max_rows);
    from = 0;
    if (!past) {
      const int start = fast_div(to > 0 ? to - 1 : 0, a.seg) * (int)a.seg.d;
      from = a.tail_of[hx] ? (start > a.tail ? start - a.tail : 0) : start;
    }
  };
  int my_from, my_to, from, to, last_from, first_to;  // of the column; of all of them: first and last row that one, and that every one sees
  bounds_of(my_token, my_from, my_to);
  bounds_of(0, from, first_to);
  bounds_of(tokens - 1, last_from, to);

  const int *table = table_of(a.c, a.Hkv, b, h);
  const int *list = past ? a.chosen + (place * a.n_past + x) * a.n_chosen : nullptr;
  const int hh = a.c.per_head ? 0 : h;
  unsigned char *tile = tiles[wave];
  const unsigned char *scales = lane < 32 ? a.c.k_scale : a.c.v_scale;
  int koff[NK], voff[NB];
  const int vrow = 4 * quad + (col >> 2);
#pragma unroll
  for (int kc = 0; kc < NK; ++kc) koff[kc] = col * kRow + (chunk_k(col, 4 * kc + quad) << 4);
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
    voff[nb] = kTileBytes + vrow * kRow + (chunk_v(vrow, 2 * nb + ((col & 3) >> 1)) << 4) + 8 * (col & 1);

  bf16x8 Q[NK];  // column col, zero beyond the live ones
  {
    const unsigned short *q = a.q + ((token0 + my_token) * a.Hq + h * a.g + my_head) * D + 8 * quad;
#pragma unroll
    for (int kc = 0; kc < NK; ++kc) {
      u32x4 y = *(const u32x4 *)(q + 32 * kc);
      if (col >= live) y = u32x4{0u, 0u, 0u, 0u};
      Q[kc] = __builtin_bit_cast(bf16x8, y);
    }
  }
  f32x4 O[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) O[nb] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_run = 0.f;

  // ---- tiles: the halves' places are looked up 64 at a time, a lane each
  int half_row = -1;           // first row of this lane's half, -1: nothing to see there
  long long half_at = 0, half_place = 0;  // its offset in k and v, and its place among the rows of the pool's heads
  auto look_up = [&](int t) {  // halves of the tiles t, t + waves, ...
    t += kChosenWaves * (lane >> 1);
    half_row = -1;
    half_at = 0;
    half_place = 0;
    const int half = 2 * t + (lane & 1);
    int row = -1;
    if (past) {
      const int entry = fast_div(half, a.block_halves);
      if (entry < a.n_chosen) {
        const int block = list[entry];
        const long long r = (long long)block * (16 * a.block_halves.d) + 16 * (half - entry * (int)a.block_halves.d);
        if (block >= 0 && r < to) row = (int)r;
      }
    } else {
      const long long r = 16ll * half + from / kChosenTile * kChosenTile;
      if (r < to && r + 16 > from) row = (int)r;
    }
    if (row < 0) return;
    int in_page;
    const int page = page_of(a.c, table, row, in_page);
    if (page < 0) return;
    half_row = row;
    half_at = page * a.c.page_bytes + hh * a.c.head_bytes + in_page * a.c.row_bytes;
    half_place = ((long long)page * a.c.heads + hh) * a.c.page_rows.d + in_page;
  };
  auto of_lane = [&](long long v, int l) {
    const unsigned lo = __builtin_amdgcn_readlane((int)v, l), hi = __builtin_amdgcn_readlane((int)(v >> 32), l);
    return (long long)(((unsigned long long)hi << 32) | lo);
  };

  u32x4 nk[NL], nv[NL];  // the wave's next tile, in flight
  int n_scale = 0;       // scale byte of row lane % 32: keys in the lower half of the wave, values in the upper
  int n_row0 = 0, n_row1 = 0;
  auto fetch = [&](int j) __attribute__((always_inline)) {  // j: number of the tile among the looked up ones
    n_row0 = __builtin_amdgcn_readlane(half_row, 2 * j);
    n_row1 = __builtin_amdgcn_readlane(half_row, 2 * j + 1);
    const long long at[2] = {of_lane(half_at, 2 * j), of_lane(half_at, 2 * j + 1)};
    const unsigned mine = (unsigned)(lane / kPieces) * (unsigned)a.c.row_bytes + (lane % kPieces) * 16;
#pragma unroll
    for (int l = 0; l < NL; ++l) {
      const long long from_row = at[l / (NL / 2)] + (l % (NL / 2)) * (RPL * a.c.row_bytes);
      nk[l] = *(const u32x4 *)(a.c.k + from_row + mine);
      nv[l] = *(const u32x4 *)(a.c.v + from_row + mine);
    }
    if constexpr (kE4m3) {
      const long long at0 = of_lane(half_place, 2 * j), at1 = of_lane(half_place, 2 * j + 1);
      n_scale = scales[(lane & 16 ? at1 : at0) + (lane & 15)];
    }
  };
  // Rows of a half that some column sees, as bits.
  auto rows_of = [&](int row) __attribute__((always_inline)) {
    if (row < 0) return 0u;
    unsigned bits = 0xffffu;
    if (row < from) bits &= 0xffffu << (from - row);
    if (row + 16 > to) bits &= (1u << (to - row)) - 1u;
    return bits & 0xffffu;
  };
  // A tile into LDS, values of rows that nobody sees as zeros (a weight of zero times NaN would be NaN).  Returns whether a value
  // is not finite.
  auto stage = [&](unsigned valid, bool look) __attribute__((always_inline)) {
    bool bad = false;
    auto not_finite = [](u32x4 y) {
      bool any = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) any |= (y[e] & 0x7f80u) == 0x7f80u || (y[e] & 0x7f800000u) == 0x7f800000u;
      return any;
    };
#pragma unroll
    for (int l = 0; l < NL; ++l) {
      const int r = RPL * l + lane / kPieces, piece = lane % kPieces;
      const u32x4 xk = nk[l], xv = nv[l];
      if constexpr (!kE4m3) {
        *(u32x4 *)(tile + r * kRow + (chunk_k(r, piece) << 4)) = xk;
        *(u32x4 *)(tile + kTileBytes + r * kRow + (chunk_v(r, piece) << 4)) = xv;
        if (look) bad |= ((valid >> r) & 1) && not_finite(xv);
      } else {
        // a scale is a power of two and e4m3 has four significant bits: the bf16 is exact below 2^128, and infinite from there on
        const float sk = __uint_as_float((unsigned)__shfl(n_scale, r) << 23), sv = __uint_as_float((unsigned)__shfl(n_scale, r + 32) << 23);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          bf16x2 yk[4], yv[4];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            yk[2 * e] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(xk[2 * half + e], sk, false);
            yk[2 * e + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(xk[2 * half + e], sk, true);
            yv[2 * e] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(xv[2 * half + e], sv, false);
            yv[2 * e + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(xv[2 * half + e], sv, true);
          }
          const int chunk = 2 * piece + half;
          *(u32x4 *)(tile + r * kRow + (chunk_k(r, chunk) << 4)) = __builtin_bit_cast(u32x4, yk);
          *(u32x4 *)(tile + kTileBytes + r * kRow + (chunk_v(r, chunk) << 4)) = __builtin_bit_cast(u32x4, yv);
          if (look) bad |= ((valid >> r) & 1) && not_finite(__builtin_bit_cast(u32x4, yv));
        }
      }
    }
    if (valid != ~0u && !((valid >> (lane & 31)) & 1)) {
#pragma unroll
      for (int e = 0; e < kRow / 32; ++e)
        *(u32x4 *)(tile + kTileBytes + (lane & 31) * kRow + (kRow / 32 * (lane >> 5) + e) * 16) = u32x4{0u, 0u, 0u, 0u};
    }
    return __builtin_amdgcn_ballot_w64(bad) != 0;
  };
  auto values = [&](int nb) __attribute__((always_inline)) {  // V^T, channels 16 nb ..
    const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4 *)(tile + voff[nb]));
    const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4 *)(tile + voff[nb] + 16 * kRow));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  auto products = [&](int row0, int row1, unsigned valid, bool mixed, bool bad) __attribute__((always_inline)) {
    f32x4 S[2];
#pragma unroll
    for (int h2 = 0; h2 < 2; ++h2) {
      S[h2] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kc = 0; kc < NK; ++kc)
        S[h2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8 *)(tile + koff[kc] + 16 * h2 * kRow), Q[kc], S[h2], 0, 0, 0);
    }
    // register r of S[h2] is row 4 quad + r of half h2
    unsigned mine = valid >> (4 * quad);  // bits r and 16 + r
    if (mixed) {
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = (h2 ? row1 : row0) + 4 * quad + r;
          if (row < my_from || row >= my_to) mine &= ~(1u << (16 * h2 + r));
        }
    }
    if (mixed || valid != ~0u) {
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (!((mine >> (16 * h2 + r)) & 1)) S[h2][r] = -INFINITY;
    }
    float mx = fmaxf(fmaxf(fmaxf(S[0][0], S[0][1]), fmaxf(S[0][2], S[0][3])), fmaxf(fmaxf(S[1][0], S[1][1]), fmaxf(S[1][2], S[1][3])));
    mx = over_quads(mx, false);
    const float m_new = fmaxf(m_run, mx);
    const float ref = m_new == -INFINITY ? 0.f : m_new;  // no row yet
    const float alpha = __builtin_amdgcn_exp2f((m_run - ref) * c);
    m_run = m_new;
    bf16x8 P, P_rest;
    float tail[2][4];  // of a weight beyond its two bf16
    float sum = 0.f;
#pragma unroll
    for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float e = __builtin_amdgcn_exp2f((S[h2][r] - ref) * c);
        sum += e;
        P[4 * h2 + r] = (__bf16)e;
        const float rest = e - (float)P[4 * h2 + r];
        P_rest[4 * h2 + r] = (__bf16)rest;
        tail[h2][r] = rest - (float)P_rest[4 * h2 + r];
      }
    l_run = l_run * alpha + sum;
    if (__builtin_amdgcn_ballot_w64(alpha != 1.f)) {  // a new maximum somewhere: rare behind the first tiles
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) O[nb] *= alpha;
    }
    bf16x8 P_tail;
#pragma unroll
    for (int e = 0; e < 8; ++e) P_tail[e] = (__bf16)tail[e / 4][e % 4];
    if (!bad) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const bf16x8 va = values(nb);
        O[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, P, O[nb], 0, 0, 0);
        O[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, P_rest, O[nb], 0, 0, 0);
        if (a.out_fp32) O[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, P_tail, O[nb], 0, 0, 0);
      }
    } else {
      // A value that is not finite in rows that some of the tokens see and others do not: token by token, the rows that it does not see as
      // zeros, and only its own columns kept.
      for (int k = 0; k < tokens; ++k) {
        int k_from, k_to;
        bounds_of(k, k_from, k_to);
        u32x4 keep;  // operand A's registers: keys 4 quad + 0 .. 3 of both halves
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = (e < 2 ? row0 : row1) + 4 * quad + 2 * (e & 1);
          keep[e] = (row >= k_from && row < k_to ? 0xffffu : 0u) | (row + 1 >= k_from && row + 1 < k_to ? 0xffff0000u : 0u);
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const bf16x8 va = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, values(nb)) & keep);
          f32x4 y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, P, O[nb], 0, 0, 0);
          y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, P_rest, y, 0, 0, 0);
          if (a.out_fp32) y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, P_tail, y, 0, 0, 0);
          if (my_token == k) O[nb] = y;
        }
      }
    }
  };

  const int per_part = past ? a.tiles_past : a.tiles_other;
  const int t_begin = part * per_part;
  int t_end = t_begin + per_part;
  {
    const long long all = past ? ((long long)a.n_chosen * a.block_halves.d + 1) / 2 : to > 0 ? (to + kChosenTile - 1) / kChosenTile - from / kChosenTile : 0;
    if (t_end > all) t_end = (int)all;
  }
  for (int t = t_begin + wave; t < t_end; t += 32 * kChosenWaves) {
    look_up(t);
    const int covered = min(32, (t_end - t + kChosenWaves - 1) / kChosenWaves);
    unsigned long long halves = __builtin_amdgcn_ballot_w64(half_row >= 0);
    if (covered < 32) halves &= (1ull << (2 * covered)) - 1;
    unsigned long long some = (halves | (halves >> 1)) & 0x5555555555555555ull;  // tiles with rows to see
    if (!some) continue;
    int j = (int)__builtin_ctzll(some) >> 1;
    some &= some - 1;
    fetch(j);
    for (;;) {
      const int row0 = n_row0, row1 = n_row1;
      const unsigned valid = rows_of(row0) | rows_of(row1) << 16;
      const bool mixed = tokens > 1 && ((row0 >= 0 && (row0 < last_from || row0 + 16 > first_to)) || (row1 >= 0 && (row1 < last_from || row1 + 16 > first_to)));
      const bool bad = stage(valid, mixed);
      const bool more = some != 0;
      if (more) {
        j = (int)__builtin_ctzll(some) >> 1;
        some &= some - 1;
        fetch(j);
      }
      products(row0, row1, valid, mixed, bad);
      if (!more) break;
    }
  }
  l_run = over_quads(l_run, true);

  // ---- the waves meet in LDS (over the tiles: everyone is done)
  __syncthreads();
  float *mg = (float *)&tiles[0][0];  // [wave][column][MS]
  if (col < live) {
    float *dst = mg + (wave * kColumns + col) * MS;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) *(f32x4 *)(dst + 16 * nb + 4 * quad) = O[nb];
    if (quad == 0) {
      dst[D] = m_run;
      dst[D + 1] = l_run;
    }
  }
  __syncthreads();
  for (int k = tid; k < live * (D / 4); k += 64 * kChosenWaves) {
    const int column = k / (D / 4), d = (k % (D / 4)) * 4;
    float top = -INFINITY;
#pragma unroll
    for (int y = 0; y < kChosenWaves; ++y) top = fmaxf(top, mg[(y * kColumns + column) * MS + D]);
    const float ref = top == -INFINITY ? 0.f : top;
    float l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int y = 0; y < kChosenWaves; ++y) {
      const float *src = mg + (y * kColumns + column) * MS;
      // 0 for a wave without rows; one whose scores are all NaN has no maximum either, and its NaN sums stay NaN
      const float wgt = __builtin_amdgcn_exp2f((src[D] - ref) * c);
      l += src[D + 1] * wgt;
      o += *(const f32x4 *)(src + d) * wgt;
    }
    const long long token = token0 + column / per;
    const int head = pass * kColumns + column % per;
    if (parts == 1) {
      store_out<D>(a, token * a.Hq + h * a.g + head, d, o, l, ref);
    } else {
      float *dst = partial_of<D>(a, past, token, x, part) + head * ws_slot_floats(D);
      *(f32x4 *)(dst + d) = o;
      if (d == 0) *(float2 *)(dst + D) = float2{top, l};
    }
  }
}

// A wave per query head whose window was shared out: its parts' partials joined.
template <int D>
__global__ __launch_bounds__(256) void paged_chosen_join_kernel(const PagedChosenArgs a, const long long first_wg) {
  constexpr int SF = D + kWsTailFloats, kLanes = D / 4, kGroups = 64 / kLanes;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const long long u = (first_wg + blockIdx.x) * 4 + wave;
  if (u >= a.total * a.Hq) return;
  const long long token = u / a.Hq;
  const int head = (int)(u - token * a.Hq), h = head / a.g;
  int hx = 0;  // h's place among the sets
  while (a.head_of[hx] != h) ++hx;
  const bool past = hx < a.n_past;
  const int parts = past ? a.parts_past : a.parts_other;
  if (parts == 1) return;
  int i, n;
  if (sequence_of(a.cu, a.B, token, i, n) < 0) return;
  const float *src = partial_of<D>(a, past, token, past ? hx : hx - a.n_past, 0) + (head - h * a.g) * SF;
  const float c = a.scale_log2e;
  const int d = lane % kLanes * 4;
  float top = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s = lane / kLanes; s < parts; s += kGroups) {
    const float *part = src + (long long)s * a.g * SF;
    const float2 ml = *(const float2 *)(part + D);
    const f32x4 y = *(const f32x4 *)(part + d);
    const float m_new = fmaxf(top, ml.x), ref = m_new == -INFINITY ? 0.f : m_new;
    const float keep = __builtin_amdgcn_exp2f((top - ref) * c), wgt = __builtin_amdgcn_exp2f((ml.x - ref) * c);
    l = l * keep + ml.y * wgt;
    o = o * keep + y * wgt;
    top = m_new;
  }
  float most = top;
#pragma unroll
  for (int sh = kLanes; sh < 64; sh <<= 1) most = fmaxf(most, __shfl_xor(most, sh));
  const float ref = most == -INFINITY ? 0.f : most, wgt = __builtin_amdgcn_exp2f((top - ref) * c);
  l *= wgt;
  o *= wgt;
#pragma unroll
  for (int sh = kLanes; sh < 64; sh <<= 1) {
    l += __shfl_xor(l, sh);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], sh);
  }
  if (lane < kLanes) store_out<D>(a, u, d, o, l, ref);
}

// Windows are shared out while there are fewer workgroups than two per compute unit of a 256-CU part, into parts of at least
// two tiles per wave.
unsigned long long plan_paged_chosen(PagedChosenArgs &a, long long max_seqlen) {
  a.passes = (a.g + kColumns - 1) / kColumns;
  a.tokens = a.g >= kColumns || max_seqlen == 1 ? 1 : kColumns / a.g;
  a.tiles = !a.cu ? a.total : a.total / a.tokens + a.B;
  const long long units_past = a.total * a.n_past * a.passes, units_other = a.tiles * a.n_other * a.passes;
  const long long halves = (long long)a.n_chosen * a.block_halves.d;
  long long window = (long long)a.seg.d + a.tail + a.tokens;
  window = window < a.max_rows ? window : a.max_rows;
  const long long tiles_past = a.n_past ? (halves + 1) / 2 : 1, tiles_other = window / kChosenTile + 2;
  const long long wanted = 512, units = units_past + units_other;
  auto share = [&](long long tiles, int &parts, int &per_part) {
    long long p = units >= wanted ? 1 : wanted / units;
    const long long most = (tiles + 2 * kChosenWaves - 1) / (2 * kChosenWaves);
    p = p < most ? p : most;
    p = p < 1 ? 1 : p;
    per_part = (int)((tiles + p - 1) / p);
    parts = (int)((tiles + per_part - 1) / per_part);
  };
  share(tiles_past, a.parts_past, a.tiles_past);
  share(tiles_other, a.parts_other, a.tiles_other);
  a.wgs_past = units_past * a.parts_past;
  a.wgs_other = units_other * a.parts_other;
  unsigned long long slots = 0;
  if (a.parts_past > 1) slots += (unsigned long long)a.total * a.n_past * a.parts_past;
  if (a.parts_other > 1) slots += (unsigned long long)a.total * a.n_other * a.parts_other;
  return slots * a.g * ws_slot_floats(a.D) * 4ull;
}

template <int D>
static hipError_t launch_chosen(const PagedChosenArgs &a, hipStream_t st) {
  const auto kern = a.c.e4m3 ? paged_chosen_kernel<D, true> : paged_chosen_kernel<D, false>;
  hipError_t e = launch_in_parts(a.wgs_past + a.wgs_other, 64 * kChosenWaves, [&](long long first, unsigned count) {
    hipLaunchKernelGGL(kern, dim3(count), dim3(64 * kChosenWaves), 0, st, a, first);
  });
  if (e != hipSuccess || (a.parts_past == 1 && a.parts_other == 1)) return e;
  return launch_in_parts((a.total * a.Hq + 3) / 4, 256, [&](long long first, unsigned count) {
    hipLaunchKernelGGL(paged_chosen_join_kernel<D>, dim3(count), dim3(256), 0, st, a, first);
  });
}

hipError_t launch_paged_chosen(const PagedChosenArgs &a, hipStream_t st) { return a.D == 128 ? launch_chosen<128>(a, st) : launch_chosen<64>(a, st); }

}  // namespace segattn
