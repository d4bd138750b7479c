// seg_attn_paged_chosen: attention of new tokens over a paged cache, long-range heads over the blocks that a list names for each token.
//
// This file's kernel takes a token and a KV head: up to 16 query heads are columns (a group of more takes a pass per 16), with the rows of the
// listed blocks or of the window.  Per tile of 32 rows -- two halves of 16, each somewhere in the pool -- a wave forms
//   S^T[key][column] = K . Q^T            v_mfma_f32_16x16x32_bf16, A = K rows, B = Q^T (registers)
//   P = exp2((S^T - m) c)                 running maximum m and sum l per column, in fp32
//   O^T[d][column] += V^T . P^T           A = V^T via ds_read_b64_tr_b16, B = P from the S^T registers
// P enters as two bf16 (what that leaves is below 2^-16 of a weight), for fp32 outputs as three: the matrix pipes idle beside the memory.
// K and V go from memory to LDS through registers, a tile ahead, because the halves lie anywhere and 8-bit rows become bf16 on the way.  Bound by
// memory where the workgroups fill the card (48 sequences of 8-bit rows, two heads with 32 blocks of 64 and six with windows up to 5K rows:
// 58 us, 4.7 TB/s, of bf16 rows 98 us, 5.5 TB/s; without the windows' unequal lengths 6.3 to 6.7), else by latencies: row count -> list -> page ->
// tile, a second round of tiles, the waves' merge (one sequence's 64 blocks: 9 us and 4 to join).
#include <math.h>

#include <type_traits>

#include "segattn_paged_chosen.h"

namespace segattn {

template <int D, bool kE4m3>
__global__ __launch_bounds__(64 * kChosenWaves, 2) void paged_chosen_kernel(const PagedChosenArgs a, const long long first_wg) {
  constexpr int NK = D / 32, NB = D / 16;
  constexpr int kRow = 2 * D, kTileBytes = kChosenTile * kRow;  // of a tile in LDS, bf16
  constexpr int kPieces = (kE4m3 ? D : 2 * D) / 16;             // 16-byte pieces of a row in memory
  constexpr int RPL = 64 / kPieces, NL = kChosenTile / RPL;     // rows per wave load, loads per tile and tensor

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
  const long long token = u / parts;
  const int hx = past ? x : a.n_past + x, h = a.head_of[hx];
  int i, n;
  const int b = sequence_of(a.cu, a.B, token, i, n);
  if (b < 0) return;
  const long long w = (long long)b * a.Hkv + h;
  const int live = min(kColumns, a.g - pass * kColumns), head0 = h * a.g + pass * kColumns;  // columns, and the first one's query head
  int from, to;
  token_window(a, w, hx, i, n, from, to);

  const int *table = table_of(a.c, a.Hkv, b, h);
  const int *list = past ? a.chosen + (token * a.n_past + x) * a.n_chosen : nullptr;
  const int hh = a.c.per_head ? 0 : h;
  unsigned char *tile = tiles[wave];
  const unsigned char *scales = lane < 32 ? a.c.k_scale : a.c.v_scale;
  int koff[NK], voff[NB];
  const int vrow = 4 * quad + (col >> 2);
#pragma unroll
  for (int kc = 0; kc < NK; ++kc) koff[kc] = col * kRow + (chunk_k<D>(col, 4 * kc + quad) << 4);
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
    voff[nb] = kTileBytes + vrow * kRow + (chunk_v<D>(vrow, 2 * nb + ((col & 3) >> 1)) << 4) + 8 * (col & 1);

  bf16x8 Q[NK];  // column col, zero beyond the live ones
  {
    const unsigned short *q = a.q + (token * a.Hq + head0 + (col < live ? col : 0)) * D + 8 * quad;
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
      nk[l] = __builtin_nontemporal_load((const u32x4 *)(a.c.k + from_row + mine));
      nv[l] = __builtin_nontemporal_load((const u32x4 *)(a.c.v + from_row + mine));
    }
    if constexpr (kE4m3) {
      const long long at0 = of_lane(half_place, 2 * j), at1 = of_lane(half_place, 2 * j + 1);
      n_scale = scales[(lane & 16 ? at1 : at0) + (lane & 15)];
    }
  };
  // A tile into LDS, values of rows that do not count as zeros (a weight of zero times NaN would be NaN).
  auto stage = [&](unsigned valid) __attribute__((always_inline)) {
#pragma unroll
    for (int l = 0; l < NL; ++l) {
      const int r = RPL * l + lane / kPieces, piece = lane % kPieces;
      const u32x4 xk = nk[l], xv = nv[l];
      if constexpr (!kE4m3) {
        *(u32x4 *)(tile + r * kRow + (chunk_k<D>(r, piece) << 4)) = xk;
        *(u32x4 *)(tile + kTileBytes + r * kRow + (chunk_v<D>(r, piece) << 4)) = xv;
      } else {
        const float sk = __uint_as_float((unsigned)__shfl(n_scale, r) << 23), sv = __uint_as_float((unsigned)__shfl(n_scale, r + 32) << 23);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int chunk = 2 * piece + half;
          *(u32x4 *)(tile + r * kRow + (chunk_k<D>(r, chunk) << 4)) = bf16_of_e4m3(xk[2 * half], xk[2 * half + 1], sk);
          *(u32x4 *)(tile + kTileBytes + r * kRow + (chunk_v<D>(r, chunk) << 4)) = bf16_of_e4m3(xv[2 * half], xv[2 * half + 1], sv);
        }
      }
    }
    if (valid != ~0u && !((valid >> (lane & 31)) & 1)) {
#pragma unroll
      for (int e = 0; e < kRow / 32; ++e)
        *(u32x4 *)(tile + kTileBytes + (lane & 31) * kRow + (kRow / 32 * (lane >> 5) + e) * 16) = u32x4{0u, 0u, 0u, 0u};
    }
  };
  auto values = [&](int nb) __attribute__((always_inline)) {  // V^T, channels 16 nb ..
    const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4 *)(tile + voff[nb]));
    const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4 *)(tile + voff[nb] + 16 * kRow));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  auto products = [&](unsigned valid) __attribute__((always_inline)) {
    f32x4 S[2];
#pragma unroll
    for (int h2 = 0; h2 < 2; ++h2) {
      S[h2] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kc = 0; kc < NK; ++kc)
        S[h2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8 *)(tile + koff[kc] + 16 * h2 * kRow), Q[kc], S[h2], 0, 0, 0);
    }
    // register r of S[h2] is row 4 quad + r of half h2
    if (valid != ~0u) {
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (!((valid >> (16 * h2 + 4 * quad + r)) & 1)) S[h2][r] = -INFINITY;
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
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const bf16x8 va = values(nb);
      O[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, P, O[nb], 0, 0, 0);
      O[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, P_rest, O[nb], 0, 0, 0);
    }
    if (a.out_fp32) {
      bf16x8 P_tail;
#pragma unroll
      for (int e = 0; e < 8; ++e) P_tail[e] = (__bf16)tail[e / 4][e % 4];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) O[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values(nb), P_tail, O[nb], 0, 0, 0);
    }
  };

  // A window is shared out evenly, in whole rounds of the waves; a list by its length.
  const int all = past ? (int)(((long long)a.n_chosen * a.block_halves.d + 1) / 2) : to > 0 ? (to + kChosenTile - 1) / kChosenTile - from / kChosenTile : 0;
  const int per_part = past ? a.tiles_past : ((all + parts - 1) / parts + kChosenWaves - 1) / kChosenWaves * kChosenWaves;
  const int t_begin = min(part * per_part, all), t_end = min(t_begin + per_part, all);
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
      const unsigned valid = half_bits(n_row0, from, to) | half_bits(n_row1, from, to) << 16;
      stage(valid);
      const bool more = some != 0;
      if (more) {
        j = (int)__builtin_ctzll(some) >> 1;
        some &= some - 1;
        fetch(j);
      }
      products(valid);
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
    if (parts == 1) {
      store_out<D>(a, token * a.Hq + head0 + column, d, o, l, ref * c);
    } else {
      float *dst = partial_of<D>(a, past, token, x, part) + (pass * kColumns + column) * ws_slot_floats(D);
      *(f32x4 *)(dst + d) = o;
      if (d == 0) *(float2 *)(dst + D) = float2{top * c, l};
    }
  }
}

// A wave per (token, query head) whose window was shared out: the parts' partials joined.  (They are few: a window is shared out only where there
// are fewer than kResident units.  One sequence's 32 heads 4.3 us, with four of them one after the other in a wave 10.4.)
template <int D>
__global__ __launch_bounds__(256) void paged_chosen_join_kernel(const PagedChosenArgs a, const int hx0, const int heads, const long long first_wg) {
  constexpr int SF = D + kWsTailFloats, kLanes = D / 4, kGroups = 64 / kLanes, kBatch = 4;
  const int lane = threadIdx.x & 63;
  const long long wave = (first_wg + blockIdx.x) * 4 + (threadIdx.x >> 6), u = wave / a.g, token = u / heads;
  if (token >= a.total) return;
  const int j = (int)(wave - u * a.g);
  const int hx = hx0 + (int)(u - token * heads), h = a.head_of[hx];
  const bool past = hx < a.n_past;
  const int parts = past ? a.parts_past : a.parts_other;
  int i, n;
  if (sequence_of(a.cu, a.B, token, i, n) < 0) return;
  const int group = lane / kLanes, d = lane % kLanes * 4;
  const float *src = partial_of<D>(a, past, token, past ? hx : hx - a.n_past, 0) + j * SF;
  float top = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = group; s0 - group < parts; s0 += kGroups * kBatch) {
    float2 ml[kBatch];
    f32x4 y[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int s = s0 + kGroups * k;
      const float *part = src + (long long)(s < parts ? s : parts - 1) * a.g * SF;
      ml[k] = *(const float2 *)(part + D);
      y[k] = *(const f32x4 *)(part + d);
    }
    float m_new = top;
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (s0 + kGroups * k < parts) m_new = fmaxf(m_new, ml[k].x);
    const float ref = m_new == -INFINITY ? 0.f : m_new, keep = __builtin_amdgcn_exp2f(top - ref);
    l *= keep;
    o *= keep;
    top = m_new;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      if (s0 + kGroups * k < parts) {
        const float wgt = __builtin_amdgcn_exp2f(ml[k].x - ref);
        l += ml[k].y * wgt;
        o += y[k] * wgt;
      }
    }
  }
  float most = top;
#pragma unroll
  for (int sh = kLanes; sh < 64; sh <<= 1) most = fmaxf(most, __shfl_xor(most, sh));
  const float ref = most == -INFINITY ? 0.f : most, wgt = __builtin_amdgcn_exp2f(top - ref);
  l *= wgt;
  o *= wgt;
#pragma unroll
  for (int sh = kLanes; sh < 64; sh <<= 1) {
    l += __shfl_xor(l, sh);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], sh);
  }
  if (lane < kLanes) store_out<D>(a, token * a.Hq + h * a.g + j, d, o, l, ref);
}

constexpr long long kListedSpace = 1ll << 30;  // bytes of partials of listed blocks at a time
constexpr long long kMostKeys = 1ll << 27;     // (sequence, PAST head, block): two words for each
constexpr long long kResident = 512;  // workgroups: two per compute unit of a 256-CU part
constexpr int kListedColumns = 384;

constexpr double kListedLaunches = 30;  // us
double row_bytes(const PagedChosenArgs &a) { return 2.0 * a.D * (a.c.e4m3 ? 1 : 2); }  // keys and values

// Bytes of partials that an entry of a list leaves.
long long entry_bytes(const PagedChosenArgs &a) { return (long long)a.listed_pieces * a.g * (a.D + 2) * 4; }

// Whether listed blocks are turned round and taken one by one, by how long both ways take (us).  Token by token: rounds of resident workgroups,
// 32 rows of a wave at a time as they come from memory, or what all rows together need of the caches.  Block by block: the launches before and
// behind, the partials written and read, and each row once.  Measured, both in us, eight KV heads of a 60K history in blocks of 64, 32 listed: 64
// tokens of four query heads a KV head 66 and 76, 128 tokens 125 and 98, 400 tokens 388 and 155 (8-bit rows: 128 tokens 74 and 86, 400
// tokens 222 and 137; heads of 64: 59 and 61, 176 and 94; one query head each: 64 tokens 66 and 64, 400 tokens 377 and 92); of an 8K history, 64
// tokens 39 and 47, 128 tokens 73 and 65; two KV heads of eight query heads, 128 tokens 38 and 56, 400 tokens 114 and 84.
bool blocks_one_by_one(const PagedChosenArgs &a, double parts, double tiles) {
  const double row = row_bytes(a), block = 16.0 * a.block_halves.d * row;
  const double entries = (double)a.total * a.n_past * a.n_chosen, listed = entries * block, all = (double)a.B * a.n_past * a.blocks * block;
  const double units = (double)a.total * a.n_past * a.passes * parts;
  const double rounds = ceil(units / kResident) * ceil(tiles / kChosenWaves) * 3.2 * row / 512;
  const double bytes = listed / (all <= 40e6 ? 14.5e6 : 8.5e6);
  const double partials = entries * entry_bytes(a);
  return kListedLaunches + (2 * partials + (listed < all ? listed : all)) / 5e6 < (rounds > bytes ? rounds : bytes);
}

// Of the windows: launches, in us, and a tile of a token, or of a unit, in us.
constexpr double kAloneLaunches = 10, kSharedLaunches = 38;
double alone_tile(const PagedChosenArgs &a) { return (0.5 + 0.9 * row_bytes(a) / 512) * 1e-3; }
double shared_tile(const PagedChosenArgs &a) { return (1.8 + row_bytes(a) / 512) * 1e-3; }

// Whether the windows of several tokens a sequence share their tiles, by how long both ways take (us, with the longest window's tiles): 128 columns
// cost what they cost however few of them are tokens', but single tokens read the rows anew, from the caches if that.  Measured, alone and
// shared, in us, windows up to 5K rows: a 130K history, eight heads, 4 tokens 16 and 31, 16 tokens 27 and 36, 32 tokens 40 and 39, 64 tokens 60 and
// 42; 48 sequences of 8-bit rows, six heads of eight, 2 tokens 114 and 158, 3 tokens 158 and 167, 4 tokens 201 and 172 (bf16 rows: 186
// and 174, 272 and 197 for three); eight of them, 4 tokens 45 and 55, 8 tokens 68 and 61.
bool windows_share_tiles(const PagedChosenArgs &a, double tiles) {
  const double bytes = row_bytes(a), alone = (double)a.total * a.n_other * tiles;
  const double shared = (double)a.n_other * (a.cu ? (double)a.total / a.wide_tokens + a.B : (double)a.total) * tiles;
  const double cached = (double)a.B * a.n_other * tiles * kChosenTile * bytes <= 40e6 ? 0.6 : 1;
  return kAloneLaunches + alone * cached * alone_tile(a) > kSharedLaunches + shared * shared_tile(a);
}

// What a plan needs of the workspace.
struct ChosenSpace {
  unsigned long long partials = 0;  // of (token, head)s whose rows are shared out, g query heads each
  unsigned long long shares = 0;    // of windows
  unsigned long long keys = 0, entries = 0;
};
unsigned long long lay_out(PagedChosenArgs &a, const ChosenSpace &s, unsigned char *ws) {
  unsigned long long at = 0;
  const auto take = [&](auto *&x, unsigned long long count) {
    x = reinterpret_cast<std::remove_reference_t<decltype(x)>>(ws + at);
    at += (count * sizeof(*x) + 255) / 256 * 256;
  };
  take(a.slots, s.partials * a.g * ws_slot_floats(a.D));
  take(a.splits, s.shares);
  take(a.wide_slots, 2 * s.shares * kWideColumns * ws_slot_floats(a.D));
  if (s.entries == 0) return at;
  take(a.cursors, s.keys + 2);
  a.counts = a.cursors + 2;
  take(a.offsets, s.keys);
  take(a.rank, s.entries);
  take(a.sorted, s.entries);
  take(a.tasks, s.entries / a.listed_tokens + (s.entries < s.keys ? s.entries : s.keys));
  take(a.listed_out, s.entries * a.listed_pieces * a.g * a.D);
  take(a.listed_sum, s.entries * a.listed_pieces * a.g);
  return at;
}

// Key tiles of a list, and of the longest window.
struct ChosenTiles {
  long long past, other;
};
ChosenTiles count_tiles(const PagedChosenArgs &a) {
  const long long halves = (long long)a.n_chosen * a.block_halves.d;
  long long window = (long long)a.seg.d + a.tail + a.wide_tokens;
  window = window < a.max_rows ? window : a.max_rows;
  return {a.n_past ? (halves + 1) / 2 : 1, window / kChosenTile + 2};
}
bool many_tokens(const PagedChosenArgs &a, long long max_seqlen) { return max_seqlen > 1 && a.g <= kColumns; }
constexpr long long kLeastPart = 2 * kChosenWaves;  // tiles
// Shares at most: as many workgroups as can be resident (D = 64: three on a compute unit, or two, by the form's registers).
long long shares_at_most(const PagedChosenArgs &a) { return a.D == 128 ? kResident : kResident * 3 / 2; }
// Shares that as many units can be cut into.
long long most_shares(long long units, long long tiles, long long resident) {
  if (units >= resident) return resident;
  const long long most = units * (2 * tiles + kUnitTiles) / kLeastShare + 1;
  return most < resident ? (most + 7) / 8 * 8 : resident;
}

unsigned long long plan_paged_chosen(PagedChosenArgs &a, long long max_seqlen, unsigned char *ws) {
  ChosenSpace space;
  a.passes = (a.g + kColumns - 1) / kColumns;
  const bool many = many_tokens(a, max_seqlen);
  a.wide_tokens = many ? kWideColumns / a.g : 1;
  a.listed_tokens = kListedColumns / a.g > 0 ? kListedColumns / a.g : 1;
  const int block_rows = 16 * (int)a.block_halves.d;
  a.blocks = (int)(((long long)a.max_rows + block_rows - 1) / block_rows);
  a.listed_pieces = (block_rows + kListedRows - 1) / kListedRows;
  long long units_past = a.total * a.n_past * a.passes;
  const ChosenTiles tiles = count_tiles(a);
  a.wide_windows = many && a.n_other > 0 && windows_share_tiles(a, tiles.other);
  a.wide_tiles = a.cu ? a.total / a.wide_tokens + a.B : a.total;
  const long long units_other = a.n_other * (a.wide_windows ? a.wide_tiles : a.total * a.passes);
  const long long units = units_past + (a.wide_windows ? 0 : units_other);
  // Windows are shared out while there are fewer workgroups than two per compute unit of a 256-CU part.
  auto share = [&](long long tiles, long long p, int &parts, int &per_part) {
    const long long most = tiles / kLeastPart;
    p = p < most ? p : most;
    p = p < 1 ? 1 : p;
    per_part = (int)((tiles + p - 1) / p);
    parts = (int)((tiles + per_part - 1) / per_part);
  };
  const long long narrow = units >= kResident || units == 0 ? 1 : kResident / units;
  share(tiles.past, narrow, a.parts_past, a.tiles_past);
  const long long keys = (long long)a.B * a.n_past * a.blocks, per_token = (long long)a.n_past * a.n_chosen, at_once = kListedSpace / entry_bytes(a);
  a.by_block = many && a.n_past > 0 && keys <= kMostKeys && per_token <= at_once && blocks_one_by_one(a, a.parts_past, a.tiles_past);
  // (windows are of all lengths up to the longest: twice as many, so that it is not waited for: 48 sequences of 8-bit rows 65 us with a workgroup each
  // and 60 with four, 30 of them 44 and 43, eight 20 and 23)
  const long long ragged = units >= kResident || units == 0 ? 1 : (kResident * 2 + units - 1) / units;
  share(tiles.other, a.wide_windows ? 1 : ragged, a.parts_other, a.tiles_other);
  if (a.by_block) {
    a.parts_past = 1;
    units_past = 0;
  }
  a.wgs_past = units_past * a.parts_past;
  a.wgs_other = units_other * a.parts_other;
  if (a.parts_past > 1) space.partials += (unsigned long long)a.total * a.n_past * a.parts_past;
  if (a.parts_other > 1) space.partials += (unsigned long long)a.total * a.n_other * a.parts_other;
  if (a.wide_windows) {
    // Shares of equal length for as many workgroups as are resident, but where the units alone are several rounds of them, a workgroup for
    // each (8 heads with windows up to 5K, up to as many new tokens: 2048 326 us in shares and 454 by units, 8192 991 and 975, 16384 1998 and 1901).
    // The runtime is asked how many are: heads of 64, bf16 pages, fp32 outputs have two on a compute unit (2048 tokens in 768 shares 165 us, in 512
    // 143), the other forms of 64 three.
    // (Without a workspace the question is only how large one may be: nothing is asked.)
    const long long most = shares_at_most(a), asked = ws ? windows_resident(a) : most, resident = asked < 8 ? kResident : asked < most ? asked / 8 * 8 : most;
    a.wide_wgs = units_other < 4 * resident ? (int)most_shares(units_other, tiles.other, resident) : 0;
    space.shares = a.wide_wgs;
  }
  if (a.by_block) {
    const long long part = at_once / per_token;
    a.part_tokens = (int)(part < a.total ? part : a.total);
    space.keys = keys;
    space.entries = a.part_tokens * per_token;
  }
  return lay_out(a, space, ws);
}

// Room for this call and every smaller one: with fewer tokens (in all, of a sequence), sequences, rows or listed blocks, which may take other
// forms.  So a form counts where what it saves, without what it costs, lets any of them take it; what it then needs grows with the sizes.
unsigned long long most_paged_chosen(PagedChosenArgs a, long long max_seqlen) {
  const bool many = many_tokens(a, max_seqlen);
  const ChosenTiles tiles = count_tiles(a);
  ChosenSpace space;
  // Rows are shared out while there are fewer than kResident units of the passes: lists in kResident / units parts, windows in 2 kResident / units,
  // rounded up, so that all parts together are fewer than 3 kResident.
  const auto parts = [](long long tiles) { return tiles / kLeastPart > 1 ? tiles / kLeastPart : 0; };
  const long long cut = a.total * (a.n_past * parts(tiles.past) + a.n_other * parts(tiles.other)), most_cut = 3 * kResident / a.passes + 1;
  space.partials = cut < most_cut ? cut : most_cut;
  const double alone = (double)a.total * a.n_other * tiles.other;
  if (many && a.n_other > 0 && kAloneLaunches + alone * (alone_tile(a) - shared_tile(a) / a.wide_tokens) > kSharedLaunches)
    space.shares = most_shares(a.n_other * (a.total / a.wide_tokens + a.B), tiles.other, shares_at_most(a));
  const double rounds = ceil((double)a.total * a.n_past * a.passes / kResident) * ceil((double)tiles.past / kChosenWaves) * 3.2 * row_bytes(a) / 512;
  const double listed = (double)a.total * a.n_past * a.n_chosen * 16.0 * a.block_halves.d * row_bytes(a) / 8.5e6;
  if (many && a.n_past > 0 && kListedLaunches < (rounds > listed ? rounds : listed)) {
    const long long keys = (long long)a.B * a.n_past * a.blocks, entries = a.total * a.n_past * a.n_chosen, at_once = kListedSpace / entry_bytes(a);
    space.keys = keys < kMostKeys ? keys : kMostKeys;
    space.entries = entries < at_once ? entries : at_once;
  }
  return lay_out(a, space, nullptr);
}

template <int D>
static hipError_t launch_chosen(const PagedChosenArgs &a, hipStream_t st) {
  hipError_t e = hipSuccess;
  if (a.by_block && (e = launch_paged_listed(a, st)) != hipSuccess) return e;
  if (a.wide_windows && (e = launch_paged_windows(a, st)) != hipSuccess) return e;
  const auto kern = a.c.e4m3 ? paged_chosen_kernel<D, true> : paged_chosen_kernel<D, false>;
  e = launch_in_parts(a.wgs_past + (a.wide_windows ? 0 : a.wgs_other), 64 * kChosenWaves, [&](long long first, unsigned count) {
    hipLaunchKernelGGL(kern, dim3(count), dim3(64 * kChosenWaves), 0, st, a, first);
  });
  const int hx0 = a.parts_past > 1 ? 0 : a.n_past, heads = (a.parts_other > 1 ? a.Hkv : a.n_past) - hx0;
  if (e != hipSuccess || heads <= 0) return e;
  return launch_in_parts((a.total * heads * a.g + 3) / 4, 256, [&](long long first, unsigned count) {
    hipLaunchKernelGGL(paged_chosen_join_kernel<D>, dim3(count), dim3(256), 0, st, a, hx0, heads, first);
  });
}

hipError_t launch_paged_chosen(const PagedChosenArgs &a, hipStream_t st) { return a.D == 128 ? launch_chosen<128>(a, st) : launch_chosen<64>(a, st); }

}  // namespace segattn
