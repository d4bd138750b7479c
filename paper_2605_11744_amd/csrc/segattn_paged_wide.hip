// seg_attn_paged_chosen, many tokens at a time: the waves of a workgroup share keys and values in LDS, and each has query columns of
// its own, 32 of them (16 for listed blocks), in the arithmetic of the kernel for single tokens.
//
// Windows: the columns are the query heads of neighbouring tokens, the rows all that one of them sees.  Listed blocks, where
// the tokens of a sequence are so many that a block is listed by several of them: the columns are the heads of tokens that
// list one block, whose rows are read once for all of them; a token's lists are turned round first (count, place, sort), each
// (token, entry) leaves a partial (acc[D], m, l) per query head, and a last launch joins a token's partials.  Which
// token lands in which column depends on the order of atomics, but no column's numbers depend on its neighbours.
//
// A chunk of 2533 tokens behind up to 60K rows, eight KV heads of four query heads, half of them long-range with 32 blocks of 64 rows: windows 185 us
// and 16 to join (73 GFLOP, 395 TFLOP/s: eight waves a compute unit do not hide a tile's chain of scores, maximum, exponentials and products),
// listed blocks 221 (0.68 GB of partials written, 3.1 TB/s), their join 119 (read, 5.7 TB/s), turning the lists round 40.
#include "segattn_paged_chosen.h"

namespace segattn {

constexpr int kListedThreads = 256;
constexpr int kWideThreads = 256;

// ---- lists turned round -------------------------------------------------------------------------
// Entry e of the list of the part's token t0 + u / n_past, head u % n_past: its key (sequence, head, block), or -1 if there is nothing to
// see; its index is u * n_chosen + e.
__device__ inline int entry_key(const PagedChosenArgs &a, int u, int e, bool ask_page) {
  const int x = u % a.n_past;
  const long long token = a.part0 + u / a.n_past;
  int i, n;
  const int b = sequence_of(a.cu, a.B, token, i, n);
  if (b < 0) return -1;
  const int block = a.chosen[(token * a.n_past + x) * a.n_chosen + e];
  const int h = a.head_of[x];
  const int to = rows_seen(a.rows, (long long)b * a.Hkv + h, i, n, a.max_rows);
  const int br = 16 * (int)a.block_halves.d;
  if (block < 0 || (long long)block * br >= to) return -1;
  if (ask_page) {
    int in_page;
    if (page_of(a.c, table_of(a.c, a.Hkv, b, h), block * br, in_page) < 0) return -1;
  }
  return (b * a.n_past + x) * a.blocks + block;
}
__global__ __launch_bounds__(256) void paged_clear_kernel(int *x, int n) {
  for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) x[i] = 0;
}
// A wave takes an entry of 64 lists of one head that belong to neighbouring tokens: they often name the same block (the first, the
// newest), and one lane counts for all that name the block of the first lane.
__device__ inline bool entry_of_thread(const PagedChosenArgs &a, int units, int &u, int &e) {
  const long long wave = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, groups = (units / a.n_past + 63) / 64;
  e = (int)(wave % a.n_chosen);
  const int rest = (int)(wave / a.n_chosen), x = rest % a.n_past, token = rest / a.n_past * 64 + lane;
  u = token * a.n_past + x;
  return rest / a.n_past < groups && token < units / a.n_past;
}
__global__ __launch_bounds__(256) void paged_count_kernel(const PagedChosenArgs a, const int units) {
  int u, e;
  const bool is = entry_of_thread(a, units, u, e);
  const int lane = threadIdx.x & 63, key = is ? entry_key(a, u, e, true) : -1;
  // who counts for this lane, and its number among those it counts for
  int leader = lane, before = 0, count = 1;
  unsigned long long left = __builtin_amdgcn_ballot_w64(key >= 0);
  for (int round = 0; round < 3 && left; ++round) {
    const int first = (int)__builtin_ctzll(left);
    const unsigned long long same = __builtin_amdgcn_ballot_w64(key == __builtin_amdgcn_readlane(key, first)) & left;
    if ((same >> lane) & 1) {
      leader = first;
      before = __popcll(same & ((1ull << lane) - 1));
      count = __popcll(same);
    }
    left &= ~same;
  }
  int rank = 0;
  if (key >= 0 && leader == lane) rank = atomicAdd(a.counts + key, count);
  rank = __shfl(rank, leader) + before;
  rank = key < 0 ? -1 : rank;
  if (is) a.rank[(long long)u * a.n_chosen + e] = rank;
}
// Places for every block's entries, and the workgroups' tasks: (key, first entry of it, entries).
__global__ __launch_bounds__(256) void paged_place_kernel(const PagedChosenArgs a, const int keys) {
  const int key = blockIdx.x * 256 + threadIdx.x, lane = threadIdx.x & 63;
  const int n = key < keys ? a.counts[key] : 0, tasks = (n + a.listed_tokens - 1) / a.listed_tokens;
  int sum = n, sum_tasks = tasks;
#pragma unroll
  for (int sh = 1; sh < 64; sh <<= 1) {
    const int up = __shfl_up(sum, sh), up_tasks = __shfl_up(sum_tasks, sh);
    if (lane >= sh) {
      sum += up;
      sum_tasks += up_tasks;
    }
  }
  int base = 0, base_tasks = 0;
  if (lane == 63 && sum > 0) {
    base = atomicAdd(a.cursors, sum);
    base_tasks = atomicAdd(a.cursors + 1, sum_tasks);
  }
  base = __shfl(base, 63) + sum - n;
  base_tasks = __shfl(base_tasks, 63) + sum_tasks - tasks;
  if (n == 0) return;
  a.offsets[key] = base;
  const int each = (n + tasks - 1) / tasks;
  for (int i = 0; i < tasks; ++i) a.tasks[base_tasks + i] = int4{key, base + i * each, min(each, n - i * each), 0};
}
__global__ __launch_bounds__(256) void paged_sort_kernel(const PagedChosenArgs a, const int units) {
  int u, e;
  if (!entry_of_thread(a, units, u, e)) return;
  const long long entry = (long long)u * a.n_chosen + e;
  const int rank = a.rank[entry], key = rank < 0 ? -1 : entry_key(a, u, e, false);
  if (key >= 0) a.sorted[a.offsets[key] + rank] = (int)entry;
}

// ---- arithmetic ------------------------------------------------------------------------------
// A wave's 32 columns, as two groups of 16: column col of group g in the lanes with lane % 16 = col.
__device__ inline unsigned two_bf16(float x, float y) {
  return __builtin_bit_cast(unsigned, bf16x2{(__bf16)x, (__bf16)y});
}
__device__ inline float low_of(unsigned x) { return __uint_as_float(x << 16); }
__device__ inline float high_of(unsigned x) { return __uint_as_float(x & 0xffff0000u); }

template <int D, bool kFp32, int NG>
struct WaveColumns {
  static constexpr int NK = D / 32, NB = D / 16, kRow = 2 * D;
  // How much a column's maximum may grow, in powers of two, before what was summed so far is scaled to the new one: weights up to 2^8 are
  // as exact as those up to 1.  (With every new maximum: a third of a window's tiles scale 64 registers.)
  static constexpr float kLag = 8.f;
  bf16x8 Q[NG][NK];
  f32x4 O[NG][NB];
  float m[NG], l[NG];  // maximum that the sums are relative to, as an exponent of two, and the lane's part of the sum

  __device__ __attribute__((always_inline)) void load(int g, const unsigned short *q, bool is) {
#pragma unroll
    for (int kc = 0; kc < NK; ++kc) {
      u32x4 y = *(const u32x4 *)(q + 32 * kc);
      if (!is) y = u32x4{0u, 0u, 0u, 0u};
      Q[g][kc] = __builtin_bit_cast(bf16x8, y);
    }
  }
  __device__ __attribute__((always_inline)) void clear() {
#pragma unroll
    for (int g = 0; g < NG; ++g) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) O[g][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
      m[g] = -INFINITY;
      l[g] = 0.f;
    }
  }
  // One tile of 32 rows in LDS: keys at `keys`, values at `keys` + values.  masked: lane's column of group g sees the rows [from, to) of row0 ..
  // and row1 .. (the two halves' first rows; beyond every `to` where there are none).
  __device__ __attribute__((always_inline)) void tile(const unsigned char *keys, const int (&koff)[NK], const int (&voff)[NB], float c, bool masked,
                                                      int row0, int row1, const int (&from)[NG], const int (&to)[NG]) {
    const int quad = (threadIdx.x >> 4) & 3;
    auto values = [&](int nb) __attribute__((always_inline)) {  // V^T, channels 16 nb ..
      const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4 *)(keys + voff[nb]));
      const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4 *)(keys + voff[nb] + 16 * kRow));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    f32x4 S[NG][2];
#pragma unroll
    for (int g = 0; g < NG; ++g) S[g][0] = S[g][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
      for (int kc = 0; kc < NK; ++kc) {
        const bf16x8 k = *(const bf16x8 *)(keys + koff[kc] + 16 * h2 * kRow);
#pragma unroll
        for (int g = 0; g < NG; ++g) S[g][h2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, Q[g][kc], S[g][h2], 0, 0, 0);
      }
    // register r of S[.][h2] is row 4 quad + r of half h2
    if (masked) {
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2) {
          const int row = (h2 ? row1 : row0) + 4 * quad;
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (row + r < from[g] || row + r >= to[g]) S[g][h2][r] = -INFINITY;
        }
    }
    u32x4 P[NG], P_rest[NG], P_tail[NG];  // eight bf16 each
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      // scores as exponents of two from here on
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[g][h2][r] *= c;
      float mx = fmaxf(fmaxf(fmaxf(S[g][0][0], S[g][0][1]), fmaxf(S[g][0][2], S[g][0][3])), fmaxf(fmaxf(S[g][1][0], S[g][1][1]), fmaxf(S[g][1][2], S[g][1][3])));
      mx = over_quads(mx, false);
      // (also where a first row is seen: infinite.  Column by column: which one lies beside it must not show in a column's roundings)
      const bool grows = mx - m[g] > kLag;
      if (__builtin_amdgcn_ballot_w64(grows)) {
        const float alpha = grows ? __builtin_amdgcn_exp2f(m[g] - mx) : 1.f;
        m[g] = grows ? mx : m[g];
        l[g] *= alpha;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) O[g][nb] *= alpha;
      }
      const float ref = m[g] == -INFINITY ? 0.f : m[g];
      float sum = 0.f;
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
          const int at = 2 * h2 + r / 2;
          const float x = __builtin_amdgcn_exp2f(S[g][h2][r] - ref), y = __builtin_amdgcn_exp2f(S[g][h2][r + 1] - ref);
          sum += x + y;
          P[g][at] = two_bf16(x, y);
          const float x_rest = x - low_of(P[g][at]), y_rest = y - high_of(P[g][at]);
          P_rest[g][at] = two_bf16(x_rest, y_rest);
          if constexpr (kFp32) P_tail[g][at] = two_bf16(x_rest - low_of(P_rest[g][at]), y_rest - high_of(P_rest[g][at]));
        }
      l[g] += sum;
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const bf16x8 va = values(nb);
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        O[g][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, __builtin_bit_cast(bf16x8, P[g]), O[g][nb], 0, 0, 0);
        O[g][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, __builtin_bit_cast(bf16x8, P_rest[g]), O[g][nb], 0, 0, 0);
        if constexpr (kFp32) O[g][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, __builtin_bit_cast(bf16x8, P_tail[g]), O[g][nb], 0, 0, 0);
      }
    }
  }
  // Values of row `row` that are not finite (v: the row in memory), for the columns that see it: whatever weight it has, the sum is not finite with
  // them, and as a product's operand they would also make NaN of the columns that weigh them with zero: tiles hold zeros in their places.
  template <bool kE4m3>
  __device__ __attribute__((always_inline)) void odd_values(const unsigned char *v, float scale, int row, const int (&from)[NG], const int (&to)[NG]) {
    const int quad = (threadIdx.x >> 4) & 3;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int d = 16 * nb + 4 * quad;
      u32x4 y = {0u, 0u, 0u, 0u};
      if constexpr (kE4m3) {
        y = bf16_of_e4m3(*(const unsigned *)(v + d), 0u, scale);
      } else {
        y[0] = *(const unsigned *)(v + 2 * d);
        y[1] = *(const unsigned *)(v + 2 * d + 4);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float z = __uint_as_float(e & 1 ? y[e / 2] & 0xffff0000u : y[e / 2] << 16);
#pragma unroll
        for (int g = 0; g < NG; ++g)
          if (!(fabsf(z) < INFINITY) && row >= from[g] && row < to[g]) O[g][nb][e] += z;
      }
    }
  }
};

// Where a lane reads its operands in a tile whose values lie `values` bytes behind its keys.
template <int D>
__device__ inline void operand_places(int values, int (&koff)[D / 32], int (&voff)[D / 16]) {
  const int lane = threadIdx.x & 63, quad = lane >> 4, col = lane & 15, vrow = 4 * quad + (col >> 2);
#pragma unroll
  for (int kc = 0; kc < D / 32; ++kc) koff[kc] = col * 2 * D + (chunk_k<D>(col, 4 * kc + quad) << 4);
#pragma unroll
  for (int nb = 0; nb < D / 16; ++nb) voff[nb] = values + vrow * 2 * D + (chunk_v<D>(vrow, 2 * nb + ((col & 3) >> 1)) << 4) + 8 * (col & 1);
}

// 16 bytes of a row of keys or values into LDS as bf16 (two chunks of an 8-bit row); zero: as zeros.  odd: values that are not finite become
// zeros too; returns whether there were some.
template <int D, bool kE4m3>
__device__ __attribute__((always_inline)) bool stage_piece(unsigned char *dst, int row, int piece, u32x4 x, int scale_byte, bool is_v, bool zero, bool odd) {
  bool any = false;
#pragma unroll
  for (int half = 0; half < (kE4m3 ? 2 : 1); ++half) {
    const int chunk = kE4m3 ? 2 * piece + half : piece;
    u32x4 y = x;
    if constexpr (kE4m3) y = bf16_of_e4m3(x[2 * half], x[2 * half + 1], __uint_as_float((unsigned)scale_byte << 23));
    if (zero) y = u32x4{0u, 0u, 0u, 0u};
    if (odd) any |= without_odd(y);
    *(u32x4 *)(dst + row * 2 * D + ((is_v ? chunk_v<D>(row, chunk) : chunk_k<D>(row, chunk)) << 4)) = y;
  }
  return any;
}

// ---- windows ---------------------------------------------------------------------------------
// A unit: the heads of wide_tokens neighbouring tokens in one window; its tiles are those that one of the tokens sees.
struct WindowUnit {
  int x, b, i, n, tokens;  // the head of the set; sequence (-1: none), first token in it, its tokens; tokens of the unit
  int all, some;           // tiles; the first ones, which only some of the tokens see (behind the start of a segment in the unit's middle)
  int cost;                // in tiles: those of `some` count one and a half times (their masks, and a look for values that are not finite)
  __device__ int tile_at(int at) const {  // the first tile of a piece that begins at `at`
    at = max(at - kUnitTiles, 0);
    return at < some + some / 2 ? at * 2 / 3 : at - some / 2;
  }
};
__device__ inline WindowUnit window_unit(const PagedChosenArgs &a, long long u) {
  WindowUnit r;
  r.x = (int)(u / a.wide_tiles);
  r.b = tile_of(a, u - r.x * a.wide_tiles, a.wide_tokens, r.i, r.n);
  r.tokens = r.all = r.some = r.cost = 0;
  if (r.b < 0) return r;
  r.tokens = min(a.wide_tokens, r.n - r.i);
  const int hx = a.n_past + r.x;
  const long long w = (long long)r.b * a.Hkv + a.head_of[hx];
  int from, last_from, to;
  token_window(a, w, hx, r.i, r.n, from, to);
  token_window(a, w, hx, r.i + r.tokens - 1, r.n, last_from, to);
  r.all = to > 0 ? (to + kChosenTile - 1) / kChosenTile - from / kChosenTile : 0;
  r.some = min((last_from + kChosenTile - 1) / kChosenTile - from / kChosenTile, r.all);
  r.cost = kUnitTiles + r.all + r.some / 2;
  return r;
}
// The units' tiles, one unit after the other, are cut into shares of one length, a workgroup each: windows are of all lengths, and with a
// workgroup for each of them, or for halves, the part waits for the longest (2500 tokens, four heads with windows up to 5K: 281 us and 26 to
// join in halves, 185 and 16 in shares).  Each workgroup finds its own: the threads sum up the units' costs, then lanes search the units
// of the thread in whose sum the share begins.
struct WindowShare {
  long long unit, at;     // the first unit, and where it begins in the order of all tiles
  long long begin, end;   // of the share
  long long length;
};
__device__ inline WindowShare window_share(const PagedChosenArgs &a, long long index) {
  __shared__ long long sm_sum[kWideThreads / 64], sm_start[2];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const long long units = a.wgs_other, each = (units + kWideThreads - 1) / kWideThreads;
  long long sum = 0;
  for (long long u = tid * each; u < min(units, (tid + 1) * each); ++u) sum += window_unit(a, u).cost;
  long long before = sum;
#pragma unroll
  for (int sh = 1; sh < 64; sh <<= 1) {
    const long long up = __shfl_up(before, sh);
    if (lane >= sh) before += up;
  }
  if (lane == 63) sm_sum[wave] = before;
  before -= sum;
  __syncthreads();
  long long all = 0;
  for (int y = 0; y < kWideThreads / 64; ++y) {
    if (y < wave) before += sm_sum[y];
    all += sm_sum[y];
  }
  all = of_lane(all, 0);  // (the same in all lanes: scalar registers)
  WindowShare s;
  s.length = max((all + a.wide_wgs - 1) / a.wide_wgs, (long long)kLeastShare);
  s.begin = index * s.length;
  s.end = min(s.begin + s.length, all);
  if (before <= s.begin && s.begin < before + sum) {  // (one thread, if the share is not empty)
    sm_start[0] = tid * each;
    sm_start[1] = before;
  }
  __syncthreads();
  s.unit = 0;
  s.at = s.end;
  if (s.begin >= s.end) return s;
  s.unit = of_lane(sm_start[0], 0);
  s.at = of_lane(sm_start[1], 0);
  while (each > 1 && s.unit < units) {
    const long long cost = s.unit + lane < units ? window_unit(a, s.unit + lane).cost : 0;
    long long upto = cost;
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) {
      const long long up = __shfl_up(upto, sh);
      if (lane >= sh) upto += up;
    }
    const unsigned long long behind = __builtin_amdgcn_ballot_w64(s.at + upto > s.begin);
    if (behind) {
      const int l = (int)__builtin_ctzll(behind);
      s.unit += l;
      s.at += of_lane(upto - cost, l);
      return s;
    }
    s.unit += 64;
    s.at += of_lane(upto, 63);
  }
  return s;
}
// The piece of a unit that share k has leaves its partials [column][ws_slot_floats(D)] in slot 2 k, or 2 k + 1 if it is the unit's first piece.
template <int D>
__device__ inline float *window_slot(const PagedChosenArgs &a, long long slot) {
  return a.wide_slots + slot * kWideColumns * ws_slot_floats(D);
}

// kShares: a share of all units' tiles, else one unit.
template <int D, bool kE4m3, bool kFp32, bool kShares>
__global__ __launch_bounds__(kWideThreads, 2) void paged_windows_kernel(const PagedChosenArgs a, const long long first_wg) {
  constexpr int NG = 2, kWaveColumns = 16 * NG, kWaves = kWideThreads / 64, NK = D / 32, NB = D / 16;
  constexpr int kRow = 2 * D, kTileBytes = kChosenTile * kRow;
  constexpr int kPieces = (kE4m3 ? D : 2 * D) / 16;   // 16-byte pieces of a row in memory
  constexpr int kHalf = 16 * kPieces;                           // of 16 rows: one, two or four waves' or all threads'
  constexpr int NP = 2 * kChosenTile * kPieces / kWideThreads;  // of a tile's keys and values, per thread
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int quad = lane >> 4, col = lane & 15;
  __shared__ __attribute__((aligned(1024))) unsigned char tiles[2][2 * kTileBytes];
  __shared__ int sm_bad[2][kWaves];

  int koff[NK], voff[NB];
  operand_places<D>(kTileBytes, koff, voff);
  int buf = 0;
  // (workgroups are dealt out to the 8 XCDs in turn; neighbouring shares read the same rows and belong into one XCD's L2)
  const float c = a.scale_log2e;
  const long long wg = first_wg + blockIdx.x, index = wg % 8 * (a.wide_wgs / 8) + wg / 8;
  WindowShare share;
  if constexpr (kShares) {
    share = window_share(a, index);
  } else {
    share.unit = wg % a.n_other * a.wide_tiles + wg / a.n_other;
    share.at = 0;
    share.end = 1;
  }
  if (kShares && tid == 0) a.splits[index].y = -1;
  long long at = share.at;
#pragma unroll 1
  for (long long u = share.unit; at < share.end && u < a.wgs_other; ++u) {
    const WindowUnit unit = window_unit(a, u);
    const int b = __builtin_amdgcn_readfirstlane(unit.b), i = __builtin_amdgcn_readfirstlane(unit.i), n = __builtin_amdgcn_readfirstlane(unit.n);
    if (!kShares) at = 1;
    if (b < 0) continue;
    const int tokens = min(a.wide_tokens, n - i), live = tokens * a.g;
    const int hx = a.n_past + __builtin_amdgcn_readfirstlane(unit.x), h = a.head_of[hx];
    const long long token0 = (a.cu ? a.cu[b] : b) + i, w = (long long)b * a.Hkv + h;
    int my_head[NG], my_from[NG], my_to[NG], my_token[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const int column = kWaveColumns * wave + 16 * g + col;
      my_token[g] = column < live ? column / a.g : 0;
      my_head[g] = column < live ? column - my_token[g] * a.g : 0;
      token_window(a, w, hx, i + my_token[g], n, my_from[g], my_to[g]);
    }
    // first and last row that one token sees, and that every one sees
    int from, first_to, last_from, to;
    token_window(a, w, hx, i, n, from, first_to);
    token_window(a, w, hx, i + tokens - 1, n, last_from, to);
    from = __builtin_amdgcn_readfirstlane(from);
    last_from = __builtin_amdgcn_readfirstlane(last_from);
    first_to = __builtin_amdgcn_readfirstlane(first_to);
    to = __builtin_amdgcn_readfirstlane(to);
    const bool idle = kWaveColumns * wave >= live;  // a wave without columns only helps to load

    const int *table = table_of(a.c, a.Hkv, b, h);
    const int hh = a.c.per_head ? 0 : h;
    WaveColumns<D, kFp32, NG> cols;
    cols.clear();
#pragma unroll
    for (int g = 0; g < NG; ++g)
      cols.load(g, a.q + ((token0 + my_token[g]) * a.Hq + h * a.g + my_head[g]) * D + 8 * quad, kWaveColumns * wave + 16 * g + col < live);

    // ---- the halves' places, 64 at a time, a lane each (every wave for itself)
    int half_row = -1;
    long long half_at = 0, half_place = 0;
    auto look_up = [&](int t) {
      half_row = -1;
      half_at = 0;
      half_place = 0;
      const long long r = 16ll * (2 * (t + (lane >> 1)) + (lane & 1)) + from / kChosenTile * kChosenTile;
      if (r >= to || r + 16 <= from) return;
      int in_page;
      const int page = page_of(a.c, table, (int)r, in_page);
      if (page < 0) return;
      half_row = (int)r;
      half_at = page * a.c.page_bytes + hh * a.c.head_bytes + in_page * a.c.row_bytes;
      half_place = ((long long)page * a.c.heads + hh) * a.c.page_rows.d + in_page;
    };

    // A wave's pieces are all of keys or all of values, and of one half.
    const unsigned char *const pool_k = a.c.k, *const pool_v = a.c.v, *const scale_k = a.c.k_scale, *const scale_v = a.c.v_scale;
    struct Flight {  // a tile's pieces on their way
      u32x4 x[NP];
      int scale[NP];
    } flight0, flight1;
    // (of the four halves of keys and values; all pieces of a thread lie in one row of them)
    auto half_of = [&](int p) __attribute__((always_inline)) { return p * (kWideThreads / kHalf) + (kHalf < kWideThreads ? wave / (kHalf / 64) : 0); };
    const int in_half = tid / kPieces % 16, piece = tid % kPieces;
    const unsigned in_memory = (unsigned)in_half * (unsigned)a.c.row_bytes + piece * 16;
    auto fetch = [&](Flight &f, int j) __attribute__((always_inline)) {
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const int half = half_of(p) % 2;
        const bool is_v = half_of(p) >= 2;
        const unsigned char *src = (is_v ? pool_v : pool_k) + of_lane(half_at, 2 * j + half);
        f.x[p] = *(const u32x4 *)(src + in_memory);
        if constexpr (kE4m3) f.scale[p] = (is_v ? scale_v : scale_k)[of_lane(half_place, 2 * j + half) + in_half];
      }
    };
    auto stage = [&](const Flight &f, int buf, unsigned valid, bool mixed) __attribute__((always_inline)) {
      bool bad = false;
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const int row = half_of(p) % 2 * 16 + in_half;
        const bool is_v = half_of(p) >= 2;
        unsigned char *dst = tiles[buf] + (is_v ? kTileBytes : 0);
        if (is_v && (mixed || valid != ~0u)) bad |= stage_piece<D, kE4m3>(dst, row, piece, f.x[p], f.scale[p], true, !((valid >> row) & 1), mixed);
        else stage_piece<D, kE4m3>(dst, row, piece, f.x[p], f.scale[p], is_v, false, false);
      }
      if (mixed) {
        const bool any = __builtin_amdgcn_ballot_w64(bad) != 0;
        if (lane == 0) sm_bad[buf][wave] = any;
      }
    };

    // ---- tiles t_begin .. t_end - 1, those without a row left out
    const int cost = __builtin_amdgcn_readfirstlane(unit.cost);
    const int begin = kShares ? (int)max(share.begin - at, 0ll) : 0, end = kShares ? (int)min(share.end - at, (long long)cost) : cost;
    const int t_begin = __builtin_amdgcn_readfirstlane(unit.tile_at(begin)), t_end = __builtin_amdgcn_readfirstlane(unit.tile_at(end));
    const bool first_piece = begin == 0, whole = !kShares || (first_piece && end == cost);
    if (kShares) {
      // (of this unit the first piece, but not all: the last one too is for some share)
      if (first_piece && !whole && tid == 0) a.splits[index] = int4{(int)u, (int)(u >> 32), (int)((at + cost - 1) / share.length), 0};
      at += cost;
    }
    for (int t = t_begin; t < t_end; t += 32) {
      look_up(t);
      unsigned long long halves = __builtin_amdgcn_ballot_w64(half_row >= 0);
      if (t_end - t < 32) halves &= (1ull << (2 * (t_end - t))) - 1;
      unsigned long long some = (halves | (halves >> 1)) & 0x5555555555555555ull;
      if (!some) continue;
      // One tile is computed, the next one waits in registers, and the one behind it is asked for: with one less in flight a tile took as
      // long as its keys needed to come.
      struct Tile {
        int j, row0, row1;
        unsigned valid;
        bool mixed;  // some tokens see all of it, others do not
      } tile0, tile1;
      auto next_tile = [&]() __attribute__((always_inline)) {
        Tile x;
        x.j = some ? (int)__builtin_ctzll(some) >> 1 : -1;
        some &= some - 1;
        const int l = x.j < 0 ? 0 : 2 * x.j;
        x.row0 = __builtin_amdgcn_readlane(half_row, l);
        x.row1 = __builtin_amdgcn_readlane(half_row, l + 1);
        x.valid = half_bits(x.row0, from, to) | half_bits(x.row1, from, to) << 16;
        x.mixed = (x.row0 >= 0 && (x.row0 < last_from || x.row0 + 16 > first_to)) || (x.row1 >= 0 && (x.row1 < last_from || x.row1 + 16 > first_to));
        return x;
      };
      auto step = [&](Tile &now, Flight &free, const Tile &then, const Flight &there) __attribute__((always_inline)) {
        const Tile behind = next_tile();  // (none behind the last one)
        if (behind.j >= 0) fetch(free, behind.j);
        if (!idle) {
          // (a half that is not there: rows behind the last one)
          cols.tile(tiles[buf], koff, voff, c, now.mixed || now.valid != ~0u, now.row0 < 0 ? 0x7fffffc0 : now.row0, now.row1 < 0 ? 0x7fffffc0 : now.row1,
                    my_from, my_to);
          bool bad = false;
          if (now.mixed)
            for (int y = 0; y < kWaves; ++y) bad |= sm_bad[buf][y] != 0;
          if (bad) {
#pragma unroll 1
            for (int r = 0; r < kChosenTile; ++r) {
              if (!((now.valid >> r) & 1)) continue;
              const int from_lane = 2 * now.j + (r >> 4);
              float scale = 1.f;
              if constexpr (kE4m3) scale = __uint_as_float((unsigned)scale_v[of_lane(half_place, from_lane) + (r & 15)] << 23);
              cols.template odd_values<kE4m3>(pool_v + of_lane(half_at, from_lane) + (long long)(r & 15) * a.c.row_bytes, scale,
                                              (r < 16 ? now.row0 : now.row1) + (r & 15), my_from, my_to);
            }
          }
        }
        buf ^= 1;
        if (then.j < 0) return false;
        stage(there, buf, then.valid, then.mixed);
        __syncthreads();
        now = behind;
        return true;
      };
      tile0 = next_tile();
      fetch(flight0, tile0.j);
      tile1 = next_tile();
      if (tile1.j >= 0) fetch(flight1, tile1.j);
      stage(flight0, buf, tile0.valid, tile0.mixed);
      __syncthreads();
      while (step(tile0, flight0, tile1, flight1) && step(tile1, flight1, tile0, flight0)) {
      }
    }

    // ---- results: a column's lanes hold four channels each
    if (idle) continue;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const float l = over_quads(cols.l[g], true);
      const int column = kWaveColumns * wave + 16 * g + col;
      if (column >= live) continue;
      if (!whole) {
        float *dst = window_slot<D>(a, 2ll * index + first_piece) + column * ws_slot_floats(D);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) *(f32x4 *)(dst + 16 * nb + 4 * quad) = cols.O[g][nb];
        if (quad == 0) *(float2 *)(dst + D) = float2{cols.m[g], l};
      } else {
        const float ref = cols.m[g] == -INFINITY ? 0.f : cols.m[g];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) store_out<D>(a, (token0 + my_token[g]) * a.Hq + h * a.g + my_head[g], 16 * nb + 4 * quad, cols.O[g][nb], l, ref);
      }
    }
  }
}

// The units whose pieces are several workgroups': of the one whose first piece is workgroup k's, some columns.
template <int D>
__global__ __launch_bounds__(256) void paged_windows_join_kernel(const PagedChosenArgs a) {
  constexpr int SF = D + kWsTailFloats, kLanes = D / 4, kEach = 256 / kLanes, kWgs = kWideColumns / kEach, kBatch = 4;
  const int k = blockIdx.x / kWgs;
  const int4 s = a.splits[k];
  if (s.y < 0) return;
  const WindowUnit unit = window_unit(a, ((long long)s.y << 32) | (unsigned)s.x);
  const int column = blockIdx.x % kWgs * kEach + threadIdx.x / kLanes, d = threadIdx.x % kLanes * 4;
  if (column >= unit.tokens * a.g) return;
  const int pieces = s.z - k + 1;
  float top = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < pieces; p0 += kBatch) {
    float2 ml[kBatch];
    f32x4 y[kBatch];
#pragma unroll
    for (int p = 0; p < kBatch; ++p) {
      const int piece = min(p0 + p, pieces - 1);
      const float *src = window_slot<D>(a, 2ll * (k + piece) + (piece == 0)) + column * SF;
      ml[p] = *(const float2 *)(src + D);
      y[p] = *(const f32x4 *)(src + d);
      if (p0 + p >= pieces) ml[p] = float2{-INFINITY, 0.f};
    }
    float m_new = top;
#pragma unroll
    for (int p = 0; p < kBatch; ++p) m_new = fmaxf(m_new, ml[p].x);
    const float ref = m_new == -INFINITY ? 0.f : m_new, keep = __builtin_amdgcn_exp2f(top - ref);
    l *= keep;
    o *= keep;
    top = m_new;
#pragma unroll
    for (int p = 0; p < kBatch; ++p) {
      if (p0 + p < pieces) {
        const float wgt = __builtin_amdgcn_exp2f(ml[p].x - ref);
        l += ml[p].y * wgt;
        o += y[p] * wgt;
      }
    }
  }
  const int token = column / a.g, hx = a.n_past + unit.x;
  const long long first = (a.cu ? a.cu[unit.b] : unit.b) + unit.i;
  store_out<D>(a, (first + token) * a.Hq + a.head_of[hx] * a.g + column - token * a.g, d, o, l, top == -INFINITY ? 0.f : top);
}

// ---- listed blocks ------------------------------------------------------------------------------
// A task: some of the entries that name one block.  Its rows go to LDS kListedRows at a time (a partial for each such piece of a
// block), and the waves take the columns 16 at a time.
template <int D, bool kE4m3, bool kFp32>
__global__ __launch_bounds__(kListedThreads, 4) void paged_listed_kernel(const PagedChosenArgs a, const long long first_wg) {
  constexpr int NG = 1, kWaveColumns = 16 * NG, NK = D / 32, NB = D / 16;
  constexpr int kRow = 2 * D, kBytes = kListedRows * kRow;
  constexpr int kPieces = (kE4m3 ? D : 2 * D) / 16;
  constexpr int NP = kListedRows * kPieces / kListedThreads;  // of the keys, and of the values, per thread
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int quad = lane >> 4, col = lane & 15;
  __shared__ __attribute__((aligned(1024))) unsigned char tiles[2 * kBytes];  // keys, then values
  __shared__ int sm_bad[4];
  const long long wg = (first_wg + blockIdx.x) / a.listed_pieces;
  const int sub = (int)((first_wg + blockIdx.x) - wg * a.listed_pieces);
  if (wg >= a.cursors[1]) return;
  const int4 task = a.tasks[wg];
  const int unit = task.x / a.blocks, block = task.x - unit * a.blocks;
  const int b = unit / a.n_past, x = unit - b * a.n_past, h = a.head_of[x];
  const int *table = table_of(a.c, a.Hkv, b, h);
  const int br = 16 * (int)a.block_halves.d;
  const int row0 = block * br + sub * kListedRows, rows = min(kListedRows, br - sub * kListedRows);
  int in_page;
  int page = page_of(a.c, table, row0, in_page);
  page = page < 0 ? 0 : page;  // (entries without a page are not listed)
  const int hh = a.c.per_head ? 0 : h;
  const long long at = page * a.c.page_bytes + hh * a.c.head_bytes + in_page * a.c.row_bytes;
  const long long place = ((long long)page * a.c.heads + hh) * a.c.page_rows.d + in_page;
  u32x4 xk[NP], xv[NP];
  int sk[NP], sv[NP];
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int row = (p * kListedThreads + tid) / kPieces;
    const int r = row < rows ? row : 0;  // (rows behind the block's last are masked)
    const long long src = at + r * a.c.row_bytes + lane % kPieces * 16;
    xk[p] = *(const u32x4 *)(a.c.k + src);
    xv[p] = *(const u32x4 *)(a.c.v + src);
    if constexpr (kE4m3) {
      sk[p] = a.c.k_scale[place + r];
      sv[p] = a.c.v_scale[place + r];
    }
  }
  const long long w = (long long)b * a.Hkv + h;
  const int first = a.cu ? a.cu[b] : b, n = a.cu ? a.cu[b + 1] - first : 1;
  int whole_to, end;  // rows that every token of the sequence sees, and that its last one does
  { int none; token_window(a, w, x, 0, n, none, whole_to); token_window(a, w, x, n - 1, n, none, end); }
  const bool edge = __builtin_amdgcn_readfirstlane((int)(row0 + kListedRows > whole_to || rows < kListedRows)) != 0;
  bool bad = false;
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int row = (p * kListedThreads + tid) / kPieces, piece = lane % kPieces;
    stage_piece<D, kE4m3>(tiles, row, piece, xk[p], sk[p], false, false, false);
    if (edge) bad |= stage_piece<D, kE4m3>(tiles + kBytes, row, piece, xv[p], sv[p], true, row >= rows || row0 + row >= end, true);
    else stage_piece<D, kE4m3>(tiles + kBytes, row, piece, xv[p], sv[p], true, false, false);
  }
  {
    const bool any = __builtin_amdgcn_ballot_w64(bad) != 0;
    if (lane == 0) sm_bad[wave] = any;
  }
  int koff[NK], voff[NB];
  operand_places<D>(kBytes, koff, voff);
  const int live = task.z * a.g;
  __syncthreads();
  const bool odd = edge && (sm_bad[0] | sm_bad[1] | sm_bad[2] | sm_bad[3]);
#pragma unroll 1
  for (int base = kWaveColumns * wave; base < live; base += 4 * kWaveColumns) {
    int my_entry[NG], my_head[NG], my_to[NG];
    int my_from[NG] = {};
    WaveColumns<D, kFp32, NG> cols;
    cols.clear();
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const int column = base + 16 * g + col, k = column < live ? column / a.g : 0;
      my_head[g] = column < live ? column - k * a.g : 0;
      my_entry[g] = a.sorted[task.y + k];
      const long long token = a.part0 + my_entry[g] / a.n_chosen / a.n_past;
      cols.load(g, a.q + (token * a.Hq + h * a.g + my_head[g]) * D + 8 * quad, column < live);
      my_to[g] = min(rows_seen(a.rows, w, (int)(token - first), n, a.max_rows), row0 + rows);
    }
#pragma unroll
    for (int t = 0; t < kListedRows / kChosenTile; ++t) {
      if (t * kChosenTile < rows)
        cols.tile(tiles + t * kChosenTile * kRow, koff, voff, a.scale_log2e, edge, row0 + kChosenTile * t, row0 + kChosenTile * t + 16, my_from, my_to);
    }
    if (odd) {
#pragma unroll 1
      for (int r = 0; r < rows && row0 + r < end; ++r) {
        float scale = 1.f;
        if constexpr (kE4m3) scale = __uint_as_float((unsigned)a.c.v_scale[place + r] << 23);
        cols.template odd_values<kE4m3>(a.c.v + at + r * a.c.row_bytes, scale, row0 + r, my_from, my_to);
      }
    }
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const float l = over_quads(cols.l[g], true);
      if (base + 16 * g + col >= live) continue;
      const long long slot = ((long long)my_entry[g] * a.listed_pieces + sub) * a.g + my_head[g];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) __builtin_nontemporal_store(cols.O[g][nb], (f32x4 *)(a.listed_out + slot * D + 16 * nb + 4 * quad));
      if (quad == 0) a.listed_sum[slot] = float2{cols.m[g], l};
    }
  }
}

constexpr int kJoinBatch = 8;  // partials of half a wave under way together
// A wave per query head of a PAST head: the partials of its token's entries.
template <int D>
__global__ __launch_bounds__(256) void paged_listed_join_kernel(const PagedChosenArgs a, const long long first_wg) {
  constexpr int kLanes = D / 4, kGroups = 64 / kLanes;
  const int lane = threadIdx.x & 63;
  const long long u = (first_wg + blockIdx.x) * 4 + (threadIdx.x >> 6);  // (token of the part, PAST head, head of the group)
  const long long unit = u / a.g;
  const int j = (int)(u - unit * a.g);
  if (unit * a.n_chosen >= a.entries) return;
  const long long token = a.part0 + unit / a.n_past;
  int i, n;
  if (sequence_of(a.cu, a.B, token, i, n) < 0) return;
  const int group = lane / kLanes, d = lane % kLanes * 4;
  float top = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  const int partials = a.n_chosen * a.listed_pieces;
  for (int e0 = 0; e0 < partials; e0 += 64) {
    float2 ml = {-INFINITY, 0.f};
    if (e0 + lane < partials && a.rank[unit * a.n_chosen + (e0 + lane) / a.listed_pieces] >= 0)
      ml = a.listed_sum[(unit * partials + e0 + lane) * a.g + j];
    float m_new = ml.x;
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) m_new = fmaxf(m_new, __shfl_xor(m_new, sh));
    m_new = fmaxf(m_new, top);
    const float ref = m_new == -INFINITY ? 0.f : m_new, keep = __builtin_amdgcn_exp2f(top - ref);
    const float wgt = __builtin_amdgcn_exp2f(ml.x - ref);  // (a partial whose scores are all NaN: 0, and its sums stay NaN)
    top = m_new;
    l = l * keep + ml.y * wgt;
    o *= keep;
    unsigned long long there = __builtin_amdgcn_ballot_w64(e0 + lane < partials && (ml.x != -INFINITY || ml.y != 0.f));
    const float *src = a.listed_out + ((unit * partials + e0) * a.g + j) * D + d;
    const int most = min(64, partials - e0);
    for (int k0 = 0; k0 < most; k0 += kGroups * kJoinBatch) {
      f32x4 y[kJoinBatch];
      float w[kJoinBatch];
#pragma unroll
      for (int k = 0; k < kJoinBatch; ++k) {  // (no branches: the loads go together; of partials that are not there some other is read)
        const int mine = k0 + kGroups * k + group;
        const bool is = mine < most && ((there >> mine) & 1);
        y[k] = __builtin_nontemporal_load((const f32x4 *)(src + (long long)(is ? mine : 0) * a.g * D));
        w[k] = __shfl(wgt, mine & 63);
        if (!is) y[k] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (!is) w[k] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < kJoinBatch; ++k) o += y[k] * w[k];
    }
  }
#pragma unroll
  for (int sh = 1; sh < 64; sh <<= 1) l += __shfl_xor(l, sh);
#pragma unroll
  for (int sh = kLanes; sh < 64; sh <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], sh);
  if (lane < kLanes) store_out<D>(a, token * a.Hq + a.head_of[(int)(unit % a.n_past)] * a.g + j, d, o, l, top == -INFINITY ? 0.f : top);
}

template <int D, bool kE4m3>
static long long resident_shares(bool fp32) {
  static ResidentCount count[2];
  const auto kern = fp32 ? paged_windows_kernel<D, kE4m3, true, true> : paged_windows_kernel<D, kE4m3, false, true>;
  return count[fp32].get((const void *)kern, kWideThreads, 0);
}
long long windows_resident(const PagedChosenArgs &a) {
  const bool fp32 = a.out_fp32 != 0;
  return a.D == 128 ? (a.c.e4m3 ? resident_shares<128, true>(fp32) : resident_shares<128, false>(fp32))
                    : (a.c.e4m3 ? resident_shares<64, true>(fp32) : resident_shares<64, false>(fp32));
}

template <int D, bool kE4m3>
static hipError_t launch_windows(const PagedChosenArgs &a, hipStream_t st) {
  const auto kern = a.wide_wgs > 0 ? (a.out_fp32 ? paged_windows_kernel<D, kE4m3, true, true> : paged_windows_kernel<D, kE4m3, false, true>)
                                   : (a.out_fp32 ? paged_windows_kernel<D, kE4m3, true, false> : paged_windows_kernel<D, kE4m3, false, false>);
  const hipError_t e = launch_in_parts(a.wide_wgs > 0 ? a.wide_wgs : a.wgs_other, kWideThreads, [&](long long first, unsigned count) {
    hipLaunchKernelGGL(kern, dim3(count), dim3(kWideThreads), 0, st, a, first);
  });
  if (e != hipSuccess || a.wide_wgs == 0) return e;
  hipLaunchKernelGGL(paged_windows_join_kernel<D>, dim3(a.wide_wgs * (kWideColumns * D / 1024)), dim3(256), 0, st, a);
  return hipGetLastError();
}
hipError_t launch_paged_windows(const PagedChosenArgs &a, hipStream_t st) {
  return a.D == 128 ? (a.c.e4m3 ? launch_windows<128, true>(a, st) : launch_windows<128, false>(a, st))
                    : (a.c.e4m3 ? launch_windows<64, true>(a, st) : launch_windows<64, false>(a, st));
}

template <int D, bool kE4m3>
static hipError_t launch_listed(PagedChosenArgs a, hipStream_t st) {
  const auto kern = a.out_fp32 ? paged_listed_kernel<D, kE4m3, true> : paged_listed_kernel<D, kE4m3, false>;
  const int keys = a.B * a.n_past * a.blocks;
  for (long long t = 0; t < a.total; t += a.part_tokens) {
    const long long n = a.total - t < a.part_tokens ? a.total - t : a.part_tokens;
    a.part0 = t;
    a.entries = n * a.n_past * a.n_chosen;
    const int units = (int)(n * a.n_past);
    const unsigned wgs = (unsigned)(((n + 63) / 64 * a.n_past * a.n_chosen + 3) / 4), key_wgs = (unsigned)((keys + 255) / 256);
    const unsigned clear_wgs = (keys + 2 + 255) / 256;
    hipLaunchKernelGGL(paged_clear_kernel, dim3(clear_wgs < 1024 ? clear_wgs : 1024), dim3(256), 0, st, a.cursors, keys + 2);
    hipLaunchKernelGGL(paged_count_kernel, dim3(wgs), dim3(256), 0, st, a, units);
    hipLaunchKernelGGL(paged_place_kernel, dim3(key_wgs), dim3(256), 0, st, a, keys);
    hipLaunchKernelGGL(paged_sort_kernel, dim3(wgs), dim3(256), 0, st, a, units);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const long long tasks = a.entries / a.listed_tokens + (a.entries < keys ? a.entries : keys);
    e = launch_in_parts(tasks * a.listed_pieces, kListedThreads, [&](long long first, unsigned count) {
      hipLaunchKernelGGL(kern, dim3(count), dim3(kListedThreads), 0, st, a, first);
    });
    if (e != hipSuccess) return e;
    e = launch_in_parts((n * a.n_past * a.g + 3) / 4, 256, [&](long long first, unsigned count) {
      hipLaunchKernelGGL(paged_listed_join_kernel<D>, dim3(count), dim3(256), 0, st, a, first);
    });
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
hipError_t launch_paged_listed(const PagedChosenArgs &a, hipStream_t st) {
  return a.D == 128 ? (a.c.e4m3 ? launch_listed<128, true>(a, st) : launch_listed<128, false>(a, st))
                    : (a.c.e4m3 ? launch_listed<64, true>(a, st) : launch_listed<64, false>(a, st));
}

}  // namespace segattn
