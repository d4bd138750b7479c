// seg_attn_decode_paged: attention of one new token per sequence over a paged cache.
//
// The g query heads of a KV head are the columns of 16-column matrix operands (16 per pass).  Per tile of
// 32 key rows a wave forms
//   S^T[key][head] = K . Q^T            v_mfma_f32_16x16x32_bf16, A = K rows, B = Q^T (registers)
//   P = exp2((S^T - m) c)               running maximum m and sum l per head (lane = head), in fp32
//   O^T[d][head] += V^T . P^T           A = V^T via ds_read_b64_tr_b16, B = P from the S^T registers
// P enters the product as a bf16 and the bf16 of what that leaves: at most 2^-16 of a weight is lost, where a bf16 output
// is rounded by up to 2^-8.  For fp32 outputs a third bf16 has the rest, so that all 24 bits count (against the formula 2^-17.2 of
// the output without it, below 2^-20 with it).  The products are idle beside the memory: fp32 outputs take as long
// without the third (696 us and 696 for 32 sequences of 4K to 64K, 192 and 194 for 24 of 1K to 32K with 8-bit rows and weights), bf16
// outputs with it 151 us instead of 143 for those without weights, so it is left out there.
//
// The work is bound by memory: every seen row is read once per 16 query heads of its KV head, so a group of up to 16 reads K and V once
// and one of 128 eight times.  The windows of all (sequence, KV
// head) pairs are cut into slices of whole tiles, found by the kernel itself from the row counts on the
// device, so a captured launch serves a cache that grows.  At the end of every window a workgroup writes one
// partial (acc[D], m, l) per query head; a second launch merges them and, where the cache keeps the weight
// of its rows, turns the stored scores into weights and adds them up.  Traced kernels on one card, 8 KV
// heads of 128: 32 sequences of 4K to 64K 700 us + 5 (as calls, untraced, 673: 6.75 TB/s; the read probe reaches 7.15), the same with
// 8-bit rows 375 + 5; 24 of 1K to 32K with 8-bit rows 143 + 5, with their weights 174 + 19.
#include "segattn_paged.h"

namespace segattn {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
#define LDS_AS __attribute__((address_space(3)))

constexpr int kPagedHeads = 16;  // query heads per pass
constexpr int kPagedWaves = 4;
// Up to so many rows of 128 channels (twice as many of 64) a workgroup takes a window by itself and there is nothing to
// join; times the windows per compute unit, up to eight, since a window that is longer than the others then weighs less.
// Kernels and the gap between them, whole and cut, 8 KV heads: five sequences of 500 rows of 128 10.4 and 14.1 us (8-bit rows
// 10.4 and 14.0), of 1000 rows of 64 10.1 and 13.0, of 1000 rows of 128 16.1 and 15.6; 100 sequences of 10 to 1000 rows of 128 42
// and 56, 128 of 100 to 2000 98 and 105, 500 of 1100 to 3000 662 and 712.  (64 of 2000 to 4000: 131 and 135, but one long
// window among short ones would be waited for.)
constexpr long long kPagedWholeRows = 512;

// Rows [first, n) of a window that the newest token (row n - 1) sees.
__device__ inline void paged_window(const PagedDecodeArgs &a, int w, int &first, int &n) {
  n = rows_held(a.rows, w, a.max_rows);
  const int h = w - fast_div(w, a.n_kv) * a.Hkv;
  first = 0;
  if (!in_set(a.heads.past, h)) {
    const int start = fast_div(n > 0 ? n - 1 : 0, a.seg) * (int)a.seg.d;
    first = in_set(a.heads.tail, h) ? (start > a.tail ? start - a.tail : 0) : start;
  }
}
__device__ inline int paged_tiles(const PagedDecodeArgs &a, int w) {
  int first, n;
  paged_window(a, w, first, n);
  return (n + kPagedTile - 1) / kPagedTile - first / kPagedTile;  // 0 for n = 0
}

// This workgroup's slice: tiles [tile, tile + count) counted from window w's first one; a count that goes beyond the
// window goes on in the next ones (not in the first form).  Every slice is a multiple of one tile per wave.  The
// first form is in the order of their numbers; the second one's order (next_window) is that of its search.
struct PagedSlice {
  int w, tile, count;
  bool by_window;
  int order;  // w's place in the order
};
__device__ inline PagedSlice paged_slice(const PagedDecodeArgs &a, int wgs) {
  const int lane = threadIdx.x & 63, me = blockIdx.x;
  constexpr int kLeast = kPagedWaves;
  auto whole = [](int tiles) { return (tiles + kPagedWaves - 1) / kPagedWaves * kPagedWaves; };
  PagedSlice s{-1, 0, 0, true, 0};
  if (a.n_windows <= kPagedLaneWindows) {
    // Few windows: each is cut by itself, into slices as long as the grid needs them, a lane per window.
    const int tiles = lane < a.n_windows ? paged_tiles(a, lane) : 0;
    int count = kLeast;
    if (!a.fits) {
      int total = tiles;
#pragma unroll
      for (int sh = 1; sh < 64; sh <<= 1) total += __shfl_xor(total, sh);
      const int spare = wgs - a.n_windows;  // sum of ceil(t / c) <= total / c + windows <= wgs
      count = whole((total + spare - 1) / spare);
      count = count < kLeast ? kLeast : count;
    }
    const int mine = (tiles + count - 1) / count;
    int incl = mine;
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) {
      const int up = __shfl_up(incl, sh);
      if (lane >= sh) incl += up;
    }
    const unsigned long long reach = __builtin_amdgcn_ballot_w64(incl > me);
    if (reach == 0) return s;
    s.w = (int)__builtin_ctzll(reach);
    s.tile = (me - __builtin_amdgcn_readlane(incl - mine, s.w)) * count;
    s.count = count;
    return s;
  }
  // Many windows: all tiles end to end, cut evenly.  A thread adds up the windows tid, tid + 256, ... (so that neighbours read
  // neighbouring counts), every wave scans the 256 sums, four a lane, and walks the windows of the one that holds the
  // slice's first tile.
  __shared__ __attribute__((aligned(16))) int sm_run[256];
  const int tid = threadIdx.x, run = (a.n_windows + 255) / 256;
  int sum = 0;
  for (int j = 0; j < run; ++j)
    if (j * 256 + tid < a.n_windows) sum += paged_tiles(a, j * 256 + tid);
  sm_run[tid] = sum;
  __syncthreads();
  int part[4], incl = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    part[j] = sm_run[4 * lane + j];
    incl += part[j];
  }
  const int mine = incl;
#pragma unroll
  for (int sh = 1; sh < 64; sh <<= 1) {
    const int up = __shfl_up(incl, sh);
    if (lane >= sh) incl += up;
  }
  const int total = __builtin_amdgcn_readlane(incl, 63);
  int count = whole((total + wgs - 1) / wgs);
  count = count < kLeast ? kLeast : count;
  if (total == 0 || me > (total - 1) / count) return s;
  const int start = me * count;  // < total
  const int L = (int)__builtin_ctzll(__builtin_amdgcn_ballot_w64(incl > start));
  int before = __builtin_amdgcn_readlane(incl - mine, L), t = 4 * L;
#pragma unroll
  for (int j = 0; j < 3; ++j) {
    const int n = __builtin_amdgcn_readlane(part[j], L);
    if (t == 4 * L + j && before + n <= start) {
      before += n;
      ++t;
    }
  }
  int w = t;  // the window that holds the tile: below n_windows, since those behind have no tiles
  for (; w + 256 < a.n_windows; w += 256) {
    const int n = paged_tiles(a, w);
    if (before + n > start) break;
    before += n;
  }
  s.w = __builtin_amdgcn_readfirstlane(w);
  s.order = t * run + s.w / 256;
  s.tile = __builtin_amdgcn_readfirstlane(start - before);
  s.count = count;
  s.by_window = false;
  return s;
}

// The window behind w in the order of the second form; n_windows or above: none.  It skips no window, and a step of the
// order per call (places of the order without a window included) numbers the slots.
__device__ inline int next_window(const PagedDecodeArgs &a, int w, int &order) {
  const int run = (a.n_windows + 255) / 256;
  ++order;
  if (w + 256 < a.n_windows) return w + 256;
  const int t = (w & 255) + 1;
  order = t * run;
  return t < 256 ? t : a.n_windows;
}

__device__ inline float over_quads(float x, bool sum) {  // over the four lanes of a column
  const float y = __shfl_xor(x, 16);
  x = sum ? x + y : fmaxf(x, y);
  const float z = __shfl_xor(x, 32);
  return sum ? x + z : fmaxf(x, z);
}

// Four channels of a head's output, and with the first ones its sum.  No row seen: zeros, and the logarithm of nothing.
template <int D>
__device__ inline void store_out(const PagedDecodeArgs &a, long long head, int d, f32x4 o, float l, float ref) {
  const float scale = l == 0.f ? 0.f : 1.f / l;
  const f32x4 r = o * scale;
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

// kInPage: page_rows is a multiple of the tile, so a tile lies in one page; otherwise every row asks the table.
// kMass: the scores are left for the weights.
// kWhole: a workgroup per window, which writes the output itself.
template <int D, bool kE4m3, bool kInPage, bool kMass, bool kWhole>
__global__ __launch_bounds__(256, 2) void paged_decode_split_kernel(const PagedDecodeArgs a) {
  constexpr int NK = D / 32, NB = D / 16;
  constexpr int kRow = 2 * D, kTileBytes = kPagedTile * kRow;  // of a tile in LDS, bf16
  constexpr int kPieces = (kE4m3 ? D : 2 * D) / 16;            // 16-byte pieces of a row in memory
  constexpr int RPL = 64 / kPieces, NL = kPagedTile / RPL;     // rows per wave load, loads per tile and tensor
  // Where a row's 16-byte chunk lies: XORed so that 16 rows read at one chunk (K), or 8 rows at two (V), meet every bank once,
  // and so do the eight lanes that write every other chunk of an 8-bit row, whose upper half is flipped against the lower one,
  // or (D = 64) of two rows, the odd one flipped.
  auto chunk_k = [](int row, int chunk) { return D == 128 ? chunk ^ (chunk >> 3) ^ (row & 15) : chunk ^ ((row >> 1) & 7) ^ (row & 1); };
  auto chunk_v = [](int row, int chunk) { return D == 128 ? chunk ^ (chunk >> 3) ^ (2 * (row & 7)) : chunk ^ (2 * ((row >> 1) & 3)) ^ (row & 1); };

  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int quad = lane >> 4, col = lane & 15;
  const float c = a.scale_log2e;
  __shared__ __attribute__((aligned(1024))) unsigned char tiles[kPagedWaves][2 * kTileBytes];
  __shared__ float sm_join[kPagedHeads][2];
  constexpr int MS = D + 4;  // floats per head of the merge area
  static_assert(kPagedWaves * 2 * kTileBytes >= (int)sizeof(float) * kPagedWaves * kPagedHeads * MS, "merge area fits the tiles");

  PagedSlice slice{(int)blockIdx.x, 0, 0x7fffffff, true, 0};
  if constexpr (!kWhole) slice = paged_slice(a, gridDim.x);
  slice.w = __builtin_amdgcn_readfirstlane(slice.w);  // the same in all lanes: what follows from them is scalar work
  slice.tile = __builtin_amdgcn_readfirstlane(slice.tile);
  slice.count = __builtin_amdgcn_readfirstlane(slice.count);
  if (slice.w < 0) return;
  const int pass = blockIdx.y, live = min(kPagedHeads, a.g - pass * kPagedHeads);
  unsigned char *tile = tiles[wave];
  const unsigned char *scales = lane < 32 ? a.c.k_scale : a.c.v_scale;
  // where this lane reads its operands; the tile's second 16 rows lie 16 kRow further on (both XORs repeat after 16 rows)
  int koff[NK], voff[NB];
  const int vrow = 4 * quad + (col >> 2);
#pragma unroll
  for (int kc = 0; kc < NK; ++kc) koff[kc] = col * kRow + (chunk_k(col, 4 * kc + quad) << 4);
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
    voff[nb] = kTileBytes + vrow * kRow + (chunk_v(vrow, 2 * nb + ((col & 3) >> 1)) << 4) + 8 * (col & 1);

  int left = slice.count;
  int order = __builtin_amdgcn_readfirstlane(slice.order);
  for (int w = slice.w, tile0 = slice.tile; left > 0 && w < a.n_windows; w = next_window(a, w, order), tile0 = 0) {
    int first, n;
    paged_window(a, w, first, n);
    first = __builtin_amdgcn_readfirstlane(first);
    n = __builtin_amdgcn_readfirstlane(n);
    const int b = fast_div(w, a.n_kv), h = w - b * a.Hkv;
    const int base = first / kPagedTile, all = (n + kPagedTile - 1) / kPagedTile - base;
    const int t_begin = base + tile0, t_end = base + min(all, tile0 + left);
    if (t_end <= t_begin) {
      if constexpr (kWhole) {  // nothing held
        for (int i = tid; i < live * (D / 4); i += 64 * kPagedWaves)
          store_out<D>(a, (long long)b * a.Hq + h * a.g + pass * kPagedHeads + i / (D / 4), i % (D / 4) * 4, f32x4{0.f, 0.f, 0.f, 0.f}, 0.f, 0.f);
        return;
      }
      continue;
    }
    left = slice.by_window ? 0 : left - (t_end - t_begin);
    const int head0 = h * a.g + pass * kPagedHeads;
    const int *table = table_of(a.c, a.Hkv, b, h);
    const int hh = a.c.per_head ? 0 : h;

    bf16x8 Q[NK];  // column col = head head0 + col, zero beyond the live ones
    {
      const unsigned short *q = a.q + ((long long)b * a.Hq + head0 + (col < live ? col : 0)) * D + 8 * quad;
#pragma unroll
      for (int kc = 0; kc < NK; ++kc) {
        u32x4 x = *(const u32x4 *)(q + 32 * kc);
        if (col >= live) x = u32x4{0u, 0u, 0u, 0u};
        Q[kc] = __builtin_bit_cast(bf16x8, x);
      }
    }
    f32x4 O[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) O[nb] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;

    u32x4 nk[NL], nv[NL];          // the wave's next tile, in flight
    int n_scale = 0;               // scale byte of row lane % 32: keys in the lower half of the wave, values in the upper
    unsigned n_valid = 0;          // rows of it that count
    int entry = 0, entry_row = 0;  // the table's entry for the tile that is fetched next (kInPage), or for this lane's row of it
    auto ask = [&](int t) __attribute__((always_inline)) {
      if constexpr (kInPage) {
        entry = table[fast_div(t * kPagedTile, a.c.page_rows)];
      } else {
        int r = t * kPagedTile + (lane & 31);
        r = r < n ? r : n - 1;
        const int i = fast_div(r, a.c.page_rows);
        entry = table[i];
        entry_row = r - i * (int)a.c.page_rows.d;
      }
    };
    auto fetch = [&](int t) __attribute__((always_inline)) {
      const int r0 = t * kPagedTile;
      unsigned valid = ~0u;
      if (r0 < first) valid &= ~0u << (first - r0);
      if (r0 + kPagedTile > n) valid &= (1u << (n - r0)) - 1u;
      const bool named = (unsigned)entry < (unsigned)a.c.n_pages;
      const int page = named ? entry : 0;  // rows without a page: some row that exists, with weight 0
      if constexpr (kInPage) {
        const int pg = __builtin_amdgcn_readfirstlane(page);
        if (!__builtin_amdgcn_readfirstlane((int)named)) valid = 0;
        const int in_page = r0 - fast_div(r0, a.c.page_rows) * (int)a.c.page_rows.d;
        const long long at = pg * a.c.page_bytes + hh * a.c.head_bytes + in_page * a.c.row_bytes;
        const unsigned mine = (unsigned)(lane / kPieces) * (unsigned)a.c.row_bytes + (lane % kPieces) * 16;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          const unsigned char *k = a.c.k + at + i * (RPL * a.c.row_bytes), *v = a.c.v + at + i * (RPL * a.c.row_bytes);
          nk[i] = __builtin_nontemporal_load((const u32x4 *)(k + mine));
          nv[i] = __builtin_nontemporal_load((const u32x4 *)(v + mine));
        }
        if constexpr (kE4m3) {
          const long long place = ((long long)pg * a.c.heads + hh) * a.c.page_rows.d + in_page + (lane & 31);
          n_scale = scales[place];
        }
      } else {
        valid &= (unsigned)__builtin_amdgcn_ballot_w64(named);
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          const int r = RPL * i + lane / kPieces;
          const long long at = __shfl(page, r) * a.c.page_bytes + hh * a.c.head_bytes + __shfl(entry_row, r) * a.c.row_bytes + (lane % kPieces) * 16;
          nk[i] = __builtin_nontemporal_load((const u32x4 *)(a.c.k + at));
          nv[i] = __builtin_nontemporal_load((const u32x4 *)(a.c.v + at));
        }
        if constexpr (kE4m3) {
          const long long place = ((long long)page * a.c.heads + hh) * a.c.page_rows.d + entry_row;
          n_scale = scales[place];
        }
      }
      n_valid = valid;
    };
    // A tile into LDS, values of rows that do not count as zeros (a weight of zero times NaN would be NaN).
    auto stage = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int r = RPL * i + lane / kPieces, piece = lane % kPieces;
        const u32x4 xk = nk[i], xv = nv[i];
        if constexpr (!kE4m3) {
          *(u32x4 *)(tile + r * kRow + (chunk_k(r, piece) << 4)) = xk;
          *(u32x4 *)(tile + kTileBytes + r * kRow + (chunk_v(r, piece) << 4)) = xv;
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
          }
        }
      }
      if (n_valid != ~0u && !((n_valid >> (lane & 31)) & 1)) {
#pragma unroll
        for (int i = 0; i < kRow / 32; ++i)
          *(u32x4 *)(tile + kTileBytes + (lane & 31) * kRow + (kRow / 32 * (lane >> 5) + i) * 16) = u32x4{0u, 0u, 0u, 0u};
      }
    };

    // Scores of a PAST head's rows for the weights, [tile][head][row of the tile]: 16 bytes a lane, written through a buffer that
    // ends with the window's scores and is empty for other heads, so that every step issues the same stores -- with a
    // branch around them the wait for the next tile would be one for the stores too.
    __amdgpu_buffer_rsrc_t score_rsrc;
    int score_at = 0;
    const int score_tile = a.g * kPagedTile * 4;  // bytes
    if constexpr (kMass) {
      const bool past = in_set(a.heads.past, h);
      float *scores = a.scores + (long long)(b * a.n_past + (past ? set_before(a.heads.past, h) : 0)) * a.g * a.score_rows;
      score_rsrc = __builtin_amdgcn_make_buffer_rsrc(scores, 0, past ? a.g * (int)a.score_rows * 4 : 0, 0x00020000);
      score_at = col < live ? ((pass * kPagedHeads + col) * kPagedTile + 4 * quad) * 4 : (int)0x80000000;  // out of range for columns without a head
    }
    auto store_scores = [&](int t, const f32x4 (&x)[2]) __attribute__((always_inline)) {
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2)
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x[h2]), score_rsrc, score_at + t * score_tile + 64 * h2, 0, 0);
    };

    auto values = [&](int nb) __attribute__((always_inline)) {  // V^T, channels 16 nb ..
      const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4 *)(tile + voff[nb]));
      const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4 *)(tile + voff[nb] + 16 * kRow));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto products = [&](int t, unsigned valid) __attribute__((always_inline)) {
      f32x4 S[2];
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2) {
        S[h2] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kc = 0; kc < NK; ++kc)
          S[h2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8 *)(tile + koff[kc] + 16 * h2 * kRow), Q[kc], S[h2], 0, 0, 0);
      }
      // register r of S[h2] is key 16 h2 + 4 quad + r
      if (valid != ~0u) {
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (!((valid >> (16 * h2 + 4 * quad + r)) & 1)) S[h2][r] = -INFINITY;
      }
      if constexpr (kMass) store_scores(t, S);
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
        for (int i = 0; i < 8; ++i) P_tail[i] = (__bf16)tail[i / 4][i % 4];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) O[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values(nb), P_tail, O[nb], 0, 0, 0);
      }
    };

    int t = t_begin + wave;
    if (t < t_end) {
      ask(t);
      fetch(t);
      ask(min(t + kPagedWaves, t_end - 1));
      if constexpr (kMass) {  // two stores that go nowhere: as many accesses behind the loads as in the loop
        const f32x4 none[2] = {};
        const int at = score_at;
        score_at = (int)0x80000000;
        store_scores(t, none);
        score_at = at;
      }
      // The last tile by itself: with the next one's loads under a condition in the loop the scales of 8-bit rows are
      // copied to where they are used as soon as they are there, and the loop waits for what it should only have asked for.
      for (; t + kPagedWaves < t_end; t += kPagedWaves) {
        const unsigned valid = n_valid;
        stage();
        fetch(t + kPagedWaves);
        ask(min(t + 2 * kPagedWaves, t_end - 1));
        products(t, valid);
      }
      stage();
      products(t, n_valid);
    }
    l_run = over_quads(l_run, true);

    // ---- this window's partial: the waves meet in LDS (over the tiles: everyone is done)
    __syncthreads();
    float *mg = (float *)&tiles[0][0];  // [wave][head][MS]
    if (col < live) {
      float *dst = mg + (wave * kPagedHeads + col) * MS;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) *(f32x4 *)(dst + 16 * nb + 4 * quad) = O[nb];
      if (quad == 0) {
        dst[D] = m_run;
        dst[D + 1] = l_run;
      }
    }
    __syncthreads();
    const long long slot = blockIdx.x + (slice.by_window ? 0 : order);  // one more with the workgroup, the window or both
    for (int i = tid; i < live * (D / 4); i += 64 * kPagedWaves) {
      const int head = i / (D / 4), d = (i % (D / 4)) * 4;
      float top = -INFINITY;
#pragma unroll
      for (int x = 0; x < kPagedWaves; ++x) top = fmaxf(top, mg[(x * kPagedHeads + head) * MS + D]);
      const float ref = top == -INFINITY ? 0.f : top;
      float l = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < kPagedWaves; ++x) {
        const float *src = mg + (x * kPagedHeads + head) * MS;
        // 0 for a wave without rows; one whose scores are all NaN has no maximum either, and its NaN sums stay NaN
        const float wgt = __builtin_amdgcn_exp2f((src[D] - ref) * c);
        l += src[D + 1] * wgt;
        const f32x4 part = *(const f32x4 *)(src + d);
        o += part * wgt;
      }
      if constexpr (kWhole) {
        store_out<D>(a, (long long)b * a.Hq + head0 + head, d, o, l, ref);
        if (kMass && d == 0) {
          sm_join[head][0] = ref;
          sm_join[head][1] = l == 0.f ? 0.f : 1.f / l;
        }
      } else {
        float *dst = a.slots + (slot * a.g + pass * kPagedHeads + head) * ws_slot_floats(D);
        *(f32x4 *)(dst + d) = o;
        if (d == 0) *(float2 *)(dst + D) = float2{top, l};
      }
    }
    if constexpr (kWhole) {
      if constexpr (kMass) {  // one pass of heads: the window's scores are this workgroup's own
        __syncthreads();
        if (in_set(a.heads.past, h)) {
          const float *scores = a.scores + (long long)(b * a.n_past + set_before(a.heads.past, h)) * a.g * a.score_rows;
          for (int r = tid; r < n; r += 64 * kPagedWaves) {
            int in_page;
            const int page = page_of(a.c, table, r, in_page);
            if (page < 0) continue;
            float sum = 0.f;
            for (int j = 0; j < live; ++j)
              sum += __builtin_amdgcn_exp2f((scores[(r / kPagedTile * a.g + j) * kPagedTile + r % kPagedTile] - sm_join[j][0]) * c) * sm_join[j][1];
            a.c.mass[row_place(a.c, page, h, in_page)] += sum;
          }
        }
      }
      return;
    }
    if (tid == 0 && pass == 0) {
      if (tile0 == 0) a.pieces[w].x = (int)slot;
      if (t_end == base + all) a.pieces[w].y = (int)slot;
    }
    __syncthreads();  // the merge area is tile space again
  }
}

// Maximum and sum of one head of a window over its partials, in the wave that asks (lanes take the partials in turn).
__device__ inline void joined_sum(const float *ml, long long stride, int count, float c, float &top, float &l) {
  const int lane = threadIdx.x & 63;
  top = -INFINITY;
  l = 0.f;
  for (int s = lane; s < count; s += 64) {
    const float2 x = *(const float2 *)(ml + s * stride);
    const float m_new = fmaxf(top, x.x), ref = m_new == -INFINITY ? 0.f : m_new;
    l = l * __builtin_amdgcn_exp2f((top - ref) * c) + x.y * __builtin_amdgcn_exp2f((x.x - ref) * c);
    top = m_new;
  }
#pragma unroll
  for (int sh = 1; sh < 64; sh <<= 1) {
    const float m2 = __shfl_xor(top, sh), l2 = __shfl_xor(l, sh);
    const float m_new = fmaxf(top, m2), ref = m_new == -INFINITY ? 0.f : m_new;
    l = l * __builtin_amdgcn_exp2f((top - ref) * c) + l2 * __builtin_amdgcn_exp2f((m2 - ref) * c);
    top = m_new;
  }
}

constexpr int kJoinBatch = 4;    // partials of a wave under way together
constexpr int kMassRows = 1024;  // rows a workgroup adds the weights of

// Workgroups 0 .. B Hq - 1: merge of one query head's partials.  The others: weights of kMassRows rows of one PAST
// head's window, from the scores that the first launch left.
template <int D>
__global__ __launch_bounds__(256) void paged_decode_join_kernel(const PagedDecodeArgs a, const int mass_chunks, const int first_wg) {
  constexpr int SF = D + kWsTailFloats;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const float c = a.scale_log2e;
  const int heads = a.B * a.Hq, wg = first_wg + (int)blockIdx.x;
  if (wg < heads) {
    const int b = wg / a.Hq, head = wg - b * a.Hq, w = b * a.Hkv + head / a.g;
    // A partial is read by D / 4 lanes, so a wave has kGroups of them at a time, and kJoinBatch of those under way.
    constexpr int kLanes = D / 4, kGroups = 64 / kLanes;
    __shared__ float sm_m[4], sm_l[4];
    __shared__ __attribute__((aligned(16))) float sm_o[4][D];
    const bool some = paged_tiles(a, w) > 0;
    const int2 piece = some ? a.pieces[w] : int2{0, -1};
    const float *ws = a.slots + ((long long)piece.x * a.g + head % a.g) * SF;
    const int count = piece.y - piece.x + 1, group = wave * kGroups + lane / kLanes, d = lane % kLanes * 4;
    float top = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = group; s0 - group < count; s0 += 4 * kGroups * kJoinBatch) {
      float2 ml[kJoinBatch];
      f32x4 x[kJoinBatch];
#pragma unroll
      for (int i = 0; i < kJoinBatch; ++i) {
        const int s = s0 + 4 * kGroups * i;
        const float *src = ws + (long long)(s < count ? s : count - 1) * a.g * SF;
        ml[i] = *(const float2 *)(src + D);
        x[i] = *(const f32x4 *)(src + d);
      }
      float m_new = top;
#pragma unroll
      for (int i = 0; i < kJoinBatch; ++i)
        if (s0 + 4 * kGroups * i < count) m_new = fmaxf(m_new, ml[i].x);
      const float ref = m_new == -INFINITY ? 0.f : m_new, keep = __builtin_amdgcn_exp2f((top - ref) * c);
      top = m_new;
      l *= keep;
      o *= keep;
#pragma unroll
      for (int i = 0; i < kJoinBatch; ++i) {
        if (s0 + 4 * kGroups * i < count) {
          const float wgt = __builtin_amdgcn_exp2f((ml[i].x - ref) * c);
          l += ml[i].y * wgt;
          o += x[i] * wgt;
        }
      }
    }
    float most = top;
#pragma unroll
    for (int sh = kLanes; sh < 64; sh <<= 1) most = fmaxf(most, __shfl_xor(most, sh));
    {
      const float wgt = __builtin_amdgcn_exp2f((top - (most == -INFINITY ? 0.f : most)) * c);
      l *= wgt;
      o *= wgt;
    }
#pragma unroll
    for (int sh = kLanes; sh < 64; sh <<= 1) {
      l += __shfl_xor(l, sh);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], sh);
    }
    if (lane == 0) {
      sm_m[wave] = most;
      sm_l[wave] = l;
    }
    if (lane < kLanes) *(f32x4 *)(&sm_o[wave][d]) = o;
    __syncthreads();
    if (tid >= kLanes) return;
    top = fmaxf(fmaxf(sm_m[0], sm_m[1]), fmaxf(sm_m[2], sm_m[3]));
    const float ref = top == -INFINITY ? 0.f : top;
    l = 0.f;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float wgt = __builtin_amdgcn_exp2f((sm_m[x] - ref) * c);
      l += sm_l[x] * wgt;
      o += *(const f32x4 *)(&sm_o[x][d]) * wgt;
    }
    store_out<D>(a, (long long)b * a.Hq + head, d, o, l, ref);
    return;
  }
  const int i = wg - heads, win = i / mass_chunks, chunk = i - win * mass_chunks;
  const int b = win / a.n_past;
  int h = 0;  // the (win % n_past)-th PAST head
  for (int k = win - b * a.n_past; h < a.Hkv; ++h)
    if (in_set(a.heads.past, h) && k-- == 0) break;
  const int w = b * a.Hkv + h, n = rows_held(a.rows, w, a.max_rows);
  if (chunk * kMassRows >= n) return;
  // A thread has four consecutive rows.  What it reads is asked for before the sums are joined, which takes a chain of loads too.
  __shared__ float sm_top[kPagedMostGroup], sm_share[kPagedMostGroup];
  const int r0 = chunk * kMassRows + 4 * tid;
  const int *table = table_of(a.c, a.Hkv, b, h);
  const int rs = r0 < n ? r0 : 0;  // (the rows up to a whole tile are there)
  const float *scores = a.scores + ((long long)win * a.score_rows + rs / kPagedTile * kPagedTile) * a.g + rs % kPagedTile;
  // A thread's rows lie in one page: their weights are one access of 16 bytes, not four that each touch all lines (24
  // sequences of 1K to 32K: 18 us instead of 25).
  const bool together = a.c.page_rows.d % 4 == 0;
  long long place[4];
  float mass[4];
  if (together) {
    int in_page;
    const int page = r0 < n ? page_of(a.c, table, r0, in_page) : -1;
    const long long at = page < 0 ? 0 : row_place(a.c, page, h, in_page);
    *(f32x4 *)mass = *(const f32x4_any *)(a.c.mass + at);
#pragma unroll
    for (int x = 0; x < 4; ++x) place[x] = page < 0 || r0 + x >= n ? -1 : at + x;
  } else {
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      int in_page;
      const int page = r0 + x < n ? page_of(a.c, table, r0 + x, in_page) : -1;
      place[x] = page < 0 ? -1 : row_place(a.c, page, h, in_page);
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) mass[x] = a.c.mass[place[x] < 0 ? 0 : place[x]];
  }
  float4 first[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) first[j] = *(const float4 *)(scores + (j < a.g ? j : 0) * kPagedTile);
  const int2 piece = a.pieces[w];
  for (int j = wave; j < a.g; j += 4) {
    float top, l;
    joined_sum(a.slots + ((long long)piece.x * a.g + j) * SF + D, (long long)a.g * SF, piece.y - piece.x + 1, c, top, l);
    if (lane == 0) {
      sm_top[j] = top == -INFINITY ? 0.f : top;
      sm_share[j] = l == 0.f ? 0.f : 1.f / l;
    }
  }
  __syncthreads();
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](float4 s, int j) __attribute__((always_inline)) {
    sum[0] += __builtin_amdgcn_exp2f((s.x - sm_top[j]) * c) * sm_share[j];
    sum[1] += __builtin_amdgcn_exp2f((s.y - sm_top[j]) * c) * sm_share[j];
    sum[2] += __builtin_amdgcn_exp2f((s.z - sm_top[j]) * c) * sm_share[j];
    sum[3] += __builtin_amdgcn_exp2f((s.w - sm_top[j]) * c) * sm_share[j];
  };
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (j < a.g) add(first[j], j);
  for (int j = 4; j < a.g; ++j) add(*(const float4 *)(scores + j * kPagedTile), j);
  if (together && place[3] >= 0) {
    *(f32x4_any *)(a.c.mass + place[0]) = *(const f32x4 *)mass + *(const f32x4 *)sum;
  } else {
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (place[x] >= 0) a.c.mass[place[x]] = mass[x] + sum[x];
  }
}

template <int D, bool kE4m3, bool kInPage, bool kMass>
static hipError_t launch_split(PagedDecodeArgs a, hipStream_t st) {
  static ResidentCount count;
  const auto kern = paged_decode_split_kernel<D, kE4m3, kInPage, kMass, false>;
  const int resident = count.get((const void *)kern, 256, 0);
  if (resident == 0) return hipErrorUnknown;
  long long grid = resident < kPagedMostWgs ? resident : kPagedMostWgs;
  const long long tiles = (a.max_rows + kPagedTile - 1) / kPagedTile;
  const long long slices = a.n_windows * ((tiles + kPagedWaves - 1) / kPagedWaves);  // at most, of the shortest length
  const int passes = (a.g + kPagedHeads - 1) / kPagedHeads;
  const long long per_cu = a.n_windows / device_cus(), whole = kPagedWholeRows * (per_cu < 1 ? 1 : per_cu > 8 ? 8 : per_cu);
  if ((long long)a.max_rows * D <= whole * 128 && !(kMass && passes > 1)) {
    hipLaunchKernelGGL((paged_decode_split_kernel<D, kE4m3, kInPage, kMass, true>), dim3((unsigned)a.n_windows, passes), dim3(256), 0, st, a);
    return hipGetLastError();
  }
  a.fits = slices <= grid;
  if (a.fits) grid = slices;
  else if (a.n_windows <= kPagedLaneWindows && grid < 2 * a.n_windows) grid = 2 * a.n_windows;  // paged_slice needs spare ones
  hipLaunchKernelGGL(kern, dim3((unsigned)grid, passes), dim3(256), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int chunks = kMass ? (a.max_rows + kMassRows - 1) / kMassRows : 0;
  const long long joins = (long long)a.B * a.Hq + (long long)a.B * a.n_past * chunks;  // < 2^30 + 2^26 + 2^24
  return launch_in_parts(joins, 256, [&](long long first, unsigned count) {
    hipLaunchKernelGGL(paged_decode_join_kernel<D>, dim3(count), dim3(256), 0, st, a, chunks, (int)first);
  });
}
template <int D, bool kE4m3, bool kInPage>
static hipError_t launch_split(const PagedDecodeArgs &a, hipStream_t st) {
  return a.scores ? launch_split<D, kE4m3, kInPage, true>(a, st) : launch_split<D, kE4m3, kInPage, false>(a, st);
}
template <int D>
static hipError_t launch_paged(const PagedDecodeArgs &a, hipStream_t st) {
  const bool in_page = a.c.page_rows.d % kPagedTile == 0;
  return a.c.e4m3 ? (in_page ? launch_split<D, true, true>(a, st) : launch_split<D, true, false>(a, st))
                  : (in_page ? launch_split<D, false, true>(a, st) : launch_split<D, false, false>(a, st));
}

hipError_t launch_paged_decode(const PagedDecodeArgs &a, hipStream_t st) {
  return a.D == 128 ? launch_paged<128>(a, st) : launch_paged<64>(a, st);
}

}  // namespace segattn
