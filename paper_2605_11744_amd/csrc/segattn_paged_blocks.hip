// seg_kv_paged_summarize and seg_kv_paged_choose: 8-bit bounds of the keys of a block, and the blocks that promise a query the most.
//
// Largest and smallest values do not depend on an order, their scale is a power of two, and a score is a sum of products of
// 8-bit whole numbers: below 2 * 128 * 2^14 in magnitude, so that it is the same however it is formed, and so is the choice.
#include <type_traits>

#include "segattn_sparse.h"

namespace segattn {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// Exponent e of the smallest scale with most <= 127 * 2^e: most = m 2^x with m in [1/2, 1) is at most 127/128 2^x, or above.
__device__ inline int scale_exponent(float most) {
  int x;
  const float m = frexpf(most, &x);
  return x - 7 + (m > 127.f / 128.f ? 1 : 0);
}
// x / 2^e rounded up, for quotients of at most 127: one above zero is 1 or more, also where it is below the smallest float.
__device__ inline int rounded_up(float x, int e) {
  const int y = (int)ceilf(ldexpf(x, -e));
  return x > 0.f && y < 1 ? 1 : y;
}
__device__ inline float finite_or_zero(float x) { return fabsf(x) < INFINITY ? x : 0.f; }

// Where block j of a window has its bounds and its scale (and the first of its rows): -1 without a page.
struct BlockAt {
  long long block, row;
};
__device__ inline BlockAt block_at(const PagedBlocksArgs &a, const int *table, int h, int j) {
  int in_page;
  const int page = page_of(a.c, table, j * (int)a.block_rows.d, in_page);
  if (page < 0) return BlockAt{-1, 0};
  const int hh = a.c.per_head ? 0 : h;
  return BlockAt{((long long)page * a.c.heads + hh) * a.per_page + fast_div(in_page, a.block_rows), row_offset(a.c, page, h, in_page)};
}

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Two bf16 as whole numbers in the same order (infinities and NaN at the ends), and back.
__device__ inline s16x2 ordered(unsigned x) {
  const s16x2 v = __builtin_bit_cast(s16x2, x);
  return __builtin_bit_cast(s16x2, x ^ (__builtin_bit_cast(unsigned, v >> 15) & 0x7fff7fffu));
}
__device__ inline float value_of(short x) { return __uint_as_float((unsigned)(unsigned short)(x ^ ((x >> 15) & 0x7fff)) << 16); }
__device__ inline s16x2 from_lane(s16x2 x, int mask) { return __builtin_bit_cast(s16x2, __shfl_xor(__builtin_bit_cast(int, x), mask)); }

// A wave per block.  Lane l has 16 bytes, kChannels channels, of the rows l / kLanes, l / kLanes + kRows, ...  The largest and smallest keys
// are found as bf16 (8-bit keys times their scales are), two at a time as whole numbers; a block in which one is not finite, or of scales
// so small that bf16 would not hold the keys, is done again in 32 bits.  The lanes of a column then share its channels out.  Bound by memory
// and by the chain row counts -> page -> rows: 152K 8-bit rows of eight heads 39.5 us, 4.1 TB/s (32 us where the last call left them in the caches);
// with keys compared one by one in 32 bits 48, with runs of blocks for a wave, the next one's rows on their way, 56 instead of the 41 of then.
// kAhead: loads of rows on their way.
template <int D, bool kE4m3, int kAhead>
__global__ __launch_bounds__(256) void paged_summarize_kernel(const PagedBlocksArgs a, const long long first_wg) {
  constexpr int kChannels = kE4m3 ? 16 : 8, kLanes = D / kChannels, kRows = 64 / kLanes, kPairs = kChannels / 2;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long unit = (first_wg + blockIdx.x) * 4 + wave;
  if (unit >= a.units) return;
  const long long win = unit / a.most;
  const int j0 = (int)(unit - win * a.most);
  const int b = (int)(win / a.n_past), h = a.past[(int)(win - (long long)b * a.n_past)];
  const long long w = (long long)b * a.Hkv + h;
  const int from = a.rows_from ? fast_div(rows_held(a.rows_from, w, a.c.cap), a.block_rows) : 0;
  const int to = fast_div(rows_held(a.rows, w, a.c.cap), a.block_rows);
  const long long j = (long long)from + j0;
  if (j >= to) return;
  const BlockAt at = block_at(a, table_of(a.c, a.Hkv, b, h), h, (int)j);
  if (at.block < 0) return;
  const int col = lane % kLanes, r0 = lane / kLanes, rows = (int)a.block_rows.d;
  const unsigned char *k = a.c.k + at.row + (long long)r0 * a.c.row_bytes + col * 16;
  const unsigned char *scales = nullptr;
  if constexpr (kE4m3) scales = a.c.k_scale + at.block * rows;  // per_page * block_rows = page_rows
  s16x2 hi[kPairs], lo[kPairs];
#pragma unroll
  for (int e = 0; e < kPairs; ++e) {
    hi[e] = s16x2{-32768, -32768};
    lo[e] = s16x2{32767, 32767};
  }
  int least_scale = 255;
  for (int r = 0; r < rows; r += kAhead * kRows) {  // rows is a multiple of 16, kRows 4, 8 or 16
    u32x4 v[kAhead];
    int sc[kAhead];  // scale bytes
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      const int row = r + x * kRows < rows ? r + x * kRows : 0;  // (once more the first ones)
      if constexpr (kE4m3) sc[x] = scales[row + r0];
      v[x] = *(const u32x4 *)(k + (long long)row * a.c.row_bytes);
    }
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      unsigned y[kPairs];
      if constexpr (kE4m3) {
        const float size = __uint_as_float((unsigned)sc[x] << 23);
        least_scale = sc[x] < least_scale ? sc[x] : least_scale;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y[2 * e] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[x][e], size, false));
          y[2 * e + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[x][e], size, true));
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = v[x][e];
      }
#pragma unroll
      for (int e = 0; e < kPairs; ++e) {
        const s16x2 z = ordered(y[e]);
        hi[e] = __builtin_elementwise_max(hi[e], z);
        lo[e] = __builtin_elementwise_min(lo[e], z);
      }
    }
  }
  // A step leaves each lane half of the pairs, until it has one: pair `pair`, and channels 2 pair and 2 pair + 1 of its 16 bytes.
  int pair = 0;
  bool writes = true;
  const auto halve = [&](auto step) __attribute__((always_inline)) {
    constexpr int sh = kLanes << decltype(step)::value, n = kPairs >> (decltype(step)::value + 1);  // pairs left
    if constexpr (sh < 64) {
      const bool upper = (lane & sh) != 0;
      if constexpr (n > 0) {
        pair += upper ? n : 0;
#pragma unroll
        for (int e = 0; e < n; ++e) {
          const s16x2 my_hi = upper ? hi[n + e] : hi[e], my_lo = upper ? lo[n + e] : lo[e];
          hi[e] = __builtin_elementwise_max(my_hi, from_lane(upper ? hi[e] : hi[n + e], sh));
          lo[e] = __builtin_elementwise_min(my_lo, from_lane(upper ? lo[e] : lo[n + e], sh));
        }
      } else {
        writes &= !upper;
        hi[0] = __builtin_elementwise_max(hi[0], from_lane(hi[0], sh));
        lo[0] = __builtin_elementwise_min(lo[0], from_lane(lo[0], sh));
      }
    }
  };
  halve(std::integral_constant<int, 0>());
  halve(std::integral_constant<int, 1>());
  halve(std::integral_constant<int, 2>());
  halve(std::integral_constant<int, 3>());
  float top[2] = {value_of(hi[0][0]), value_of(hi[0][1])}, bottom[2] = {value_of(lo[0][0]), value_of(lo[0][1])};
  const bool odd = (kE4m3 && least_scale < 16) || !(fabsf(top[0]) < INFINITY) || !(fabsf(top[1]) < INFINITY) || !(fabsf(bottom[0]) < INFINITY) ||
                   !(fabsf(bottom[1]) < INFINITY);
  if (__builtin_amdgcn_ballot_w64(odd)) {
    float t[kChannels], u[kChannels];
#pragma unroll
    for (int e = 0; e < kChannels; ++e) {
      t[e] = -INFINITY;
      u[e] = INFINITY;
    }
#pragma unroll 1
    for (int r = 0; r < rows; r += kRows) {
      const u32x4 v = *(const u32x4 *)(k + (long long)r * a.c.row_bytes);
      float x[kChannels];
      if constexpr (kE4m3) {
        const float size = ldexpf(1.f, (int)scales[r + r0] - 127);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const f32x2 p = __builtin_amdgcn_cvt_pk_f32_fp8(v[e], false), q = __builtin_amdgcn_cvt_pk_f32_fp8(v[e], true);
          x[4 * e] = p[0] * size;
          x[4 * e + 1] = p[1] * size;
          x[4 * e + 2] = q[0] * size;
          x[4 * e + 3] = q[1] * size;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[2 * e] = __uint_as_float(v[e] << 16);
          x[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
        }
      }
#pragma unroll
      for (int e = 0; e < kChannels; ++e) {
        const float y = finite_or_zero(x[e]);
        t[e] = fmaxf(t[e], y);
        u[e] = fminf(u[e], y);
      }
    }
#pragma unroll
    for (int e = 0; e < kChannels; ++e) {
#pragma unroll
      for (int sh = kLanes; sh < 64; sh <<= 1) {
        t[e] = fmaxf(t[e], __shfl_xor(t[e], sh));
        u[e] = fminf(u[e], __shfl_xor(u[e], sh));
      }
      if (e / 2 == pair) {
        top[e % 2] = t[e];
        bottom[e % 2] = u[e];
      }
    }
  }
  float most = fmaxf(fmaxf(fabsf(top[0]), fabsf(bottom[0])), fmaxf(fabsf(top[1]), fabsf(bottom[1])));
#pragma unroll
  for (int sh = 1; sh < 64; sh <<= 1) most = fmaxf(most, __shfl_xor(most, sh));
  int exponent = most > 0.f ? scale_exponent(most) : kLeastBoundExponent;
  exponent = exponent < kLeastBoundExponent ? kLeastBoundExponent : exponent;
  if (!writes) return;
  const int up0 = rounded_up(top[0], exponent), up1 = rounded_up(top[1], exponent);
  const int down0 = -rounded_up(-bottom[0], exponent), down1 = -rounded_up(-bottom[1], exponent);
  signed char *dst = a.bounds + at.block * (2 * D) + kChannels * col + 2 * pair;
  *(unsigned short *)dst = (unsigned short)((up0 & 255) | (up1 & 255) << 8);
  *(unsigned short *)(dst + D) = (unsigned short)((down0 & 255) | (down1 & 255) << 8);
  if (lane == 0) a.scale[at.block] = (unsigned char)(exponent + 127);
}

hipError_t launch_paged_summarize(const PagedBlocksArgs &a, hipStream_t st) {
  const int at_once = 64 * 16 / (a.D * (a.c.e4m3 ? 1 : 2));  // rows of a load
  const bool few = (int)a.block_rows.d <= 4 * at_once;
  const auto of = [&](auto few_kernel, auto many_kernel) { return few ? few_kernel : many_kernel; };
  const auto kern = a.D == 128 ? (a.c.e4m3 ? of(paged_summarize_kernel<128, true, 4>, paged_summarize_kernel<128, true, 8>)
                                           : of(paged_summarize_kernel<128, false, 4>, paged_summarize_kernel<128, false, 8>))
                               : (a.c.e4m3 ? of(paged_summarize_kernel<64, true, 4>, paged_summarize_kernel<64, true, 8>)
                                           : of(paged_summarize_kernel<64, false, 4>, paged_summarize_kernel<64, false, 8>));
  return launch_in_parts((a.units + 3) / 4, 256, [&](long long first, unsigned count) {
    hipLaunchKernelGGL(kern, dim3(count), dim3(256), 0, st, a, first);
  });
}

// ---- choice ------------------------------------------------------------------------------------
// A block's place among the blocks of a token: larger is better, 0 without a page.  The score's units are 2^-32 of what the
// definition says, so that no scale of bf16 keys leaves the normal floats.
__device__ inline unsigned order_key(int dot, int scale) {
  const float x = (float)dot * ldexpf(1.f, scale - 127 - 32);
  const unsigned bits = __float_as_uint(x);
  return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}

// Scores of 16 query rows (tokens of a sequence times a group's heads, padded to a power of two) against 16 blocks at a time:
//   S[query][block] = [q+ | q-] . [upper | lower]     v_mfma_i32_16x16x64_i8, A = queries, B = bounds, K = 2 D
// and then the largest over a token's heads.  GP: heads of a token in a tile, a power of two up to 16; a group of more takes passes
// of 16.
constexpr int kScoreSets = 4;
template <int D>
struct QueryRows {
  static constexpr int NK = D / 64;
  i32x4 up[NK], down[NK];  // this lane's 16 channels of every 64, of row lane % 16: what is above zero, and what is below
  int shift;               // rounded: q * 2^shift

  __device__ __attribute__((always_inline)) void round(const unsigned short *q) {
#pragma unroll
    for (int kc = 0; kc < NK; ++kc) {
      up[kc] = down[kc] = i32x4{0, 0, 0, 0};
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const u32x4 v = *(const u32x4 *)(q + 64 * kc + 8 * half);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int x0 = (int)rintf(ldexpf(finite_or_zero(__uint_as_float(v[e] << 16)), shift));
          const int x1 = (int)rintf(ldexpf(finite_or_zero(__uint_as_float(v[e] & 0xffff0000u)), shift));
          const int word = 2 * half + e / 2, at8 = 16 * (e % 2);
          up[kc][word] |= ((x0 > 0 ? x0 : 0) << at8) | ((x1 > 0 ? x1 : 0) << (at8 + 8));
          down[kc][word] |= ((x0 < 0 ? x0 & 255 : 0) << at8) | ((x1 < 0 ? x1 & 255 : 0) << (at8 + 8));
        }
      }
    }
  }
};

// The blocks [first, hi) of the tokens t .. t + here - 1 of sequence b and the PAST head h, by `waves` waves of which this is number
// `wave`: emit(number of the token, block, key).  QT: sets of 16 query rows that share a block's bounds (1 in passes).
template <int D, int GP, int QT, typename Emit>
__device__ __attribute__((always_inline)) void score_blocks(const PagedChooseArgs &a, long long t, int here, int b, int h, int hi, int wave, int waves, Emit emit) {
  constexpr int NK = D / 64, kAtOnce = QT > 1 ? 1 : 2;  // groups of 16 blocks under way together
  const int lane = threadIdx.x & 63, quad = lane >> 4, col = lane & 15;
  const int *table = table_of(a.k.c, a.k.Hkv, b, h);
  const int passes = GP < 16 ? 1 : (a.g + 15) / 16;
  const int head = col % GP;  // of this lane's query row
  // A set's queries (of head 0), and the scale of every token's.
  auto queries = [&](int qt, int &shift) __attribute__((always_inline)) {
    const int token = qt * (16 / GP) + col / GP;
    const unsigned short *q0 = a.q + ((t + (token < here ? token : 0)) * a.Hq + h * a.g) * D + 16 * quad;
    float most = 0.f;  // the largest magnitude
    for (int p = 0; p < passes; ++p) {
      if (p * 16 + head < a.g) {
        const unsigned short *q = q0 + (p * 16 + head) * D;
#pragma unroll
        for (int kc = 0; kc < NK; ++kc)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const u32x4 v = *(const u32x4 *)(q + 64 * kc + 8 * half);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              most = fmaxf(most, fmaxf(fabsf(finite_or_zero(__uint_as_float(v[e] << 16))), fabsf(finite_or_zero(__uint_as_float(v[e] & 0xffff0000u)))));
          }
      }
    }
#pragma unroll
    for (int sh = 1; sh < GP; sh <<= 1) most = fmaxf(most, __shfl_xor(most, sh));
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    shift = most > 0.f ? -scale_exponent(most) : 0;
    return q0;
  };
  QueryRows<D> rows[QT];
  const unsigned short *q0 = nullptr;
  // (rows beyond the group repeat the pass's head 0, which the largest value does not notice)
  auto take = [&](int p) __attribute__((always_inline)) { rows[0].round(q0 + (p * 16 + (p * 16 + head < a.g ? head : 0)) * D); };
  if constexpr (QT > 1) {  // each of the workgroup's four waves rounds a set (all of them by every wave: 2533 tokens 79 us instead of 63)
    static_assert(QT == 4, "");
    __shared__ i32x4 sm_rows[QT][2 * NK][64];
    const int mine = threadIdx.x >> 6;
    q0 = queries(mine, rows[0].shift);
    take(0);
    __syncthreads();  // (the tokens before are read)
#pragma unroll
    for (int kc = 0; kc < NK; ++kc) {
      sm_rows[mine][kc][lane] = rows[0].up[kc];
      sm_rows[mine][NK + kc][lane] = rows[0].down[kc];
    }
    __syncthreads();
#pragma unroll
    for (int qt = 0; qt < QT; ++qt)
#pragma unroll
      for (int kc = 0; kc < NK; ++kc) {
        rows[qt].up[kc] = sm_rows[qt][kc][lane];
        rows[qt].down[kc] = sm_rows[qt][NK + kc][lane];
      }
  } else {
    q0 = queries(0, rows[0].shift);
    take(0);
  }
  const int step = 16 * kAtOnce * waves;
  for (int j0 = a.first + 16 * kAtOnce * wave; j0 < hi; j0 += step) {
    i32x4 bd[kAtOnce][2 * NK];
    int scale[kAtOnce];
    bool named[kAtOnce];
#pragma unroll
    for (int x = 0; x < kAtOnce; ++x) {
      const int j = j0 + 16 * x + col;
      const long long at = j < hi ? block_at(a.k, table, h, j).block : -1;
      named[x] = at >= 0;
      const signed char *bounds = a.k.bounds + (named[x] ? at : 0) * (2 * D) + 16 * quad;
#pragma unroll
      for (int kc = 0; kc < 2 * NK; ++kc) bd[x][kc] = *(const i32x4 *)(bounds + 64 * kc);
      scale[x] = a.k.scale[named[x] ? at : 0];
    }
#pragma unroll
    for (int x = 0; x < kAtOnce; ++x) {
      const int j = j0 + 16 * x + col;
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        int best[4];
        for (int p = 0; p < passes; ++p) {
          if (passes > 1) take(p);
          i32x4 S = {0, 0, 0, 0};
#pragma unroll
          for (int kc = 0; kc < NK; ++kc) {
            S = __builtin_amdgcn_mfma_i32_16x16x64_i8(rows[qt].up[kc], bd[x][kc], S, 0, 0, 0);
            S = __builtin_amdgcn_mfma_i32_16x16x64_i8(rows[qt].down[kc], bd[x][NK + kc], S, 0, 0, 0);
          }
          // register r of S: query row 4 quad + r, block col
#pragma unroll
          for (int r = 0; r < 4; ++r) best[r] = p == 0 || S[r] > best[r] ? S[r] : best[r];
        }
        // the largest over the rows of a token
#pragma unroll
        for (int sh = 1; sh < (GP < 4 ? GP : 4); sh <<= 1)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if ((r & sh) == 0) best[r] = best[r] > best[r + sh] ? best[r] : best[r + sh];
        int top = best[0];
        if constexpr (GP >= 8) {
          const int y = __shfl_xor(top, 16);
          top = top > y ? top : y;
        }
        if constexpr (GP >= 16) {
          const int y = __shfl_xor(top, 32);
          top = top > y ? top : y;
        }
        if (j < hi) {
#pragma unroll
          for (int r = 0; r < 4; r += GP < 4 ? GP : 4) {
            const int tok = qt * (16 / GP) + (4 * quad + r) / GP;
            if (tok < here && (GP <= 4 || (4 * quad) % GP == 0)) emit(tok, j, named[x] ? order_key(GP <= 2 ? best[r] : top, scale[x]) : 0u);
          }
        }
      }
    }
  }
}

// The next tokens of a tile that belong to one sequence: b, and `here` of them from token t on, of which the last sees the blocks up to
// `hi` - 1 behind the newest ones (0: all of its blocks are taken, nothing is scored).  false: behind the last sequence.
__device__ inline bool tile_tokens(const PagedChooseArgs &a, long long t, long long t_end, int h, int &b, int &here, int &i, int &n, int &hi) {
  b = sequence_of(a.cu, a.k.B, t, i, n);
  if (b < 0) return false;
  here = (int)(t_end - t < n - i ? t_end - t : n - i);
  const int seen = rows_seen(a.k.rows, (long long)b * a.k.Hkv + h, i + here - 1, n, a.max_rows);
  const int own = seen > 0 ? fast_div(seen - 1, a.k.block_rows) : -1;
  hi = own + 1 > a.n_chosen ? own - a.recent + 1 : 0;
  return true;
}

// Keys to the workspace, where they do not fit LDS.  One token each: bound by memory behind the chain row counts -> page -> bounds (64 sequences
// of up to 64K rows, eight heads, 72 MB of bounds: 23 us, 3.1 TB/s).  Many tokens: QT sets of 16 query rows meet each group of bounds in registers
// (2533 tokens of four heads behind up to 60K rows 43 us, 0.39 POP/s; a set at a time 107), and what bounds it is the work on the sums -- the
// largest of a token's heads, the order's key, a store each -- which is a few times that of the products.
template <int D, int GP, int QT>
__global__ __launch_bounds__(256) void paged_score_kernel(const PagedChooseArgs a, const long long t_first, const long long first_wg, const int wgs_per_unit) {
  const long long wg = first_wg + blockIdx.x, unit = wg / wgs_per_unit, tile = unit / a.k.n_past;
  const int share = (int)(wg - unit * wgs_per_unit), ph = (int)(unit - tile * a.k.n_past), h = a.k.past[ph];
  long long t = t_first + tile * a.tile;
  const long long t_end = t + a.tile < a.total ? t + a.tile : a.total;
  int b, here, i, n, hi;
  for (; t < t_end && tile_tokens(a, t, t_end, h, b, here, i, n, hi); t += here) {
    if (hi <= a.first) continue;
    score_blocks<D, GP, QT>(a, t, here, b, h, hi, (threadIdx.x >> 6) + 4 * share, 4 * wgs_per_unit,
                        [&](int tok, int j, unsigned key) { a.keys[((t + tok - t_first) * a.k.n_past + ph) * a.stride + j] = key; });
  }
}

// What a list holds besides the picks among [lo, hi): everything where the blocks are few (0 picks left), else the first and the newest ones.
// By `threads` threads of which this is number `me`.
__device__ inline int list_frame(const PagedChooseArgs &a, int seen, int *out, int me, int threads, int &hi) {
  const int own = seen > 0 ? fast_div(seen - 1, a.k.block_rows) : -1;
  hi = own - a.recent + 1;
  if (own + 1 <= a.n_chosen) {
    for (int x = me; x < a.n_chosen; x += threads) out[x] = x <= own ? x : -1;
    return 0;
  }
  const int picks = a.n_chosen - a.first - a.recent;
  for (int x = me; x < a.first + a.recent; x += threads) out[x < a.first ? x : picks + x] = x < a.first ? x : hi + x - a.first;
  return picks;
}

// The `picks` largest of the keys of the blocks [first, hi), more of them than picks, into out[0 ..] in the blocks' order; among equals the
// lower block.  A lane keeps kHeld keys in registers.  By a team of kWaves waves (1: no barriers) of which this is number `wave`, each with a run of the blocks.  The keys are
// counted in 256 bins that span them, then those of the bin in which the last pick lies in as many, until a bin's end lies between two
// picks or the bins are single keys: two or three times.
template <int kWaves>
struct Team {
  int bins[256];
  unsigned most[kWaves], least[kWaves];
  int above[kWaves], equal[kWaves];
  unsigned base;  // of the bin
  int bin_above, bin_in;
};
template <int kWaves, int kHeld = 8, typename Keys>
__device__ __attribute__((always_inline)) void pick_blocks(const Keys keys, int first, int hi, int picks, int *out, Team<kWaves> &sm, int wave) {
  const int lane = threadIdx.x & 63, me = wave * 64 + lane;
  // (one wave: its LDS accesses are done in order, but the compiler has to leave them so -- what another lane writes, it sees no reason for)
  const auto meet = [] {
    if constexpr (kWaves > 1) {
      __syncthreads();
    } else {
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
  };
  // this wave's run, in whole rounds of 64 blocks
  const int rounds = (hi - first + 64 * kWaves - 1) / (64 * kWaves);
  const int from = first + wave * rounds * 64, to = min(hi, from + rounds * 64);
  unsigned held[kHeld];
#pragma unroll
  for (int r = 0; r < kHeld; ++r) held[r] = from + 64 * r + lane < to ? (unsigned)keys[from + 64 * r + lane] : 0u;
  const auto each = [&](auto what) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < kHeld; ++r)
      if (from + 64 * r < to) what(from + 64 * r + lane < to, held[r], from + 64 * r + lane);
    for (int j = from + 64 * kHeld; j < to; j += 64) what(j + lane < to, j + lane < to ? (unsigned)keys[j + lane] : 0u, j + lane);
  };
  unsigned most = 0u, least = ~0u;
  each([&](bool is, unsigned key, int) {
    most = is && key > most ? key : most;
    least = is && key < least ? key : least;
  });
#pragma unroll
  for (int sh = 1; sh < 64; sh <<= 1) {
    const unsigned y = __shfl_xor(most, sh), z = __shfl_xor(least, sh);
    most = y > most ? y : most;
    least = z < least ? z : least;
  }
  if constexpr (kWaves > 1) {
    if (lane == 0) {
      sm.most[wave] = most;
      sm.least[wave] = least;
    }
    __syncthreads();
    for (int y = 0; y < kWaves; ++y) {
      most = max(most, sm.most[y]);
      least = min(least, sm.least[y]);
    }
  }
  // keys from `end` on are picks; those of [base, end) are looked at, `left` of them are picks
  unsigned base = least, span = most - least;
  int left = picks;
  bool exact = false;
  for (;;) {
    const int bits = span == 0 ? 0 : 32 - __clz(span), shift = bits > 8 ? bits - 8 : 0;
    for (int x = me; x < 256; x += 64 * kWaves) sm.bins[x] = 0;
    meet();
    each([&](bool is, unsigned key, int) {
      if (is && key >= base && key - base <= span) atomicAdd(&sm.bins[(key - base) >> shift], 1);
    });
    meet();
    if (wave == 0) {
      int c[4], sum = 0;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        c[x] = sm.bins[255 - (4 * lane + x)];
        sum += c[x];
      }
      int before = sum;
#pragma unroll
      for (int sh = 1; sh < 64; sh <<= 1) {
        const int up = __shfl_up(before, sh);
        if (lane >= sh) before += up;
      }
      before -= sum;
      if (before < left && before + sum >= left) {  // one lane: the bin of the last pick is among its four
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          if (before < left && before + c[x] >= left) {
            sm.base = base + ((unsigned)(255 - (4 * lane + x)) << shift);
            sm.bin_above = before;
            sm.bin_in = c[x];
            before = 0x40000000;  // found
          } else {
            before += c[x];
          }
        }
      }
    }
    meet();
    base = sm.base;
    left -= sm.bin_above;
    exact = sm.bin_in == left;
    if (exact || shift == 0) break;
    span = (1u << shift) - 1;
    meet();  // the bins are read
  }
  // the blocks with keys from `base` on (exact), or above it and of those that equal it the first `left`
  const auto above = [&](unsigned key) { return exact ? key >= base : key > base; };
  int place = 0, equals = 0;
  if constexpr (kWaves > 1) {
    int n_above = 0, n_equal = 0;
    each([&](bool is, unsigned key, int) {
      n_above += __popcll(__builtin_amdgcn_ballot_w64(is && above(key)));
      n_equal += __popcll(__builtin_amdgcn_ballot_w64(is && !exact && key == base));
    });
    if (lane == 0) {
      sm.above[wave] = n_above;
      sm.equal[wave] = n_equal;
    }
    __syncthreads();
    for (int y = 0; y < wave; ++y) {
      place += sm.above[y];
      equals += sm.equal[y];
    }
  }
  if (exact) left = 0;
  each([&](bool is, unsigned key, int j) {
    const bool is_above = is && above(key), is_equal = is && !exact && key == base;
    const unsigned long long ups = __builtin_amdgcn_ballot_w64(is_above), eqs = __builtin_amdgcn_ballot_w64(is_equal), below = (1ull << lane) - 1;
    const int eq = equals + __popcll(eqs & below);
    if (is_above || (is_equal && eq < left)) out[place + __popcll(ups & below) + (eq < left ? eq : left)] = j;
    place += __popcll(ups);
    equals += __popcll(eqs);
  });
}

// Scores and choice in one launch: a tile's keys stay in LDS.  A token's picks are found by one wave where the tile has several tokens, by
// all waves together where it has one.
template <int D, int GP>
__global__ __launch_bounds__(256) void paged_choose_kernel(const PagedChooseArgs a, const long long first_wg) {
  constexpr int kThreads = 256, kWaves = kThreads / 64;
  extern __shared__ unsigned sm_keys[];  // [token of the tile][stride]
  __shared__ union {
    Team<kWaves> all;
    Team<1> one[kWaves];
  } sm;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const long long unit = first_wg + blockIdx.x, tile = unit / a.k.n_past;
  const int ph = (int)(unit - tile * a.k.n_past), h = a.k.past[ph];
  long long t = tile * a.tile;
  const long long t_end = t + a.tile < a.total ? t + a.tile : a.total;
  int b, here, i, n, all_hi;
  for (; t < t_end && tile_tokens(a, t, t_end, h, b, here, i, n, all_hi); t += here) {
    if (all_hi > a.first)
      score_blocks<D, GP, 1>(a, t, here, b, h, all_hi, wave, kWaves, [&](int tok, int j, unsigned key) { sm_keys[tok * a.stride + j] = key; });
    __syncthreads();
    const bool together = here == 1;
    for (int tok = together ? 0 : wave; tok < here; tok += together ? 1 : kWaves) {
      int *out = a.chosen + ((t + tok) * a.k.n_past + ph) * a.n_chosen;
      const int seen = rows_seen(a.k.rows, (long long)b * a.k.Hkv + h, i + tok, n, a.max_rows);
      int hi;
      const int picks = list_frame(a, seen, out, together ? tid : lane, together ? kThreads : 64, hi);
      if (picks == 0) continue;
      if (together) pick_blocks<kWaves>(sm_keys, a.first, hi, picks, out + a.first, sm.all, wave);
      else pick_blocks<1>(sm_keys + tok * a.stride, a.first, hi, picks, out + a.first, sm.one[wave], 0);
    }
    __syncthreads();  // the keys are read
  }
}

// The choice from keys in the workspace: a workgroup per (token, PAST head), or (kAlone) a wave.  Bound by the latencies of its two or three
// rounds of counting: 10132 lists of 32 from up to 970 keys 23 us, 512 lists from up to 1024 keys 7.
template <int kThreads, bool kAlone>
__global__ __launch_bounds__(kThreads) void paged_select_kernel(const PagedChooseArgs a, const long long t_first, const long long units, const long long first_wg) {
  constexpr int kTeams = kAlone ? kThreads / 64 : 1, kWaves = kThreads / 64 / kTeams;
  __shared__ Team<kWaves> sm[kTeams];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), team = kAlone ? wave : 0, me = kAlone ? threadIdx.x & 63 : threadIdx.x;
  const long long u = (first_wg + blockIdx.x) * kTeams + team, t = t_first + u / a.k.n_past;
  if (u >= units) return;
  const int ph = (int)(u % a.k.n_past);
  int i, n;
  const int b = sequence_of(a.cu, a.k.B, t, i, n);
  if (b < 0) return;
  const int seen = rows_seen(a.k.rows, (long long)b * a.k.Hkv + a.k.past[ph], i, n, a.max_rows);
  int *out = a.chosen + (t * a.k.n_past + ph) * a.n_chosen;
  int hi;
  const int picks = list_frame(a, seen, out, me, 64 * kWaves, hi);
  if (picks) pick_blocks<kWaves, kAlone ? 16 : 8>(a.keys + u * a.stride, a.first, hi, picks, out + a.first, sm[team], kAlone ? 0 : wave);
}

template <int D, int GP>
static hipError_t launch_choose(const PagedChooseArgs &a, hipStream_t st) {
  if (a.in_lds) {
    const size_t lds = (size_t)a.tile * a.stride * 4;
    return launch_in_parts((a.total + a.tile - 1) / a.tile * a.k.n_past, 256, [&](long long first, unsigned count) {
      hipLaunchKernelGGL((paged_choose_kernel<D, GP>), dim3(count), dim3(256), lds, st, a, first);
    });
  }
  for (long long t = 0; t < a.total; t += a.part) {
    const long long n = a.total - t < a.part ? a.total - t : a.part, units = n * a.k.n_past, tiles = (n + a.tile - 1) / a.tile * a.k.n_past;
    // enough workgroups to fill the card, none with fewer than 128 blocks (3 a compute unit and 6: 64 sequences of up to 64K rows, eight heads,
    // 28.7 us and 30.4 with the choice; 2533 tokens of four heads 63 and 65)
    const long long groups = (a.stride + 127) / 128;
    long long share = (3 * device_cus() + tiles - 1) / tiles;
    share = share < 1 ? 1 : share > groups ? groups : share;
    PagedChooseArgs part = a;
    part.total = t + n;
    hipError_t e = launch_in_parts(tiles * share, 256, [&](long long first, unsigned count) {
      if (a.tile > 16 / GP) hipLaunchKernelGGL((paged_score_kernel<D, GP, GP < 16 ? kScoreSets : 1>), dim3(count), dim3(256), 0, st, part, t, first, (int)share);
      else hipLaunchKernelGGL((paged_score_kernel<D, GP, 1>), dim3(count), dim3(256), 0, st, part, t, first, (int)share);
    });
    if (e != hipSuccess) return e;
    const bool few = units < 2 * device_cus(), many = units >= 16 * device_cus();
    e = launch_in_parts(many ? (units + 3) / 4 : units, few ? 1024 : 256, [&](long long first, unsigned count) {
      if (few) hipLaunchKernelGGL((paged_select_kernel<1024, false>), dim3(count), dim3(1024), 0, st, a, t, units, first);
      else if (many) hipLaunchKernelGGL((paged_select_kernel<256, true>), dim3(count), dim3(256), 0, st, a, t, units, first);
      else hipLaunchKernelGGL((paged_select_kernel<256, false>), dim3(count), dim3(256), 0, st, a, t, units, first);
    });
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Tokens of a tile: one where no sequence has more; as many as 16 query rows hold, or several times as many where the sequences have them.
void plan_paged_choose(PagedChooseArgs &a, long long max_seqlen) {
  const int gp = a.g <= 1 ? 1 : a.g <= 2 ? 2 : a.g <= 4 ? 4 : a.g <= 8 ? 8 : 16, set = 16 / gp;
  a.in_lds = a.stride <= kChoiceInLds;
  a.tile = max_seqlen == 1 ? 1 : !a.in_lds && gp < 16 && max_seqlen >= 2 * kScoreSets * set ? kScoreSets * set : set;
}

template <int D>
static hipError_t launch_choose(const PagedChooseArgs &a, hipStream_t st) {
  return a.g <= 1 ? launch_choose<D, 1>(a, st) : a.g <= 2 ? launch_choose<D, 2>(a, st) : a.g <= 4 ? launch_choose<D, 4>(a, st)
         : a.g <= 8 ? launch_choose<D, 8>(a, st) : launch_choose<D, 16>(a, st);
}
hipError_t launch_paged_choose(const PagedChooseArgs &a, hipStream_t st) {
  return a.k.D == 128 ? launch_choose<128>(a, st) : launch_choose<64>(a, st);
}

}  // namespace segattn
