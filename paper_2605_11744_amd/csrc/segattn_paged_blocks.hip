// seg_kv_paged_summarize and seg_kv_paged_choose: 8-bit bounds of the keys of a block, and the blocks that promise a query the most.
//
// Largest and smallest values do not depend on an order, their scale is a power of two, and a score is a sum of products of
// 8-bit whole numbers: below 2 * 128 * 2^14 in magnitude, so that it is the same however it is formed, and so is the choice.
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

// A wave per block.  Lane l has channels 8 (l % L) .. + 7 (L = D / 8 lanes a row) of the rows l / L, l / L + 64 / L, ...
template <int D, bool kE4m3>
__global__ __launch_bounds__(256) void paged_summarize_kernel(const PagedBlocksArgs a, const long long first_wg) {
  constexpr int kLanes = D / 8, kRows = 64 / kLanes;
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
  const unsigned char *k = a.c.k + at.row + (long long)r0 * a.c.row_bytes + col * (kE4m3 ? 8 : 16);
  const unsigned char *scales = nullptr;
  if constexpr (kE4m3) scales = a.c.k_scale + at.block * rows + r0;  // per_page * block_rows = page_rows
  float hi[8], lo[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    hi[e] = -INFINITY;
    lo[e] = INFINITY;
  }
  auto take = [&](const float *x) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float y = finite_or_zero(x[e]);
      hi[e] = fmaxf(hi[e], y);
      lo[e] = fminf(lo[e], y);
    }
  };
#pragma unroll 4
  for (int r = 0; r < rows; r += kRows) {  // rows is a multiple of 16, kRows 4 or 8
    float x[8];
    if constexpr (kE4m3) {
      const u32x2 v = *(const u32x2 *)(k + (long long)r * a.c.row_bytes);
      const float size = ldexpf(1.f, (int)scales[r] - 127);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const f32x2 p = __builtin_amdgcn_cvt_pk_f32_fp8(v[e], false), q = __builtin_amdgcn_cvt_pk_f32_fp8(v[e], true);
        x[4 * e] = p[0] * size;
        x[4 * e + 1] = p[1] * size;
        x[4 * e + 2] = q[0] * size;
        x[4 * e + 3] = q[1] * size;
      }
    } else {
      const u32x4 v = *(const u32x4 *)(k + (long long)r * a.c.row_bytes);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[2 * e] = __uint_as_float(v[e] << 16);
        x[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
      }
    }
    take(x);
  }
  float most = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
#pragma unroll
    for (int sh = kLanes; sh < 64; sh <<= 1) {
      hi[e] = fmaxf(hi[e], __shfl_xor(hi[e], sh));
      lo[e] = fminf(lo[e], __shfl_xor(lo[e], sh));
    }
    most = fmaxf(most, fmaxf(fabsf(hi[e]), fabsf(lo[e])));
  }
#pragma unroll
  for (int sh = 1; sh < kLanes; sh <<= 1) most = fmaxf(most, __shfl_xor(most, sh));
  int exponent = most > 0.f ? scale_exponent(most) : kLeastBoundExponent;
  exponent = exponent < kLeastBoundExponent ? kLeastBoundExponent : exponent;
  if (r0 != 0) return;
  u32x2 up = {0u, 0u}, down = {0u, 0u};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int u = (int)ceilf(ldexpf(hi[e], -exponent)), d = (int)floorf(ldexpf(lo[e], -exponent));
    up[e / 4] |= (unsigned)(u & 255) << (8 * (e % 4));
    down[e / 4] |= (unsigned)(d & 255) << (8 * (e % 4));
  }
  signed char *dst = a.bounds + at.block * (2 * D) + 8 * col;
  *(u32x2 *)dst = up;
  *(u32x2 *)(dst + D) = down;
  if (col == 0) a.scale[at.block] = (unsigned char)(exponent + 127);
}

hipError_t launch_paged_summarize(const PagedBlocksArgs &a, hipStream_t st) {
  const auto kern = a.D == 128 ? (a.c.e4m3 ? paged_summarize_kernel<128, true> : paged_summarize_kernel<128, false>)
                               : (a.c.e4m3 ? paged_summarize_kernel<64, true> : paged_summarize_kernel<64, false>);
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
// and then the largest over a token's heads.  Units are (tile of tokens, PAST head); a tile's tokens belong to one sequence.
// GP: heads of a token in a tile, a power of two up to 16; a group of more takes passes of 16.
template <int D, int GP>
__global__ __launch_bounds__(256) void paged_score_kernel(const PagedChooseArgs a, const long long t_first, const long long first_wg, const int wgs_per_unit) {
  constexpr int NK = D / 64, kTokens = 16 / GP;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, quad = lane >> 4, col = lane & 15;
  const long long wg = first_wg + blockIdx.x, unit = wg / wgs_per_unit;
  const int share = (int)(wg - unit * wgs_per_unit);
  const long long tile = unit / a.k.n_past;
  const int ph = (int)(unit - tile * a.k.n_past), h = a.k.past[ph];
  // tokens t0 .. of the part; a tile may meet the ends of sequences: every row of queries has its own
  const long long t0 = t_first + tile * kTokens;
  if (t0 >= a.total) return;
  // sequence of the tile's tokens: tiles go over the tokens end to end, so up to kTokens sequences share one; each is scored
  // by itself
  long long t = t0;
  const long long t_end = t0 + kTokens < a.total ? t0 + kTokens : a.total;
  while (t < t_end) {
    int i, n;
    const int b = sequence_of(a.cu, a.k.B, t, i, n);
    if (b < 0) return;  // behind the last sequence
    const int here = (int)(t_end - t < n - i ? t_end - t : n - i);  // tokens of it in the tile
    const long long w = (long long)b * a.k.Hkv + h;
    const int seen = rows_seen(a.k.rows, w, i + here - 1, n, a.max_rows);  // of the last one
    const int own = seen > 0 ? fast_div(seen - 1, a.k.block_rows) : -1;
    const int hi = own + 1 > a.n_chosen ? own - a.recent + 1 : 0;  // blocks [first, hi) are scored
    if (hi > a.first) {
      const int *table = table_of(a.k.c, a.k.Hkv, b, h);
      // the largest magnitude of every token's queries
      float most = 0.f;
      const int passes = (a.g + 15) / 16;
      const int token = col / GP, head = col % GP;  // of this lane's query row
      const bool mine = token < here;
      for (int p = 0; p < passes; ++p) {
        if (mine && p * 16 + head < a.g) {
          const unsigned short *q = a.q + ((t + token) * a.Hq + h * a.g + p * 16 + head) * D + 16 * quad;
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
      const int shift = most > 0.f ? -scale_exponent(most) : 0;
      for (int j0 = a.first + 16 * (wave + 4 * share); j0 < hi; j0 += 64 * wgs_per_unit) {
        const int j = j0 + col;
        const BlockAt at = j < hi ? block_at(a.k, table, h, j) : BlockAt{-1, 0};
        const signed char *bounds = a.k.bounds + (at.block < 0 ? 0 : at.block) * (2 * D) + 16 * quad;
        i32x4 bd[2 * NK];
#pragma unroll
        for (int kc = 0; kc < 2 * NK; ++kc) bd[kc] = *(const i32x4 *)(bounds + 64 * kc);
        const int scale = a.k.scale[at.block < 0 ? 0 : at.block];
        int best[4] = {-0x7fffffff - 1, -0x7fffffff - 1, -0x7fffffff - 1, -0x7fffffff - 1};
        for (int p = 0; p < passes; ++p) {
          const bool live = mine && p * 16 + head < a.g;
          const unsigned short *q = a.q + ((t + (mine ? token : 0)) * a.Hq + h * a.g + (live ? p * 16 + head : 0)) * D + 16 * quad;
          i32x4 S = {0, 0, 0, 0};
#pragma unroll
          for (int kc = 0; kc < NK; ++kc) {
            i32x4 up = {0, 0, 0, 0}, down = {0, 0, 0, 0};
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const u32x4 v = *(const u32x4 *)(q + 64 * kc + 8 * half);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int x0 = (int)rintf(ldexpf(finite_or_zero(__uint_as_float(v[e] << 16)), shift));
                const int x1 = (int)rintf(ldexpf(finite_or_zero(__uint_as_float(v[e] & 0xffff0000u)), shift));
                const int word = 2 * half + e / 2, at8 = 16 * (e % 2);
                up[word] |= ((x0 > 0 ? x0 : 0) << at8) | ((x1 > 0 ? x1 : 0) << (at8 + 8));
                down[word] |= ((x0 < 0 ? x0 & 255 : 0) << at8) | ((x1 < 0 ? x1 & 255 : 0) << (at8 + 8));
              }
            }
            S = __builtin_amdgcn_mfma_i32_16x16x64_i8(up, bd[kc], S, 0, 0, 0);
            S = __builtin_amdgcn_mfma_i32_16x16x64_i8(down, bd[NK + kc], S, 0, 0, 0);
          }
          // register r of S: query row 4 quad + r, block col.  The rows beyond the group repeat its head 0 of the pass
#pragma unroll
          for (int r = 0; r < 4; ++r) best[r] = S[r] > best[r] ? S[r] : best[r];
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
            const int tok = (4 * quad + r) / GP;
            if (tok < here && (GP <= 4 || (4 * quad) % GP == 0))
              a.keys[((t + tok - t_first) * a.k.n_past + ph) * a.stride + j] =
                  at.block < 0 ? 0u : order_key(GP <= 2 ? best[r] : top, scale);
          }
        }
      }
    }
    t += here;
  }
}

// A workgroup per (token, PAST head): the n-th largest key digit by digit, then a walk in order.
__global__ __launch_bounds__(256) void paged_select_kernel(const PagedChooseArgs a, const long long t_first, const long long first_wg) {
  __shared__ int sm_hist[256], sm_count[4][2];
  __shared__ unsigned sm_digit;
  __shared__ int sm_left;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const long long u = first_wg + blockIdx.x, t = t_first + u / a.k.n_past;
  const int ph = (int)(u % a.k.n_past);
  int i, n;
  const int b = sequence_of(a.cu, a.k.B, t, i, n);
  if (b < 0) return;
  const int seen = rows_seen(a.k.rows, (long long)b * a.k.Hkv + a.k.past[ph], i, n, a.max_rows);
  const int own = seen > 0 ? fast_div(seen - 1, a.k.block_rows) : -1;
  int *out = a.chosen + (t * a.k.n_past + ph) * a.n_chosen;
  if (own + 1 <= a.n_chosen) {
    for (int x = tid; x < a.n_chosen; x += 256) out[x] = x <= own ? x : -1;
    return;
  }
  const int lo = a.first, hi = own - a.recent + 1, picks = a.n_chosen - a.first - a.recent;  // of [lo, hi): more than picks
  for (int x = tid; x < a.first + a.recent; x += 256) out[x < a.first ? x : picks + x] = x < a.first ? x : hi + x - a.first;
  if (picks == 0) return;
  const unsigned *keys = a.keys + u * a.stride;
  unsigned top = 0;  // digits of the picks-th largest key found so far
  int left = picks;  // picks among the keys with these digits
  for (int digit = 3; digit >= 0; --digit) {
    sm_hist[tid] = 0;
    __syncthreads();
    for (int j = lo + tid; j < hi; j += 256) {
      const unsigned key = keys[j];
      if (digit == 3 || (key >> (8 * digit + 8)) == top) atomicAdd(&sm_hist[(key >> (8 * digit)) & 255], 1);
    }
    __syncthreads();
    if (wave == 0) {  // the digit below which fewer than `left` keys lie above
      int c[4], sum = 0;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        c[x] = sm_hist[255 - (4 * lane + x)];
        sum += c[x];
      }
      int incl = sum;
#pragma unroll
      for (int sh = 1; sh < 64; sh <<= 1) {
        const int up = __shfl_up(incl, sh);
        if (lane >= sh) incl += up;
      }
      int before = incl - sum;
      if (before < left && incl >= left) {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          if (before < left && before + c[x] >= left) {
            sm_digit = 255 - (4 * lane + x);
            sm_left = left - before;
            before = 0x40000000;  // found
          } else {
            before += c[x];
          }
        }
      }
    }
    __syncthreads();
    top = (top << 8) | sm_digit;
    left = sm_left;
    __syncthreads();
  }
  // the blocks above `top`, and the first `left` that equal it
  int taken = 0, equals = 0;
  for (int j0 = lo; j0 < hi; j0 += 256) {
    const int j = j0 + tid;
    const unsigned key = j < hi ? keys[j] : 0u;
    const bool equal = j < hi && key == top;
    const unsigned long long eq = __builtin_amdgcn_ballot_w64(equal), above = __builtin_amdgcn_ballot_w64(j < hi && key > top);
    if (lane == 0) {
      sm_count[wave][0] = __popcll(above);
      sm_count[wave][1] = __popcll(eq);
    }
    __syncthreads();
    int at = taken, eq_at = equals;
    for (int x = 0; x < 4; ++x) {
      if (x < wave) {
        at += sm_count[x][0];
        eq_at += sm_count[x][1];
      }
      taken += sm_count[x][0];
      equals += sm_count[x][1];
    }
    const unsigned long long below = (1ull << lane) - 1;
    at += __popcll(above & below);
    eq_at += __popcll(eq & below);
    if ((j < hi && key > top) || (equal && eq_at < left)) out[a.first + at + (eq_at < left ? eq_at : left)] = j;
    __syncthreads();
  }
}

template <int D>
static hipError_t launch_scores(const PagedChooseArgs &a, long long t, long long n, hipStream_t st) {
  const int gp = a.g <= 1 ? 1 : a.g <= 2 ? 2 : a.g <= 4 ? 4 : a.g <= 8 ? 8 : 16;
  const long long units = (n + 16 / gp - 1) / (16 / gp) * a.k.n_past;
  // enough workgroups to fill the card, none with fewer than 64 blocks
  const long long groups = (a.max_rows / a.k.block_rows.d + 63) / 64;
  long long share = (2 * device_cus() + units - 1) / units;
  share = share < 1 ? 1 : share > groups ? (groups < 1 ? 1 : groups) : share;
  const auto kern = gp == 1 ? paged_score_kernel<D, 1> : gp == 2 ? paged_score_kernel<D, 2> : gp == 4 ? paged_score_kernel<D, 4>
                    : gp == 8 ? paged_score_kernel<D, 8> : paged_score_kernel<D, 16>;
  PagedChooseArgs part = a;
  part.total = t + n;
  return launch_in_parts(units * share, 256, [&](long long first, unsigned count) {
    hipLaunchKernelGGL(kern, dim3(count), dim3(256), 0, st, part, t, first, (int)share);
  });
}

hipError_t launch_paged_choose(const PagedChooseArgs &a, hipStream_t st) {
  for (long long t = 0; t < a.total; t += a.part) {
    const long long n = a.total - t < a.part ? a.total - t : a.part;
    hipError_t e = a.k.D == 128 ? launch_scores<128>(a, t, n, st) : launch_scores<64>(a, t, n, st);
    if (e != hipSuccess) return e;
    e = launch_in_parts(n * a.k.n_past, 256, [&](long long first, unsigned count) {
      hipLaunchKernelGGL(paged_select_kernel, dim3(count), dim3(256), 0, st, a, t, first);
    });
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace segattn
