// seg_kv_paged_append: new tokens enter a paged cache.
//
// Queries are turned by their positions and written to q_out; keys are turned and values taken as they are, and
// both go to the next free rows of their sequence, as bf16 or as e4m3.  An e4m3 row has a scale of its own, the
// smallest power of two 2^e with max |x| <= 448 * 2^e: dividing by it is exact, so a stored value is the
// element rounded once, and e4m3's range loses less than a factor of two of the 2^15 that it spans.  With a
// row: its position, and a weight of zero.  Every input is read and every output written once; bound by
// memory (20K tokens of 32 + 8 heads of 128 into 8-bit rows 82 us = 5.7 TB/s), a generation step by the chain row
// count -> page -> store (48 sequences 5 us).
#include <utility>

#include "segattn_rotate.h"

namespace segattn {

constexpr int kAppendRows = 4;  // (prompts into an 8-bit cache 100 us with 16, 90 with 4, 91 with 2, 99 with 1)

// Exponent e of the scale of a row whose largest finite magnitude is `most`, as the byte e + 127: the binary
// exponent of most minus that of 448 = 1.75 * 2^8, one more where the significand is above 1.75.  Rows
// of zeros have scale 1, tiny ones 2^-119 (so that 1 / scale stays a normal float).
__device__ inline int scale_byte(float most) {
  const unsigned bits = __float_as_uint(most);
  if (bits == 0) return 127;
  const int e = (int)((bits + 0x1fffffu) >> 23) - 8;
  return e < 8 ? 8 : e;
}
__device__ inline float finite_magnitude(float x) {
  const float m = fabsf(x);
  return m < INFINITY ? m : 0.f;  // also 0 for NaN
}
// Eight elements as e4m3: x times 1 / scale is exact, the conversion rounds to nearest even.  e4m3 has no
// infinity: what is not finite becomes NaN.
__device__ inline uint2 e4m3_of(const float *x, float inverse) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = fabsf(x[i]) < INFINITY ? x[i] * inverse : __uint_as_float(0x7fc00000u);
  int a = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  a = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], a, true);
  int b = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
  b = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], b, true);
  return uint2{(unsigned)a, (unsigned)b};
}

// The new row count of window w = b * Hkv + h.
__device__ inline void count_rows(const PagedAppendArgs &a, int w) {
  if (w >= a.B * a.Hkv) return;
  const int b = w / a.Hkv;
  const long long held = rows_held(a.rows, w, a.c.cap);
  const long long sum = held + (a.cu ? a.cu[b + 1] - a.cu[b] : 1);
  a.rows_out[w] = sum < held ? (int)held : sum < a.c.cap ? (int)sum : a.c.cap;
}

// A workgroup takes up to kAppendRows consecutive tokens.  First it finds every token's sequence and every
// (token, head)'s row, and forms the sines, in LDS; then its threads walk over the units of the queries, the
// keys and the values.  The D / 16 threads of a row are neighbours in one wave, which finds an e4m3 row's
// largest magnitude by exchanges between lanes.
template <int D, bool kE4m3, bool kInterleaved>
__global__ __launch_bounds__(256) void paged_append_kernel(const PagedAppendArgs a, const int tokens_per_wg, const int token_wgs, const int first_wg) {
  constexpr int kUnits = D / 16;
  __shared__ __attribute__((aligned(16))) float sm_sn[kAppendRows][64], sm_cs[kAppendRows][64];
  __shared__ int sm_seq[kAppendRows], sm_index[kAppendRows];
  __shared__ int2 sm_row[kAppendRows * kMaxKvHeads];  // page (or -1) and row in it
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int wg = first_wg + (int)blockIdx.x;
  if (wg >= token_wgs) {
    count_rows(a, (wg - token_wgs) * 256 + tid);
    return;
  }
  const int t0 = wg * tokens_per_wg;
  const int n = a.total - t0 < tokens_per_wg ? a.total - t0 : tokens_per_wg;
  // sequence of token t: as many sequences end at or before t
  for (int r = wave; r < n; r += 4) {
    int b = t0 + r, i = 0;
    if (a.cu) {
      b = 0;
      for (int s0 = 0; s0 < a.B; s0 += 64) {
        const bool before = s0 + lane < a.B && a.cu[s0 + lane + 1] <= t0 + r;
        b += __popcll(__builtin_amdgcn_ballot_w64(before));
      }
      b = b < a.B ? b : a.B - 1;
      i = t0 + r - a.cu[b];
    }
    if (lane == 0) {
      sm_seq[r] = b;
      sm_index[r] = i;
    }
  }
  __syncthreads();
  for (int j = tid; j < n * a.Hkv; j += 256) {
    const int r = j / a.Hkv, h = j - r * a.Hkv, b = sm_seq[r];
    const long long row = (long long)rows_held(a.rows, (long long)b * a.Hkv + h, a.c.cap) + sm_index[r];
    int in_page = 0, page = -1;
    if (sm_index[r] >= 0 && row < a.c.cap) page = page_of(a.c, table_of(a.c, a.Hkv, b, h), (int)row, in_page);
    sm_row[j] = int2{page, in_page};
  }
  const int pairs = a.rot.pairs;
  for (int i = tid; i < n * pairs; i += 256) {
    const int r = i / pairs, c = i - r * pairs;
    const double position = (double)((a.pos0 ? a.pos0[sm_seq[r]] : 0) + sm_index[r]);
    const float2 sc = turn_of(position, a.rot.turns[c], 0, a.rot.magnitude);
    sm_sn[r][c] = sc.x;
    sm_cs[r][c] = sc.y;
  }
  __syncthreads();
  if (a.count_rows == 1) {  // one token per sequence: nobody else reads this sequence's counts
    for (int h = tid; h < a.Hkv; h += 256) {
      const long long w = (long long)sm_seq[0] * a.Hkv + h;
      const int held = rows_held(a.rows, w, a.c.cap);
      a.rows_out[w] = held < a.c.cap ? held + 1 : a.c.cap;
    }
  }
  if (a.q_out) {
    const int per_token = a.Hq * kUnits;
    for (int j = tid; j < n * per_token; j += 256) {
      const int r = j / per_token, u = j - r * per_token, unit = u % kUnits;
      int lo, hi;
      unit_channels<8>(unit, pairs, D, lo, hi);
      const long long at = ((long long)(t0 + r) * a.Hq + u / kUnits) * D;
      u32x4 x = load_piece(a.q + at + lo), y = load_piece(a.q + at + hi);
      if (8 * unit < pairs) turn_pieces<8, kInterleaved>(x, y, unit, pairs, sm_sn[r], sm_cs[r]);
      store_piece(a.q_out + at + lo, x);
      store_piece(a.q_out + at + hi, y);
    }
  }
  const int per_token = a.Hkv * kUnits, per_tensor = n * per_token;
  for (int j = tid; j < 2 * per_tensor; j += 256) {  // the keys' units, then the values'
    const bool is_v = j >= per_tensor;
    const int jj = is_v ? j - per_tensor : j;
    const int r = jj / per_token, u = jj - r * per_token, head = u / kUnits, unit = u % kUnits;
    int lo = 16 * unit, hi = lo + 8;
    if (!is_v) unit_channels<8>(unit, pairs, D, lo, hi);
    const unsigned short *src = (is_v ? a.v : a.k) + ((long long)(t0 + r) * a.Hkv + head) * D;
    const u32x4 x_lo = load_piece(src + lo), x_hi = load_piece(src + hi);
    const int2 at = sm_row[r * a.Hkv + head];
    int byte = 0;
    float x[16];
    if constexpr (kE4m3) {
      {
        float p[8], q[8];
        numbers_of(x_lo, p);
        numbers_of(x_hi, q);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[e] = p[e];
          x[8 + e] = q[e];
        }
      }
      if (!is_v && 8 * unit < pairs) turn_unit<8, kInterleaved>(x, unit, pairs, sm_sn[r], sm_cs[r]);
      float most = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) most = fmaxf(most, finite_magnitude(x[e]));
#pragma unroll
      for (int sh = 1; sh < kUnits; sh <<= 1) most = fmaxf(most, __shfl_xor(most, sh));
      byte = scale_byte(most);
    }
    if (at.x < 0) continue;
    unsigned char *dst = (is_v ? a.c.v : a.c.k) + row_offset(a.c, at.x, head, at.y);
    const long long place = row_place(a.c, at.x, head, at.y);
    if constexpr (kE4m3) {
      const float inverse = __uint_as_float((unsigned)(254 - byte) << 23);  // 2^-e
      *(uint2 *)(dst + lo) = e4m3_of(x, inverse);
      *(uint2 *)(dst + hi) = e4m3_of(x + 8, inverse);
      if (unit == 0) (is_v ? a.c.v_scale : a.c.k_scale)[place] = (unsigned char)byte;
    } else {
      u32x4 p = x_lo, q = x_hi;
      if (!is_v && 8 * unit < pairs) turn_pieces<8, kInterleaved>(p, q, unit, pairs, sm_sn[r], sm_cs[r]);
      store_piece((unsigned short *)dst + lo, p);
      store_piece((unsigned short *)dst + hi, q);
    }
    if (unit == 0 && !is_v) {
      if (a.c.pos) a.c.pos[place] = (int)((a.pos0 ? a.pos0[sm_seq[r]] : 0) + sm_index[r]);
      if (a.c.mass) a.c.mass[place] = 0.f;
    }
  }
}

__global__ __launch_bounds__(256) void paged_count_kernel(const PagedAppendArgs a) {
  count_rows(a, blockIdx.x * 256 + threadIdx.x);
}

hipError_t launch_paged_append(const PagedAppendArgs &args, hipStream_t st) {
  PagedAppendArgs a = args;
  int per = a.total / 1024;
  per = per < 1 ? 1 : per > kAppendRows ? kAppendRows : per;
  const int wgs = (a.total + per - 1) / per;
  // Counts that are updated in place can only be written when every token has found its row: by the token's
  // own workgroup where a sequence has one token, else by a launch of its own.
  const bool in_place = a.rows == a.rows_out;
  a.count_rows = !in_place ? 2 : (a.cu == nullptr && per == 1) ? 1 : 0;
  const int count_wgs = (a.B * a.Hkv + 255) / 256, grid = wgs + (a.count_rows == 2 ? count_wgs : 0);
  const auto of = [&](auto turned) { return a.rot.interleaved ? turned.second : turned.first; };
  const auto kern = a.D == 128 ? (a.c.e4m3 ? of(std::make_pair(paged_append_kernel<128, true, false>, paged_append_kernel<128, true, true>))
                                           : of(std::make_pair(paged_append_kernel<128, false, false>, paged_append_kernel<128, false, true>)))
                               : (a.c.e4m3 ? of(std::make_pair(paged_append_kernel<64, true, false>, paged_append_kernel<64, true, true>))
                                           : of(std::make_pair(paged_append_kernel<64, false, false>, paged_append_kernel<64, false, true>)));
  const hipError_t e = launch_in_parts(grid, 256, [&](long long first, unsigned count) {
    hipLaunchKernelGGL(kern, dim3(count), dim3(256), 0, st, a, per, wgs, (int)first);
  });
  if (e != hipSuccess || a.count_rows != 0) return e;
  hipLaunchKernelGGL(paged_count_kernel, dim3(count_wgs), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace segattn
