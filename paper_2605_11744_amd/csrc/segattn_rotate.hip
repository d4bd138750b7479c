// seg_rope_rotate: queries and keys of a layer (or their gradients) turned by their positions.
//
// Pair i of a token at position p becomes magnitude * (a cos - b sin, a sin + b cos) with the angle p * f_i; the
// frequencies f_i are the host's business (scaled ones too).  Backward is the same with the negative angle.
// Every element is read and written once; bound by memory.
#include "segattn_rotate.h"

namespace segattn {

constexpr int kRotateRows = 16;

// A workgroup turns up to kRotateRows consecutive tokens: its threads form the sines and cosines of every
// (token, pair) once, in LDS, then walk over the tokens' units in memory order.  Few tokens per workgroup, many workgroups:
// 32K tokens of 32 + 8 heads of 128 took 136 us with 16 tokens, 122 with 4, 118 with 2 (109 with rows marked as not worth
// keeping: 6.2 TB/s).  Units requested before the sines are formed, or several of a thread at once, are no faster (112).
template <typename T, bool kInterleaved>
__global__ __launch_bounds__(256) void rotate_kernel(const RotateArgs a, const int tokens_per_wg, const long long first_wg) {
  constexpr int P = 16 / sizeof(T);
  __shared__ __attribute__((aligned(16))) float sm_sn[kRotateRows][64], sm_cs[kRotateRows][64];
  const int tid = threadIdx.x;
  const long long t0 = (first_wg + blockIdx.x) * tokens_per_wg;
  const int n = a.total - t0 < tokens_per_wg ? (int)(a.total - t0) : tokens_per_wg;
  const int pairs = a.rot.pairs;
  for (int i = tid; i < n * pairs; i += 256) {
    const int r = i / pairs, c = i - r * pairs;
    const long long t = t0 + r, b = t / a.rows;
    const double position = (double)(a.pos ? a.pos[t] : (a.pos0 ? a.pos0[b] : 0) + (t - b * a.rows));
    const float2 sc = turn_of(position, a.rot.turns[c], a.rot.back, a.rot.magnitude);
    sm_sn[r][c] = sc.x;
    sm_cs[r][c] = sc.y;
  }
  __syncthreads();
  const int per_head = a.D / (2 * P);
  auto walk = [&](const T *from, long long stride, T *to, long long to_stride, int heads) __attribute__((always_inline)) {
    const int per_token = heads * per_head;
    int r = tid / per_token, u = tid - r * per_token;
    const int dr = 256 / per_token, du = 256 - dr * per_token;
    while (r < n) {
      const int head = u / per_head, unit = u - head * per_head;
      int c_lo, c_hi;
      unit_channels<P>(unit, pairs, a.D, c_lo, c_hi);
      const T *src = from + (t0 + r) * stride + head * a.D;
      T *dst = to + (t0 + r) * to_stride + head * a.D;
      u32x4 lo = load_piece(src + c_lo), hi = load_piece(src + c_hi);
      if (P * unit < pairs) turn_pieces<P, kInterleaved>(lo, hi, unit, pairs, sm_sn[r], sm_cs[r]);
      store_piece(dst + c_lo, lo);
      store_piece(dst + c_hi, hi);
      r += dr;
      u += du;
      if (u >= per_token) {
        u -= per_token;
        ++r;
      }
    }
  };
  if (a.q) walk((const T *)a.q, a.q_stride, (T *)a.q_out, a.q_out_stride, a.Hq);
  if (a.k) walk((const T *)a.k, a.k_stride, (T *)a.k_out, a.k_out_stride, a.Hkv);
}

hipError_t launch_rotate(const RotateArgs &a, bool fp32, hipStream_t st) {
  // At most 320 units for 256 threads: 1 token of 32 + 8 heads of 128, 10 of 4 + 4 of 64 -- which take
  // 15 us for 27000 tokens, 23 with 2, 39 with 1 -- and fewer where compute units would be idle.  (32K tokens of the former: 320
  // units 105.7 us, 640 108.4, 1280 112.6.)
  const long long units = ((a.q ? a.Hq : 0) + (a.k ? a.Hkv : 0)) * (long long)a.D * (fp32 ? 4 : 2) / 32;
  long long per = 320 / units;
  if (per > a.total / 1024) per = a.total / 1024;
  per = per < 1 ? 1 : per > kRotateRows ? kRotateRows : per;
  const long long blocks = (a.total + per - 1) / per;
  const auto kern = fp32 ? (a.rot.interleaved ? rotate_kernel<float, true> : rotate_kernel<float, false>)
                         : (a.rot.interleaved ? rotate_kernel<unsigned short, true> : rotate_kernel<unsigned short, false>);
  return launch_in_parts(blocks, 256, [&](long long first, unsigned count) {
    hipLaunchKernelGGL(kern, dim3(count), dim3(256), 0, st, a, (int)per, first);
  });
}

}  // namespace segattn
