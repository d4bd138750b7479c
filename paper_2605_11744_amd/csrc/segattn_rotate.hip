// seg_rope_rotate: queries and keys of a layer (or their gradients) turned by their positions.
//
// Pair i of a token at position p becomes magnitude * (a cos - b sin, a sin + b cos) with the angle p * f_i; the
// frequencies f_i are the host's business (scaled ones too).  Backward is the same with the negative angle.
// Every element is read and written once; bound by memory.
#include "segattn_rotate.h"

namespace segattn {

constexpr int kRotateRows = 16;

// A workgroup turns up to kRotateRows consecutive tokens: its threads form the sines and cosines of every
// (token, pair) once, in LDS, then walk over the tokens' units in memory order.
template <typename T>
__global__ __launch_bounds__(256) void rotate_kernel(const RotateArgs a, const int tokens_per_wg) {
  __shared__ __attribute__((aligned(16))) float sm_sn[kRotateRows][64], sm_cs[kRotateRows][64];
  const int tid = threadIdx.x;
  const long long t0 = (long long)blockIdx.x * tokens_per_wg;
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
  const int per_head = a.D / 16;
  auto walk = [&](const T *from, long long stride, T *to, long long to_stride, int heads) __attribute__((always_inline)) {
    const int per_token = heads * per_head;
    int r = tid / per_token, u = tid - r * per_token;
    const int dr = 256 / per_token, du = 256 - dr * per_token;
    while (r < n) {
      const int head = u / per_head, unit = u - head * per_head;
      int lo, hi;
      unit_channels(unit, pairs, a.rot.interleaved, lo, hi);
      const T *src = from + (t0 + r) * stride + head * a.D;
      T *dst = to + (t0 + r) * to_stride + head * a.D;
      float x[16];
      load8(src + lo, x);
      load8(src + hi, x + 8);
      if (8 * unit < pairs) turn_unit(x, &sm_sn[r][8 * unit], &sm_cs[r][8 * unit], a.rot.interleaved);
      store8(dst + lo, x);
      store8(dst + hi, x + 8);
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
  // fewer tokens per workgroup where sixteen would leave compute units idle
  long long per = a.total / 1024;
  per = per < 1 ? 1 : per > kRotateRows ? kRotateRows : per;
  const long long blocks = (a.total + per - 1) / per;
  if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
  if (fp32) hipLaunchKernelGGL(rotate_kernel<float>, dim3((unsigned)blocks), dim3(256), 0, st, a, (int)per);
  else hipLaunchKernelGGL(rotate_kernel<unsigned short>, dim3((unsigned)blocks), dim3(256), 0, st, a, (int)per);
  return hipGetLastError();
}

}  // namespace segattn
