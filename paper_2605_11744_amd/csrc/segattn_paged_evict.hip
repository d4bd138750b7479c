// seg_kv_paged_evict: of every PAST head that holds more than `keep` rows the `keep` with the largest keys stay.
//
// A row's key is the bits of its accumulated weight (weights are not negative, so their bits order as they do;
// what is negative or NaN counts as 0), or the largest of all where its position is among the `recent` newest
// or the `first` first ones.  Equal keys: the lower row stays.  Rows that stay and lie at or behind row `keep`
// move, in order, into the places below that become free: attention does not depend on the order of rows, a row
// is moved at most once, and no place that is read is written, so all rows move at once.
//
// select: one workgroup per window finds the key of rank `keep` by counting, a byte of the key at a time, then lists
// the free places and the rows that go there.  move: copies them, many workgroups per window.  Bound by the
// bytes of the moved rows where many move, else by the passes over the keys.
#include "segattn_paged.h"

namespace segattn {

constexpr unsigned kSureKey = 0xffffffffu;
constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;

__device__ inline unsigned evict_key(const PagedEvictArgs &a, int newest, float mass, int pos) {
  if ((long long)pos > (long long)newest - a.recent || (a.first > 0 && pos < a.first)) return kSureKey;
  return mass > 0.f ? __float_as_uint(mass) : 0u;
}

__global__ __launch_bounds__(kSelectThreads) void paged_select_kernel(const PagedEvictArgs a) {
  const int w = blockIdx.x, b = w / a.Hkv, h = w - b * a.Hkv;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  __shared__ int sm_hist[256], sm_part[kSelectWaves], sm_part2[kSelectWaves];
  __shared__ int sm_pick[2];
  const int n = rows_held(a.rows, w, a.max_rows);
  __syncthreads();  // rows may be rows_out
  const bool evicts = in_set(a.heads.past, h) && n > a.keep;
  if (tid == 0) {
    a.rows_out[w] = evicts ? a.keep : a.rows[w];
    if (!evicts) a.moves[w] = 0;
  }
  if (!evicts) return;
  const int *table = table_of(a.c, a.Hkv, b, h);
  int newest = -0x7fffffff - 1;
  for (int r = tid; r < n; r += kSelectThreads) {
    int in_page;
    const int page = page_of(a.c, table, r, in_page);
    if (page < 0) continue;
    const int pos = a.c.pos[row_place(a.c, page, h, in_page)];
    newest = pos > newest ? pos : newest;
  }
#pragma unroll
  for (int sh = 1; sh < 64; sh <<= 1) {
    const int x = __shfl_xor(newest, sh);
    newest = x > newest ? x : newest;
  }
  if (lane == 0) sm_part[wave] = newest;
  __syncthreads();
  newest = sm_part[0];
#pragma unroll
  for (int x = 1; x < kSelectWaves; ++x) newest = sm_part[x] > newest ? sm_part[x] : newest;
  __syncthreads();
  auto key_of = [&](int r) __attribute__((always_inline)) {  // a row without a page: the lowest
    int in_page;
    const int page = page_of(a.c, table, r, in_page);
    if (page < 0) return 0u;
    const long long place = row_place(a.c, page, h, in_page);
    return evict_key(a, newest, a.c.mass[place], a.c.pos[place]);
  };
  // The key of rank keep, a byte at a time from the top: among the rows that agree with it so far, count by the next
  // byte and walk down to the one in which the rank falls.
  unsigned edge = 0;
  int rank = a.keep;  // the edge's rank among the rows that agree with it
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) sm_hist[tid] = 0;
    __syncthreads();
    for (int r = tid; r < n; r += kSelectThreads) {
      const unsigned key = key_of(r);
      if (shift == 24 || (key >> (shift + 8)) == (edge >> (shift + 8))) atomicAdd(&sm_hist[(key >> shift) & 255], 1);
    }
    __syncthreads();
    if (wave == 0) {  // lane i has the counts of bytes 255 - 4 i .. 252 - 4 i
      int own[4], sum = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        own[j] = sm_hist[255 - 4 * lane - j];
        sum += own[j];
      }
      int incl = sum;
#pragma unroll
      for (int sh = 1; sh < 64; sh <<= 1) {
        const int up = __shfl_up(incl, sh);
        if (lane >= sh) incl += up;
      }
      int above = incl - sum;
      if (above < rank && rank <= incl) {
        int j = 0;
        while (j < 3 && above + own[j] < rank) above += own[j++];
        sm_pick[0] = 255 - 4 * lane - j;
        sm_pick[1] = rank - above;
      }
    }
    __syncthreads();
    edge |= (unsigned)sm_pick[0] << shift;
    rank = sm_pick[1];
    __syncthreads();
  }
  // `rank` rows with the edge's key stay.  Wave x lists a run of rows of its own: first how many edge keys lie before it.
  const int run = (n + kSelectThreads - 1) / kSelectThreads * 64;
  const int r0 = wave * run, r1 = r0 + run < n ? r0 + run : n;
  int ties = 0;
  for (int r = r0; r < r1; r += 64) ties += __popcll(__builtin_amdgcn_ballot_w64(r + lane < r1 && key_of(r + lane) == edge));
  if (lane == 0) sm_part[wave] = ties;
  __syncthreads();
  int ties_before = 0;
  for (int x = 0; x < wave; ++x) ties_before += sm_part[x];
  __syncthreads();
  const unsigned long long below = (1ull << lane) - 1;
  int places = 0, movers = 0;
  int *place_list = a.lists + (long long)w * 2 * a.most_moves, *mover_list = place_list + a.most_moves;
  for (int pass = 0; pass < 2; ++pass) {
    int seen = ties_before;
    for (int r = r0; r < r1; r += 64) {
      const bool in = r + lane < r1;
      const unsigned key = in ? key_of(r + lane) : 0u;
      const unsigned long long tie = __builtin_amdgcn_ballot_w64(in && key == edge);
      const bool stays = in && (key > edge || (key == edge && seen + __popcll(tie & below) < rank));
      seen += __popcll(tie);
      const bool is_place = in && !stays && r + lane < a.keep, is_mover = stays && r + lane >= a.keep;
      const unsigned long long pm = __builtin_amdgcn_ballot_w64(is_place), mm = __builtin_amdgcn_ballot_w64(is_mover);
      if (pass == 1) {
        const int ip = places + __popcll(pm & below), im = movers + __popcll(mm & below);
        if (is_place && ip < a.most_moves) place_list[ip] = r + lane;
        if (is_mover && im < a.most_moves) mover_list[im] = r + lane;
      }
      places += __popcll(pm);
      movers += __popcll(mm);
    }
    if (pass == 1) break;
    if (lane == 0) {
      sm_part[wave] = places;
      sm_part2[wave] = movers;
    }
    __syncthreads();
    places = movers = 0;
    int all = 0;
    for (int x = 0; x < kSelectWaves; ++x) {
      if (x < wave) {
        places += sm_part[x];
        movers += sm_part2[x];
      }
      all += sm_part2[x];
    }
    if (tid == 0) a.moves[w] = all < a.most_moves ? all : a.most_moves;
  }
}

// D * 2 (D for e4m3) bytes of keys and values per row, 16 a lane.
__global__ __launch_bounds__(256) void paged_move_kernel(const PagedEvictArgs a) {
  const int w = blockIdx.x, b = w / a.Hkv, h = w - b * a.Hkv;
  const int count = a.moves[w];
  const int pieces = (a.c.e4m3 ? a.D : 2 * a.D) / 16, per = 256 / (2 * pieces);  // lanes per tensor, rows at a time
  const int piece = threadIdx.x % pieces, is_v = (threadIdx.x / pieces) & 1, mine = threadIdx.x / (2 * pieces);
  const int *table = table_of(a.c, a.Hkv, b, h);
  const int *place_list = a.lists + (long long)w * 2 * a.most_moves, *mover_list = place_list + a.most_moves;
  unsigned char *pool = is_v ? a.c.v : a.c.k;
  for (int i = blockIdx.y * per + mine; i < count; i += gridDim.y * per) {
    int to_row, of_row;
    const int to = page_of(a.c, table, place_list[i], to_row), of = page_of(a.c, table, mover_list[i], of_row);
    if (to < 0 || of < 0) continue;
    *(uint4 *)(pool + row_offset(a.c, to, h, to_row) + 16 * piece) = *(const uint4 *)(pool + row_offset(a.c, of, h, of_row) + 16 * piece);
    if (piece == 0) {
      const long long p1 = row_place(a.c, to, h, to_row), p0 = row_place(a.c, of, h, of_row);
      if (a.c.e4m3) (is_v ? a.c.v_scale : a.c.k_scale)[p1] = (is_v ? a.c.v_scale : a.c.k_scale)[p0];
      if (is_v) a.c.mass[p1] = a.c.mass[p0];
      else a.c.pos[p1] = a.c.pos[p0];
    }
  }
}

hipError_t launch_paged_evict(const PagedEvictArgs &a, hipStream_t st) {
  const int windows = a.B * a.Hkv;
  hipLaunchKernelGGL(paged_select_kernel, dim3(windows), dim3(kSelectThreads), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.most_moves == 0) return e;
  int wgs = 4096 / windows;
  const int most = (a.most_moves + 7) / 8;
  wgs = wgs < 1 ? 1 : wgs > most ? most : wgs;
  hipLaunchKernelGGL(paged_move_kernel, dim3(windows, wgs), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace segattn
