// seg_kv_paged_evict: of every PAST head that holds more than `keep` rows the `keep` with the largest keys stay.
//
// A row's key is one more than the bits of its accumulated weight (weights are not negative, so their bits order as they
// do; what is negative or NaN counts as 0), or above all of those where its position is among the `recent` newest, the
// newest highest, or the `first` first ones.  Key 0 is a row without a page: it is not there, so it neither stays nor is
// a place, and as many rows stay as have a page below row `keep`.  Equal keys: the lower row stays.  Rows that stay and
// lie at or behind row `keep` move, in order, into the places below that become free: attention does not depend on the
// order of rows, a row is moved at most once, and no place that is read is written, so all rows move at once.
//
// select: one workgroup per window finds the key of the last rank that stays by counting, a byte of the key at a time, then lists
// the free places and the rows that go there.  move: copies them, many workgroups per window.  Bound by the
// bytes of the moved rows where many move, else by the passes over the keys: 96 windows of up to 32768 rows to 16384, 48 us
// for the selection and 83 for 0.38 GB of moves (4.6 TB/s); 32 windows of 1100 to 1279 rows to 1024, 10.9 and 4.3.
#include "segattn_paged.h"

namespace segattn {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr unsigned kNewestKey = 0xffffffffu, kFirstKey = 0x80000000u;  // of the newest position, of the first ones
constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;
constexpr int kHeldRows = 32 * kSelectThreads;  // rows whose keys fit the select kernel's LDS
constexpr int kCopies = 4;  // of the histogram: neighbouring lanes count in different ones
constexpr int kAtOnce = 4;  // rows of a lane that are under way together

// The select kernel walks over a window's keys seven times, so they are formed once (a key costs a look into the
// table and two loads) and kept: in LDS (kHeld; the positions in registers until the newest is known), or for longer windows in
// the workspace.  Wave x has a run of consecutive rows, 64 at a time.  The histogram is kept kCopies times: weights share
// few exponents, protected rows all but their low bits, and lanes that count the same byte in one word wait for each other.  (Of 11 bits at
// a time, in one copy: 5.5K rows, 901 of them protected, 18.3 us instead of 17.1.)
//
// One compute unit works on a window, and a vector instruction more per 64 rows is 0.25 us more for 32768.  kInPage:
// page_rows is a multiple of 64, so 64 rows lie in one page and are found with scalar instructions.
template <bool kHeld, bool kInPage>
__global__ __launch_bounds__(kSelectThreads) void paged_select_kernel(const PagedEvictArgs a, const int first_window) {
  const int w = first_window + blockIdx.x, b = w / a.Hkv, h = w - b * a.Hkv;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  extern __shared__ unsigned sm_keys[];
  __shared__ int sm_hist[256 * kCopies];
  __shared__ __attribute__((aligned(16))) int sm_part[kSelectWaves][4];
  __shared__ int sm_pick[3];
  const int n = rows_held(a.rows, w, a.max_rows);
  __syncthreads();  // rows may be rows_out
  const bool past = in_set(a.heads.past, h), evicts = past && n > a.keep;
  if (tid == 0) {
    const int rows = a.rows[w];
    a.rows_out[w] = past && rows > a.budget ? a.budget : rows;
    if (!evicts) a.moves[w] = 0;
  }
  if (!evicts) return;
  unsigned *keys;
  if constexpr (kHeld) keys = sm_keys;
  else keys = a.keys + (long long)w * a.key_rows;
  const int *table = table_of(a.c, a.Hkv, b, h);
  const int run = (n + kSelectThreads - 1) / kSelectThreads * 64;
  const int r0 = wave * run, r1 = r0 + run < n ? r0 + run : n;

  // First the weights' bits, and the newest position; then the rows that stay for their position's sake.
  constexpr int kNowhere = -0x7fffffff - 1;
  int newest = kNowhere, holes = 0;  // holes: the wave's rows below row keep that have no page
  const int lo_end = a.keep < r1 ? a.keep : r1;
  // Places of rows r + 64 i + lane, i < kAtOnce, or -1: of the first one of 64 (kInPage) or of the row.  kInPage: the
  // table's entries for 64 steps of the wave are asked at once, one a lane.
  long long place[kAtOnce];
  int entry = -1;
  auto ask = [&](int r) __attribute__((always_inline)) {
    if constexpr (kInPage) {
      if ((r - r0) % (64 * 64) == 0) {
        int in_page;
        const int row = r + 64 * lane;
        entry = row < r1 ? page_of(a.c, table, row, in_page) : -1;
      }
    }
  };
  auto find = [&](int r) __attribute__((always_inline)) {
    if constexpr (kInPage) {
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int row = r + 64 * i, page = __builtin_amdgcn_readlane(entry, ((row - r0) >> 6) & 63);
        const int in_page = row - fast_div(row, a.c.page_rows) * (int)a.c.page_rows.d;
        place[i] = page < 0 ? -1 : row_place(a.c, page, h, in_page);
      }
    } else {
      int page[kAtOnce], in_page[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int row = r + 64 * i + lane;
        page[i] = page_of(a.c, table, row < n ? row : n - 1, in_page[i]);
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) place[i] = page[i] < 0 ? -1 : row_place(a.c, page[i], h, in_page[i]);
    }
  };
  const int beside = kInPage ? lane : 0;  // (a page has room for all 64 rows, also behind the last one)
  auto form_weights = [&](int r, int (&pos)[kAtOnce]) __attribute__((always_inline)) {  // positions: kNowhere for a row without one
    ask(r);
    find(r);
    float mass[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      pos[i] = (a.c.pos + (place[i] < 0 ? 0 : place[i]))[place[i] < 0 ? 0 : beside];
      mass[i] = (a.c.mass + (place[i] < 0 ? 0 : place[i]))[place[i] < 0 ? 0 : beside];
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const bool held = place[i] >= 0 && r + 64 * i + lane < r1;
      if (r + 64 * i < r0 + run) keys[r + 64 * i + lane] = (held && mass[i] > 0.f ? __float_as_uint(mass[i]) : 0u) + held;
      holes += __popcll(__builtin_amdgcn_ballot_w64(place[i] < 0 && r + 64 * i + lane < lo_end));
      if (!held) pos[i] = kNowhere;
      newest = pos[i] > newest ? pos[i] : newest;
    }
  };
  constexpr int kBatches = kHeldRows / kSelectThreads / kAtOnce;  // of a wave's rows, where their keys fit LDS
  int kept_pos[kHeld ? kBatches : 1][kAtOnce];
  if constexpr (kHeld) {
#pragma unroll
    for (int y = 0; y < kBatches; ++y) {
      if (64 * kAtOnce * y >= run) break;
      form_weights(r0 + 64 * kAtOnce * y, kept_pos[y]);
    }
  } else {
    for (int r = r0; r < r0 + run; r += 64 * kAtOnce) form_weights(r, kept_pos[0]);
  }
#pragma unroll
  for (int sh = 1; sh < 64; sh <<= 1) {
    const int x = __shfl_xor(newest, sh);
    newest = x > newest ? x : newest;
  }
  if (lane == 0) *(int2 *)sm_part[wave] = int2{newest, holes};
  __syncthreads();
  int rank = a.keep;  // rows that stay; below, the edge's rank among the rows that agree with it
#pragma unroll
  for (int x = 0; x < kSelectWaves; ++x) {
    const int2 of = *(const int2 *)sm_part[x];
    newest = of.x > newest ? of.x : newest;
    rank -= of.y;
  }
  if (rank == 0) {  // no place below row keep is there
    if (tid == 0) a.moves[w] = 0;
    return;
  }
  // positions above newest - recent stay, as a bound that an int holds
  const int above = (long long)newest - a.recent < kNowhere ? kNowhere : newest - a.recent;
  const unsigned of_newest = kNewestKey - (unsigned)newest;
  const int from = a.first > 0 ? a.first : kNowhere;
  auto sure = [&](int r, const int (&pos)[kAtOnce]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i)
      if ((pos[i] > above || pos[i] < from) && pos[i] != kNowhere)
        keys[r + 64 * i + lane] = pos[i] > above ? (unsigned)pos[i] + of_newest : kFirstKey;
  };
  if constexpr (kHeld) {
#pragma unroll
    for (int y = 0; y < kBatches; ++y) {
      if (64 * kAtOnce * y >= run) break;
      sure(r0 + 64 * kAtOnce * y, kept_pos[y]);
    }
  } else {
    for (int r = r0; r < r1; r += 64 * kAtOnce) {
      int pos[kAtOnce];
      if (run > 64 * 64) ask(r);
      find(r);
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
        pos[i] = place[i] >= 0 && r + 64 * i + lane < r1 ? (a.c.pos + place[i])[beside] : kNowhere;
      sure(r, pos);
    }
  }
  // (a wave reads only the keys that it wrote itself: no barrier)
  // body(row of lane 0, key) for 64 rows at a time, in order.  The rows from n on have key 0 too.
  auto over_rows = [&](auto body) __attribute__((always_inline)) {
    int r = r0;
    for (; r + 64 * 4 <= r0 + run; r += 64 * 4) {
      unsigned key[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) key[i] = keys[r + 64 * i + lane];
#pragma unroll
      for (int i = 0; i < 4; ++i) body(r + 64 * i, key[i]);
    }
    for (; r < r0 + run; r += 64) body(r, keys[r + lane]);
  };
  // The key of the last row that stays, a byte at a time from the top: among the rows that agree with it so far, count by the next
  // byte and walk down to the one in which the rank falls.
  unsigned edge = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
#pragma unroll
    for (int i = 0; i < 256 * kCopies / kSelectThreads; ++i) sm_hist[i * kSelectThreads + tid] = 0;
    __syncthreads();
    const unsigned agree = shift == 24 ? 0u : ~0u << (shift + 8);
    over_rows([&](int, unsigned key) __attribute__((always_inline)) {
      if (((key ^ edge) & agree) == 0) atomicAdd(&sm_hist[((key >> shift) & 255) * kCopies + lane % kCopies], 1);
    });
    __syncthreads();
    if (tid < 256) {
      int sum = 0;
#pragma unroll
      for (int i = 0; i < kCopies; ++i) sum += sm_hist[tid * kCopies + (i + tid) % kCopies];
      sm_hist[tid * kCopies] = sum;
    }
    __syncthreads();
    if (wave == 0) {  // lane i has the counts of bytes 255 - 4 i .. 252 - 4 i
      int own[4], sum = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        own[j] = sm_hist[(255 - 4 * lane - j) * kCopies];
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
        int j = 0, in_byte = own[0];
#pragma unroll
        for (int x = 1; x < 4; ++x)
          if (j == x - 1 && above + in_byte < rank) {
            above += in_byte;
            in_byte = own[x];
            j = x;
          }
        sm_pick[0] = 255 - 4 * lane - j;
        sm_pick[1] = rank - above;
        sm_pick[2] = rank - above == in_byte;
      }
    }
    __syncthreads();
    edge |= (unsigned)sm_pick[0] << shift;
    rank = sm_pick[1];
    if (sm_pick[2] && edge) {  // all rows that agree so far stay: those above the key before the lowest such one
      --edge;
      rank = 0;
      break;
    }
  }
  // `rank` rows with the edge's key stay, the lowest ones.  Every wave counts its rows above the edge and on it, below
  // row keep and from there on; what the waves before it counted says where its places and movers are listed.
  int over_lo = 0, on_lo = 0, over_hi = 0, on_hi = 0;
  over_rows([&](int r, unsigned key) __attribute__((always_inline)) {
    const unsigned long long over = __builtin_amdgcn_ballot_w64(key > edge), on = __builtin_amdgcn_ballot_w64(key == edge);
    const unsigned long long lo = r + 64 <= a.keep ? ~0ull : r >= a.keep ? 0ull : (1ull << (a.keep - r)) - 1;
    over_lo += __popcll(over & lo);
    on_lo += __popcll(on & lo);
    over_hi += __popcll(over & ~lo);
    on_hi += __popcll(on & ~lo);
  });
  if (lane == 0) *(int4 *)sm_part[wave] = int4{over_lo + holes, on_lo, over_hi, on_hi};
  __syncthreads();
  // lane x < kSelectWaves: wave x's counts; seen: rows on the edge before its rows
  const int4 part = *(const int4 *)sm_part[lane % kSelectWaves];
  auto before_wave = [&](int v) __attribute__((always_inline)) {  // sum over the lanes below, of those kSelectWaves
    int incl = v;
#pragma unroll
    for (int sh = 1; sh < kSelectWaves; sh <<= 1) {
      const int up = __shfl_up(incl, sh, kSelectWaves);
      if (lane % kSelectWaves >= sh) incl += up;
    }
    return incl - v;
  };
  auto of_wave = [&](int v, int x) __attribute__((always_inline)) { return __builtin_amdgcn_readlane(v, x); };
  const int on_before = before_wave(part.y + part.w);
  const int first = (lane % kSelectWaves) * run, lo_rows = min(max(a.keep - first, 0), run);
  const int own_places = lo_rows - part.x - min(max(rank - on_before, 0), part.y);
  const int own_movers = part.z + min(max(rank - on_before - part.y, 0), part.w);
  const int places_before = before_wave(own_places), movers_before = before_wave(own_movers);
  int seen = of_wave(on_before, wave), places = of_wave(places_before, wave), movers = of_wave(movers_before, wave);
  if (tid == 0) {
    const int all = of_wave(movers_before + own_movers, kSelectWaves - 1);
    a.moves[w] = all < a.most_moves ? all : a.most_moves;
  }
  auto before = [](unsigned long long m) __attribute__((always_inline)) {  // set bits of lanes below this one
    return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0u));
  };
  int2 *place_list = a.lists + (long long)w * 2 * a.most_moves, *mover_list = place_list + a.most_moves;
  auto found = [&](int r) __attribute__((always_inline)) {  // row r + lane
    int2 at;
    if constexpr (kInPage) {
      at.x = __builtin_amdgcn_readlane(entry, ((r - r0) >> 6) & 63);
      at.y = r - fast_div(r, a.c.page_rows) * (int)a.c.page_rows.d + lane;
    } else {
      at.x = page_of(a.c, table, r + lane < n ? r + lane : n - 1, at.y);
    }
    return at;
  };
  over_rows([&](int r, unsigned key) __attribute__((always_inline)) {
    unsigned long long stays = __builtin_amdgcn_ballot_w64(key > edge);
    const unsigned long long tie = __builtin_amdgcn_ballot_w64(key == edge);
    if (tie) {
      stays |= __builtin_amdgcn_ballot_w64(key == edge && seen + before(tie) < rank);
      seen += __popcll(tie);
    }
    const unsigned long long lo = r + 64 <= a.keep ? ~0ull : r >= a.keep ? 0ull : (1ull << (a.keep - r)) - 1;
    unsigned long long pm = ~stays & lo;
    const unsigned long long mm = stays & ~lo;
    if (holes) pm &= __builtin_amdgcn_ballot_w64(key != 0);
    if (kInPage && run > 64 * 64) ask(r);
    if (pm) {
      const int i = places + before(pm);
      const int2 at = found(r);
      if (((pm >> lane) & 1) && i < a.most_moves) place_list[i] = at;
      places += __popcll(pm);
    }
    if (mm) {
      const int i = movers + before(mm);
      const int2 at = found(r);
      if (((mm >> lane) & 1) && i < a.most_moves) mover_list[i] = at;
      movers += __popcll(mm);
    }
  });
}

// Rows of keys and values (2 D bytes each, D as e4m3), 16 bytes a lane; kMovesAtOnce rows of a lane are under way
// together, since each is a chain of accesses: lists, row.  The lists hold pages, which the select kernel has at hand: with row
// numbers in them, looked up in the table here, 12 prompts of 2.4K to 14K rows took 137 us instead of 133.
constexpr int kMovesAtOnce = 4;
__global__ __launch_bounds__(256) void paged_move_kernel(const PagedEvictArgs a) {
  const int w = blockIdx.x, b = w / a.Hkv, h = w - b * a.Hkv;
  const int count = a.moves[w];
  const int pieces = (a.c.e4m3 ? a.D : 2 * a.D) / 16, per = 256 / (2 * pieces);  // lanes per tensor, rows at a time
  const int piece = threadIdx.x % pieces, is_v = (threadIdx.x / pieces) & 1, mine = threadIdx.x / (2 * pieces);
  const int2 *place_list = a.lists + (long long)w * 2 * a.most_moves, *mover_list = place_list + a.most_moves;
  unsigned char *pool = is_v ? a.c.v : a.c.k;
  unsigned char *scale = is_v ? a.c.v_scale : a.c.k_scale;
  unsigned *per_row = is_v ? (unsigned *)a.c.mass : (unsigned *)a.c.pos;  // of a row, the lanes of its values take the one along, those of its keys the other
  for (int i0 = blockIdx.y * per * kMovesAtOnce + mine; i0 < count; i0 += gridDim.y * per * kMovesAtOnce) {
    int2 to[kMovesAtOnce], of[kMovesAtOnce];
    u32x4 x[kMovesAtOnce];
    unsigned beside[kMovesAtOnce];
    unsigned char byte[kMovesAtOnce];
#pragma unroll
    for (int m = 0; m < kMovesAtOnce; ++m) {
      const int i = i0 + m * per < count ? i0 + m * per : i0;
      to[m] = place_list[i];
      of[m] = mover_list[i];
    }
#pragma unroll
    for (int m = 0; m < kMovesAtOnce; ++m) {
      x[m] = __builtin_nontemporal_load((const u32x4 *)(pool + row_offset(a.c, of[m].x, h, of[m].y) + 16 * piece));
      if (piece == 0) {
        const long long from = row_place(a.c, of[m].x, h, of[m].y);
        beside[m] = per_row[from];
        if (a.c.e4m3) byte[m] = scale[from];
      }
    }
#pragma unroll
    for (int m = 0; m < kMovesAtOnce; ++m) {
      if (i0 + m * per < count) {
        __builtin_nontemporal_store(x[m], (u32x4 *)(pool + row_offset(a.c, to[m].x, h, to[m].y) + 16 * piece));
        if (piece == 0) {
          const long long place = row_place(a.c, to[m].x, h, to[m].y);
          per_row[place] = beside[m];
          if (a.c.e4m3) scale[place] = byte[m];
        }
      }
    }
  }
}

bool evict_keys_held(long long max_rows) { return max_rows <= kHeldRows; }

hipError_t launch_paged_evict(const PagedEvictArgs &a, hipStream_t st) {
  const int windows = a.B * a.Hkv;
  const bool in_page = a.c.page_rows.d % 64 == 0;
  const auto kern = a.keys ? (in_page ? paged_select_kernel<false, true> : paged_select_kernel<false, false>)
                           : (in_page ? paged_select_kernel<true, true> : paged_select_kernel<true, false>);
  int lds = 0;
  if (!a.keys) {
    static std::atomic<bool> allowed[2];
    if (!allowed[in_page].load(std::memory_order_acquire)) {
      const hipError_t e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, kHeldRows * 4);
      if (e != hipSuccess) return e;
      allowed[in_page].store(true, std::memory_order_release);
    }
    if (a.most_moves) lds = (a.max_rows + kSelectThreads - 1) / kSelectThreads * kSelectThreads * 4;  // else no window can hold more than it may: nothing is selected
  }
  const hipError_t e = launch_in_parts(windows, kSelectThreads, [&](long long first, unsigned count) {
    hipLaunchKernelGGL(kern, dim3(count), dim3(kSelectThreads), lds, st, a, (int)first);
  });
  if (e != hipSuccess || a.most_moves == 0) return e;
  int wgs = 16384 / windows;
  const int at_once = kMovesAtOnce * 256 / (a.D * (a.c.e4m3 ? 2 : 4) / 16);  // rows of a workgroup
  const int most = (a.most_moves + at_once - 1) / at_once;
  wgs = wgs < 1 ? 1 : wgs > most ? most : wgs;
  hipLaunchKernelGGL(paged_move_kernel, dim3(windows, wgs), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace segattn
