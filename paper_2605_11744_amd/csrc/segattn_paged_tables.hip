// seg_kv_paged_reserve and seg_kv_paged_release: tables of a paged cache kept on the device.
//
// A page is free where no table names it (users <= 0), so a pool needs no list of free pages that calls would have to keep in order: the
// free ones are counted, ranked by their number and handed out in the order of the entries that lack one.  Whole
// numbers only, and no result depends on the order in which workgroups run.
// There is little to move: bound by launches and by dependent reads (row counts -> entries -> pages).  Prompts of 404K tokens, eight heads, take
// 31 us in four launches, 13 of them for the 26 MB of slots; releasing of 64 tables of eight heads 5.5.
#include "segattn_sparse.h"

namespace segattn {

// Entries [from, to) of a head that m new tokens behind `rows` rows want.
__device__ inline void wanted_entries(const PagedTablesArgs &a, int b, int h, int m, int &from, int &to) {
  const int rows = rows_held(a.rows, (long long)b * a.Hkv + h, a.c.cap);
  const int end = rows + m;  // (fits the table: checked before)
  int first = rows;
  if (a.newest && !in_set(a.heads.past, h)) {
    const int start = fast_div(end - 1, a.seg) * (int)a.seg.d;
    const int seen = in_set(a.heads.tail, h) ? (start > a.tail ? start - a.tail : 0) : start;
    first = seen > first ? seen : first;
  }
  from = fast_div(first, a.c.page_rows);
  to = fast_div(end - 1, a.c.page_rows) + 1;
}
__device__ inline int new_tokens(const PagedTablesArgs &a, int b) {
  if (!a.cu) return 1;
  const int m = a.cu[b + 1] - a.cu[b];
  return m < 0 ? 0 : m < a.longest ? m : a.longest;
}

constexpr int kTableThreads = 256;

// Whether the rows of sequence b fit its table with m new ones, by the threads of a workgroup (all of them get the answer).
__device__ inline bool rows_fit(const PagedTablesArgs &a, int b, int m) {
  bool bad = false;
  for (int h = threadIdx.x; h < a.Hkv; h += blockDim.x) bad |= (long long)rows_held(a.rows, (long long)b * a.Hkv + h, a.c.cap) + m > a.c.cap;
  return !__syncthreads_or(bad);
}

// The missing entries of table row w (a sequence's or, with per_head, a head's), in order: `found(index of the entry among them, its place
// in the table)`, by all threads of the workgroup, and their number.  -1: the rows do not fit the table.
template <typename Found>
__device__ inline int missing_entries(const PagedTablesArgs &a, long long w, Found found) {
  __shared__ int sm_from[kMaxKvHeads], sm_to[kMaxKvHeads], sm_count[kTableThreads / 64];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int b = a.c.per_head ? (int)(w / a.Hkv) : (int)w, h0 = a.c.per_head ? (int)(w - (long long)b * a.Hkv) : 0, heads = a.c.per_head ? 1 : a.Hkv;
  const int m = new_tokens(a, b);
  if (m == 0) return 0;
  if (!rows_fit(a, b, m)) return -1;
  for (int k = tid; k < heads; k += kTableThreads) wanted_entries(a, b, h0 + k, m, sm_from[k], sm_to[k]);
  __syncthreads();
  int from = sm_from[0], to = sm_to[0];
  for (int k = 1; k < heads; ++k) {
    from = sm_from[k] < from ? sm_from[k] : from;
    to = sm_to[k] > to ? sm_to[k] : to;
  }
  const long long base = w * a.c.max_pages;
  int count = 0;
  for (int e0 = from; e0 < to; e0 += kTableThreads) {
    const int e = e0 + tid;
    bool missing = false;
    if (e < to) {
      bool wanted = false;
      for (int k = 0; k < heads; ++k) wanted |= e >= sm_from[k] && e < sm_to[k];
      missing = wanted && (unsigned)a.table[base + e] >= (unsigned)a.c.n_pages;
    }
    const unsigned long long votes = __builtin_amdgcn_ballot_w64(missing);
    if (lane == 0) sm_count[wave] = __popcll(votes);
    __syncthreads();
    int before = count;
    for (int x = 0; x < kTableThreads / 64; ++x) {
      if (x < wave) before += sm_count[x];
      count += sm_count[x];
    }
    if (missing) found(before + __popcll(votes & ((1ull << lane) - 1)), base + e);
    __syncthreads();
  }
  return count;
}

// Workgroups 0 .. chunks - 1: free pages among kTablePages.  The others: entries that a table row lacks.
__global__ __launch_bounds__(kTableThreads) void paged_need_kernel(const PagedTablesArgs a, const long long first_wg) {
  __shared__ int sm_sum[kTableThreads / 64];
  const int tid = threadIdx.x;
  const long long wg = first_wg + blockIdx.x;
  if (wg >= a.chunks) {
    const int n = missing_entries(a, wg - a.chunks, [](int, long long) {});
    if (tid == 0) a.need[wg - a.chunks] = n;
    return;
  }
  int n = 0;
#pragma unroll
  for (int i = 0; i < kTablePages / kTableThreads; ++i) {
    const long long page = wg * kTablePages + i * kTableThreads + tid;
    n += __popcll(__builtin_amdgcn_ballot_w64(page < a.c.n_pages && a.users[page < a.c.n_pages ? page : 0] <= 0));
  }
  if ((tid & 63) == 0) sm_sum[tid >> 6] = n;
  __syncthreads();
  if (tid == 0) {
    for (int x = 1; x < kTableThreads / 64; ++x) n += sm_sum[x];
    a.free_of[wg] = n;
  }
}

// Sums over the threads before this one, and over all of the workgroup's.
template <int kThreads, typename T>
__device__ inline T sum_before(T x, T &all, T *sm) {  // sm [kThreads / 64]
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  T incl = x;
#pragma unroll
  for (int sh = 1; sh < 64; sh <<= 1) {
    const T up = __shfl_up(incl, sh);
    if (lane >= sh) incl += up;
  }
  __syncthreads();
  if (lane == 63) sm[wave] = incl;
  __syncthreads();
  all = 0;
  T before = incl - x;
  for (int y = 0; y < kThreads / 64; ++y) {
    if (y < wave) before += sm[y];
    all += sm[y];
  }
  return before;
}

// Workgroups 0 .. chunks - 1: the free pages among kTablePages, to their ranks.  The last one: which sequences are granted what they lack,
// and where their rows' pages begin.
__global__ __launch_bounds__(kTableThreads) void paged_grant_kernel(const PagedTablesArgs a) {
  __shared__ int sm_int[kTableThreads / 64];
  __shared__ long long sm_long[kTableThreads / 64];
  constexpr int kEach = kTablePages / kTableThreads;
  const int tid = threadIdx.x, wg = blockIdx.x;
  const int upto = wg < a.chunks ? wg : a.chunks;
  int sum = 0, base;
  for (int x = tid; x < upto; x += kTableThreads) sum += a.free_of[x];
  sum_before<kTableThreads>(sum, base, sm_int);  // base: free pages before this chunk; for the last workgroup all of them
  if (wg < a.chunks) {
    const long long first = (long long)wg * kTablePages + tid * kEach;
    unsigned is_free = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) is_free |= (first + i < a.c.n_pages && a.users[first + i < a.c.n_pages ? first + i : 0] <= 0 ? 1u : 0u) << i;
    int all, at = base + sum_before<kTableThreads>((int)__popc(is_free), all, sm_int);
    for (; is_free; is_free &= is_free - 1) a.free[at++] = (int)(first + __builtin_ctz(is_free));
    return;
  }
  const long long there = base;
  const int rows = a.c.per_head ? a.Hkv : 1;  // table rows of a sequence
  long long before = 0;                       // pages that the sequences so far lack
  for (int b0 = 0; b0 < a.B; b0 += kTableThreads) {
    const int b = b0 + tid;
    long long need = 0;
    bool fits = true;
    if (b < a.B)
      for (int r = 0; r < rows; ++r) {
        const int n = a.need[(long long)b * rows + r];
        fits &= n >= 0;
        need += n > 0 ? n : 0;
      }
    if (!fits) need = 0;
    long long all, at = before + sum_before<kTableThreads>(need, all, sm_long);
    if (b < a.B) {
      const bool ok = fits && (need == 0 || at + need <= there);
      a.granted[b] = ok;
      for (int r = 0; r < rows; ++r) {  // where the row's pages begin, below n_pages; -1: it gets none
        const int n = a.need[(long long)b * rows + r];
        a.need[(long long)b * rows + r] = ok && n > 0 ? (int)at : -1;
        at += n > 0 ? n : 0;
      }
    }
    before += all;
  }
}

__global__ __launch_bounds__(kTableThreads) void paged_assign_kernel(const PagedTablesArgs a, const long long first_wg) {
  const long long w = first_wg + blockIdx.x;
  const int base = a.need[w];
  if (base < 0) return;
  missing_entries(a, w, [&](int i, long long place) {
    const int page = a.free[base + i];
    a.table[place] = page;
    a.users[page] = 1;
  });
}

// Where the row of a token will be.  (Without branches, so that the loads of several go together.)
__device__ inline long long slot_of(const PagedTablesArgs &a, int h, int b, int i, bool granted) {
  const long long row = (long long)rows_held(a.rows, (long long)b * a.Hkv + h, a.c.cap) + i;
  const bool fits = granted && row < a.c.cap;
  const int e = fast_div(fits ? (int)row : 0, a.c.page_rows), page = table_of(a.c, a.Hkv, b, h)[e];
  const long long slot = row_place(a.c, page, h, (int)row - e * (int)a.c.page_rows.d);
  return fits && (unsigned)page < (unsigned)a.c.n_pages ? slot : -1;
}

// 256 tokens: each thread finds one's sequence, then they walk over the (token, head) pairs.
__global__ __launch_bounds__(kTableThreads) void paged_slots_kernel(const PagedTablesArgs a, const long long first_wg) {
  __shared__ int sm_b[kTableThreads], sm_i[kTableThreads];
  const int tid = threadIdx.x;
  const long long t0 = (first_wg + blockIdx.x) * kTableThreads;
  int i = 0, n, b = -1;
  if (t0 + tid < a.total) b = sequence_of(a.cu, a.B, t0 + tid, i, n);
  sm_b[tid] = b < 0 ? -1 : a.granted[b] ? 2 * b + 1 : 2 * b;
  sm_i[tid] = i;
  __syncthreads();
#pragma unroll 8
  for (int x = tid; x < kTableThreads * a.Hkv; x += kTableThreads) {
    const int t = fast_div(x, a.heads_div), h = x - t * a.Hkv, s = sm_b[t];
    const long long slot = slot_of(a, h, s < 0 ? 0 : s >> 1, sm_i[t], s & 1);
    if (s >= 0) a.slots[t0 * a.Hkv + x] = slot;
  }
}

// The same in one workgroup, for the few pages of a step: a thread per sequence counts what it lacks, and the pool is searched only until there
// are as many free pages.  (Four launches take 19 us for a step of 48 sequences, this one 11.)
constexpr int kSmallThreads = 1024;
__global__ __launch_bounds__(kSmallThreads) void paged_reserve_small_kernel(const PagedTablesArgs a) {
  __shared__ int sm_free[kSmallReserve], sm_int[kSmallThreads / 64];
  __shared__ long long sm_long[kSmallThreads / 64];
  const int tid = threadIdx.x, rows = a.c.per_head ? a.Hkv : 1;
  // entries of sequence b that are missing, in order: visit(place in the table)
  const auto missing = [&](int b, int m, auto visit) {
    for (int r = 0; r < rows; ++r) {
      const long long base = ((long long)b * rows + r) * a.c.max_pages;
      int last = -1;
      for (;;) {
        int next = 0x7fffffff;  // the first wanted entry behind the last one
        for (int k = 0; k < (a.c.per_head ? 1 : a.Hkv); ++k) {
          int from, to;
          wanted_entries(a, b, a.c.per_head ? r : k, m, from, to);
          from = from > last ? from : last + 1;
          if (from < to && from < next) next = from;
        }
        if (next == 0x7fffffff) break;
        if ((unsigned)a.table[base + next] >= (unsigned)a.c.n_pages) visit(base + next);
        last = next;
      }
    }
  };
  // (at most kSmallThreads sequences)
  const int b = tid, m = b < a.B ? new_tokens(a, b) : 0;
  bool fits = true;
  if (m > 0)
    for (int h = 0; h < a.Hkv; ++h) fits &= (long long)rows_held(a.rows, (long long)b * a.Hkv + h, a.c.cap) + m <= a.c.cap;
  int need = 0;
  if (m > 0 && fits) missing(b, m, [&](long long) { ++need; });
  int wanted;  // below kSmallReserve: the host has checked
  const int at = sum_before<kSmallThreads>(need, wanted, sm_int);
  int there = 0;
  constexpr int kEach = 8;
  for (long long p0 = 0; p0 < a.c.n_pages && there < wanted; p0 += kSmallThreads * kEach) {
    const long long first = p0 + tid * kEach;
    unsigned is_free = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) is_free |= (first + i < a.c.n_pages && a.users[first + i < a.c.n_pages ? first + i : 0] <= 0 ? 1u : 0u) << i;
    int all, place = there + sum_before<kSmallThreads>((int)__popc(is_free), all, sm_int);
    for (; is_free && place < wanted; is_free &= is_free - 1) sm_free[place++] = (int)(first + __builtin_ctz(is_free));
    there += all;
  }
  __syncthreads();
  const bool ok = fits && (need == 0 || at + need <= there);
  if (b < a.B) {
    a.granted[b] = ok;
    int place = at;
    if (ok && need > 0)
      missing(b, m, [&](long long entry) {
        const int page = sm_free[place++];
        a.table[entry] = page;
        a.users[page] = 1;
      });
  }
  if (!a.slots) return;
  __threadfence_block();
  __syncthreads();
  for (long long x = tid; x < a.total * a.Hkv; x += kSmallThreads) {  // total * Hkv < 2^31
    const int t = fast_div((int)x, a.heads_div), h = (int)x - t * a.Hkv;
    int i, n;
    const int s = sequence_of(a.cu, a.B, t, i, n);
    if (s >= 0) a.slots[x] = slot_of(a, h, s, i, a.granted[s] != 0);
  }
}

hipError_t launch_paged_reserve(const PagedTablesArgs &a, hipStream_t st) {
  if (a.small) {
    hipLaunchKernelGGL(paged_reserve_small_kernel, dim3(1), dim3(kSmallThreads), 0, st, a);
    return hipGetLastError();
  }
  const long long table_rows = a.c.per_head ? (long long)a.B * a.Hkv : a.B;
  hipError_t e = launch_in_parts(a.chunks + table_rows, kTableThreads, [&](long long first, unsigned count) {
    hipLaunchKernelGGL(paged_need_kernel, dim3(count), dim3(kTableThreads), 0, st, a, first);
  });
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(paged_grant_kernel, dim3(a.chunks + 1), dim3(kTableThreads), 0, st, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  e = launch_in_parts(table_rows, kTableThreads, [&](long long first, unsigned count) {
    hipLaunchKernelGGL(paged_assign_kernel, dim3(count), dim3(kTableThreads), 0, st, a, first);
  });
  if (e != hipSuccess || !a.slots) return e;
  return launch_in_parts((a.total + kTableThreads - 1) / kTableThreads, kTableThreads, [&](long long first, unsigned count) {
    hipLaunchKernelGGL(paged_slots_kernel, dim3(count), dim3(kTableThreads), 0, st, a, first);
  });
}

// A workgroup takes kTableThreads entries of a table.
__global__ __launch_bounds__(kTableThreads) void paged_release_kernel(const PagedTablesArgs a, const long long first_wg, const int chunks) {
  __shared__ int sm_from[kMaxKvHeads], sm_to[kMaxKvHeads];
  const long long wg = first_wg + blockIdx.x, w = wg / chunks;
  const int tid = threadIdx.x, e = (int)(wg - w * chunks) * kTableThreads + tid;
  const int heads = a.c.per_head ? 1 : a.Hkv;
  for (int k = tid; k < heads; k += kTableThreads) {
    const long long window = w * heads + k;
    const int h = (int)(window % a.Hkv), n = rows_held(a.rows, window, a.c.cap);
    int first = 0;
    if (!in_set(a.heads.past, h)) {
      const int start = fast_div(n > 0 ? n - 1 : 0, a.seg) * (int)a.seg.d;
      first = in_set(a.heads.tail, h) ? (start > a.tail ? start - a.tail : 0) : start;
    }
    sm_from[k] = fast_div(first, a.c.page_rows);
    sm_to[k] = n == 0 ? 0 : fast_div(n - 1, a.c.page_rows) + 1;
  }
  __syncthreads();
  if (e >= a.c.max_pages) return;
  int *entry = a.table + w * a.c.max_pages + e;
  const int page = *entry;
  if ((unsigned)page >= (unsigned)a.c.n_pages) return;
  bool keep = false;
  for (int k = 0; k < heads; ++k) keep |= e >= sm_from[k] && e < sm_to[k];
  if (keep) return;
  *entry = -1;
  atomicSub(a.users + page, 1);
}

hipError_t launch_paged_release(const PagedTablesArgs &a, hipStream_t st) {
  const int chunks = (a.c.max_pages + kTableThreads - 1) / kTableThreads;
  const long long windows = a.c.per_head ? (long long)a.B * a.Hkv : a.B;
  return launch_in_parts(windows * chunks, kTableThreads, [&](long long first, unsigned count) {
    hipLaunchKernelGGL(paged_release_kernel, dim3(count), dim3(kTableThreads), 0, st, a, first, chunks);
  });
}

}  // namespace segattn
