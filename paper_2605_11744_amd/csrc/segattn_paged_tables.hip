// seg_kv_paged_reserve and seg_kv_paged_release: tables of a paged cache kept on the device.
//
// A page is free where no table names it (users <= 0), so a pool needs no list of free pages that calls would have to keep in order: the
// free ones are counted, ranked by their number and handed out in the order of the entries that lack one.  Whole
// numbers only, and no result depends on the order in which workgroups run.
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
  return m > 0 ? m : 0;
}

constexpr int kTableThreads = 256;

// The missing entries of sequence b, in order: `found(index of the entry among them, its place in the table)`, by all threads of the
// workgroup, and their number.  -1: the rows do not fit the table.
template <typename Found>
__device__ inline int missing_entries(const PagedTablesArgs &a, int b, Found found) {
  __shared__ int sm_from[kMaxKvHeads], sm_to[kMaxKvHeads], sm_bad, sm_count[kTableThreads / 64];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int m = new_tokens(a, b);
  __syncthreads();
  if (tid == 0) sm_bad = 0;
  __syncthreads();
  if (m == 0) return 0;
  for (int h = tid; h < a.Hkv; h += kTableThreads) {
    const long long end = (long long)rows_held(a.rows, (long long)b * a.Hkv + h, a.c.cap) + m;
    if (end > a.c.cap) sm_bad = 1;
    else wanted_entries(a, b, h, m, sm_from[h], sm_to[h]);
  }
  __syncthreads();
  if (sm_bad) return -1;
  int from = sm_from[0], to = sm_to[0];
  for (int h = 1; h < a.Hkv; ++h) {
    from = sm_from[h] < from ? sm_from[h] : from;
    to = sm_to[h] > to ? sm_to[h] : to;
  }
  const int span = to - from;
  const long long all = a.c.per_head ? (long long)a.Hkv * span : span;
  const long long base = (long long)b * a.c.max_pages * (a.c.per_head ? a.Hkv : 1);
  int count = 0;
  for (long long j0 = 0; j0 < all; j0 += kTableThreads) {
    const long long j = j0 + tid;
    bool missing = false;
    long long place = 0;
    if (j < all) {
      const int h = a.c.per_head ? (int)(j / span) : 0, e = from + (int)(j - (long long)h * span);
      place = base + (long long)h * a.c.max_pages + e;
      bool wanted = false;
      if (a.c.per_head) wanted = e >= sm_from[h] && e < sm_to[h];
      else
        for (int k = 0; k < a.Hkv; ++k) wanted |= e >= sm_from[k] && e < sm_to[k];
      missing = wanted && (unsigned)a.table[place] >= (unsigned)a.c.n_pages;
    }
    const unsigned long long votes = __builtin_amdgcn_ballot_w64(missing);
    if (lane == 0) sm_count[wave] = __popcll(votes);
    __syncthreads();
    int before = count;
    for (int x = 0; x < kTableThreads / 64; ++x) {
      if (x < wave) before += sm_count[x];
      count += sm_count[x];
    }
    if (missing) found(before + __popcll(votes & ((1ull << lane) - 1)), place);
    __syncthreads();
  }
  return count;
}

// Workgroups 0 .. chunks - 1: free pages among kTablePages.  The others: entries that a sequence lacks.
__global__ __launch_bounds__(kTableThreads) void paged_need_kernel(const PagedTablesArgs a, const long long first_wg) {
  __shared__ int sm_sum[kTableThreads / 64];
  const int tid = threadIdx.x;
  const long long wg = first_wg + blockIdx.x;
  if (wg >= a.chunks) {
    const int b = (int)(wg - a.chunks);
    const int n = missing_entries(a, b, [](int, long long) {});
    if (tid == 0) a.need[b] = n;
    return;
  }
  int n = 0;
  for (int i = 0; i < kTablePages / kTableThreads; ++i) {
    const long long page = wg * kTablePages + i * kTableThreads + tid;
    n += __popcll(__builtin_amdgcn_ballot_w64(page < a.c.n_pages && a.users[page] <= 0));
  }
  if ((tid & 63) == 0) sm_sum[tid >> 6] = n;
  __syncthreads();
  if (tid == 0) {
    for (int x = 1; x < kTableThreads / 64; ++x) n += sm_sum[x];
    a.free_of[wg] = n;
  }
}

__device__ inline int sum_over_workgroup(int x, int *sm) {  // sm [kTableThreads / 64]
#pragma unroll
  for (int sh = 1; sh < 64; sh <<= 1) x += __shfl_xor(x, sh);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = x;
  __syncthreads();
  x = 0;
  for (int i = 0; i < kTableThreads / 64; ++i) x += sm[i];
  return x;
}

// Workgroups 0 .. chunks - 1: the free pages among kTablePages, to their ranks.  The last one: which sequences are granted what they lack,
// and where their pages begin.
__global__ __launch_bounds__(kTableThreads) void paged_grant_kernel(const PagedTablesArgs a) {
  __shared__ int sm_sum[kTableThreads / 64], sm_count[kTableThreads / 64];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, wg = blockIdx.x;
  const int upto = wg < a.chunks ? wg : a.chunks;
  int sum = 0;
  for (int x = tid; x < upto; x += kTableThreads) sum += a.free_of[x];
  int base = sum_over_workgroup(sum, sm_sum);  // free pages before this chunk; for the last workgroup all of them
  if (wg < a.chunks) {
    for (int i = 0; i < kTablePages / kTableThreads; ++i) {
      const long long page = (long long)wg * kTablePages + i * kTableThreads + tid;
      const bool is_free = page < a.c.n_pages && a.users[page] <= 0;
      const unsigned long long votes = __builtin_amdgcn_ballot_w64(is_free);
      if (lane == 0) sm_count[wave] = __popcll(votes);
      __syncthreads();
      int at = base + __popcll(votes & ((1ull << lane) - 1));
      for (int x = 0; x < kTableThreads / 64; ++x) {
        if (x < wave) at += sm_count[x];
        base += sm_count[x];
      }
      if (is_free) a.free[at] = (int)page;
      __syncthreads();
    }
    return;
  }
  const long long there = base;
  long long before = 0;  // pages that the sequences so far lack
  for (int b0 = 0; b0 < a.B; b0 += kTableThreads) {
    const int b = b0 + tid, need = b < a.B ? a.need[b] : 0;
    // sums of entries of up to 256 sequences can pass 32 bits
    long long incl = need > 0 ? need : 0;
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) {
      const long long up = __shfl_up(incl, sh);
      if (lane >= sh) incl += up;
    }
    __shared__ long long sm_wave[kTableThreads / 64];
    __syncthreads();
    if (lane == 63) sm_wave[wave] = incl;
    __syncthreads();
    long long sum_all = 0;
    for (int x = 0; x < kTableThreads / 64; ++x) {
      if (x < wave) incl += sm_wave[x];
      sum_all += sm_wave[x];
    }
    if (b < a.B) {
      const bool ok = need == 0 || (need > 0 && before + incl <= there);
      a.granted[b] = ok;
      a.need[b] = ok && need > 0 ? (int)(before + incl - need) : -1;  // (below n_pages)
    }
    before += sum_all;
  }
}

__global__ __launch_bounds__(kTableThreads) void paged_assign_kernel(const PagedTablesArgs a) {
  const int b = blockIdx.x, base = a.need[b];
  if (base < 0) return;
  missing_entries(a, b, [&](int i, long long place) {
    const int page = a.free[base + i];
    a.table[place] = page;
    a.users[page] = 1;
  });
}

__global__ __launch_bounds__(kTableThreads) void paged_slots_kernel(const PagedTablesArgs a, const long long first_wg) {
  const long long x = (first_wg + blockIdx.x) * kTableThreads + threadIdx.x, t = x / a.Hkv;
  const int h = (int)(x - t * a.Hkv);
  if (t >= a.total) return;
  int i, n;
  const int b = sequence_of(a.cu, a.B, t, i, n);
  if (b < 0) return;
  long long slot = -1;
  const long long row = (long long)rows_held(a.rows, (long long)b * a.Hkv + h, a.c.cap) + i;
  if (a.granted[b] && row < a.c.cap) {
    int in_page;
    const int page = page_of(a.c, table_of(a.c, a.Hkv, b, h), (int)row, in_page);
    if (page >= 0) slot = row_place(a.c, page, h, in_page);
  }
  a.slots[x] = slot;
}

hipError_t launch_paged_reserve(const PagedTablesArgs &a, hipStream_t st) {
  hipError_t e = launch_in_parts((long long)a.chunks + a.B, kTableThreads, [&](long long first, unsigned count) {
    hipLaunchKernelGGL(paged_need_kernel, dim3(count), dim3(kTableThreads), 0, st, a, first);
  });
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(paged_grant_kernel, dim3(a.chunks + 1), dim3(kTableThreads), 0, st, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL(paged_assign_kernel, dim3(a.B), dim3(kTableThreads), 0, st, a);
  if ((e = hipGetLastError()) != hipSuccess || !a.slots) return e;
  return launch_in_parts((a.total * a.Hkv + kTableThreads - 1) / kTableThreads, kTableThreads, [&](long long first, unsigned count) {
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
