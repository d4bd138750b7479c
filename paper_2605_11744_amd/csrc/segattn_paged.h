// Internal declarations of the operators around a paged cache: rotation by position, append, decode
// attention, eviction by weight (not part of the ABI).
#pragma once
#include "segattn_internal.h"

namespace segattn {

// A pool of pages and the table that names the pages of every sequence, as kernels see it.  A row is found by
// its number r inside the (sequence, KV head): entry r / page_rows of the table, row r % page_rows of that page.
// An entry outside 0 .. n_pages - 1 names no page: nothing is read or written there.
struct PagedCache {
  unsigned char *k, *v, *k_scale, *v_scale;
  float *mass;
  int *pos;
  const int *table;
  long long page_bytes, head_bytes, row_bytes;  // strides of k and v
  FastDiv page_rows;
  int n_pages, max_pages;
  int per_head;  // 1: a page holds rows of one KV head, and every head has a table of its own
  int heads;     // KV heads in a page: Hkv or 1
  int cap;       // rows a table can name: max_pages * page_rows, below 2^31
  int e4m3;
};

// Which KV heads have the PAST / the TAIL bit.
struct HeadSets {
  unsigned past[kMaxKvHeads / 32], tail[kMaxKvHeads / 32];
};
__host__ __device__ inline bool in_set(const unsigned (&set)[kMaxKvHeads / 32], int h) { return (set[h >> 5] >> (h & 31)) & 1; }
__device__ inline int set_before(const unsigned (&set)[kMaxKvHeads / 32], int h) {  // members below h
  int n = 0;
#pragma unroll
  for (int i = 0; i < kMaxKvHeads / 32; ++i) {
    const int left = h - 32 * i;
    if (left > 0) n += __popc(set[i] & (left >= 32 ? ~0u : (1u << left) - 1u));
  }
  return n;
}

__device__ inline const int *table_of(const PagedCache &c, int Hkv, int b, int h) {
  return c.table + (c.per_head ? (long long)b * Hkv + h : (long long)b) * c.max_pages;
}
// Page of row `row` (0 <= row), or -1; `in_page`: the row's number inside it.
__device__ inline int page_of(const PagedCache &c, const int *table, int row, int &in_page) {
  const int i = fast_div(row, c.page_rows);
  in_page = row - i * (int)c.page_rows.d;
  if (i >= c.max_pages) return -1;
  const int page = table[i];
  return (unsigned)page < (unsigned)c.n_pages ? page : -1;
}
// Byte offset of a row in k and v, and its place in the arrays that hold one value per row.
__device__ inline long long row_offset(const PagedCache &c, int page, int h, int in_page) {
  return page * c.page_bytes + (c.per_head ? 0 : h) * c.head_bytes + in_page * c.row_bytes;
}
__device__ inline long long row_place(const PagedCache &c, int page, int h, int in_page) {
  return ((long long)page * c.heads + (c.per_head ? 0 : h)) * c.page_rows.d + in_page;
}
__device__ inline int rows_held(const int *rows, long long w, int most) {
  const int n = rows[w];
  return n < 0 ? 0 : n < most ? n : most;
}

// A launch has fewer than 2^32 threads in a dimension (more are taken modulo 2^32, without an error): a longer row of
// workgroups goes in several.  launch(first, count) starts workgroups first .. first + count - 1.
template <typename Launch>
hipError_t launch_in_parts(long long workgroups, int threads, Launch launch) {
  const long long most = ((1ll << 32) - 1) / threads;
  for (long long first = 0; first < workgroups; first += most) {
    const long long count = workgroups - first < most ? workgroups - first : most;
    launch(first, (unsigned)count);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ---- rotation ---------------------------------------------------------------------------------
struct RotaryArgs {
  int pairs;            // rotary_dim / 2; 0: nothing is turned
  int interleaved;
  int back;             // 1: by the negative angle
  float magnitude;
  double turns[64];     // turns per position of every pair: frequency / (2 pi)
};
struct RotateArgs {
  const void *q, *k;
  void *q_out, *k_out;
  long long q_stride, k_stride, q_out_stride, k_out_stride;  // elements between token rows
  const long long *pos0;  // [B] or nullptr
  const long long *pos;   // [tokens] or nullptr
  long long total;        // tokens
  int rows;               // tokens per sequence
  int Hq, Hkv, D;
  RotaryArgs rot;
};

// ---- append -----------------------------------------------------------------------------------
struct PagedAppendArgs {
  PagedCache c;
  RotaryArgs rot;
  const unsigned short *q, *k, *v;
  unsigned short *q_out;  // nullptr: no queries
  const int *cu;          // [B+1]; nullptr: token t is the one of sequence t
  const long long *pos0;  // [B] or nullptr
  const int *rows;
  int *rows_out;
  int total, B, Hq, Hkv, D;
  int count_rows;         // the token kernel also writes rows_out: 1 each workgroup its sequence's, 2 workgroups behind the others
};

// ---- decode -----------------------------------------------------------------------------------
constexpr int kPagedTile = 32;        // key rows per tile
constexpr int kPagedMostWgs = 1024;   // the workspace has slots for as many workgroups
constexpr int kPagedMostGroup = 128;  // query heads of a KV head
constexpr int kPagedLaneWindows = 64; // up to so many windows a wave finds its slice by itself, one window a lane
struct PagedDecodeArgs {
  PagedCache c;
  HeadSets heads;
  const unsigned short *q;
  const int *rows;      // [B, Hkv]
  void *out;
  float *lse;
  int2 *pieces;         // workspace: first and last slot of every window
  float *slots;         // workspace: partials [slot][g][ws_slot_floats(D)]
  float *scores;        // workspace: [B, n_past][score_rows / tile][g][tile], or nullptr
  long long score_rows;
  int B, Hq, Hkv, g, D, n_windows, n_past;
  int max_rows, tail;
  FastDiv seg, n_kv;
  int fits;             // every window's shortest slices fit the grid
  float scale, scale_log2e;
  int out_fp32;
};

// ---- eviction ---------------------------------------------------------------------------------
struct PagedEvictArgs {
  PagedCache c;
  HeadSets heads;
  const int *rows;
  int *rows_out;
  int *moves;           // workspace: rows to move of every window
  unsigned *keys;       // workspace: [window][key_rows], or nullptr where they fit the kernel's LDS
  long long key_rows;
  int2 *lists;          // workspace: [window][2][most_moves]: freed places, then the rows that go there, as (page, row in it)
  int B, Hkv, D;
  int budget;           // rows that a PAST head may hold afterwards
  int max_rows, keep, recent, first, most_moves;  // keep: the budget, max_rows at most
};

hipError_t launch_rotate(const RotateArgs &a, bool fp32, hipStream_t st);
hipError_t launch_paged_append(const PagedAppendArgs &a, hipStream_t st);
hipError_t launch_paged_decode(const PagedDecodeArgs &a, hipStream_t st);
bool evict_keys_held(long long max_rows);  // the keys of so many rows need no workspace
hipError_t launch_paged_evict(const PagedEvictArgs &a, hipStream_t st);

}  // namespace segattn
