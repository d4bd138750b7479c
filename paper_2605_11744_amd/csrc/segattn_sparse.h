// Internal declarations of the operators for sparse attention over a paged cache: tables kept on the device, bounds of
// blocks, choice of blocks, attention over them (not part of the ABI).
#pragma once
#include "segattn_paged.h"

namespace segattn {

// ---- tables -----------------------------------------------------------------------------------
constexpr int kTablePages = 4096;  // pages whose users a workgroup looks at
struct PagedTablesArgs {
  PagedCache c;
  HeadSets heads;
  int *table, *users;
  const int *cu;         // [B+1]; nullptr: one token of every sequence
  const int *rows;
  int *granted;
  long long *slots;      // or nullptr
  int *need;             // workspace: [table rows] entries that each lacks (-1: the rows do not fit), then where its pages begin in `free`
  int *free_of;          // workspace: [chunks] free pages among kTablePages
  int *free;             // workspace: [n_pages] free pages, ascending
  long long total;
  int B, Hkv, newest, tail, chunks;
  int longest;           // most new tokens of a sequence
  int small;             // by one workgroup
  FastDiv seg, heads_div;
};
constexpr long long kSmallReserve = 4096;  // entries that one workgroup hands out
hipError_t launch_paged_reserve(const PagedTablesArgs &a, hipStream_t st);
hipError_t launch_paged_release(const PagedTablesArgs &a, hipStream_t st);

// ---- blocks -----------------------------------------------------------------------------------
// Exponent of a block's smallest scale: bounds of smaller keys round to -1, 0 and 1.  (Scores are compared as 2^(e - 32) times whole numbers
// below 2^22, which are normal floats from here up to bf16's largest.)
constexpr int kLeastBoundExponent = -80;
struct PagedBlocksArgs {
  PagedCache c;
  signed char *bounds;  // [page][heads][blocks][2][D]
  unsigned char *scale; // [page][heads][blocks]
  const int *rows_from; // or nullptr
  const int *rows;
  long long units;      // B * n_past * most
  int most;             // blocks of a window, at most
  int B, Hkv, n_past, D;
  FastDiv n_past_div;
  int per_page;         // blocks of a page
  FastDiv block_rows;
  unsigned char past[kMaxKvHeads];  // the PAST heads, ascending
};
hipError_t launch_paged_summarize(const PagedBlocksArgs &a, hipStream_t st);

struct PagedChooseArgs {
  PagedBlocksArgs k;
  const unsigned short *q;
  const int *cu;
  int *chosen;
  unsigned *keys;       // workspace: [token of the part][n_past][stride]
  long long total, stride;
  int part;             // tokens whose keys the workspace holds
  int tile;             // tokens of a tile
  int in_lds;           // a tile's keys fit LDS: no workspace is used
  int Hq, g, max_rows, n_chosen, first, recent;
};
constexpr long long kChoiceInLds = 256;  // blocks
void plan_paged_choose(PagedChooseArgs &a, long long max_seqlen);
hipError_t launch_paged_choose(const PagedChooseArgs &a, hipStream_t st);

// ---- attention over chosen blocks ---------------------------------------------------------------
struct PagedChosenArgs {
  PagedCache c;
  const unsigned short *q;
  const int *cu, *rows, *chosen;
  void *out;
  float *lse;
  float *slots;         // workspace: partials [token][head of the set][part][g], PAST heads before the others
  // Many tokens at a time: tiles of windows, and listed blocks turned round, a part of the tokens after the other.
  int wide_windows, by_block;
  int wide_tokens;      // tokens whose heads are the columns of a window's workgroup
  long long wide_tiles; // of that many tokens, in all sequences (some are empty)
  int wide_wgs;         // workgroups that the windows' tiles are shared out to, a multiple of 8; 0: a workgroup for each of wide_tokens tokens
  int4 *splits;         // of each of them: the unit whose first piece is its (two words, -1: none), the workgroup of the last piece
  float *wide_slots;    // partials of pieces, two of kWideColumns columns for each
  int listed_tokens;    // most tokens of a task
  int listed_pieces;    // of a block, kListedRows rows each
  int blocks;           // of a window
  int part_tokens;      // of a part
  long long part0, entries;       // first token, and entries of the lists
  int *cursors, *counts;          // workspace: entries and tasks so far; entries of a key (sequence, PAST head, block); together
  int *offsets, *rank, *sorted;   // where a key's entries lie in `sorted`; an entry's number in its key, -1: sees nothing
  int4 *tasks;                    // (key, first of its entries in `sorted`, entries)
  float *listed_out;              // [entry][piece][g][D]
  float2 *listed_sum;             // [entry][piece][g]: maximum, sum
  long long total;
  int B, Hq, Hkv, g, D, n_past, n_other, n_chosen, max_rows, tail;
  int passes;           // of 16 columns over a token's query heads
  int parts_past, parts_other;    // workgroups that share a window
  int tiles_past, tiles_other;    // key tiles of a part
  long long wgs_past, wgs_other;
  FastDiv seg, block_halves;      // block_halves: half tiles of 16 rows in a block
  float scale, scale_log2e;
  int out_fp32;
  unsigned char head_of[kMaxKvHeads];  // PAST heads, then the others, ascending
  unsigned char tail_of[kMaxKvHeads];  // the same order: 1 with the TAIL bit
};
constexpr int kChosenTile = 32;
constexpr int kWideColumns = 128;  // of a window's workgroup
constexpr int kUnitTiles = 2;      // what a window's workgroup takes to begin and to end, in tiles
constexpr int kLeastShare = 4;     // tiles
constexpr int kListedRows = 64;
// Shares the windows out (parts, tiles, workgroups) and lays the workspace out from `ws` on; returns its bytes.
unsigned long long plan_paged_chosen(PagedChosenArgs &a, long long max_seqlen, unsigned char *ws);
// Bytes that no plan of these sizes, or of smaller ones, exceeds (of a planned call's arguments).
unsigned long long most_paged_chosen(PagedChosenArgs a, long long max_seqlen);
// Workgroups of the kernel for windows in shares that the device holds at once (0: could not be asked).
long long windows_resident(const PagedChosenArgs &a);
hipError_t launch_paged_windows(const PagedChosenArgs &a, hipStream_t st);
hipError_t launch_paged_listed(const PagedChosenArgs &a, hipStream_t st);
hipError_t launch_paged_chosen(const PagedChosenArgs &a, hipStream_t st);

// The sequence of token t of a packed batch, or -1 (behind the last one); i: its number there, n: the sequence's tokens.
__device__ inline int sequence_of(const int *cu, int B, long long t, int &i, int &n) {
  if (!cu) {
    i = 0;
    n = 1;
    return t < B ? (int)t : -1;
  }
  if (t >= cu[B]) return -1;
  int lo = 0, hi = B;  // cu[lo] <= t < cu[hi]
  while (hi - lo > 1) {
    const int mid = lo + (hi - lo) / 2;
    if (cu[mid] <= t) lo = mid;
    else hi = mid;
  }
  i = (int)t - cu[lo];
  n = cu[lo + 1] - cu[lo];
  return i >= 0 && i < n ? lo : -1;
}
// Rows of window w up to and with that of token i of n: the token's own is the last.
__device__ inline int rows_seen(const int *rows, long long w, int i, int n, int max_rows) {
  const long long end = (long long)rows[w] - n + i + 1;
  return end < 0 ? 0 : end < max_rows ? (int)end : max_rows;
}

}  // namespace segattn
