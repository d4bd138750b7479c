// C ABI of the operators around a paged cache: argument validation and launches.
#include <math.h>
#include <string.h>

#include "segattn_sparse.h"

using namespace segattn;

namespace {

constexpr unsigned long long kAlign = 256;
constexpr long long kMostRows = (1ll << 31) - 4096;

unsigned long long align_up(unsigned long long x) { return (x + kAlign - 1) / kAlign * kAlign; }
bool misaligned(const void *p, size_t to) { return (uintptr_t)p % to != 0; }
segattn_status hip_status(hipError_t e) { return e == hipSuccess ? SEGATTN_OK : SEGATTN_EHIP; }

// Work for a stream of another device than the current one would run there on the current one's pointers.
bool foreign(void *stream) {
  if (!stream) return false;
  hipDevice_t of = 0;
  int now = 0;
  if (hipStreamGetDevice((hipStream_t)stream, &of) != hipSuccess || hipGetDevice(&now) != hipSuccess) {
    (void)hipGetLastError();
    return true;
  }
  return of != now;
}

bool build_rotary(const segattn_rope *r, int D, RotaryArgs &out) {
  memset(&out, 0, sizeof(out));
  const int n = r->rotary_dim ? r->rotary_dim : D;
  if (n < 16 || n > D || n % 16) return false;
  if (r->interleaved < 0 || r->interleaved > 1) return false;
  if (!r->inv_freq && (!(r->theta > 0.0) || isinf(r->theta))) return false;
  if (!(r->magnitude >= 0.0) || isinf(r->magnitude)) return false;
  const int kind = r->inv_freq ? SEGATTN_ROPE_PLAIN : r->scaling;
  if (kind < SEGATTN_ROPE_PLAIN || kind > SEGATTN_ROPE_BY_INDEX) return false;
  if (kind != SEGATTN_ROPE_PLAIN && (!(r->factor > 0.0) || isinf(r->factor))) return false;
  const double two_pi = 6.283185307179586476925286766559;
  double from = 0.0, to = 0.0;  // BY_INDEX: the pairs between which the scaling sets in
  if (kind == SEGATTN_ROPE_BY_ROTATIONS || kind == SEGATTN_ROPE_BY_INDEX) {
    if (!(r->trained_len > 0.0) || isinf(r->trained_len) || !(r->low > 0.0) || !(r->high > r->low) || isinf(r->high)) return false;
    if (kind == SEGATTN_ROPE_BY_INDEX) {
      if (r->theta == 1.0) return false;
      from = fmax(0.0, floor(n * log(r->trained_len / (two_pi * r->high)) / (2.0 * log(r->theta))));
      to = fmin(n - 1.0, ceil(n * log(r->trained_len / (two_pi * r->low)) / (2.0 * log(r->theta))));
    }
  }
  const double step = r->inv_freq ? 0.0 : -2.0 * log(r->theta) / n;
  out.pairs = n / 2;
  out.interleaved = r->interleaved;
  out.magnitude = r->magnitude > 0.0 ? (float)r->magnitude : 1.f;
  for (int i = 0; i < n / 2; ++i) {
    double f = r->inv_freq ? r->inv_freq[i] : exp(i * step);  // (half the time of a pow per pair: 0.6 us of every call)
    double kept = 1.0;  // share of the unscaled frequency
    if (kind == SEGATTN_ROPE_LINEAR) kept = 0.0;
    if (kind == SEGATTN_ROPE_BY_ROTATIONS) kept = fmin(1.0, fmax(0.0, (r->trained_len * f / two_pi - r->low) / (r->high - r->low)));
    if (kind == SEGATTN_ROPE_BY_INDEX) kept = 1.0 - fmin(1.0, fmax(0.0, (i - from) / fmax(to - from, 1e-3)));
    if (kind != SEGATTN_ROPE_PLAIN) f *= kept + (1.0 - kept) / r->factor;
    if (!isfinite(f)) return false;
    out.turns[i] = f / two_pi;
  }
  return true;
}

bool build_pages(const segattn_pages *g, const Problem &p, PagedCache &c) {
  if (!g || !g->k || !g->v || !g->table) return false;
  if (g->page_rows < 1 || g->n_pages < 1 || g->max_pages < 1 || g->per_head < 0 || g->per_head > 1) return false;
  if (g->type != SEGATTN_PAGES_BF16 && g->type != SEGATTN_PAGES_E4M3) return false;
  const long long size = g->type == SEGATTN_PAGES_E4M3 ? 1 : 2, heads = g->per_head ? 1 : p.Hkv;
  if ((long long)g->max_pages * g->page_rows >= kMostRows) return false;
  long long row = g->row_stride, head = g->head_stride, page = g->page_stride;
  if (row == 0 && head == 0 && page == 0) {  // dense [n_pages][heads][page_rows][D]
    row = p.D;
    head = row * g->page_rows;
    page = head * heads;
  }
  // 16-byte pieces; offsets inside a tile in 32 bits, and of the whole pool in 63
  if (row < p.D || row * size > (1ll << 26) || row * size % 16) return false;
  if (page < 0 || page >= (1ll << 40) || page * size % 16) return false;
  if (g->per_head) head = 0;
  else if ((heads > 1 && head < 1) || head < 0 || head >= (1ll << 40) || head * size % 16) return false;
  if (page == 0 && g->n_pages > 1) return false;
  if ((double)g->n_pages * page * size > 4e18) return false;
  if (misaligned(g->k, 16) || misaligned(g->v, 16) || misaligned(g->table, 4) || misaligned(g->mass, 4) || misaligned(g->pos, 4)) return false;
  if (g->type == SEGATTN_PAGES_E4M3 && (!g->k_scale || !g->v_scale)) return false;
  memset(&c, 0, sizeof(c));
  c.k = (unsigned char *)g->k;
  c.v = (unsigned char *)g->v;
  c.k_scale = g->k_scale;
  c.v_scale = g->v_scale;
  c.mass = g->mass;
  c.pos = g->pos;
  c.table = g->table;
  c.page_bytes = page * size;
  c.head_bytes = head * size;
  c.row_bytes = row * size;
  c.page_rows = fast_div_by(g->page_rows);
  c.n_pages = g->n_pages;
  c.max_pages = g->max_pages;
  c.per_head = g->per_head;
  c.heads = (int)heads;
  c.cap = g->max_pages * g->page_rows;
  c.e4m3 = g->type == SEGATTN_PAGES_E4M3;
  return true;
}

// The configuration as the paged operators take it: no validation mode, no retrieval mode.
bool build_paged(const segattn_config *cfg, Problem &p) {
  return build_problem(cfg, false, p) && !cfg->fp32_check && cfg->retrieved_capacity == 0 &&
         (long long)p.B * p.Hkv < (1ll << 24);
}

void fill_heads(const Problem &p, HeadSets &s) {
  memset(&s, 0, sizeof(s));
  for (int h = 0; h < p.Hkv; ++h) {
    if (p.policy[h] & SEGATTN_PAST) s.past[h >> 5] |= 1u << (h & 31);
    if (p.policy[h] & SEGATTN_TAIL) s.tail[h >> 5] |= 1u << (h & 31);
  }
}

struct DecodeSpace {
  unsigned long long pieces, slots, scores, total;  // offsets, and all of it
  long long score_rows;
};
bool decode_space(const Problem &p, const PagedCache &c, int64_t max_rows, int accumulate, DecodeSpace &s) {
  if (max_rows < 1 || max_rows > c.cap || accumulate < 0 || accumulate > 1 || p.g > kPagedMostGroup) return false;
  if (accumulate && (!c.mass || p.n_past == 0)) return false;
  if (accumulate && (max_rows + kPagedTile) * p.g >= (1ll << 29)) return false;  // the scores of a window are addressed by 31 bits
  const unsigned long long windows = (unsigned long long)p.B * p.Hkv;
  if ((long long)p.B * p.Hq >= (1ll << 30)) return false;  // (the partials of as many heads would be 290 GB)
  if (windows * ((max_rows + kPagedTile - 1) / kPagedTile + 1) >= (1ull << 31)) return false;
  s.pieces = 0;
  s.slots = align_up(windows * 8ull);
  s.scores = align_up(s.slots + (kPagedMostWgs + windows + 256) * p.g * ws_slot_floats(p.D) * 4ull);
  s.score_rows = accumulate ? (max_rows + kPagedTile - 1) / kPagedTile * kPagedTile : 0;
  s.total = s.scores + align_up((unsigned long long)p.B * p.n_past * p.g * s.score_rows * 4ull);
  return s.total < (1ull << 46);
}

struct EvictSpace {
  unsigned long long lists, keys, total;
  long long most_moves, key_rows;
};
bool evict_space(const Problem &p, const PagedCache &c, int64_t max_rows, int64_t keep, EvictSpace &s) {
  if (!c.mass || !c.pos || p.n_past == 0 || max_rows < 1 || max_rows > c.cap || keep < 1) return false;
  // a row moves from behind the budget into a place below it
  s.most_moves = max_rows <= keep ? 0 : max_rows - keep < keep ? max_rows - keep : keep;
  const unsigned long long windows = (unsigned long long)p.B * p.Hkv;
  s.lists = align_up(windows * 4ull);
  s.keys = align_up(s.lists + windows * 2ull * s.most_moves * 8ull);
  s.key_rows = s.most_moves == 0 || evict_keys_held(max_rows) ? 0 : (max_rows + 1023) / 1024 * 1024;
  s.total = s.keys + align_up(windows * 4ull * s.key_rows);
  return s.total < (1ull << 46);
}

// Two different buffers of `bytes` that share some of them.
bool overlap(const void *a, const void *b, unsigned long long bytes) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x != y && x < y + bytes && y < x + bytes;
}

// Rows of two strided tensors, `rows` each, that share bytes.  (Of tensors with different strides only the whole ranges
// are compared, so parts of rows that lie between each other's are taken for shared ones.)
bool rows_overlap(const void *x, long long x_row, long long x_stride, const void *y, long long y_row, long long y_stride, long long rows) {
  const uintptr_t from_x = (uintptr_t)x, from_y = (uintptr_t)y;
  const __int128 end_x = from_x + (__int128)(rows - 1) * x_stride + x_row, end_y = from_y + (__int128)(rows - 1) * y_stride + y_row;
  if (from_x >= end_y || from_y >= end_x) return false;
  if (x_stride != y_stride) return true;
  const long long off = (long long)(from_y - from_x) % x_stride, at = off < 0 ? off + x_stride : off;  // y's rows in x's
  return at < x_row || at + y_row > x_stride;
}

// One of the outputs shares bytes with another one or with an input.
struct Bytes {
  const void *at;
  unsigned long long count;
};
template <size_t kOuts, size_t kIns>
bool shared_bytes(const Bytes (&outs)[kOuts], const Bytes (&ins)[kIns]) {
  const auto meet = [](const Bytes &x, const Bytes &y) {
    const unsigned __int128 from_x = (uintptr_t)x.at, from_y = (uintptr_t)y.at;
    return x.at && y.at && x.count && y.count && from_x < from_y + y.count && from_y < from_x + x.count;
  };
  for (size_t i = 0; i < kOuts; ++i) {
    for (size_t j = 0; j < i; ++j)
      if (meet(outs[i], outs[j])) return true;
    for (size_t j = 0; j < kIns; ++j)
      if (meet(outs[i], ins[j])) return true;
  }
  return false;
}

unsigned long long table_entries(const Problem &p, const PagedCache &c) {
  return (unsigned long long)p.B * (c.per_head ? p.Hkv : 1) * c.max_pages;
}
// One of the outputs shares bytes with the table or with an array of the pool that holds a value per row.
template <size_t kOuts>
bool shared_with_pool(const Bytes (&outs)[kOuts], const Problem &p, const PagedCache &c) {
  const unsigned long long rows = (unsigned long long)c.n_pages * c.heads * c.page_rows.d;
  const Bytes pool[] = {{c.table, 4 * table_entries(p, c)}, {c.e4m3 ? c.k_scale : nullptr, rows}, {c.e4m3 ? c.v_scale : nullptr, rows},
                        {c.mass, 4 * rows}, {c.pos, 4 * rows}};
  return shared_bytes(outs, pool);
}

// A packed batch of new tokens; one without any is a batch too.
bool batch_size_fits(const Problem &p, int64_t total, int64_t max_seqlen) {
  if (max_seqlen < 1 || max_seqlen >= kMostRows) return false;
  return total == 0 || (total >= max_seqlen && total < kMostRows && total <= (long long)p.B * max_seqlen);
}
bool batch_fits(const Problem &p, const int32_t *cu_seqlens, int64_t total, int64_t max_seqlen) {
  if (!batch_size_fits(p, total, max_seqlen)) return false;
  return cu_seqlens ? !misaligned(cu_seqlens, 4) : total == p.B && max_seqlen == 1;
}

struct ReserveSpace {
  unsigned long long free_of, free, total;
  long long chunks;
};
bool reserve_space(const Problem &p, const PagedCache &c, ReserveSpace &s) {
  if ((c.per_head ? (long long)p.Hkv : 1ll) * c.max_pages >= kMostRows) return false;
  s.chunks = ((long long)c.n_pages + kTablePages - 1) / kTablePages;
  s.free_of = align_up(4ull * p.B * (c.per_head ? p.Hkv : 1));
  s.free = align_up(s.free_of + 4ull * s.chunks);
  s.total = s.free + align_up(4ull * c.n_pages);
  return true;
}

// Whether one workgroup does it all.  A thread of it goes through a sequence's entries one after the other, 0.25 us for each and head that wants
// it (tables per head: 0.6), and looks at them twice.  Measured, one workgroup and four launches, in us, eight heads: 256 sequences with an entry
// each 13 and 19 (tables per head 19 and 21), 8 with 4 entries 15 and 18 (25 and 18), 4 with 5 16 and 16, 2 with 6 19 and 16, one with 21
// 50 and 16 (100 and 17); one head, 2560 entries, 1454 and 22.
bool reserve_by_one_workgroup(const Problem &p, const PagedCache &c, int64_t total, int64_t max_seqlen) {
  // a row range of m rows meets (m + page_rows - 2) / page_rows + 1 entries at most
  const long long entries = (max_seqlen + c.page_rows.d - 2) / c.page_rows.d + 1;
  return p.B <= 256 && c.n_pages <= (1 << 18) && total * p.Hkv <= 2560 && (long long)p.B * p.Hkv * entries <= kSmallReserve &&
         p.Hkv * entries <= (c.per_head ? 10 : 40);
}

void fill_tables(const Problem &p, const segattn_pages *pages, PagedTablesArgs &a) {
  fill_heads(p, a.heads);
  a.table = const_cast<int32_t *>(pages->table);  // (the caller's device memory; the two calls that write it say so)
  a.B = p.B;
  a.Hkv = p.Hkv;
  a.tail = p.T;
  a.seg = fast_div_by(p.S);
}

bool build_blocks(const segattn_blocks *g, const Problem &p, const PagedCache &c, bool bounds, PagedBlocksArgs &a) {
  if (!g || g->block_rows < 16 || g->block_rows % 16 || (long long)c.page_rows.d % g->block_rows) return false;
  if (bounds && (!g->bounds || !g->scale || misaligned(g->bounds, 16))) return false;
  a.c = c;
  a.bounds = g->bounds;
  a.scale = g->scale;
  a.B = p.B;
  a.Hkv = p.Hkv;
  a.D = p.D;
  a.n_past = p.n_past;
  a.per_page = (int)(c.page_rows.d / g->block_rows);
  a.block_rows = fast_div_by(g->block_rows);
  for (int i = 0; i < p.n_past; ++i) a.past[i] = (unsigned char)p.order[i];
  return true;
}
Bytes bounds_bytes(const PagedBlocksArgs &a) { return Bytes{a.bounds, (unsigned long long)a.c.n_pages * a.c.heads * a.per_page * 2 * a.D}; }
Bytes scale_bytes(const PagedBlocksArgs &a) { return Bytes{a.scale, (unsigned long long)a.c.n_pages * a.c.heads * a.per_page}; }

constexpr long long kMostChosen = 4096, kMostListed = 65536;
constexpr unsigned long long kChoiceSpace = 256ull << 20;  // keys of as many tokens as fit are formed at a time, of one at least
bool choose_space(const Problem &p, const PagedBlocksArgs &k, int64_t total, int64_t max_rows, int32_t n_chosen, PagedChooseArgs &a,
                  unsigned long long &bytes) {
  if (p.n_past == 0 || p.g > kPagedMostGroup || total < 0 || total >= kMostRows || max_rows < 1 || max_rows > k.c.cap) return false;
  if (n_chosen < 1 || n_chosen > kMostChosen) return false;
  a.stride = (max_rows + k.block_rows.d - 1) / k.block_rows.d;
  const unsigned long long per_token = 4ull * p.n_past * a.stride;
  unsigned long long part = kChoiceSpace / per_token;
  part = part < 16 ? 16 : part;
  a.part = (int)(part < (unsigned long long)total ? part : total);
  // (not of whole tokens, so that a call's bytes cover those of fewer tokens or rows)
  const unsigned long long all = (unsigned long long)total * per_token, most = kChoiceSpace > 16 * per_token ? kChoiceSpace : 16 * per_token;
  bytes = align_up(all < most ? all : most);
  bytes = bytes ? bytes : kAlign;
  return true;
}

bool chosen_space(const Problem &p, const PagedCache &c, const segattn_blocks *blocks, const int32_t *cu_seqlens, int64_t total,
                  int64_t max_seqlen, int64_t max_rows, int32_t n_chosen, void *ws, PagedChosenArgs &a, unsigned long long &bytes) {
  PagedBlocksArgs k;
  memset(&k, 0, sizeof(k));
  if (!build_blocks(blocks, p, c, false, k)) return false;
  if (p.g > kPagedMostGroup || max_rows < 1 || max_rows > c.cap) return false;
  if (p.n_past && (n_chosen < 1 || n_chosen > kMostListed || (long long)n_chosen * blocks->block_rows >= kMostRows)) return false;
  a.c = c;
  a.total = total;
  a.B = p.B;
  a.Hq = p.Hq;
  a.Hkv = p.Hkv;
  a.g = p.g;
  a.D = p.D;
  a.n_past = p.n_past;
  a.n_other = p.Hkv - p.n_past;
  a.n_chosen = p.n_past ? n_chosen : 0;
  a.max_rows = (int)max_rows;
  a.tail = p.T;
  a.seg = fast_div_by(p.S);
  a.block_halves = fast_div_by(blocks->block_rows / 16);
  a.scale = p.scale;
  a.scale_log2e = p.scale_log2e;
  a.out_fp32 = p.out_fp32;
  a.cu = cu_seqlens;
  for (int i = 0; i < p.Hkv; ++i) {
    a.head_of[i] = (unsigned char)p.order[i];
    a.tail_of[i] = (p.policy[p.order[i]] & SEGATTN_TAIL) != 0;
  }
  bytes = kAlign;
  if (total == 0) return true;
  const unsigned long long planned = plan_paged_chosen(a, max_seqlen, (unsigned char *)ws), most = most_paged_chosen(a, max_seqlen);
  bytes = align_up(most > planned ? most : planned);  // (never less than what is laid out)
  bytes = bytes ? bytes : kAlign;
  return true;
}

}  // namespace

extern "C" {

segattn_status seg_rope_rotate(const segattn_config *cfg, const segattn_rope *rope, const void *q, int64_t q_stride,
                               const void *k, int64_t k_stride, int64_t rows, const int64_t *pos0, const int64_t *pos,
                               int32_t inverse, int32_t fp32, void *q_out, int64_t q_out_stride, void *k_out,
                               int64_t k_out_stride, void *stream) {
  Problem p;
  if (!build_problem(cfg, false, p) || !rope) return SEGATTN_EINVAL;
  RotateArgs a;
  memset(&a, 0, sizeof(a));
  if (!build_rotary(rope, p.D, a.rot)) return SEGATTN_EINVAL;
  if ((!q && !k) || (q != nullptr) != (q_out != nullptr) || (k != nullptr) != (k_out != nullptr)) return SEGATTN_EINVAL;
  if (rows < 1 || rows >= kMostRows || (long long)p.B * rows >= kMostRows || (pos0 && pos)) return SEGATTN_EINVAL;
  if (inverse < 0 || inverse > 1 || fp32 < 0 || fp32 > 1) return SEGATTN_EINVAL;
  const long long of_q = (long long)p.Hq * p.D, of_k = (long long)p.Hkv * p.D, size = fp32 ? 4 : 2;
  struct {
    const void *at;
    int64_t *stride;
    long long dense;
  } tensors[] = {{q, &q_stride, of_q}, {q_out, &q_out_stride, of_q}, {k, &k_stride, of_k}, {k_out, &k_out_stride, of_k}};
  for (auto &t : tensors) {
    if (!t.at) continue;
    if (*t.stride == 0) *t.stride = t.dense;
    if (*t.stride < t.dense || *t.stride >= (1ll << 32) || *t.stride * size % 16 || misaligned(t.at, 16)) return SEGATTN_EINVAL;
  }
  // in place only row by row: another place or stride would write over rows that are still to be read
  const long long total = (long long)p.B * rows;
  for (int out = 1; out < 4; out += 2) {
    for (int other = 0; other < 4; ++other) {
      const auto &x = tensors[out], &y = tensors[other];
      if (out == other || !x.at || !y.at || (other == out - 1 && x.at == y.at && *x.stride == *y.stride)) continue;
      if (rows_overlap(x.at, x.dense * size, *x.stride * size, y.at, y.dense * size, *y.stride * size, total)) return SEGATTN_EINVAL;
    }
  }
  if (misaligned(pos0, 8) || misaligned(pos, 8) || foreign(stream)) return SEGATTN_EINVAL;
  a.q = q;
  a.k = k;
  a.q_out = q_out;
  a.k_out = k_out;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.q_out_stride = q_out_stride;
  a.k_out_stride = k_out_stride;
  a.pos0 = (const long long *)pos0;
  a.pos = (const long long *)pos;
  a.total = total;
  a.rows = (int)rows;
  a.Hq = p.Hq;
  a.Hkv = p.Hkv;
  a.D = p.D;
  a.rot.back = inverse;
  return hip_status(launch_rotate(a, fp32 != 0, (hipStream_t)stream));
}

segattn_status seg_kv_paged_append(const segattn_config *cfg, const segattn_pages *pages, const segattn_rope *rope,
                                   const void *q, const void *k, const void *v, const int32_t *cu_seqlens, int64_t total,
                                   int64_t max_seqlen, const int64_t *pos0, const int32_t *rows, void *q_out,
                                   int32_t *rows_out, void *stream) {
  Problem p;
  PagedAppendArgs a;
  memset(&a, 0, sizeof(a));
  if (!build_paged(cfg, p) || !build_pages(pages, p, a.c)) return SEGATTN_EINVAL;
  if (rope && !build_rotary(rope, p.D, a.rot)) return SEGATTN_EINVAL;
  if (!k || !v || !rows || !rows_out || (q != nullptr) != (q_out != nullptr)) return SEGATTN_EINVAL;
  if (q && !rope && q != q_out) return SEGATTN_EINVAL;  // nothing to do but a copy
  if (max_seqlen < 1 || total < max_seqlen || total >= kMostRows || (!cu_seqlens && (total != p.B || max_seqlen != 1))) return SEGATTN_EINVAL;
  if (total > (long long)p.B * max_seqlen) return SEGATTN_EINVAL;
  if (misaligned(q, 16) || misaligned(q_out, 16) || misaligned(k, 16) || misaligned(v, 16) || misaligned(rows, 4) ||
      misaligned(rows_out, 4) || misaligned(cu_seqlens, 4) || misaligned(pos0, 8))
    return SEGATTN_EINVAL;
  if (overlap(rows, rows_out, 4ull * p.B * p.Hkv) || overlap(q, q_out, 2ull * total * p.Hq * p.D) || foreign(stream)) return SEGATTN_EINVAL;
  const long long q_bytes = 2ll * total * p.Hq * p.D, k_bytes = 2ll * total * p.Hkv * p.D;
  if (q_out && (rows_overlap(q_out, q_bytes, q_bytes, k, k_bytes, k_bytes, 1) || rows_overlap(q_out, q_bytes, q_bytes, v, k_bytes, k_bytes, 1)))
    return SEGATTN_EINVAL;
  a.q = (const unsigned short *)q;
  a.k = (const unsigned short *)k;
  a.v = (const unsigned short *)v;
  a.q_out = rope ? (unsigned short *)q_out : nullptr;
  a.cu = max_seqlen == 1 && total == p.B ? nullptr : cu_seqlens;  // one token each
  a.pos0 = (const long long *)pos0;
  a.rows = rows;
  a.rows_out = rows_out;
  a.total = (int)total;
  a.B = p.B;
  a.Hq = p.Hq;
  a.Hkv = p.Hkv;
  a.D = p.D;
  return hip_status(launch_paged_append(a, (hipStream_t)stream));
}

size_t seg_attn_decode_paged_workspace_bytes(const segattn_config *cfg, const segattn_pages *pages, int64_t max_rows,
                                             int32_t accumulate) {
  Problem p;
  PagedCache c;
  DecodeSpace s;
  if (!build_paged(cfg, p) || !build_pages(pages, p, c) || !decode_space(p, c, max_rows, accumulate, s)) return 0;
  return (size_t)s.total;
}

segattn_status seg_attn_decode_paged(const segattn_config *cfg, const segattn_pages *pages, const void *q,
                                     const int32_t *rows, int64_t max_rows, int32_t accumulate, void *out, float *lse,
                                     void *workspace, size_t workspace_bytes, void *stream) {
  Problem p;
  PagedDecodeArgs a;
  DecodeSpace s;
  memset(&a, 0, sizeof(a));
  if (!build_paged(cfg, p) || !build_pages(pages, p, a.c) || !decode_space(p, a.c, max_rows, accumulate, s)) return SEGATTN_EINVAL;
  if (!q || !rows || !out || !lse || !workspace || workspace_bytes < s.total) return SEGATTN_EINVAL;
  if (misaligned(q, 16) || misaligned(rows, 4) || misaligned(out, p.out_fp32 ? 4 : 2) || misaligned(lse, 4) ||
      misaligned(workspace, kAlign) || foreign(stream))
    return SEGATTN_EINVAL;
  unsigned char *ws = (unsigned char *)workspace;
  a.q = (const unsigned short *)q;
  a.rows = rows;
  a.out = out;
  a.lse = lse;
  a.pieces = (int2 *)(ws + s.pieces);
  a.slots = (float *)(ws + s.slots);
  a.scores = accumulate ? (float *)(ws + s.scores) : nullptr;
  a.score_rows = s.score_rows;
  fill_heads(p, a.heads);
  a.B = p.B;
  a.Hq = p.Hq;
  a.Hkv = p.Hkv;
  a.g = p.g;
  a.D = p.D;
  a.n_windows = p.B * p.Hkv;
  a.n_past = p.n_past;
  a.max_rows = (int)max_rows;
  a.tail = p.T;
  a.seg = fast_div_by(p.S);
  a.n_kv = fast_div_by(p.Hkv);
  a.scale = p.scale;
  a.scale_log2e = p.scale_log2e;
  a.out_fp32 = p.out_fp32;
  return hip_status(launch_paged_decode(a, (hipStream_t)stream));
}

size_t seg_kv_paged_evict_workspace_bytes(const segattn_config *cfg, const segattn_pages *pages, int64_t max_rows,
                                          int64_t keep_rows) {
  Problem p;
  PagedCache c;
  EvictSpace s;
  if (!build_paged(cfg, p) || !build_pages(pages, p, c) || !evict_space(p, c, max_rows, keep_rows, s)) return 0;
  return (size_t)s.total;
}

segattn_status seg_kv_paged_evict(const segattn_config *cfg, const segattn_pages *pages, const int32_t *rows,
                                  int64_t max_rows, int64_t keep_rows, int64_t keep_recent, int64_t keep_first,
                                  int32_t *rows_out, void *workspace, size_t workspace_bytes, void *stream) {
  Problem p;
  PagedEvictArgs a;
  EvictSpace s;
  memset(&a, 0, sizeof(a));
  if (!build_paged(cfg, p) || !build_pages(pages, p, a.c) || !evict_space(p, a.c, max_rows, keep_rows, s)) return SEGATTN_EINVAL;
  if (keep_recent < 0 || keep_first < 0 || keep_recent > keep_rows || keep_first > keep_rows - keep_recent) return SEGATTN_EINVAL;
  if (!rows || !rows_out || !workspace || workspace_bytes < s.total) return SEGATTN_EINVAL;
  if (misaligned(rows, 4) || misaligned(rows_out, 4) || misaligned(workspace, kAlign) ||
      overlap(rows, rows_out, 4ull * p.B * p.Hkv) || foreign(stream))
    return SEGATTN_EINVAL;
  unsigned char *ws = (unsigned char *)workspace;
  a.rows = rows;
  a.rows_out = rows_out;
  a.moves = (int *)ws;
  a.lists = (int2 *)(ws + s.lists);
  a.keys = s.key_rows ? (unsigned *)(ws + s.keys) : nullptr;
  a.key_rows = s.key_rows;
  fill_heads(p, a.heads);
  a.B = p.B;
  a.Hkv = p.Hkv;
  a.D = p.D;
  a.max_rows = (int)max_rows;
  a.budget = (int)(keep_rows < kMostRows ? keep_rows : kMostRows);
  a.keep = a.budget < a.max_rows ? a.budget : a.max_rows;
  a.recent = (int)(keep_recent < kMostRows ? keep_recent : kMostRows);
  a.first = (int)(keep_first < kMostRows ? keep_first : kMostRows);
  a.most_moves = (int)s.most_moves;
  return hip_status(launch_paged_evict(a, (hipStream_t)stream));
}

size_t seg_kv_paged_reserve_workspace_bytes(const segattn_config *cfg, const segattn_pages *pages) {
  Problem p;
  PagedCache c;
  ReserveSpace s;
  if (!build_paged(cfg, p) || !build_pages(pages, p, c) || !reserve_space(p, c, s)) return 0;
  return (size_t)s.total;
}

segattn_status seg_kv_paged_reserve(const segattn_config *cfg, const segattn_pages *pages, int32_t *users,
                                    const int32_t *cu_seqlens, int64_t total, int64_t max_seqlen, const int32_t *rows,
                                    int32_t newest_only, int32_t *granted, int64_t *slots, void *workspace,
                                    size_t workspace_bytes, void *stream) {
  Problem p;
  PagedTablesArgs a;
  ReserveSpace s;
  memset(&a, 0, sizeof(a));
  if (!build_paged(cfg, p) || !build_pages(pages, p, a.c) || !reserve_space(p, a.c, s)) return SEGATTN_EINVAL;
  if (!users || !rows || !granted || !workspace || workspace_bytes < s.total || newest_only < 0 || newest_only > 1) return SEGATTN_EINVAL;
  if (!batch_fits(p, cu_seqlens, total, max_seqlen)) return SEGATTN_EINVAL;
  if (misaligned(users, 4) || misaligned(rows, 4) || misaligned(granted, 4) || misaligned(slots, 8) || misaligned(workspace, kAlign) ||
      foreign(stream))
    return SEGATTN_EINVAL;
  const Bytes outs[] = {{pages->table, 4 * table_entries(p, a.c)}, {users, 4ull * a.c.n_pages}, {granted, 4ull * p.B},
                        {slots, 8ull * total * p.Hkv}, {workspace, s.total}};
  const Bytes ins[] = {{rows, 4ull * p.B * p.Hkv}, {cu_seqlens, 4ull * (p.B + 1ull)}};
  if (shared_bytes(outs, ins)) return SEGATTN_EINVAL;
  unsigned char *ws = (unsigned char *)workspace;
  fill_tables(p, pages, a);
  a.users = users;
  a.cu = cu_seqlens;
  a.rows = rows;
  a.granted = granted;
  a.slots = (long long *)slots;
  a.need = (int *)ws;
  a.free_of = (int *)(ws + s.free_of);
  a.free = (int *)(ws + s.free);
  a.total = total;
  a.newest = newest_only;
  a.chunks = (int)s.chunks;
  a.heads_div = fast_div_by(p.Hkv);
  a.longest = (int)max_seqlen;
  a.small = reserve_by_one_workgroup(p, a.c, total, max_seqlen);
  return hip_status(launch_paged_reserve(a, (hipStream_t)stream));
}

segattn_status seg_kv_paged_release(const segattn_config *cfg, const segattn_pages *pages, int32_t *users, const int32_t *rows,
                                    void *stream) {
  Problem p;
  PagedTablesArgs a;
  memset(&a, 0, sizeof(a));
  if (!build_paged(cfg, p) || !build_pages(pages, p, a.c)) return SEGATTN_EINVAL;
  if (!users || !rows || misaligned(users, 4) || misaligned(rows, 4) || foreign(stream)) return SEGATTN_EINVAL;
  const Bytes outs[] = {{pages->table, 4 * table_entries(p, a.c)}, {users, 4ull * a.c.n_pages}};
  const Bytes ins[] = {{rows, 4ull * p.B * p.Hkv}};
  if (shared_bytes(outs, ins)) return SEGATTN_EINVAL;
  fill_tables(p, pages, a);
  a.users = users;
  a.rows = rows;
  return hip_status(launch_paged_release(a, (hipStream_t)stream));
}

segattn_status seg_kv_paged_summarize(const segattn_config *cfg, const segattn_pages *pages, const segattn_blocks *blocks,
                                      const int32_t *rows_from, const int32_t *rows, int64_t max_new, void *stream) {
  Problem p;
  PagedCache c;
  PagedBlocksArgs a;
  memset(&a, 0, sizeof(a));
  if (!build_paged(cfg, p) || !build_pages(pages, p, c) || !build_blocks(blocks, p, c, true, a)) return SEGATTN_EINVAL;
  if (p.n_past == 0 || !rows || max_new < 1 || max_new >= kMostRows) return SEGATTN_EINVAL;
  if (misaligned(rows_from, 4) || misaligned(rows, 4) || foreign(stream)) return SEGATTN_EINVAL;
  const Bytes outs[] = {bounds_bytes(a), scale_bytes(a)};
  const Bytes ins[] = {{rows, 4ull * p.B * p.Hkv}, {rows_from, 4ull * p.B * p.Hkv}};
  if (shared_bytes(outs, ins) || shared_with_pool(outs, p, c)) return SEGATTN_EINVAL;
  a.rows_from = rows_from;
  a.rows = rows;
  a.most = (int)((max_new + blocks->block_rows - 1) / blocks->block_rows);
  a.units = (long long)p.B * p.n_past * a.most;
  if (a.units >= (1ll << 40)) return SEGATTN_EINVAL;
  return hip_status(launch_paged_summarize(a, (hipStream_t)stream));
}

size_t seg_kv_paged_choose_workspace_bytes(const segattn_config *cfg, const segattn_pages *pages, const segattn_blocks *blocks,
                                           int64_t total, int64_t max_rows, int32_t n_chosen) {
  Problem p;
  PagedCache c;
  PagedChooseArgs a;
  unsigned long long bytes;
  memset(&a, 0, sizeof(a));
  if (!build_paged(cfg, p) || !build_pages(pages, p, c) || !build_blocks(blocks, p, c, true, a.k)) return 0;
  return choose_space(p, a.k, total, max_rows, n_chosen, a, bytes) ? (size_t)bytes : 0;
}

segattn_status seg_kv_paged_choose(const segattn_config *cfg, const segattn_pages *pages, const segattn_blocks *blocks, const void *q,
                                   const int32_t *cu_seqlens, int64_t total, int64_t max_seqlen, const int32_t *rows,
                                   int64_t max_rows, int32_t n_chosen, int32_t keep_first, int32_t keep_recent, int32_t *chosen,
                                   void *workspace, size_t workspace_bytes, void *stream) {
  Problem p;
  PagedCache c;
  PagedChooseArgs a;
  unsigned long long bytes;
  memset(&a, 0, sizeof(a));
  if (!build_paged(cfg, p) || !build_pages(pages, p, c) || !build_blocks(blocks, p, c, true, a.k)) return SEGATTN_EINVAL;
  if (!batch_fits(p, cu_seqlens, total, max_seqlen) || !choose_space(p, a.k, total, max_rows, n_chosen, a, bytes)) return SEGATTN_EINVAL;
  if (keep_first < 0 || keep_recent < 1 || keep_first > n_chosen - keep_recent || keep_recent > n_chosen) return SEGATTN_EINVAL;
  if ((total > 0 && (!q || !chosen)) || !rows || !workspace || workspace_bytes < bytes) return SEGATTN_EINVAL;
  if (misaligned(q, 16) || misaligned(rows, 4) || misaligned(chosen, 4) || misaligned(workspace, kAlign) || foreign(stream)) return SEGATTN_EINVAL;
  const Bytes outs[] = {{chosen, 4ull * total * p.n_past * n_chosen}, {workspace, bytes}};
  const Bytes ins[] = {{q, 2ull * total * p.Hq * p.D}, {rows, 4ull * p.B * p.Hkv}, {cu_seqlens, 4ull * (p.B + 1ull)},
                       bounds_bytes(a.k), scale_bytes(a.k)};
  if (shared_bytes(outs, ins) || shared_with_pool(outs, p, c)) return SEGATTN_EINVAL;
  if (total == 0) return SEGATTN_OK;
  a.q = (const unsigned short *)q;
  a.cu = cu_seqlens;
  a.k.rows = rows;
  a.chosen = chosen;
  a.keys = (unsigned *)workspace;
  a.total = total;
  a.Hq = p.Hq;
  a.g = p.g;
  a.max_rows = (int)max_rows;
  a.n_chosen = n_chosen;
  a.first = keep_first;
  a.recent = keep_recent;
  plan_paged_choose(a, max_seqlen);
  return hip_status(launch_paged_choose(a, (hipStream_t)stream));
}

size_t seg_attn_paged_chosen_workspace_bytes(const segattn_config *cfg, const segattn_pages *pages, const segattn_blocks *blocks,
                                             int64_t total, int64_t max_seqlen, int64_t max_rows, int32_t n_chosen) {
  Problem p;
  PagedCache c;
  PagedChosenArgs a;
  unsigned long long bytes;
  memset(&a, 0, sizeof(a));
  if (!build_paged(cfg, p) || !build_pages(pages, p, c)) return 0;
  if (!batch_size_fits(p, total, max_seqlen)) return 0;
  // (without cu_seqlens a sequence has one token, and then nothing depends on them)
  return chosen_space(p, c, blocks, (const int32_t *)4, total, max_seqlen, max_rows, n_chosen, nullptr, a, bytes) ? (size_t)bytes : 0;
}

segattn_status seg_attn_paged_chosen(const segattn_config *cfg, const segattn_pages *pages, const segattn_blocks *blocks, const void *q,
                                     const int32_t *cu_seqlens, int64_t total, int64_t max_seqlen, const int32_t *rows,
                                     int64_t max_rows, const int32_t *chosen, int32_t n_chosen, void *out, float *lse,
                                     void *workspace, size_t workspace_bytes, void *stream) {
  Problem p;
  PagedCache c;
  PagedChosenArgs a;
  unsigned long long bytes;
  memset(&a, 0, sizeof(a));
  if (!build_paged(cfg, p) || !build_pages(pages, p, c) || !batch_fits(p, cu_seqlens, total, max_seqlen)) return SEGATTN_EINVAL;
  if (!chosen_space(p, c, blocks, cu_seqlens, total, max_seqlen, max_rows, n_chosen, workspace, a, bytes)) return SEGATTN_EINVAL;
  if ((total > 0 && (!q || !out || !lse || (p.n_past && !chosen))) || !rows || !workspace || workspace_bytes < bytes) return SEGATTN_EINVAL;
  if (misaligned(q, 16) || misaligned(rows, 4) || misaligned(chosen, 4) || misaligned(out, p.out_fp32 ? 4 : 2) || misaligned(lse, 4) ||
      misaligned(workspace, kAlign) || foreign(stream))
    return SEGATTN_EINVAL;
  const unsigned long long heads = (unsigned long long)total * p.Hq;
  const Bytes outs[] = {{out, heads * p.D * (p.out_fp32 ? 4 : 2)}, {lse, heads * 4}, {workspace, bytes}};
  const Bytes ins[] = {{q, heads * p.D * 2}, {rows, 4ull * p.B * p.Hkv}, {cu_seqlens, 4ull * (p.B + 1ull)},
                       {p.n_past ? chosen : nullptr, 4ull * total * p.n_past * n_chosen}};
  if (shared_bytes(outs, ins) || shared_with_pool(outs, p, c)) return SEGATTN_EINVAL;
  if (total == 0) return SEGATTN_OK;
  a.q = (const unsigned short *)q;
  a.rows = rows;
  a.chosen = chosen;
  a.out = out;
  a.lse = lse;
  return hip_status(launch_paged_chosen(a, (hipStream_t)stream));
}

}  // extern "C"
