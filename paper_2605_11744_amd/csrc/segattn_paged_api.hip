// C ABI of the operators around a paged cache: argument validation and launches.
#include <math.h>
#include <string.h>

#include "segattn_paged.h"

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

}  // extern "C"
