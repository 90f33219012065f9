// Host entry points of the paged cache: argument validation, the division of
// an attention call into blocks, then the kernels' launch functions.  Nothing
// here allocates memory or synchronises a stream.
#include <algorithm>

#include "paged.h"

namespace starkv {

namespace {

bool at(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
size_t up256(size_t x) { return (x + 255) / 256 * 256; }
starkv_status hip_status(int err) { return err ? STARKV_E_HIP : STARKV_OK; }

}  // namespace

starkv_status check_paged(const starkv_paged* c, PagedView* v) {
  if (!c) return STARKV_E_NULL;
  if (c->dtype != STARKV_F32 && c->dtype != STARKV_BF16) return STARKV_E_DTYPE;
  if (c->n_layers < 1 || c->n_layers > 4096) return STARKV_E_SHAPE;
  if (c->G < 1 || c->G > STARKV_MAX_GROUPS || c->H < c->G || c->H % c->G != 0 || c->H > 4096)
    return STARKV_E_SHAPE;
  if (c->d != 64 && c->d != 128) return STARKV_E_SHAPE;
  const int P = c->page_tokens;
  if (P < 16 || P > 1024 || (P & (P - 1))) return STARKV_E_SHAPE;
  if (c->n_pages < 1 || c->n_pages > kMaxTokens || c->n_slots < 1 || c->n_slots > (1 << 20) ||
      c->max_pages < 1 || (int64_t)c->max_pages * P > kMaxTokens || c->reserved != 0)
    return STARKV_E_SHAPE;
  const int64_t esz = c->dtype == STARKV_F32 ? 4 : 2;
  const int64_t st[4] = {c->layer_stride, c->page_stride, c->group_stride, c->token_stride};
  if (c->token_stride < c->d) return STARKV_E_SHAPE;
  for (int64_t s : st) {
    if (s < 0 || s > INT64_MAX / 8) return STARKV_E_SHAPE;
    if (s * esz % 16) return STARKV_E_ALIGN;
  }
  if (c->token_stride * esz >= 1 << 28) return STARKV_E_SHAPE;   // 32-bit offsets within 8 rows
  if (!c->k || !c->v || !c->table || !c->len || !c->refs) return STARKV_E_NULL;
  if (!at(c->k, 16) || !at(c->v, 16) || !at(c->table, 4) || !at(c->len, 4) || !at(c->refs, 4))
    return STARKV_E_ALIGN;
  if (v) {
    v->k = static_cast<char*>(c->k);
    v->v = static_cast<char*>(c->v);
    v->table = c->table;
    v->len = c->len;
    v->refs = c->refs;
    v->ls = c->layer_stride * esz;
    v->ps = c->page_stride * esz;
    v->gs = c->group_stride * esz;
    v->ts = c->token_stride * esz;
    v->n_layers = c->n_layers;
    v->H = c->H;
    v->G = c->G;
    v->d = c->d;
    v->esz = (int)esz;
    v->P = P;
    v->psh = 0;
    while ((1 << v->psh) < P) ++v->psh;
    v->n_pages = c->n_pages;
    v->n_slots = c->n_slots;
    v->max_pages = c->max_pages;
    v->cap = c->max_pages * P;
  }
  return STARKV_OK;
}

starkv_status check_slots(const PagedView& v, const int32_t* slots, int32_t n, bool once) {
  if (n < 0 || n > kMaxSeqs) return STARKV_E_PARAM;
  if (n == 0) return STARKV_OK;
  if (!slots) return STARKV_E_NULL;
  int32_t seen[kMaxSeqs];
  for (int i = 0; i < n; ++i) {
    if (slots[i] < 0 || slots[i] >= v.n_slots) return STARKV_E_PARAM;
    seen[i] = slots[i];
  }
  if (once) {
    std::sort(seen, seen + n);
    for (int i = 1; i < n; ++i)
      if (seen[i] == seen[i - 1]) return STARKV_E_PARAM;
  }
  return STARKV_OK;
}

PagesWs pages_ws(const PagedView& v, int n, int64_t most) {
  PagesWs w;
  w.most_fresh = (int64_t)n * ((most + v.P - 1) / v.P + 1);
  w.fresh = 0;
  w.info = up256((size_t)w.most_fresh * 4);
  w.old = w.info + up256((size_t)n * 16);
  w.bytes = w.old + up256((size_t)n * v.max_pages * 4);
  return w;
}

namespace {

// rows[b] >= 0 query (or written) tokens per sequence, into a RowList.
starkv_status take_rows(const PagedView& v, const int32_t* slots, const int32_t* rows, int n,
                        RowList* r) {
  int64_t tot = 0;
  r->n = n;
  r->row0[0] = 0;
  for (int b = 0; b < n; ++b) {
    if (rows[b] < 0 || rows[b] > v.cap) return STARKV_E_PARAM;
    tot += rows[b];
    if (tot > kMaxTokens) return STARKV_E_PARAM;
    r->slot[b] = slots ? slots[b] : 0;
    r->row0[b + 1] = (int32_t)tot;
  }
  return STARKV_OK;
}

}  // namespace

namespace {

// How many splits a (layer, group, row tile)'s steps are divided into, at
// most `most`, in a call of n sequences.
int split_count(const AttendShape& s, int n, int d, int esz, int64_t steps, int64_t most) {
  if (s.units == 0) return 1;
  if (!s.many) {
    // bound by HBM: splits of at least two steps for each of a block's waves
    // (four in the kernel for 32 rows, whose blocks take longer to end).
    // Measured, 256 against 512 tokens: one sequence of 13,711 tokens 13.7 and
    // 15.6 us, eight trees of four tokens (28 rows) 47.8 and 34.3
    const int64_t least = s.row_tile == 32 ? 16 : 8;
    // and of so many blocks in all that each CU has two, which keep HBM busy.
    // 512 against 1,024 blocks: 28 layers of 4 trees of 4 tokens 126 and 148
    // us, 64 sequences of one token 85 and 92, float32 trees of up to 13 tokens
    // 37 and 40; 12 sequences of 3,000 to 9,000 tokens 62 and 54
    const int64_t blocks = 512;
    // of several sequences, whose lengths may be far from each other, none of
    // over 3,200 tokens (float32: 1,536), or one long sequence would hold up
    // the rest (two layers of 18 trees of 3 tokens over 215 to 30,867 140 us
    // without and 128 with; float32, eight trees over 1,664 to 39,197 tokens
    // 442 and 355), as far as 4,096 blocks go: the bound on the lengths may be
    // a whole table row, of which little is in use, and every split has its
    // place in the workspace
    const int64_t longest = esz == 2 ? 100 : 48;
    const int64_t even = n > 1 ? std::min((steps + longest - 1) / longest, 4096 / s.units) : 1;
    const int64_t ns = std::min((steps + least - 1) / least, std::max(even, blocks / s.units));
    return (int)std::max<int64_t>(1, std::min(ns, most));
  }
  const int64_t top = std::min(steps, most);
  if (n > 1) {
    // lengths that only the device knows: it divides the steps itself, into
    // at most this many splits
    return (int)std::min(top, std::max<int64_t>(1, 1024 / s.units));
  }
  // bound by the matrix units: rounds of the 512 blocks that the card holds,
  // each as long as a split's steps and the four that a block's start and
  // end are worth; joining costs two steps and one per 10 MB of partial sums
  double best = 0;
  int best_ns = 1;
  const int64_t last = std::min<int64_t>(top, std::max<int64_t>(1, 4096 / s.units));
  for (int64_t ns = 1; ns <= last;) {
    const int64_t per = (steps + ns - 1) / ns;
    double cost = (double)((s.units * ns + 511) / 512) * (double)(per + 4);
    if (ns > 1) cost += 2 + (double)(s.units * ns) * s.row_tile * d * 8 / 10e6;
    if (ns == 1 || cost < best) {
      best = cost;
      best_ns = (int)ns;
    }
    if (per == 1) break;
    ns = (steps + per - 2) / (per - 1);   // the least with shorter splits; between them none is cheaper
  }
  return best_ns;
}

}  // namespace

starkv_status attend_shape(const PagedView& v, const int32_t* rows, int n, int32_t max_len,
                           int32_t window, int32_t sinks, AttendShape* s, int32_t* tile0) {
  if (n < 0 || n > kMaxSeqs) return STARKV_E_PARAM;
  if (n > 0 && !rows) return STARKV_E_NULL;
  if (max_len < 1 || max_len > kMaxTokens) return STARKV_E_PARAM;
  const int hpg = v.H / v.G;
  int64_t tot = 0, most = 0;
  for (int b = 0; b < n; ++b) {
    if (rows[b] < 0 || rows[b] > v.cap) return STARKV_E_PARAM;
    tot += rows[b];
    most = std::max<int64_t>(most, rows[b]);
  }
  if (tot > kMaxTokens) return STARKV_E_PARAM;
  s->n_rows = (int)tot;
  const int64_t R = most * hpg;
  s->many = v.esz == 2 && R > 32;
  s->row_tile = s->many ? 128 : v.esz == 2 && R > 16 ? 32 : 16;
  int64_t tiles = 0;
  for (int b = 0; b < n; ++b) {
    if (tile0) tile0[b] = (int32_t)tiles;
    tiles += ((int64_t)rows[b] * hpg + s->row_tile - 1) / s->row_tile;
  }
  if (tile0) tile0[n] = (int32_t)tiles;
  s->units = tiles * v.n_layers * v.G;
  // Splits for the tokens that one row tile may see.  The workspace is that
  // of a call without a window, whose splits bound those of one with it.
  const int64_t len = std::min<int64_t>(max_len, v.cap);
  const int step = s->many ? 64 : 32;
  const int most_split = split_count(*s, n, v.d, v.esz, (len + step - 1) / step, INT32_MAX);
  const int64_t row_tokens = (s->row_tile + hpg - 1) / hpg + 1;
  const int64_t seen = window ? std::min<int64_t>(len, (int64_t)window + sinks + row_tokens + 2 * step)
                              : len;
  const int64_t steps = std::max<int64_t>(1, (seen + step - 1) / step);
  s->n_split = split_count(*s, n, v.d, v.esz, steps, most_split);
  s->chunk = (int)((steps + s->n_split - 1) / s->n_split * step);
  // (up to 1.6 blocks to a tile's split, each of 256 of a launch's 2^32
  // threads; and a sequence's rows stay below 2^31)
  if (s->units > 1 << 23) return STARKV_E_PARAM;
  s->n_tiles = (int)tiles;
  s->seq_tiles = (int)std::max<int64_t>(1, (R + s->row_tile - 1) / s->row_tile);
  s->stat_off = s->steps_off = s->ws_bytes = 0;
  s->steps = (int)steps;
  s->balance = s->many && n > 1 && s->n_split > 1;
  if (most_split > 1) {
    const size_t rec = (size_t)s->units * most_split * s->row_tile;
    s->stat_off = up256(rec * v.d * sizeof(float));
    s->steps_off = s->stat_off + up256(rec * 2 * sizeof(float));
    s->ws_bytes = s->steps_off + 256;
  }
  return STARKV_OK;
}

namespace {

starkv_status attend(const starkv_paged* cache, const int32_t* slots, int32_t n,
                     const int32_t* rows, int32_t max_len, AttendCall* c, size_t ws_bytes,
                     void* stream) {
  PagedView v;
  starkv_status st = check_paged(cache, &v);
  if (st != STARKV_OK) return st;
  if ((st = check_slots(v, slots, n, false)) != STARKV_OK) return st;
  if ((st = attend_shape(v, rows, n, max_len, c->words ? 0 : c->window, c->sinks, &c->s,
                         c->tile0)) != STARKV_OK) return st;
  if (c->words)
    for (int b = 0; b < n; ++b)
      if (rows[b] > 64 * c->words) return STARKV_E_PARAM;
  if ((st = take_rows(v, slots, rows, n, &c->r)) != STARKV_OK) return st;
  if (c->s.n_rows == 0) return STARKV_OK;
  if (!c->q || !c->out || (c->words && !c->mask)) return STARKV_E_NULL;
  if (!at(c->q, 16) || !at(c->out, 16) || !at(c->lse, 4) || !at(c->mask, 8))
    return STARKV_E_ALIGN;
  if (c->s.ws_bytes) {
    if (!c->ws || ws_bytes < c->s.ws_bytes) return STARKV_E_WORKSPACE;
    if (!at(c->ws, 16)) return STARKV_E_ALIGN;
  }
  return hip_status(launch_attend(v, *c, stream));
}

starkv_status write(const starkv_paged* cache, const int32_t* slots, int32_t n,
                    const int32_t* rows, const void* k, const void* vv,
                    const starkv_kv_layout* lay, const int32_t* grown, void* stream) {
  PagedView v;
  starkv_status st = check_paged(cache, &v);
  if (st != STARKV_OK) return st;
  if ((st = check_slots(v, slots, n, true)) != STARKV_OK) return st;
  if (n == 0) return STARKV_OK;
  if (!rows || !lay) return STARKV_E_NULL;
  RowList r;
  if ((st = take_rows(v, slots, rows, n, &r)) != STARKV_OK) return st;
  r.grown = grown;
  if (lay->layer_stride < 0 || lay->group_stride < 0 || lay->token_stride < 0)
    return STARKV_E_SHAPE;
  if (r.row0[n] == 0) return STARKV_OK;
  if (!k || !vv) return STARKV_E_NULL;
  const int64_t e = v.esz;
  if (lay->layer_stride > INT64_MAX / 8 || lay->group_stride > INT64_MAX / 8 ||
      lay->token_stride > INT64_MAX / 8)
    return STARKV_E_SHAPE;
  if (lay->layer_stride * e % 16 || lay->group_stride * e % 16 || lay->token_stride * e % 16 ||
      !at(k, 16) || !at(vv, 16) || !at(grown, 4))
    return STARKV_E_ALIGN;
  return hip_status(launch_pages_write(v, r, k, vv, *lay, stream));
}

starkv_status compact(const starkv_paged* cache, const int32_t* slots, int32_t n,
                      const int32_t* span, const int32_t* idx, int64_t idx_layer_stride, int32_t B,
                      const int32_t* counts, int32_t tail, const int32_t* grown, int32_t* status,
                      void* ws, size_t ws_bytes, void* stream) {
  PagedView v;
  starkv_status st = check_paged(cache, &v);
  if (st != STARKV_OK) return st;
  if ((st = check_slots(v, slots, n, true)) != STARKV_OK) return st;
  if (B < 0 || tail < 0 || (int64_t)B + tail > kMaxTokens) return STARKV_E_BUDGET;
  if (idx_layer_stride < 0) return STARKV_E_SHAPE;
  if (n == 0) return STARKV_OK;
  if (!status || (B > 0 && !idx)) return STARKV_E_NULL;
  SeqList s;
  s.n = n;
  s.grown = grown;
  for (int b = 0; b < n; ++b) {
    if (span && (span[b] < 0 || span[b] > kMaxTokens)) return STARKV_E_PARAM;
    s.slot[b] = slots[b];
    s.num[b] = span ? span[b] : 0;
  }
  if (!at(status, 4) || !at(idx, 4) || !at(counts, 4) || !at(grown, 4))
    return STARKV_E_ALIGN;
  const PagesWs w = pages_ws(v, n, (int64_t)B + tail);
  if (!ws || ws_bytes < w.bytes) return STARKV_E_WORKSPACE;
  if (!at(ws, 16)) return STARKV_E_ALIGN;
  return hip_status(launch_pages_compact(v, s, span == nullptr, idx, idx_layer_stride, B, counts,
                                         tail, w, status, ws, stream));
}

}  // namespace

}  // namespace starkv

using namespace starkv;

extern "C" {

starkv_status starkv_pages_init(const starkv_paged* cache, void* stream) {
  PagedView v;
  const starkv_status st = check_paged(cache, &v);
  if (st != STARKV_OK) return st;
  return hip_status(launch_pages_init(v, stream));
}

size_t starkv_pages_workspace_bytes(const starkv_paged* cache, int32_t n, int32_t most) {
  PagedView v;
  if (check_paged(cache, &v) != STARKV_OK || n < 0 || n > kMaxSeqs || most < 0 ||
      most > kMaxTokens)
    return 0;
  return pages_ws(v, n, most).bytes;
}

starkv_status starkv_pages_grow(const starkv_paged* cache, const int32_t* slots, int32_t n,
                                const int32_t* add, int32_t* status, void* ws, size_t ws_bytes,
                                void* stream) {
  PagedView v;
  starkv_status st = check_paged(cache, &v);
  if (st != STARKV_OK) return st;
  if ((st = check_slots(v, slots, n, true)) != STARKV_OK) return st;
  if (n == 0) return STARKV_OK;
  if (!add || !status) return STARKV_E_NULL;
  SeqList s;
  s.n = n;
  int32_t most = 0;
  for (int b = 0; b < n; ++b) {
    if (add[b] < 0 || add[b] > kMaxTokens) return STARKV_E_PARAM;
    s.slot[b] = slots[b];
    s.num[b] = add[b];
    most = std::max(most, add[b]);
  }
  if (!at(status, 4)) return STARKV_E_ALIGN;
  const PagesWs w = pages_ws(v, n, most);
  if (!ws || ws_bytes < w.bytes) return STARKV_E_WORKSPACE;
  if (!at(ws, 16)) return STARKV_E_ALIGN;
  return hip_status(launch_pages_grow(v, s, w, status, ws, stream));
}

starkv_status starkv_pages_write(const starkv_paged* cache, const int32_t* slots, int32_t n,
                                 const int32_t* rows, const void* k, const void* v,
                                 const starkv_kv_layout* lay, void* stream) {
  return write(cache, slots, n, rows, k, v, lay, nullptr, stream);
}

starkv_status starkv_pages_write_grown(const starkv_paged* cache, const int32_t* slots, int32_t n,
                                       const int32_t* rows, const void* k, const void* v,
                                       const starkv_kv_layout* lay, const int32_t* grown,
                                       void* stream) {
  if (n > 0 && !grown) return STARKV_E_NULL;
  return write(cache, slots, n, rows, k, v, lay, grown, stream);
}

starkv_status starkv_pages_fork(const starkv_paged* cache, const int32_t* src,
                                const int32_t* dst, int32_t n, void* stream) {
  PagedView v;
  starkv_status st = check_paged(cache, &v);
  if (st != STARKV_OK) return st;
  if ((st = check_slots(v, src, n, false)) != STARKV_OK) return st;
  if ((st = check_slots(v, dst, n, true)) != STARKV_OK) return st;
  if (n == 0) return STARKV_OK;
  SeqList s;
  s.n = n;
  int32_t from[kMaxSeqs];
  std::copy(src, src + n, from);
  std::sort(from, from + n);
  for (int i = 0; i < n; ++i) {
    if (std::binary_search(from, from + n, dst[i])) return STARKV_E_PARAM;
    s.slot[i] = dst[i];
    s.num[i] = src[i];
  }
  return hip_status(launch_pages_fork(v, s, stream));
}

starkv_status starkv_pages_free(const starkv_paged* cache, const int32_t* slots, int32_t n,
                                int32_t keep_first, int32_t keep_last, void* stream) {
  PagedView v;
  starkv_status st = check_paged(cache, &v);
  if (st != STARKV_OK) return st;
  if ((st = check_slots(v, slots, n, true)) != STARKV_OK) return st;
  if (keep_first < 0 || keep_last < 0) return STARKV_E_PARAM;
  if (n == 0) return STARKV_OK;
  SeqList s;
  s.n = n;
  std::copy(slots, slots + n, s.slot);
  std::fill(s.num, s.num + n, 0);
  return hip_status(launch_pages_free(v, s, keep_first, keep_last, stream));
}

starkv_status starkv_pages_compact(const starkv_paged* cache, const int32_t* slots, int32_t n,
                                   const int32_t* span, const int32_t* idx,
                                   int64_t idx_layer_stride, int32_t B, const int32_t* counts,
                                   int32_t tail, int32_t* status, void* ws, size_t ws_bytes,
                                   void* stream) {
  return compact(cache, slots, n, span, idx, idx_layer_stride, B, counts, tail, nullptr, status, ws,
                 ws_bytes, stream);
}

starkv_status starkv_pages_compact_grown(const starkv_paged* cache, const int32_t* slots,
                                         int32_t n, const int32_t* span, const int32_t* idx,
                                         int64_t idx_layer_stride, int32_t B,
                                         const int32_t* counts, int32_t tail,
                                         const int32_t* grown, int32_t* status, void* ws,
                                         size_t ws_bytes, void* stream) {
  if (n > 0 && !grown) return STARKV_E_NULL;
  return compact(cache, slots, n, span, idx, idx_layer_stride, B, counts, tail, grown, status, ws,
                 ws_bytes, stream);
}

size_t starkv_attend_workspace_bytes(const starkv_paged* cache, const int32_t* rows, int32_t n,
                                     int32_t max_len) {
  PagedView v;
  AttendShape s;
  if (check_paged(cache, &v) != STARKV_OK ||
      attend_shape(v, rows, n, max_len, 0, 0, &s, nullptr) != STARKV_OK)
    return 0;
  return s.ws_bytes;
}

starkv_status starkv_attend_tree(const starkv_paged* cache, const int32_t* slots, int32_t n,
                                 const int32_t* rows, const void* q, const uint64_t* mask,
                                 int32_t words, int32_t max_len, void* out, float* lse, void* ws,
                                 size_t ws_bytes, void* stream) {
  if (words < 1 || words > STARKV_MAX_DRAFT_WORDS) return STARKV_E_PARAM;
  AttendCall c;
  c.q = q;
  c.out = out;
  c.lse = lse;
  c.ws = ws;
  c.mask = mask;
  c.words = words;
  c.window = c.sinks = 0;
  return attend(cache, slots, n, rows, max_len, &c, ws_bytes, stream);
}

starkv_status starkv_attend_window(const starkv_paged* cache, const int32_t* slots, int32_t n,
                                   const int32_t* rows, const void* q, int32_t window,
                                   int32_t sinks, int32_t max_len, void* out, float* lse,
                                   void* ws, size_t ws_bytes, void* stream) {
  if (window < 0 || window > kMaxTokens || sinks < 0 || sinks > kMaxTokens)
    return STARKV_E_PARAM;
  AttendCall c;
  c.q = q;
  c.out = out;
  c.lse = lse;
  c.ws = ws;
  c.mask = nullptr;
  c.words = 0;
  c.window = window ? window : (int32_t)kMaxTokens;   // no window: longer than any sequence
  c.sinks = window ? sinks : 0;
  return attend(cache, slots, n, rows, max_len, &c, ws_bytes, stream);
}

}  // extern "C"
