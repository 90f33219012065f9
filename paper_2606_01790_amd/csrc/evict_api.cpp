// Host entry points that read rows back out of a paged cache, add up attention
// weights and evict by them: argument validation and the division of the work,
// then the kernels' launch functions.  Nothing here allocates memory or
// synchronises a stream.
#include <algorithm>

#include "evict.h"

namespace starkv {

namespace {

bool at(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
size_t up256(size_t x) { return (x + 255) / 256 * 256; }
starkv_status hip_status(int err) { return err ? STARKV_E_HIP : STARKV_OK; }

}  // namespace

starkv_status mass_shape(const PagedView& v, const int32_t* rows, int n, int32_t max_len,
                         MassShape* s) {
  if (n < 0 || n > kMaxSeqs) return STARKV_E_PARAM;
  if (n > 0 && !rows) return STARKV_E_NULL;
  if (max_len < 1 || max_len > kMaxTokens) return STARKV_E_PARAM;
  const int64_t hpg = v.H / v.G;
  int64_t tot = 0, most = 0;
  for (int b = 0; b < n; ++b) {
    if (rows[b] < 0 || rows[b] > v.cap || rows[b] * hpg > 1 << 30) return STARKV_E_PARAM;
    tot += rows[b];
    most = std::max<int64_t>(most, rows[b]);
  }
  if (tot > kMaxTokens) return STARKV_E_PARAM;
  s->n_rows = (int)tot;
  const int64_t R = most * hpg;
  // up to 32 rows of a group stay in a wave's registers while it reads K once; of more
  // the tokens do (56 rows over 13,711 tokens in 28 layers: 100 us by tokens, and 183 with
  // four blocks of 16 rows in registers)
  s->many = R > 32;
  s->row_blocks = (int)std::max<int64_t>(1, (R + 15) / 16);
  const int64_t len = std::min<int64_t>(max_len, v.cap);
  const int64_t pairs = std::max<int64_t>(1, (int64_t)v.n_layers * n);
  s->n_split = 1;
  s->ws_bytes = 0;
  if (!s->many) {
    // tiles of four parts of every group (of 256 tokens where there are fewer than four
    // groups, so that a wave has more than one: three rows of one group, 8 sequences of
    // 13,711 tokens in 4 layers, 43 us with four parts and 30 so), or of one where those
    // are too few for the card, or the groups' sums would fill LDS
    const int part = mass_part(v.fp4, v.row);
    const int most = v.G < 4 ? kMassTile : v.fp4 && v.G > 32 ? part : 4 * part;
    s->tile = pairs * ((len + most - 1) / most) >= 512 ? most : part;
    s->tiles = (int)((len + s->tile - 1) / s->tile);
    s->blocks = (int)std::min<int64_t>(pairs * s->tiles, 1 << 20);   // (the launch takes what the card holds)
    return STARKV_OK;
  }
  s->tile = kMassTile;
  s->tiles = (int)((len + s->tile - 1) / s->tile);
  s->blocks = (int)std::max<int64_t>(1, std::min<int64_t>(s->tiles, (1 << 22) / pairs));
  // splits of a tile's (group, 32 rows) products until there are 2,048 blocks, of at
  // least four products (100 rows over 100 tokens: 33 us with at least 16, and 20 so),
  // or 4,096 of at least 16, whose last round is shorter (40 rows of 4 sequences of 1,000
  // to 4,000 tokens in 28 layers 207 and 188 us; but 8 rows over 13,711, of which it
  // would leave four products, 100 and 109); a multiple of the 8 XCDs, each of which then
  // reads the same eighth of Q for every tile (2,755 rows over 13,711 tokens: 32, 40 or
  // 48 splits 287 us, 37 298, 16 290, 9 310)
  const int64_t products = v.G * ((R + 31) / 32), units = pairs * s->tiles;
  s->n_split = (int)std::clamp<int64_t>(
      std::max(std::min(2048 / units, products / 4), std::min(4096 / units, products / 16)), 1, 64);
  if (s->n_split > 8) s->n_split &= ~7;
  if (s->n_split > 1)
    s->ws_bytes = (size_t)units * s->n_split * s->tile * sizeof(float);
  return STARKV_OK;
}

EvictWs evict_ws(const PagedView& v, int n, int64_t want, int recent) {
  EvictWs w;
  w.pages = pages_ws(v, n, want + recent);
  w.counts = w.pages.bytes;
  w.stay = w.counts + up256((size_t)n * 4);
  w.kept = w.stay + up256((size_t)n * 4);
  w.bytes = w.kept + up256((size_t)v.n_layers * n * (want + recent) * 4);
  return w;
}

namespace {

starkv_status add(const starkv_paged* cache, const int32_t* slots, int32_t n,
                  const int32_t* rows, const void* q, const float* lse, int32_t window,
                  int32_t sinks, int32_t max_len, const float* mass, float* out,
                  const int32_t* grown, void* ws, size_t ws_bytes, void* stream) {
  PagedView v;
  starkv_status st = check_paged(cache, &v);
  if (st != STARKV_OK) return st;
  if ((st = check_slots(v, slots, n, true)) != STARKV_OK) return st;
  if (window < 0 || window > kMaxTokens || sinks < 0 || sinks > kMaxTokens) return STARKV_E_PARAM;
  MassCall c;
  if ((st = mass_shape(v, rows, n, max_len, &c.s)) != STARKV_OK) return st;
  if ((st = take_rows(v, slots, rows, n, &c.r)) != STARKV_OK) return st;
  c.r.grown = grown;
  if (c.s.n_rows == 0) return STARKV_OK;
  if (!q || !lse || !mass || !out) return STARKV_E_NULL;
  if (!at(q, 16) || !at(lse, 4) || !at(mass, 4) || !at(out, 4) || !at(grown, 4))
    return STARKV_E_ALIGN;
  if (c.s.ws_bytes) {
    if (!ws || ws_bytes < c.s.ws_bytes) return STARKV_E_WORKSPACE;
    if (!at(ws, 16)) return STARKV_E_ALIGN;
  }
  c.q = q;
  c.lse = lse;
  c.mass = mass;
  c.out = out;
  c.part = static_cast<float*>(ws);
  c.window = window ? window : (int32_t)kMaxTokens;
  c.sinks = window ? sinks : 0;
  return hip_status(launch_mass_add(v, c, stream));
}

}  // namespace

}  // namespace starkv

using namespace starkv;

extern "C" {

starkv_status starkv_pages_read(const starkv_paged* cache, const int32_t* slots, int32_t n,
                                const int32_t* rows, void* k, void* v,
                                const starkv_kv_layout* lay, void* stream) {
  PagedView view;
  starkv_status st = check_paged(cache, &view);
  if (st != STARKV_OK) return st;
  if ((st = check_slots(view, slots, n, false)) != STARKV_OK) return st;
  if (n == 0) return STARKV_OK;
  if (!rows || !lay) return STARKV_E_NULL;
  RowList r;
  if ((st = take_rows(view, slots, rows, n, &r)) != STARKV_OK) return st;
  if (lay->layer_stride < 0 || lay->group_stride < 0 || lay->token_stride < 0)
    return STARKV_E_SHAPE;
  if (r.row0[n] == 0) return STARKV_OK;
  if ((st = check_new_rows(view, k, v, *lay)) != STARKV_OK) return st;
  return hip_status(launch_pages_read(view, r, k, v, *lay, stream));
}

size_t starkv_mass_workspace_bytes(const starkv_paged* cache, const int32_t* rows, int32_t n,
                                   int32_t max_len) {
  PagedView v;
  MassShape s;
  if (check_paged(cache, &v) != STARKV_OK || mass_shape(v, rows, n, max_len, &s) != STARKV_OK)
    return 0;
  return s.ws_bytes;
}

starkv_status starkv_mass_add(const starkv_paged* cache, const int32_t* slots, int32_t n,
                              const int32_t* rows, const void* q, const float* lse,
                              int32_t window, int32_t sinks, int32_t max_len, const float* mass,
                              float* out, void* ws, size_t ws_bytes, void* stream) {
  return add(cache, slots, n, rows, q, lse, window, sinks, max_len, mass, out, nullptr, ws,
             ws_bytes, stream);
}

starkv_status starkv_mass_add_grown(const starkv_paged* cache, const int32_t* slots, int32_t n,
                                    const int32_t* rows, const void* q, const float* lse,
                                    int32_t window, int32_t sinks, int32_t max_len,
                                    const float* mass, float* out, const int32_t* grown, void* ws,
                                    size_t ws_bytes, void* stream) {
  if (n > 0 && !grown) return STARKV_E_NULL;
  return add(cache, slots, n, rows, q, lse, window, sinks, max_len, mass, out, grown, ws,
             ws_bytes, stream);
}

starkv_status starkv_mass_fork(const starkv_paged* cache, const int32_t* src, const int32_t* dst,
                               int32_t n, float* mass, void* stream) {
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
  if (!mass) return STARKV_E_NULL;
  if (!at(mass, 4)) return STARKV_E_ALIGN;
  return hip_status(launch_mass_fork(v, s, mass, stream));
}

size_t starkv_evict_workspace_bytes(const starkv_paged* cache, int32_t n, int32_t keep,
                                    int32_t sinks, int32_t recent) {
  PagedView v;
  if (check_paged(cache, &v) != STARKV_OK || n < 0 || n > kMaxSeqs || keep < 0 || sinks < 0 ||
      recent < 0 || (int64_t)keep + sinks + recent > kMaxTokens)
    return 0;
  return evict_ws(v, n, (int64_t)sinks + keep, recent).bytes;
}

starkv_status starkv_pages_evict(const starkv_paged* cache, const int32_t* slots, int32_t n,
                                 float* mass, int32_t keep, int32_t sinks, int32_t recent,
                                 int32_t* idx, int32_t* status, void* ws, size_t ws_bytes,
                                 void* stream) {
  PagedView v;
  starkv_status st = check_paged(cache, &v);
  if (st != STARKV_OK) return st;
  if ((st = check_slots(v, slots, n, true)) != STARKV_OK) return st;
  if (keep < 0 || sinks < 0 || recent < 0 || (int64_t)keep + sinks + recent > kMaxTokens)
    return STARKV_E_BUDGET;
  if (n == 0) return STARKV_OK;
  const int want = sinks + keep;
  if (!mass || !status || (want > 0 && !idx)) return STARKV_E_NULL;
  if (!at(mass, 4) || !at(idx, 4) || !at(status, 4)) return STARKV_E_ALIGN;
  const EvictWs w = evict_ws(v, n, want, recent);
  if (!ws || ws_bytes < w.bytes) return STARKV_E_WORKSPACE;
  if (!at(ws, 16)) return STARKV_E_ALIGN;
  char* p = static_cast<char*>(ws);
  EvictCall c;
  c.s.n = n;
  std::copy(slots, slots + n, c.s.slot);
  std::fill(c.s.num, c.s.num + n, 0);
  c.mass = mass;
  c.keep = keep;
  c.sinks = sinks;
  c.recent = recent;
  c.idx = idx;
  c.counts = reinterpret_cast<int32_t*>(p + w.counts);
  c.stay = reinterpret_cast<int32_t*>(p + w.stay);
  c.kept = reinterpret_cast<float*>(p + w.kept);
  c.s.grown = c.stay;
  c.s.kept = KeptMasses{c.kept, mass};
  int err = launch_evict_select(v, c, stream);
  if (!err)
    err = launch_pages_compact(v, c.s, true, idx, (int64_t)n * want, want, c.counts, recent,
                               w.pages, status, ws, stream);
  return hip_status(err);
}

}  // extern "C"
