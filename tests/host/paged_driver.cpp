// The host unit of the paged cache with stub launches, built with the address
// and undefined-behaviour sanitizers: the division of attention calls into
// blocks over many shapes, and what the launch functions receive.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "paged.h"

using namespace starkv;

static int launches = 0;
static AttendCall last;
static PagesWs last_ws;

namespace starkv {
int launch_pages_init(const PagedView&, void*) { return ++launches, 0; }
int launch_pages_grow(const PagedView&, const SeqList&, const PagesWs& w, int32_t*, void*, void*) {
  last_ws = w;
  return ++launches, 0;
}
int launch_pages_write(const PagedView&, const RowList&, const void*, const void*,
                       const starkv_kv_layout&, void*) {
  return ++launches, 0;
}
int launch_pages_fork(const PagedView&, const SeqList&, void*) { return ++launches, 0; }
int launch_pages_free(const PagedView&, const SeqList&, int, int, void*) { return ++launches, 0; }
int launch_pages_compact(const PagedView&, const SeqList&, bool, const int32_t*, int64_t, int,
                         const int32_t*, int, const PagesWs& w, int32_t*, void*, void*) {
  last_ws = w;
  return ++launches, 0;
}
int launch_attend(const PagedView&, const AttendCall& c, void*) {
  last = c;
  return ++launches, 0;
}
}  // namespace starkv

#define CHECK(x)                                                   \
  do {                                                             \
    if (!(x)) {                                                    \
      std::printf("line %d: %s\n", __LINE__, #x);                  \
      std::exit(1);                                                \
    }                                                              \
  } while (0)

int main() {
  std::mt19937 rng(7);
  const auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
  alignas(16) static char mem[64];
  long checked = 0;
  for (int it = 0; it < 20000; ++it) {
    starkv_paged c{};
    c.G = 1 << pick(0, 4);
    c.H = c.G * pick(1, 20);
    c.n_layers = pick(0, 3) ? 1 : pick(1, 60);
    c.d = pick(0, 1) ? 64 : 128;
    c.dtype = pick(0, 3) ? STARKV_BF16 : STARKV_F32;
    c.page_tokens = 16 << pick(0, 6);
    c.n_pages = pick(1, 5000);
    c.n_slots = pick(1, 300);
    c.max_pages = pick(1, 4000);
    if ((int64_t)c.max_pages * c.page_tokens > kMaxTokens) continue;
    c.token_stride = c.d;
    c.group_stride = c.d * c.page_tokens;
    c.page_stride = c.group_stride * c.G;
    c.layer_stride = c.page_stride * c.n_pages;
    c.k = c.v = mem;
    c.table = c.len = c.refs = reinterpret_cast<int32_t*>(mem);
    const int cap = c.max_pages * c.page_tokens;
    const int n = pick(0, 2) ? pick(0, 12) : pick(0, kMaxSeqs);
    const int most = pick(0, 2) ? pick(1, 64) : pick(1, 9000);
    std::vector<int32_t> rows(n), slots(n);
    for (int b = 0; b < n; ++b) {
      rows[b] = std::min(pick(0, most), cap);
      slots[b] = pick(0, c.n_slots - 1);
    }
    const int max_len = pick(0, 3) ? pick(1, 50000) : pick(1, (int)kMaxTokens);
    const size_t ws = starkv_attend_workspace_bytes(&c, rows.data(), n, max_len);
    const int window = pick(0, 1) ? pick(1, 9000) : 0, sinks = pick(0, 300);
    const int before = launches;
    const starkv_status st = starkv_attend_window(&c, slots.data(), n, rows.data(), mem, window, sinks,
                                                  max_len, mem, nullptr, ws ? mem : nullptr, ws, nullptr);
    if (st != STARKV_OK) {
      CHECK(st == STARKV_E_PARAM && launches == before);   // too many blocks for one launch
      continue;
    }
    if (launches == before) {
      for (int r : rows) CHECK(r == 0);
      continue;
    }
    ++checked;
    const AttendShape& s = last.s;
    const int hpg = c.H / c.G, step = s.many ? 64 : 32;
    CHECK(s.row_tile % 16 == 0 && s.n_split >= 1 && s.chunk >= 1 && s.chunk % step == 0);
    // every row has a tile of its sequence, and no tile is of two sequences
    int64_t tiles = 0, tot = 0;
    for (int b = 0; b < n; ++b) {
      CHECK(last.tile0[b] == tiles && last.r.row0[b] == tot && last.r.slot[b] == slots[b]);
      tiles += ((int64_t)rows[b] * hpg + s.row_tile - 1) / s.row_tile;
      tot += rows[b];
    }
    CHECK(last.tile0[n] == tiles && last.r.row0[n] == tot && s.n_tiles == tiles && s.n_rows == tot);
    CHECK(s.units == tiles * c.n_layers * c.G);
    // the splits cover the steps, and their records fit the workspace
    CHECK((int64_t)s.n_split * s.chunk >= (int64_t)s.steps * step);
    if (s.n_split > 1) {
      const size_t rec = (size_t)s.units * s.n_split * s.row_tile;
      CHECK(rec * c.d * 4 <= s.stat_off && s.stat_off + rec * 8 <= s.steps_off);
      CHECK(s.steps_off + sizeof(int) <= s.ws_bytes && s.ws_bytes == ws);
    }
    CHECK(!s.balance || s.n_split > 1);
    // the pages' workspace: the records of n sequences behind the free pages
    const size_t need = starkv_pages_workspace_bytes(&c, n, most);
    const PagesWs w = pages_ws(PagedView{nullptr, nullptr, nullptr, nullptr, nullptr, 0, 0, 0, 0, 0, 0, 0,
                                         0, 0, c.page_tokens, 0, c.n_pages, c.n_slots, c.max_pages, cap},
                               n, most);
    CHECK(need == w.bytes && w.info >= (size_t)w.most_fresh * 4 && w.old >= w.info + (size_t)n * 16);
    CHECK(w.bytes >= w.old + (size_t)n * c.max_pages * 4);
  }
  CHECK(checked > 5000);
  std::printf("%ld calls checked\n", checked);
  return 0;
}
