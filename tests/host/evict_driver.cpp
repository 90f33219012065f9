// The host units of the paged cache and of eviction with stub launches, built with
// the address and undefined-behaviour sanitizers and with locals that start as a
// pattern where the compiler can: the division of calls that add weights over many
// shapes, the layout of an eviction's workspace, and what the launches receive.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <vector>

#include "evict.h"

using namespace starkv;

#define CHECK(x)                                  \
  do {                                            \
    if (!(x)) {                                   \
      std::printf("line %d: %s\n", __LINE__, #x); \
      std::exit(1);                               \
    }                                             \
  } while (0)

static int launches = 0;
static MassCall mass;
static EvictCall evict;
static SeqList forked, compacted;
static RowList read_rows;
static PagesWs compact_ws;
static int compact_b, compact_tail;
static const int32_t* compact_counts;

namespace starkv {
int launch_pages_init(const PagedView&, void*) { return 0; }
int launch_pages_grow(const PagedView&, const SeqList&, const PagesWs&, int32_t*, void*, void*) { return 0; }
int launch_pages_write(const PagedView&, const RowList&, const void*, const void*, const starkv_kv_layout&,
                       void*) {
  return 0;
}
int launch_pages_read(const PagedView&, const RowList& r, void*, void*, const starkv_kv_layout&, void*) {
  read_rows = r;
  return ++launches, 0;
}
int launch_pages_fork(const PagedView&, const SeqList&, void*) { return 0; }
int launch_pages_free(const PagedView&, const SeqList&, int, int, void*) { return 0; }
int launch_pages_compact(const PagedView&, const SeqList& s, bool whole, const int32_t*, int64_t ls, int B,
                         const int32_t* counts, int tail, const PagesWs& w, int32_t*, void*, void*) {
  CHECK(whole && ls == (int64_t)s.n * B);
  compacted = s;
  compact_b = B;
  compact_tail = tail;
  compact_counts = counts;
  compact_ws = w;
  return ++launches, 0;
}
int launch_attend(const PagedView&, const AttendCall&, void*) { return 0; }
int launch_mass_add(const PagedView&, const MassCall& c, void*) {
  mass = c;
  return ++launches, 0;
}
int launch_mass_fork(const PagedView&, const SeqList& s, float*, void*) {
  forked = s;
  return ++launches, 0;
}
int launch_evict_select(const PagedView&, const EvictCall& c, void*) {
  evict = c;
  return ++launches, 0;
}
}  // namespace starkv

int main() {
  std::mt19937 rng(11);
  const auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
  alignas(16) static char mem[64];
  float* f32 = reinterpret_cast<float*>(mem);
  long checked = 0, split = 0;
  for (int it = 0; it < 20000; ++it) {
    starkv_paged c;
    std::memset(&c, 0, sizeof c);
    c.G = 1 << pick(0, 6);
    c.H = c.G * pick(1, 20);
    if (c.H > 4096) continue;
    c.n_layers = pick(0, 3) ? 1 : pick(0, 1) ? pick(1, 60) : pick(1, 4096);
    c.d = pick(0, 1) ? 64 : 128;
    c.dtype = pick(0, 2) == 0 ? STARKV_FP4 : pick(0, 2) ? STARKV_BF16 : STARKV_F32;
    c.page_tokens = 16 << pick(0, 6);
    c.n_pages = pick(1, 5000);
    c.n_slots = pick(300, 600);
    c.max_pages = pick(1, 4000);
    if ((int64_t)c.max_pages * c.page_tokens > kMaxTokens) continue;
    c.token_stride = c.dtype == STARKV_FP4 ? c.d / 2 : c.d;
    c.group_stride = 17 * c.d * c.page_tokens;
    c.page_stride = c.group_stride * c.G;
    c.layer_stride = c.page_stride * c.n_pages;
    c.k = c.v = mem;
    c.table = c.len = c.refs = reinterpret_cast<int32_t*>(mem);
    PagedView v;
    CHECK(check_paged(&c, &v) == STARKV_OK);
    CHECK(v.fp4 == (c.dtype == STARKV_FP4) && v.esz == (c.dtype == STARKV_F32 ? 4 : 2));
    CHECK(v.row == (v.fp4 ? c.d / 2 : c.d * v.esz) && v.ts == v.row && v.row % 16 == 0);
    const int cap = c.max_pages * c.page_tokens;
    const int n = pick(0, 2) ? pick(0, 12) : pick(0, kMaxSeqs);
    const int most = pick(0, 2) ? pick(1, 64) : pick(1, 9000);
    std::vector<int32_t> rows(n), slots(n);
    int64_t tot = 0;
    for (int b = 0; b < n; ++b) {
      rows[b] = std::min(pick(0, most), cap);
      slots[b] = b;
      tot += rows[b];
    }
    const int max_len = pick(0, 3) ? pick(1, 50000) : pick(1, (int)kMaxTokens);
    const size_t ws = starkv_mass_workspace_bytes(&c, rows.data(), n, max_len);
    const int window = pick(0, 1) ? pick(1, 9000) : 0, sinks = pick(0, 300);
    int before = launches;
    CHECK(starkv_mass_add(&c, slots.data(), n, rows.data(), mem, f32, window, sinks, max_len, f32, f32,
                          ws ? mem : nullptr, ws, nullptr) == STARKV_OK);
    CHECK(launches == before + (tot > 0));
    if (tot > 0) {
      ++checked;
      const MassShape& s = mass.s;
      const int hpg = c.H / c.G;
      int64_t R = 0, at = 0;
      for (int b = 0; b < n; ++b) {
        R = std::max<int64_t>(R, (int64_t)rows[b] * hpg);
        CHECK(mass.r.row0[b] == at && mass.r.slot[b] == slots[b]);
        at += rows[b];
      }
      CHECK(mass.r.n == n && mass.r.row0[n] == tot && s.n_rows == tot);
      const int64_t pairs = (int64_t)c.n_layers * n, len = std::min(max_len, cap);
      CHECK(s.many == (R > 32));
      CHECK((int64_t)s.tiles * s.tile >= len && (int64_t)(s.tiles - 1) * s.tile < len);
      CHECK(s.blocks >= 1 && s.n_split >= 1);
      if (s.many) {
        CHECK(s.tile == 256 && s.blocks <= s.tiles && pairs * s.blocks * s.n_split <= 1 << 22);
        CHECK(s.n_split <= 64 && (s.n_split < 8 || s.n_split % 8 == 0));
        CHECK(s.n_split == 1 || pairs * s.tiles * s.n_split <= 4096);
        CHECK(s.ws_bytes == (s.n_split > 1 ? (size_t)pairs * s.n_split * s.tiles * 256 * 4 : 0));
        split += s.n_split > 1;
      } else {
        const int part = v.fp4 ? 64 : v.row == 128 ? 32 : 16;
        CHECK((s.tile == part || s.tile == (c.G < 4 ? 256 : 4 * part)) && s.n_split == 1 && s.ws_bytes == 0);
        CHECK((int64_t)s.row_blocks * 16 >= R && s.row_blocks <= 2);
        CHECK(2 * c.G * s.tile * 4 <= 64 * 1024);       // LDS
      }
      CHECK(s.ws_bytes == ws && (!ws || mass.part == f32));
      CHECK(mass.window == (window ? window : (int)kMaxTokens) && mass.sinks == (window ? sinks : 0));
      if (ws)
        CHECK(starkv_mass_add(&c, slots.data(), n, rows.data(), mem, f32, window, sinks, max_len, f32, f32, mem,
                              ws - 1, nullptr) == STARKV_E_WORKSPACE);
    }
    // an eviction's workspace: the compaction's, then counts, marks and masses
    const int keep = pick(0, 5000), recent = pick(0, 300), want = keep + sinks;
    const size_t need = starkv_evict_workspace_bytes(&c, n, keep, sinks, recent);
    const EvictWs w = evict_ws(v, n, want, recent);
    CHECK(need == w.bytes && w.pages.bytes == starkv_pages_workspace_bytes(&c, n, want + recent));
    CHECK(w.counts >= w.pages.bytes && w.stay >= w.counts + (size_t)n * 4 && w.kept >= w.stay + (size_t)n * 4);
    CHECK(w.bytes >= w.kept + (size_t)c.n_layers * n * (want + recent) * 4 && w.kept % 16 == 0);
    before = launches;
    int32_t* i32 = c.len;
    CHECK(starkv_pages_evict(&c, slots.data(), n, f32, keep, sinks, recent, i32, i32, mem, need, nullptr) ==
          STARKV_OK);
    CHECK(launches == before + (n ? 2 : 0));
    if (n) {
      CHECK(evict.keep == keep && evict.sinks == sinks && evict.recent == recent && evict.s.n == n);
      CHECK(compacted.n == n && compacted.grown == evict.stay && compact_counts == evict.counts);
      CHECK(compact_b == want && compact_tail == recent && compact_ws.bytes == w.pages.bytes);
      CHECK(compacted.kept.from == evict.kept && compacted.kept.to == f32);
      CHECK((char*)evict.counts == mem + w.counts && (char*)evict.stay == mem + w.stay &&
            (char*)evict.kept == mem + w.kept);
      for (int b = 0; b < n; ++b) CHECK(evict.s.slot[b] == b && evict.s.num[b] == 0 && compacted.slot[b] == b);
    }
    starkv_kv_layout lay{0, 128, 128};
    before = launches;
    CHECK(starkv_pages_read(&c, slots.data(), n, rows.data(), mem, mem, &lay, nullptr) == STARKV_OK);
    CHECK(launches == before + (tot > 0));
    if (tot > 0) CHECK(read_rows.n == n && read_rows.row0[n] == tot && read_rows.grown == nullptr);
    if (n >= 2) {
      CHECK(starkv_mass_fork(&c, slots.data(), slots.data() + 1, 1, f32, nullptr) == STARKV_OK);
      CHECK(forked.n == 1 && forked.slot[0] == 1 && forked.num[0] == 0);
    }
  }
  CHECK(checked > 5000 && split > 300);
  std::printf("%ld calls checked\n", checked);
  return 0;
}
