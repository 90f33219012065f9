// The host unit of the paged cache with stub launches that read what the kernels' lists
// are made of, built so that every local that nobody has set holds a pattern:
// each call hands over defined values only.
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "paged.h"

using namespace starkv;

#define CHECK(x)                                  \
  do {                                            \
    if (!(x)) {                                   \
      std::printf("line %d: %s\n", __LINE__, #x); \
      std::exit(1);                               \
    }                                             \
  } while (0)

static int launches = 0;
static const int32_t slots[3] = {4, 0, 2}, other[3] = {1, 1, 3}, tokens[3] = {7, 0, 20};
alignas(16) static char mem[64];

static void check_rows(const RowList& r, bool grown) {
  CHECK(r.n == 3 && r.row0[0] == 0);
  for (int i = 0; i < 3; ++i) CHECK(r.slot[i] == slots[i] && r.row0[i + 1] - r.row0[i] == tokens[i]);
  CHECK(r.grown == (grown ? reinterpret_cast<int32_t*>(mem) : nullptr));
  ++launches;
}
static void check_seqs(const SeqList& s, const int32_t* num, bool grown) {
  CHECK(s.n == 3);
  for (int i = 0; i < 3; ++i) CHECK(s.slot[i] == slots[i] && s.num[i] == (num ? num[i] : 0));
  CHECK(s.grown == (grown ? reinterpret_cast<int32_t*>(mem) : nullptr));
  ++launches;
}
static bool behind_a_grow = false;
static const int32_t* spans = nullptr;

namespace starkv {
int launch_pages_init(const PagedView&, void*) { return 0; }
int launch_pages_grow(const PagedView&, const SeqList& s, const PagesWs&, int32_t*, void*, void*) {
  return check_seqs(s, tokens, false), 0;
}
int launch_pages_write(const PagedView&, const RowList& r, const void*, const void*,
                       const starkv_kv_layout&, void*) {
  return check_rows(r, behind_a_grow), 0;
}
int launch_pages_fork(const PagedView&, const SeqList& s, void*) {
  return check_seqs(s, other, false), 0;
}
int launch_pages_free(const PagedView&, const SeqList& s, int, int, void*) {
  return check_seqs(s, nullptr, false), 0;
}
int launch_pages_compact(const PagedView&, const SeqList& s, bool whole, const int32_t*, int64_t, int,
                         const int32_t*, int, const PagesWs&, int32_t*, void*, void*) {
  CHECK(whole == (spans == nullptr));
  return check_seqs(s, spans, behind_a_grow), 0;
}
int launch_attend(const PagedView&, const AttendCall& c, void*) {
  CHECK(c.tile0[0] == 0 && c.tile0[3] == c.s.n_tiles && c.lse == nullptr);
  return check_rows(c.r, false), 0;
}
}  // namespace starkv

int main() {
  starkv_paged c;
  std::memset(&c, 0, sizeof c);
  c.n_layers = c.G = 1;
  c.H = 2;
  c.d = 64;
  c.dtype = STARKV_BF16;
  c.page_tokens = 16;
  c.n_pages = 10;
  c.n_slots = 5;
  c.max_pages = 4;
  c.layer_stride = c.page_stride = c.group_stride = 1024;
  c.token_stride = 64;
  c.k = c.v = mem;
  c.table = c.len = c.refs = reinterpret_cast<int32_t*>(mem);
  int32_t* i32 = c.len;
  starkv_kv_layout lay{1024, 64, 64};
  const size_t big = 1 << 20;
  CHECK(starkv_pages_grow(&c, slots, 3, tokens, i32, mem, big, nullptr) == STARKV_OK);
  CHECK(starkv_pages_write(&c, slots, 3, tokens, mem, mem, &lay, nullptr) == STARKV_OK);
  CHECK(starkv_pages_fork(&c, other, slots, 3, nullptr) == STARKV_OK);
  CHECK(starkv_pages_free(&c, slots, 3, 2, 1, nullptr) == STARKV_OK);
  CHECK(starkv_pages_compact(&c, slots, 3, nullptr, i32, 0, 2, nullptr, 1, i32, mem, big, nullptr) ==
        STARKV_OK);
  CHECK(starkv_attend_window(&c, slots, 3, tokens, mem, 0, 0, 64, mem, nullptr, mem, big, nullptr) ==
        STARKV_OK);
  behind_a_grow = true;
  spans = tokens;
  CHECK(starkv_pages_write_grown(&c, slots, 3, tokens, mem, mem, &lay, i32, nullptr) == STARKV_OK);
  CHECK(starkv_pages_compact_grown(&c, slots, 3, tokens, i32, 0, 2, nullptr, 0, i32, i32, mem, big,
                                   nullptr) == STARKV_OK);
  CHECK(launches == 8);
  std::printf("%d lists checked\n", launches);
  return 0;
}
