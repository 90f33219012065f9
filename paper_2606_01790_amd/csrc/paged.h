// Internal declarations of the paged cache, shared by its host entry points
// and kernels.  Free of HIP types, so the host unit compiles with a plain
// C++ compiler.
#pragma once

#include <cstddef>
#include <cstdint>

#include "starkv_paged.h"

namespace starkv {

constexpr int kMaxSeqs = STARKV_MAX_SEQS;
constexpr int64_t kMaxTokens = 1 << 26;

// A validated cache, with what the kernels derive from it.
struct PagedView {
  char* k;
  char* v;
  int32_t* table;
  int32_t* len;
  int32_t* refs;
  int64_t ls, ps, gs, ts;   // byte strides
  int n_layers, H, G, d, esz;
  int P, psh;               // page tokens and their logarithm
  int n_pages, n_slots, max_pages;
  int cap;                  // tokens of a table row
  int row = 0;              // bytes of a K (or V) row in its page
  // 4 bits: esz is that of q, out and the rows given, bf16.  A block's P rows
  // are followed, from byte P*row, by their scales, d/32 bytes each
  bool fp4 = false;
};

// The masses that stay in an eviction, [n_layers][n][B + tail], and the cache's.
struct KeptMasses {
  const float* from = nullptr;
  float* to = nullptr;
};

// The sequences of a call, passed to the kernels by value.
struct SeqList {
  int32_t n;
  int32_t slot[kMaxSeqs];
  int32_t num[kMaxSeqs];    // per sequence: tokens added, a span, or the slot forked from
  const int32_t* grown = nullptr;   // compact, device: the status of the grow before it, if any
  KeptMasses kept;                  // compact: that move too, if any
};

// Rows of the sequences of a call: sequence b has rows [row0[b], row0[b+1]).
struct RowList {
  int32_t n;
  int32_t slot[kMaxSeqs];
  int32_t row0[kMaxSeqs + 1];
  const int32_t* grown = nullptr;   // device: the status of the grow that made the rows, if any
};

starkv_status check_paged(const starkv_paged* c, PagedView* v);
// rows[b] >= 0 query (or written, or read) tokens per sequence, into a list.
starkv_status take_rows(const PagedView& v, const int32_t* slots, const int32_t* rows, int n,
                        RowList* r);
// The strides and addresses of new rows (bytes of an element: v.esz).
starkv_status check_new_rows(const PagedView& v, const void* k, const void* vv,
                             const starkv_kv_layout& lay);
// n slots of the cache, each at most once if `once`.
starkv_status check_slots(const PagedView& v, const int32_t* slots, int32_t n, bool once);

// Workspace of grow and compact, byte offsets: the free pages found, the
// pages to copy (grow) or the sequences' extents (compact), and the table
// rows as they were (compact).
struct PagesWs {
  size_t fresh, info, old, bytes;
  int64_t most_fresh;
};
PagesWs pages_ws(const PagedView& v, int n, int64_t most);

int launch_pages_init(const PagedView& v, void* stream);
int launch_pages_grow(const PagedView& v, const SeqList& s, const PagesWs& w, int32_t* status,
                      void* ws, void* stream);
int launch_pages_write(const PagedView& v, const RowList& r, const void* k, const void* vv,
                       const starkv_kv_layout& lay, void* stream);
int launch_pages_read(const PagedView& v, const RowList& r, void* k, void* vv,
                      const starkv_kv_layout& lay, void* stream);
int launch_pages_fork(const PagedView& v, const SeqList& s, void* stream);
int launch_pages_free(const PagedView& v, const SeqList& s, int keep_first, int keep_last,
                      void* stream);
int launch_pages_compact(const PagedView& v, const SeqList& s, bool whole, const int32_t* idx,
                         int64_t idx_ls, int B, const int32_t* counts, int tail,
                         const PagesWs& w, int32_t* status, void* ws, void* stream);

// How an attention call is divided.  The query rows of a (sequence, group)
// are its tokens' heads of the group, r = i*(H/G) + head; a block takes a
// tile of row_tile of them and one split of the cached tokens.
struct AttendShape {
  bool many;        // the kernel for many rows
  int n_rows;       // query tokens of the call
  int row_tile;     // rows of a block
  int n_tiles;      // row tiles of one (layer, group), over all sequences
  int seq_tiles;    // the most of one sequence
  int n_split;      // splits of the tokens
  int chunk;        // tokens that a split takes at least
  int steps;        // the most steps that a row tile walks
  bool balance;     // the device divides the steps (several sequences)
  int64_t units;    // n_layers * G * n_tiles
  size_t stat_off;  // bytes: the partial statistics behind the partial outputs
  size_t steps_off; // the device's steps of a split
  size_t ws_bytes;
};

struct AttendCall {
  RowList r;
  int32_t tile0[kMaxSeqs + 1];   // first row tile of each sequence
  AttendShape s;
  const void* q;
  void* out;
  float* lse;
  void* ws;
  const uint64_t* mask;   // tree, or NULL
  int words;
  int window, sinks;      // no mask: window > 0
};

// The shape of a call over `rows` (window 0: none, or a tree), and the first
// tile of each sequence.
starkv_status attend_shape(const PagedView& v, const int32_t* rows, int n, int32_t max_len,
                           int32_t window, int32_t sinks, AttendShape* s, int32_t* tile0);
int launch_attend(const PagedView& v, const AttendCall& c, void* stream);

}  // namespace starkv
