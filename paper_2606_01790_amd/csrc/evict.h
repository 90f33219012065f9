// Internal declarations of eviction by accumulated attention weight, shared by
// its host entry points and kernels.  Free of HIP types.
#pragma once

#include "paged.h"

namespace starkv {

// Tokens of a part of a tile, which a wave of the kernel for few rows works on at a time,
// by the bytes of a row: 4 KB of K, but 8 of float32 rows of 128 and 2 of 4-bit rows of 64
// (4 bits with 32 tokens: 28 layers of 40,941 99 us and not 79); and the most tokens of a
// tile, in either kernel.  A tile of few rows is one or four parts, or kMassTile, and the
// launch refuses others.
constexpr int mass_part(bool fp4, int row) { return fp4 ? 64 : row == 128 ? 32 : 16; }
constexpr int kMassTile = 256;

// How a call that adds weights is divided.  Few rows: `blocks` blocks take the tiles
// of all sequences and layers in turn.  Many rows: `blocks` of each (layer,
// sequence) take its tiles in turn, n_split of them share a tile's products, and
// their sums are joined afterwards.
struct MassShape {
  bool many;       // the kernel for many rows
  int n_rows;      // query tokens of the call
  int tile;        // tokens of a tile
  int tiles;       // tiles of a sequence, by the bound on the lengths
  int row_blocks;  // few rows: 16-row blocks of a group, at most
  int blocks;
  int n_split;
  size_t ws_bytes; // the splits' sums, float [n_layers][n][n_split][tiles*tile]
};

struct MassCall {
  RowList r;
  MassShape s;
  const void* q;
  const float* lse;
  const float* mass;
  float* out;
  float* part;
  int window, sinks;   // no window: longer than any sequence
};

starkv_status mass_shape(const PagedView& v, const int32_t* rows, int n, int32_t max_len,
                         MassShape* s);
int launch_mass_add(const PagedView& v, const MassCall& c, void* stream);
int launch_mass_fork(const PagedView& v, const SeqList& s, float* mass, void* stream);

// Workspace of an eviction, byte offsets behind the compaction's.
struct EvictWs {
  PagesWs pages;
  size_t counts, stay;  // int32 [n]: kept tokens but for the recent ones; STARKV_SEQ_SHORT or OK
  size_t kept;          // float [n_layers][n][sinks + keep + recent]: masses that stay
  size_t bytes;
};
EvictWs evict_ws(const PagedView& v, int n, int64_t want, int recent);

struct EvictCall {
  SeqList s;
  float* mass;
  int keep, sinks, recent;
  int32_t* idx;
  int32_t* counts;
  int32_t* stay;
  float* kept;
};
int launch_evict_select(const PagedView& v, const EvictCall& c, void* stream);

}  // namespace starkv
