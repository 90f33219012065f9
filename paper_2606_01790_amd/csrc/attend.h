// What the attention kernels over a paged cache share: the call's arguments
// on the device, the rows and the cached tokens of a block, and who sees
// whom.
#pragma once

#include "device_common.h"
#include "paged.h"

namespace starkv {

struct AttendArgs {
  const char* q;
  char* out;
  float* lse;
  float* part;            // partial outputs, [units][n_split][row_tile][d]
  float2* stat;           // partial (max, sum), [units][n_split][row_tile]
  const uint64_t* mask;
  int words, window, sinks;
  int n_split, chunk, n_tiles, n_rows;
  int most_steps;         // the most steps of a row tile
  int* steps;             // the steps of a split that the device chose, or NULL
  float scale;            // log2(e) / sqrt(d)
};

// Tables and lengths do not change while a kernel reads them: uniform reads go
// through the scalar cache.
typedef __attribute__((address_space(4))) int32_t const_i32;
__device__ inline const const_i32* const_ints(const int32_t* p) {
  return (const const_i32*)(uintptr_t)p;
}

struct AttendLists {      // with PagedView and AttendArgs below 4 KB of kernel arguments
  RowList r;
  int32_t tile0[kMaxSeqs + 1];
};

// The last b with first[b] <= k: the sequence of row tile k (sequences
// without rows have no tile and are passed over).  The list lies among the
// kernel's arguments, which vector loads fetch from memory every time: all
// steps are uniform, so that they go through the scalar cache.
__device__ inline int tile_owner(const int32_t* first, int n, int k) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= k) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// Blocks are dealt to the 8 XCDs round-robin by number.  Work items that
// follow each other share K and V: each XCD takes `run` of them in turn, so
// that its L2 holds what they read, and all XCDs move through the items
// together, whose costs differ from end to end.
__device__ inline unsigned xcd_item(unsigned block, unsigned run) {
  const unsigned xcd = block & 7, i = block >> 3;
  return (i / run * 8 + xcd) * run + i % run;
}

// The cached tokens of one row tile.  They are walked in steps of TT tokens:
// first the sinks' [0, ns*TT), then the window's from lo on, both from
// multiples of TT, so that no step is in both.
struct TokenSpan {
  int n, T, row0;        // sequence length, query tokens, first query row of the call
  int lo, hi;            // the window part is [lo, hi), lo a multiple of TT
  int ns, nt;            // steps of the sinks, steps in all
  int per;               // steps of a split
};

template <int TT>
__device__ inline TokenSpan token_span(const PagedView& v, const AttendArgs& a,
                                       const AttendLists& s, int b, int tile, int row_tile,
                                       int chosen = 0) {
  TokenSpan t;
  const int hpg = v.H / v.G;
  t.n = min(max(const_ints(v.len)[s.r.slot[b]], 0), v.cap);
  t.row0 = s.r.row0[b];
  t.T = s.r.row0[b + 1] - t.row0;
  const int r0 = (tile - s.tile0[b]) * row_tile;
  const int i0 = r0 / hpg, i1 = min((r0 + row_tile - 1) / hpg, t.T - 1);
  int lo = 0, sinks = 0;
  t.hi = t.n;
  if (!a.mask) {
    t.hi = min(t.n, max(t.n - t.T + i1 + 1, 0));
    lo = max(t.n - t.T + i0 - a.window + 1, 0);
    sinks = a.sinks;
  }
  t.lo = min(lo, t.hi) / TT * TT;
  t.ns = (min(sinks, t.lo) + TT - 1) / TT;
  t.nt = t.ns + (t.hi - t.lo + TT - 1) / TT;
  // a split takes chunk tokens, or more where the lengths exceed the bound
  // that the number of splits was made for
  t.per = max(chosen ? chosen : (a.chunk + TT - 1) / TT, (t.nt + a.n_split - 1) / a.n_split);
  return t;
}

// The steps of a split, for sequences whose lengths only the device knows:
// the least with which the blocks of all splits fit the `slots` that the card
// holds at a time, or as many times as leave about 96 steps to a block.  The
// lanes of a wave take a sequence each.
template <int TT>
__device__ inline int balanced_steps(const PagedView& v, const AttendArgs& a, const AttendLists& s,
                                     int slots) {
  constexpr int kPer = kMaxSeqs / 64;
  const int lane = threadIdx.x & 63;
  int tiles[kPer], steps[kPer], work = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int b = lane + 64 * j;
    tiles[j] = steps[j] = 0;
    if (b < s.r.n) {
      tiles[j] = s.tile0[b + 1] - s.tile0[b];
      const int n = min(max(v.len[s.r.slot[b]], 0), v.cap);
      steps[j] = min((n + TT - 1) / TT, a.most_steps);
    }
    work += tiles[j] * steps[j];
  }
  const auto all = [](int x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
    return x;
  };
  work = all(work);
  const int lgs = v.n_layers * v.G;
  const float rounds = fmaxf(1.f, rintf((float)work * (float)lgs / (float)(slots * 96)));
  const int target = max(1, (int)((float)slots * rounds / (float)lgs));   // blocks of a (layer, group)
  int per = max(4, (work + target - 1) / target);
  for (int i = 0; i < 16; ++i) {
    int blocks = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) blocks += tiles[j] * ((steps[j] + per - 1) / per);
    if (all(blocks) <= target) break;
    per += max(1, per >> 4);
  }
  return __builtin_amdgcn_readfirstlane(per);
}

// Token of step u's first.
template <int TT>
__device__ inline int step_token(const TokenSpan& t, int u) {
  return u < t.ns ? u * TT : t.lo + (u - t.ns) * TT;
}

// The low k bits, k clamped to [0, 32].
__device__ inline uint32_t low_bits(int k) {
  return k >= 32 ? 0xFFFFFFFFu : k <= 0 ? 0u : (1u << k) - 1u;
}

// Which of the 32 cached tokens from t0 on query token i of the sequence
// sees, bit by bit: those of a tree's mask, or of a window and the sinks.
__device__ inline uint32_t seen_bits(const AttendArgs& a, const TokenSpan& s, int i, int t0) {
  uint32_t in = low_bits(s.n - t0);
  if (a.mask) {
    const int j0 = t0 - (s.n - s.T);            // the first token's number among the drafted
    const int j = max(j0, 0), w = j >> 6, sh = j & 63;
    uint64_t m = 0;
    if (j0 > -32 && w < a.words) {
      const uint64_t* row = a.mask + (size_t)(s.row0 + i) * a.words + w;
      m = row[0] >> sh;
      if (sh > 32 && w + 1 < a.words) m |= row[1] << (64 - sh);
    }
    m &= low_bits(s.T - j);                     // bits behind the last drafted token
    const int before = min(max(-j0, 0), 32);    // tokens before the drafted ones: all seen
    return in & (low_bits(before) | (uint32_t)(m << before));
  }
  const int p = s.n - s.T + i;
  in &= low_bits(p + 1 - t0);
  return in & ~(low_bits(p - a.window + 1 - t0) & ~low_bits(a.sinks - t0));
}

// The tokens that query tokens i0..i1 all see, but for dropped ones: [lo, hi),
// and [0, sinks).
struct AllSee {
  int lo, hi, sinks;
};
__device__ inline AllSee all_see(const AttendArgs& a, const TokenSpan& s, int i0, int i1) {
  if (a.mask) return AllSee{0, s.n - s.T, 0};
  const int p0 = s.n - s.T + i0, p1 = s.n - s.T + i1;
  return AllSee{p1 - a.window + 1, min(p0 + 1, s.n), min(a.sinks, p0 + 1)};
}
template <int TT>
__device__ inline bool sees_step(const AllSee& w, int t0) {
  return t0 + TT <= w.hi && (t0 >= w.lo || t0 + TT <= w.sinks);
}

// Columns [c, c + 4) of a finished row (of [n_layers][n_rows][H]): o / l in
// the cache's type, and with its first columns the row's log-sum-exp.
template <typename T>
__device__ inline void store_out(const AttendArgs& a, int d, size_t row, int c, float M, float L,
                                 f32x4 O) {
  const bool none = M == -INFINITY && L == 0.f;     // the row sees nothing
  typedef T T4 __attribute__((ext_vector_type(4)));
  T4 o;
  const float inv = none ? 0.f : 1.f / L;
#pragma unroll
  for (int j = 0; j < 4; ++j) o[j] = (T)(O[j] * inv);
  *reinterpret_cast<T4*>(a.out + (row * d + c) * sizeof(T)) = o;
  if (c == 0 && a.lse)
    a.lse[row] = none ? -INFINITY : fmaf(M, a.scale, __builtin_amdgcn_logf(L)) * 0.6931471805599453f;
}

// The same of row r of a (sequence, group) whose first query row is row0.
template <typename T>
__device__ inline void store_row(const AttendArgs& a, const PagedView& v, int layer, int g, int hpg,
                                 int row0, int r, int c, float M, float L, f32x4 O) {
  const size_t row = ((size_t)layer * a.n_rows + row0 + r / hpg) * v.H + g * hpg + r % hpg;
  store_out<T>(a, v.d, row, c, M, L, O);
}

// The kernel for many rows (attend_many.hip); the splits are joined after it.
int launch_attend_many(const PagedView& v, const AttendArgs& a, const AttendLists& l,
                       const AttendShape& s, hipStream_t st);

}  // namespace starkv
