// The pages of a paged cache: growing, writing, forking, freeing and
// compacting sequences.  The bookkeeping (table, lengths, reference counts)
// is integer work on a few kilobytes, bounded by the chain of dependent
// loads and block barriers of one block; the moves of K and V rows are bound
// by HBM and run 16 bytes per thread, whole rows contiguous.
//
// A page is free when its reference count is 0, so there is no free list to
// keep in order: one block scans the counts from page 0 up and takes the
// lowest free pages, which makes every call's result a function of the
// state alone.  Counts change by integer atomics, whose order does not
// matter; a call reads the counts that it decides by before it changes any.
#include <algorithm>
#include <type_traits>

#include "device_common.h"
#include "paged.h"

namespace starkv {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kScan = 8;          // reference counts per thread of a scan step
constexpr int kLowFresh = 1024;   // fresh pages kept in LDS
constexpr int64_t kMaxBlocks = (1 << 24) - 1;   // of 256 threads: a launch has under 2^32 of them

__device__ inline bool is_page(const PagedView& v, int32_t p) { return p >= 0 && p < v.n_pages; }
__device__ inline int seq_len(const PagedView& v, int slot) {
  return min(max(v.len[slot], 0), v.cap);
}
__device__ inline int pages_of(const PagedView& v, int64_t tokens) {
  return (int)((tokens + v.P - 1) >> v.psh);
}
__device__ inline int32_t* table_row(const PagedView& v, int slot) {
  return v.table + (size_t)slot * v.max_pages;
}

// The lists of a call, by value.  A launch pays for the bytes of its
// arguments, so short lists travel in short structs (one slot freed: 5.2 us
// of the host's time with the long struct, 4.3 with the short one).
constexpr int kShort = 16;
template <int N>
struct Seqs {
  int32_t n;
  int32_t slot[N], num[N];
  explicit Seqs(const SeqList& s) : n(s.n) {
    for (int i = 0; i < n; ++i) {
      slot[i] = s.slot[i];
      num[i] = s.num[i];
    }
  }
};
template <int N>
struct Rows {
  int32_t n;
  int32_t slot[N], row0[N + 1];
  explicit Rows(const RowList& r) : n(r.n) {
    for (int i = 0; i < n; ++i) slot[i] = r.slot[i];
    for (int i = 0; i <= n; ++i) row0[i] = r.row0[i];
  }
};

// The sequence (or tile, or row range) that item k belongs to: the last b
// with first[b] <= k.
__device__ inline int owner_of(const int32_t* first, int n, int k) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= k) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// Which of the kScan pages from p0 on are free, bit by bit.
__device__ inline unsigned free_pages(const PagedView& v, int p0) {
  unsigned m = 0;
#pragma unroll
  for (int j = 0; j < kScan; ++j)
    if (p0 + j < v.n_pages && v.refs[p0 + j] == 0) m |= 1u << j;
  return m;
}

// The fresh pages of a call, the first in LDS and the rest in the workspace.
struct Fresh {
  int32_t* low;
  int32_t* rest;
  __device__ inline void put(int i, int page) const {
    if (i < kLowFresh) low[i] = page;
    else rest[i] = page;
  }
  __device__ inline int at(int i) const { return i < kLowFresh ? low[i] : rest[i]; }
};

// The pages that the sequences need, thread b's `need` behind those of the
// threads before it, *excl: the lowest free ones, ascending.  Returns how many
// there are, at most what is needed.  `m`: the thread's first free_pages, read
// while the needs were worked out and counted with them.  A round looks at 8,192
// pages, 4.2 us where the search has to go on (a grow by one page: 8 us, behind
// 65,536 taken pages 39, behind a million 538).
__device__ int take_pages(const PagedView& v, int need, unsigned m, const Fresh& fresh, int (*sh)[2],
                          int* excl) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int inc0 = wave_incl_scan(need), inc1 = wave_incl_scan(__popc(m));
  if (lane == 63) {
    sh[w][0] = inc0;
    sh[w][1] = inc1;
  }
  __syncthreads();
  int before0 = 0, before1 = 0, total = 0, tot = 0;
#pragma unroll
  for (int i = 0; i < kPlanThreads / 64; ++i) {
    if (i < w) {
      before0 += sh[i][0];
      before1 += sh[i][1];
    }
    total += sh[i][0];
    tot += sh[i][1];
  }
  *excl = before0 + inc0 - need;
  int r = before1 + inc1 - __popc(m), found = 0, base = 0;
  for (;;) {
    while (m) {
      const int j = __ffs(m) - 1;
      m &= m - 1;
      if (r < total) fresh.put(r, base + (int)threadIdx.x * kScan + j);
      ++r;
    }
    found += tot;
    base += kPlanThreads * kScan;
    if (found >= total || base >= v.n_pages) break;
    m = free_pages(v, base + (int)threadIdx.x * kScan);
    r = found + block_excl_scan(__popc(m), &sh[0][0], &tot);
  }
  __syncthreads();   // the fresh pages are read by other threads of the block
  return min(found, total);
}

__global__ __launch_bounds__(256) void init_kernel(PagedView v) {
  const int64_t n = (int64_t)v.n_slots * v.max_pages, step = (int64_t)gridDim.x * blockDim.x;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += step) v.table[i] = -1;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < v.n_pages; i += step)
    v.refs[i] = 0;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < v.n_slots; i += step)
    v.len[i] = 0;
}

// Pages for the new tokens (4 to 5 us: the arguments, a length, its table
// entry, the page's count, the scan and the writes, one after the other).
// info[b]: the page to copy from (or -1), to, and the rows to copy.
template <int N>
__global__ __launch_bounds__(kPlanThreads) void grow_plan(PagedView v, Seqs<N> s, int32_t* rest,
                                                          i32x4* info, int32_t* status) {
  __shared__ int pre[kMaxSeqs], first[kMaxSeqs], ok[kMaxSeqs], sh[kPlanThreads / 64][2];
  __shared__ int32_t low[kLowFresh];
  const Fresh fresh{low, rest};
  const int b = threadIdx.x;
  const unsigned free0 = free_pages(v, b * kScan);
  int need = 0, col = 0, part = 0, st = STARKV_SEQ_OK, old = -1, len1 = 0;
  if (b < s.n) {
    const int len0 = seq_len(v, s.slot[b]), add = s.num[b];
    const int64_t to = (int64_t)len0 + add;
    col = pages_of(v, len0);
    part = len0 & (v.P - 1);
    if (to > v.cap) {
      st = STARKV_SEQ_RANGE;
    } else if (add > 0) {
      len1 = (int)to;
      if (part) {
        // the partly filled last page: replaced where it is shared.  Where it
        // was dropped there is no page to go on in: a fresh one would bring
        // back the dropped tokens, with rows that nobody wrote
        old = table_row(v, s.slot[b])[col - 1];
        if (!is_page(v, old)) st = STARKV_SEQ_RANGE;
        else if (v.refs[old] > 1) --col;
        else old = -1;
      }
      if (st == STARKV_SEQ_OK) need = pages_of(v, to) - col;
    } else {
      len1 = len0;
    }
  }
  int excl;
  const int found = take_pages(v, need, free0, fresh, sh, &excl);
  if (b < s.n) {
    if (need > 0 && excl + need > found) st = STARKV_SEQ_NO_PAGES;
    pre[b] = excl;
    first[b] = col;
    ok[b] = st == STARKV_SEQ_OK;
    status[b] = st;
    const bool copy = ok[b] && old >= 0;
    info[b] = i32x4{copy ? old : -1, copy ? fresh.at(excl) : -1, part, 0};
    if (ok[b]) v.len[s.slot[b]] = len1;
    if (copy) atomicSub(&v.refs[old], 1);
  }
  __syncthreads();
  for (int k = threadIdx.x; k < found; k += kPlanThreads) {
    const int o = owner_of(pre, s.n, k);
    if (!ok[o]) continue;
    const int page = fresh.at(k);
    table_row(v, s.slot[o])[first[o] + (k - pre[o])] = page;
    v.refs[page] = 1;
  }
}

// 4-bit caches are those whose rows are two or four vectors: their scales, as
// many bytes, lie behind the block's rows and move along.
template <int VPR>
struct ScaleRow {
  using type = uint32_t;
};
template <>
struct ScaleRow<2> {
  using type = uint16_t;
};
template <int VPR>
constexpr bool kScaled = VPR <= 4;

// Rows [0, part) of a replaced page, one (sequence, group, layer) per block (16
// forks with 28 or 35 rows in 28 layers: 10.4 us, 5.6 TB/s read and written;
// with nothing to copy 2; with 35 rows 10 in bf16, 17 in float32, 5 in 4 bits).
template <int VPR>
__global__ __launch_bounds__(256) void grow_copy(PagedView v, const i32x4* info) {
  const i32x4 c = info[blockIdx.x];
  if (c[0] < 0) return;
  const int64_t base = (int64_t)blockIdx.z * v.ls + (int64_t)blockIdx.y * v.gs;
  const int64_t from = base + (int64_t)c[0] * v.ps, to = base + (int64_t)c[1] * v.ps;
  for (int i = threadIdx.x; i < c[2] * VPR; i += 256) {
    const int64_t off = (int64_t)(i / VPR) * v.ts + (i % VPR) * 16;
    const i32x4 kk = *reinterpret_cast<const i32x4*>(v.k + from + off);
    const i32x4 vv = *reinterpret_cast<const i32x4*>(v.v + from + off);
    *reinterpret_cast<i32x4*>(v.k + to + off) = kk;
    *reinterpret_cast<i32x4*>(v.v + to + off) = vv;
  }
  if constexpr (kScaled<VPR>) {
    using S = typename ScaleRow<VPR>::type;
    for (int i = threadIdx.x; i < c[2]; i += 256) {
      const int64_t off = (int64_t)v.P * v.row + (int64_t)i * sizeof(S);
      const S ks = *reinterpret_cast<const S*>(v.k + from + off);
      const S vs = *reinterpret_cast<const S*>(v.v + from + off);
      *reinterpret_cast<S*>(v.k + to + off) = ks;
      *reinterpret_cast<S*>(v.v + to + off) = vs;
    }
  }
}

struct WriteArgs {
  const char* k;
  const char* v;
  int64_t ls, gs, ts;   // byte strides
  const int32_t* grown;
};

// 16-byte vectors of K and V, one per thread (or, where a launch cannot hold
// as many threads, several).  The page of a token must belong to its sequence
// alone: a shared one is left as it is.  So is a sequence that the grow before
// it left unchanged: its last tokens are not the ones to write.  (One token of
// 16 sequences in 28 layers: 3.6 us, a chain of four loads; a prompt of 13,711
// tokens in 28 layers 241 us, 6.5 TB/s read and written, in one 9.)
template <int VPR, int N>
__global__ __launch_bounds__(256) void write_kernel(PagedView v, Rows<N> r, WriteArgs a) {
  const int64_t n = (int64_t)r.row0[r.n] * v.G * VPR;
  const int layer = blockIdx.y;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int part = (int)(i % VPR);
    const int64_t rg = i / VPR;
    const int g = (int)(rg % v.G), row = (int)(rg / v.G);
    const int b = owner_of(r.row0, r.n, row);
    if (a.grown && a.grown[b] != STARKV_SEQ_OK) continue;
    const int t = seq_len(v, r.slot[b]) - r.row0[b + 1] + row;
    if (t < 0) continue;
    const int page = table_row(v, r.slot[b])[t >> v.psh];
    if (!is_page(v, page) || v.refs[page] > 1) continue;
    const int64_t from = (int64_t)layer * a.ls + (int64_t)g * a.gs + (int64_t)row * a.ts + part * 16;
    const int64_t to = (int64_t)layer * v.ls + (int64_t)page * v.ps + (int64_t)g * v.gs +
                       (int64_t)(t & (v.P - 1)) * v.ts + part * 16;
    *reinterpret_cast<i32x4*>(v.k + to) = *reinterpret_cast<const i32x4*>(a.k + from);
    *reinterpret_cast<i32x4*>(v.v + to) = *reinterpret_cast<const i32x4*>(a.v + from);
  }
}

// The same into a 4-bit cache: a thread takes 16 bytes, eight elements, of K and
// of V, and four neighbours the 32 elements that share a scale.  Their largest
// magnitude, as an integer (which orders infinities and NaN above all numbers),
// gives the scale by its exponent, one more where the mantissa is over 1.75; the
// hardware's conversion divides by it, exactly, and rounds to the nearest, ties to
// the even code.  Bound by HBM (13,711 tokens in 28 layers, 786 MB read and 209
// written: 195 us, 5.1 TB/s).
__device__ inline uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true));   // lanes 1 0 3 2
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true));  // lanes 2 3 0 1
}
__device__ inline uint32_t quantise(const i32x4& x, uint32_t* scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  uint32_t top = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w)
    top = max(top, max((uint32_t)x[w] << 16 & 0x7FFF0000u, (uint32_t)x[w] & 0x7FFF0000u));
  top = quad_max(top);
  const uint32_t byte = min(max((int)((top + 0x1FFFFFu) >> 23) - 2, 2), 252);
  *scale = top >= 0x7F800000u ? 255u : byte;
  const float s = __uint_as_float(byte << 23);
  uint32_t code = 0;
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2, (uint32_t)x[0]), s, 0);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2, (uint32_t)x[1]), s, 1);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2, (uint32_t)x[2]), s, 2);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2, (uint32_t)x[3]), s, 3);
  return code;
}

template <int D, int N>
__global__ __launch_bounds__(256) void write_fp4(PagedView v, Rows<N> r, WriteArgs a) {
  constexpr int VPR = D / 8;
  const int64_t n = (int64_t)r.row0[r.n] * v.G * VPR;
  const int layer = blockIdx.y;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int part = (int)(i % VPR);
    const int64_t rg = i / VPR;
    const int g = (int)((uint32_t)rg % (uint32_t)v.G), row = (int)((uint32_t)rg / (uint32_t)v.G);
    // the rows first, whether they are to be written or not: their way overlaps that of
    // the page (the tokens above took 241 us one after the other).  They are read once,
    // past the caches
    const int64_t from = (int64_t)layer * a.ls + (int64_t)g * a.gs + (int64_t)row * a.ts + part * 16;
    const i32x4 kk = __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(a.k + from));
    const i32x4 vv = __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(a.v + from));
    const int b = owner_of(r.row0, r.n, row);
    if (a.grown && a.grown[b] != STARKV_SEQ_OK) continue;
    const int t = seq_len(v, r.slot[b]) - r.row0[b + 1] + row;
    if (t < 0) continue;
    const int page = table_row(v, r.slot[b])[t >> v.psh];
    if (!is_page(v, page) || v.refs[page] > 1) continue;
    const int64_t block = (int64_t)layer * v.ls + (int64_t)page * v.ps + (int64_t)g * v.gs;
    const int in_page = t & (v.P - 1);
    const int64_t to = block + (int64_t)in_page * (D / 2) + part * 4;
    const int64_t sto = block + (int64_t)v.P * (D / 2) + in_page * (D / 32) + part / 4;
    uint32_t ks, vs;
    const uint32_t kc = quantise(kk, &ks);
    const uint32_t vc = quantise(vv, &vs);
    *reinterpret_cast<uint32_t*>(v.k + to) = kc;
    *reinterpret_cast<uint32_t*>(v.v + to) = vc;
    if (part % 4 == 0) {
      v.k[sto] = (char)ks;
      v.v[sto] = (char)vs;
    }
  }
}

// The rows of tokens out of their pages, 16 bytes of K and of V per thread; of a
// 4-bit cache the bf16 numbers that four bytes stand for.  What has no page gives
// zeros.  Bound by HBM: 13,711 tokens in 28 layers of bf16 254 us (1,572 MB, 6.2 TB/s), of
// float32 512 (6.1), out of 4 bits 150 (995 MB, 6.6), 237 with the rows written through the caches, where they took the place of the
// pages.
struct ReadArgs {
  char* k;
  char* v;
  int64_t ls, gs, ts;   // byte strides
};
__device__ inline i32x4 dequantise(uint32_t w, uint32_t byte) {
  const float s = __uint_as_float(byte << 23);
  return i32x4{__builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0)),
               __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1)),
               __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2)),
               __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3))};
}
// VPR: 16-byte vectors of a row in the pool
template <int VPR, int N>
__global__ __launch_bounds__(256) void read_kernel(PagedView v, Rows<N> r, ReadArgs a) {
  constexpr bool F4 = kScaled<VPR>;
  constexpr int kOut = F4 ? 4 * VPR : VPR;     // vectors of a row given back
  const int64_t n = (int64_t)r.row0[r.n] * v.G * kOut;
  const int layer = blockIdx.y;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int part = (int)(i % kOut);
    const int64_t rg = i / kOut;
    const int g = (int)((uint32_t)rg % (uint32_t)v.G), row = (int)((uint32_t)rg / (uint32_t)v.G);
    const int b = owner_of(r.row0, r.n, row);
    const int t = seq_len(v, r.slot[b]) - r.row0[b + 1] + row;
    const int page = t < 0 ? -1 : table_row(v, r.slot[b])[t >> v.psh];
    i32x4 kk{0, 0, 0, 0}, vv{0, 0, 0, 0};
    if (is_page(v, page)) {
      const int64_t block = (int64_t)layer * v.ls + (int64_t)page * v.ps + (int64_t)g * v.gs;
      const int in_page = t & (v.P - 1);
      if constexpr (F4) {
        const int64_t from = block + (int64_t)in_page * (16 * VPR) + part * 4;
        const int64_t at = block + (int64_t)v.P * (16 * VPR) + in_page * VPR + part / 4;
        kk = dequantise(*reinterpret_cast<const uint32_t*>(v.k + from), (uint8_t)v.k[at]);
        vv = dequantise(*reinterpret_cast<const uint32_t*>(v.v + from), (uint8_t)v.v[at]);
      } else {
        const int64_t from = block + (int64_t)in_page * v.ts + part * 16;
        kk = *reinterpret_cast<const i32x4*>(v.k + from);
        vv = *reinterpret_cast<const i32x4*>(v.v + from);
      }
    }
    const int64_t to = (int64_t)layer * a.ls + (int64_t)g * a.gs + (int64_t)row * a.ts + part * 16;
    __builtin_nontemporal_store(kk, reinterpret_cast<i32x4*>(a.k + to));
    __builtin_nontemporal_store(vv, reinterpret_cast<i32x4*>(a.v + to));
  }
}

// Sequence s.slot[b] becomes a fork of s.num[b], one pair per block.  No
// slot is read and written by the same call.  (1.5 to 3 us, as free below:
// lengths, table entries, counts, one after the other.)
template <int N>
__global__ __launch_bounds__(256) void fork_kernel(PagedView v, Seqs<N> s) {
  const int b = blockIdx.x, dst = s.slot[b], src = s.num[b];
  const int had = pages_of(v, seq_len(v, dst)), has = pages_of(v, seq_len(v, src));
  int32_t* to = table_row(v, dst);
  const int32_t* from = table_row(v, src);
  for (int j = threadIdx.x; j < max(had, has); j += 256) {
    const int old = j < had ? to[j] : -1;
    const int page = j < has ? from[j] : -1;
    if (is_page(v, old)) atomicSub(&v.refs[old], 1);
    if (is_page(v, page)) atomicAdd(&v.refs[page], 1);
    to[j] = page;
  }
  __syncthreads();   // every thread has read the length
  if (threadIdx.x == 0) v.len[dst] = seq_len(v, src);
}

template <int N>
__global__ __launch_bounds__(256) void free_kernel(PagedView v, Seqs<N> s, int keep_first,
                                                   int keep_last) {
  const int slot = s.slot[blockIdx.x], len0 = seq_len(v, slot);
  // dropped tokens: [lo, hi)
  const int lo = min(keep_first, len0), hi = len0 - min(keep_last, len0);
  const int p1 = pages_of(v, len0);
  int32_t* row = table_row(v, slot);
  for (int j = pages_of(v, lo) + (int)threadIdx.x; j < p1; j += 256) {
    if (min((int64_t)(j + 1) << v.psh, (int64_t)len0) > hi) break;
    if (is_page(v, row[j])) atomicSub(&v.refs[row[j]], 1);
    row[j] = -1;
  }
  __syncthreads();
  if (keep_last == 0 && threadIdx.x == 0) v.len[slot] = lo;
}

// Fresh pages for the kept tokens; the table rows as they were into old[].
// info[b]: length, a, count (or -1: the sequence stays) and the first fresh
// page's column.  (5.7 us, as grow_plan's, 0.2 of them for the tail's pages.)
template <int N>
__global__ __launch_bounds__(kPlanThreads) void compact_plan(PagedView v, Seqs<N> s, bool whole,
                                                             int B, const int32_t* counts,
                                                             int tail, const int32_t* grown,
                                                             int32_t* rest, i32x4* info,
                                                             int32_t* old, int32_t* status) {
  __shared__ int pre[kMaxSeqs], first[kMaxSeqs], last[kMaxSeqs], end[kMaxSeqs], lost[kMaxSeqs];
  __shared__ int sh[kPlanThreads / 64][2];
  __shared__ int32_t low[kLowFresh];
  const Fresh fresh{low, rest};
  const int b = threadIdx.x, lane = threadIdx.x & 63;
  const unsigned free0 = free_pages(v, b * kScan);
  // Tails of a few pages are looked at by the sequence's thread, beside its
  // other table entry; longer ones by a wave, 64 pages at a time.
  const bool few = tail <= 3 * v.P;
  if (!few) {
    for (int o = threadIdx.x >> 6; o < s.n; o += kPlanThreads / 64) {
      const int n = seq_len(v, s.slot[o]);
      const int32_t* row = table_row(v, s.slot[o]);
      bool gone = false;
      if (tail <= n)
        for (int j = ((n - tail) >> v.psh) + lane; j < pages_of(v, n); j += 64) gone |= !is_page(v, row[j]);
      gone = __any(gone);
      if (lane == 0) lost[o] = gone;
    }
    __syncthreads();
  }
  int need = 0, col = 0, st = STARKV_SEQ_OK, len0 = 0, a = 0, cnt = 0, len1 = 0;
  if (b < s.n) {
    len0 = seq_len(v, s.slot[b]);
    const int span = whole ? len0 : min(s.num[b], len0);
    a = len0 - span;
    cnt = counts ? min(max(counts[b], 0), B) : B;
    const int64_t to = (int64_t)a + cnt + tail;
    // token a's page keeps the tokens before a: not where it was dropped
    bool gone = cnt + tail > 0 && (a & (v.P - 1)) &&
                !is_page(v, table_row(v, s.slot[b])[a >> v.psh]);
    // and a dropped token of the tail has no row: a row of zeros in its place
    // would be seen by the attentions, which did not see the token
    if (!few) {
      gone |= lost[b] != 0;
    } else if (tail > 0 && tail <= len0) {
      const int j0 = (len0 - tail) >> v.psh, j1 = (len0 - 1) >> v.psh;
#pragma unroll
      for (int j = 0; j < 4; ++j)      // tails of at most 3 P tokens end within four pages
        if (j0 + j <= j1) gone |= !is_page(v, table_row(v, s.slot[b])[j0 + j]);
    }
    // (the grow's status before this call's own, which may be written over it)
    if (grown) st = grown[b];
    if (st != STARKV_SEQ_OK) {
      // its last tokens are not those that the call is about: it stays
    } else if (tail > span || to > v.cap || gone) {
      st = STARKV_SEQ_RANGE;
    } else {
      len1 = (int)to;
      // nothing kept of the span: no page changes, the later ones are let go
      col = cnt + tail > 0 ? a >> v.psh : pages_of(v, a);
      need = pages_of(v, to) - col;
    }
  }
  int excl;
  const int found = take_pages(v, need, free0, fresh, sh, &excl);
  if (b < s.n) {
    if (need > 0 && excl + need > found) st = STARKV_SEQ_NO_PAGES;
    const bool ok = st == STARKV_SEQ_OK;
    pre[b] = excl;
    first[b] = ok ? col : -1;
    last[b] = pages_of(v, len0);
    end[b] = pages_of(v, len1);
    status[b] = st;
    info[b] = i32x4{len0, a, ok ? cnt : -1, col};
    if (ok) v.len[s.slot[b]] = len1;
  }
  __syncthreads();
  // a wave per sequence: the old entries kept aside and let go
  for (int o = threadIdx.x >> 6; o < s.n; o += kPlanThreads / 64) {
    if (first[o] < 0) continue;
    int32_t* row = table_row(v, s.slot[o]);
    for (int j = first[o] + lane; j < last[o]; j += 64) {
      const int page = row[j];
      old[(size_t)o * v.max_pages + j] = page;
      if (is_page(v, page)) atomicSub(&v.refs[page], 1);
      if (j >= end[o]) row[j] = -1;
    }
  }
  __syncthreads();
  for (int k = threadIdx.x; k < found; k += kPlanThreads) {
    const int o = owner_of(pre, s.n, k);
    if (first[o] < 0) continue;
    const int page = fresh.at(k);
    table_row(v, s.slot[o])[first[o] + (k - pre[o])] = page;
    v.refs[page] = 1;
  }
}

struct MoveArgs {
  const i32x4* info;
  const int32_t* old;
  const int32_t* idx;
  int64_t idx_ls;
  int B, tail, chunks;
  KeptMasses kept;
};

// The kept rows into the fresh pages, one vector of K and of V per thread
// (28 layers, 2,723 rows kept of 13,711: 49 us, 6.5 TB/s read and written; four
// vectors per thread with ordinary stores 61, against 52 on that card; of 128 elements
// in float32 101, in 4 bits 22, and of 64 in 4 bits 17, with their scales).  The rows
// are not read again here, so the stores bypass the caches.
template <int VPR, int N>
__global__ __launch_bounds__(256) void compact_move(PagedView v, Seqs<N> s, MoveArgs m) {
  const int chunk = blockIdx.x % m.chunks;
  const int rest = blockIdx.x / m.chunks;
  const int g = rest % v.G, b = rest / v.G, layer = blockIdx.y;
  const i32x4 info = m.info[b];
  const int len0 = info[0], a = info[1], cnt = info[2];
  if (cnt < 0) return;
  if (m.kept.from && chunk == 0 && g == 0) {      // (an eviction's masses move with the rows)
    const float* from = m.kept.from + ((size_t)layer * s.n + b) * (m.B + m.tail);
    float* to = m.kept.to + ((size_t)layer * v.n_slots + s.slot[b]) * v.cap;
    for (int i = threadIdx.x; i < cnt + m.tail; i += 256) to[i] = from[i];
  }
  const int r0 = info[3] << v.psh;                 // the first fresh page's first token
  const int64_t nvec = ((int64_t)a + cnt + m.tail - r0) * VPR;
  const int32_t* idx = m.idx + (int64_t)layer * m.idx_ls + (int64_t)b * m.B;
  const int32_t* old = m.old + (size_t)b * v.max_pages;
  const int32_t* row = table_row(v, s.slot[b]);
  const int64_t base = (int64_t)layer * v.ls + (int64_t)g * v.gs;
  const int picks = len0 - a - m.tail;             // idx is over [0, picks)
  for (int64_t vec = (int64_t)chunk * 256 + threadIdx.x; vec < nvec; vec += (int64_t)m.chunks * 256) {
    const int r = r0 + (int)(vec / VPR), part = (int)(vec % VPR);
    int t = r;
    if (r >= a + cnt) {
      t = len0 - m.tail + (r - a - cnt);
    } else if (r >= a) {
      const int pick = idx[r - a];
      t = pick >= 0 && pick < picks ? a + pick : -1;
    }
    i32x4 kk{0, 0, 0, 0}, vv{0, 0, 0, 0};
    const int page = t >= 0 ? old[t >> v.psh] : -1;
    if (is_page(v, page)) {
      const int64_t from = base + (int64_t)page * v.ps + (int64_t)(t & (v.P - 1)) * v.ts + part * 16;
      kk = *reinterpret_cast<const i32x4*>(v.k + from);
      vv = *reinterpret_cast<const i32x4*>(v.v + from);
    }
    const int64_t to = base + (int64_t)row[r >> v.psh] * v.ps + (int64_t)(r & (v.P - 1)) * v.ts + part * 16;
    __builtin_nontemporal_store(kk, reinterpret_cast<i32x4*>(v.k + to));
    __builtin_nontemporal_store(vv, reinterpret_cast<i32x4*>(v.v + to));
    if constexpr (kScaled<VPR>) {
      if (part == 0) {
        using S = typename ScaleRow<VPR>::type;
        S ks = 0, vs = 0;
        if (is_page(v, page)) {
          const int64_t from = base + (int64_t)page * v.ps + (int64_t)v.P * v.row +
                               (int64_t)(t & (v.P - 1)) * sizeof(S);
          ks = *reinterpret_cast<const S*>(v.k + from);
          vs = *reinterpret_cast<const S*>(v.v + from);
        }
        const int64_t sto = base + (int64_t)row[r >> v.psh] * v.ps + (int64_t)v.P * v.row +
                            (int64_t)(r & (v.P - 1)) * sizeof(S);
        *reinterpret_cast<S*>(v.k + sto) = ks;
        *reinterpret_cast<S*>(v.v + sto) = vs;
      }
    }
  }
}

template <int I>
using Int = std::integral_constant<int, I>;
// f(16-byte vectors of a row), f(the call's list)
template <typename F>
void by_row_vectors(const PagedView& v, F f) {
  switch (v.row / 16) {
    case 2: f(Int<2>{}); break;
    case 4: f(Int<4>{}); break;
    case 8: f(Int<8>{}); break;
    case 16: f(Int<16>{}); break;
    default: f(Int<32>{}); break;
  }
}
template <typename F>
void with_list(const SeqList& s, F f) {
  if (s.n <= kShort) f(Seqs<kShort>(s));
  else f(Seqs<kMaxSeqs>(s));
}
template <typename F>
void with_list(const RowList& r, F f) {
  if (r.n <= kShort) f(Rows<kShort>(r));
  else f(Rows<kMaxSeqs>(r));
}

}  // namespace

int launch_pages_init(const PagedView& v, void* stream) {
  const int64_t n = std::max<int64_t>((int64_t)v.n_slots * v.max_pages, v.n_pages);
  const int blocks = (int)std::min<int64_t>((n + 255) / 256, 2048);
  init_kernel<<<blocks, 256, 0, reinterpret_cast<hipStream_t>(stream)>>>(v);
  return (int)hipGetLastError();
}

int launch_pages_grow(const PagedView& v, const SeqList& s, const PagesWs& w, int32_t* status,
                      void* ws, void* stream) {
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  char* p = static_cast<char*>(ws);
  i32x4* info = reinterpret_cast<i32x4*>(p + w.info);
  with_list(s, [&](const auto& l) {
    grow_plan<<<1, kPlanThreads, 0, st>>>(v, l, reinterpret_cast<int32_t*>(p + w.fresh), info, status);
  });
  by_row_vectors(v, [&](auto vpr) {
    grow_copy<decltype(vpr)::value><<<dim3(s.n, v.G, v.n_layers), 256, 0, st>>>(v, info);
  });
  return (int)hipGetLastError();
}

int launch_pages_write(const PagedView& v, const RowList& r, const void* k, const void* vv,
                       const starkv_kv_layout& lay, void* stream) {
  WriteArgs a{static_cast<const char*>(k), static_cast<const char*>(vv), lay.layer_stride * v.esz,
              lay.group_stride * v.esz, lay.token_stride * v.esz, r.grown};
  const int64_t nvec = (int64_t)r.row0[r.n] * v.G * (v.d * v.esz / 16);
  const dim3 grid((unsigned)std::min((nvec + 255) / 256, kMaxBlocks), v.n_layers);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (v.fp4) {
    with_list(r, [&](const auto& l) {
      if (v.d == 128) write_fp4<128><<<grid, 256, 0, st>>>(v, l, a);
      else write_fp4<64><<<grid, 256, 0, st>>>(v, l, a);
    });
    return (int)hipGetLastError();
  }
  by_row_vectors(v, [&](auto vpr) {
    if constexpr (!kScaled<decltype(vpr)::value>)
      with_list(r, [&](const auto& l) {
        write_kernel<decltype(vpr)::value><<<grid, 256, 0, st>>>(v, l, a);
      });
  });
  return (int)hipGetLastError();
}

int launch_pages_read(const PagedView& v, const RowList& r, void* k, void* vv,
                      const starkv_kv_layout& lay, void* stream) {
  ReadArgs a{static_cast<char*>(k), static_cast<char*>(vv), lay.layer_stride * v.esz,
             lay.group_stride * v.esz, lay.token_stride * v.esz};
  const int64_t nvec = (int64_t)r.row0[r.n] * v.G * (v.d * v.esz / 16);
  const dim3 grid((unsigned)std::min((nvec + 255) / 256, kMaxBlocks), v.n_layers);
  by_row_vectors(v, [&](auto vpr) {
    with_list(r, [&](const auto& l) {
      read_kernel<decltype(vpr)::value>
          <<<grid, 256, 0, reinterpret_cast<hipStream_t>(stream)>>>(v, l, a);
    });
  });
  return (int)hipGetLastError();
}

int launch_pages_fork(const PagedView& v, const SeqList& s, void* stream) {
  with_list(s, [&](const auto& l) {
    fork_kernel<<<s.n, 256, 0, reinterpret_cast<hipStream_t>(stream)>>>(v, l);
  });
  return (int)hipGetLastError();
}

int launch_pages_free(const PagedView& v, const SeqList& s, int keep_first, int keep_last,
                      void* stream) {
  with_list(s, [&](const auto& l) {
    free_kernel<<<s.n, 256, 0, reinterpret_cast<hipStream_t>(stream)>>>(v, l, keep_first, keep_last);
  });
  return (int)hipGetLastError();
}

int launch_pages_compact(const PagedView& v, const SeqList& s, bool whole, const int32_t* idx,
                         int64_t idx_ls, int B, const int32_t* counts, int tail,
                         const PagesWs& w, int32_t* status, void* ws, void* stream) {
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  char* p = static_cast<char*>(ws);
  MoveArgs m;
  m.info = reinterpret_cast<const i32x4*>(p + w.info);
  m.old = reinterpret_cast<const int32_t*>(p + w.old);
  m.idx = idx;
  m.idx_ls = idx_ls;
  m.B = B;
  m.tail = tail;
  m.kept = s.kept;
  with_list(s, [&](const auto& l) {
    compact_plan<<<1, kPlanThreads, 0, st>>>(v, l, whole, B, counts, tail, s.grown,
                                             reinterpret_cast<int32_t*>(p + w.fresh),
                                             reinterpret_cast<i32x4*>(p + w.info),
                                             reinterpret_cast<int32_t*>(p + w.old), status);
  });
  if (B + tail > 0) {
    // the most rows of a sequence: the kept ones and the first page's before them
    const int vpr_n = v.row / 16;
    const int64_t nvec = ((int64_t)B + tail + v.P - 1) * vpr_n;
    const int64_t per = (int64_t)s.n * v.G;      // at most 2^14
    m.chunks = (int)std::min<int64_t>({(nvec + 255) / 256, kMaxBlocks / per, 65535});
    by_row_vectors(v, [&](auto vpr) {
      with_list(s, [&](const auto& l) {
        compact_move<decltype(vpr)::value>
            <<<dim3((unsigned)(per * m.chunks), v.n_layers), 256, 0, st>>>(v, l, m);
      });
    });
  }
  return (int)hipGetLastError();
}

}  // namespace starkv
