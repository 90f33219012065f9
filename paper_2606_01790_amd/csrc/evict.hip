// Eviction by accumulated attention weight: of a sequence's masses the largest,
// in the order of their tokens, and the masses moved to where the compaction
// moved their rows.
//
// One block of 16 waves works on a (layer, sequence).  The masses become 32-bit
// keys in the order of the numbers, a wave keeps a range of tokens' keys in its
// registers, and the largest threshold that K keys reach is found bit by bit: the
// lanes of a wave are counted by a ballot, so a round is a compare and a count of
// bits per 64 keys and one barrier, whatever the distribution of the masses.  It
// ends early where the count is met.
#include <algorithm>

#include "device_common.h"
#include "evict.h"

namespace starkv {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;

// The lists of a call, by value, as for the pages.
struct Slots {
  int32_t n;
  int32_t slot[kMaxSeqs];
  int32_t from[kMaxSeqs];
};

struct EvictArgs {
  float* mass;
  int keep, sinks, recent;
  int32_t* idx;
  int32_t* counts;
  int32_t* stay;
  float* kept;
};

__device__ inline int seq_len(const PagedView& v, int slot) {
  return min(max(v.len[slot], 0), v.cap);
}
__device__ inline float* mass_row(const PagedView& v, float* mass, int layer, int slot) {
  return mass + ((size_t)layer * v.n_slots + slot) * v.cap;
}

// Sinks above all, then NaN, then the masses; 0: not to be kept.
constexpr uint32_t kSink = ~0u, kNan = ~0u - 1;
__device__ inline uint32_t key_of(const PagedView& v, const int32_t* table, const float* mass,
                                  int t, int span, int sinks) {
  if (t >= span) return 0;
  const int page = table[t >> v.psh];
  if (page < 0 || page >= v.n_pages) return 0;
  if (t < sinks) return kSink;
  const float m = mass[t];
  return m != m ? kNan : fkey(m + 0.f);      // (-0 counts as 0)
}

// The keys of a wave's tokens [first, first + 64 * count): in N registers a lane,
// or (N = 0) read again each time.
template <int N>
struct Keys {
  uint32_t k[N > 0 ? N : 1];
  const PagedView& v;
  const int32_t* table;
  const float* mass;
  int first, count, span, sinks;

  __device__ inline uint32_t read(int j) const {
    return key_of(v, table, mass, first + 64 * j + (int)(threadIdx.x & 63), span, sinks);
  }
  __device__ inline void load() {
#pragma unroll
    for (int j = 0; j < N; ++j) k[j] = j < count ? read(j) : 0;
  }
  // f(key, j) for each of them, in the order of the tokens
  template <typename F>
  __device__ inline void each(F f) const {
    if constexpr (N > 0) {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (j < count) f(k[j], j);
    } else {
      for (int j = 0; j < count; ++j) f(read(j), j);
    }
  }
  __device__ inline int at_least(uint32_t bound) const {
    int c = 0;
    each([&](uint32_t x, int) { c += __popcll(__ballot(x >= bound)); });
    return c;
  }
};

// The sum over the block of a count that is the same in all lanes of a wave, and
// (before) over the waves before this one.
__device__ inline int block_total(int c, int* sh, int* before = nullptr) {
  const int w = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) sh[w] = c;
  __syncthreads();
  int all = 0, pre = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    const int x = sh[i];
    if (i < w) pre += x;
    all += x;
  }
  if (before) *before = pre;
  return all;
}

template <int N>
__device__ void select(const PagedView& v, const EvictArgs& a, int b, int layer, int n_seqs,
                       int slot, int n, int (*sh)[kWaves]) {
  const int want = a.sinks + a.keep, span = n - a.recent;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int per = (span + kThreads - 1) / kThreads;          // groups of 64 tokens of a wave
  const float* mass = mass_row(v, a.mass, layer, slot);
  Keys<N> keys{{}, v, v.table + (size_t)slot * v.max_pages, mass, w * per * 64, per, span, a.sinks};
  keys.load();
  int turn = 0;                                              // the LDS counts of rounds by turns
  const int here = block_total(keys.at_least(1), sh[turn++ % 3]);
  const int sunk = block_total(keys.at_least(kSink), sh[turn++ % 3]);
  const int K = here - sunk <= a.keep ? here : sunk + a.keep;
  uint32_t T = 1;
  if (K < here) {
    T = 0;
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t next = T | 1u << bit;
      const int c = block_total(keys.at_least(next), sh[turn++ % 3]);
      if (c >= K) T = next;
      if (c == K) break;
    }
  }
  // all above T, and of those at T the first ones
  const int above = T == kSink ? 0 : keys.at_least(T + 1), level = keys.at_least(T) - above;
  int above_before, level_before;
  const int most = K - block_total(above, sh[turn++ % 3], &above_before);
  block_total(level, sh[turn++ % 3], &level_before);
  int pos = above_before + min(level_before, most), seen = level_before;
  const size_t row = (size_t)layer * n_seqs + b;
  int32_t* idx = a.idx + row * want;
  float* kept = a.kept + row * (want + a.recent);
  if (K > 0)
    keys.each([&](uint32_t x, int j) {
      const uint64_t below = (1ull << lane) - 1;
      const uint64_t tie = __ballot(x == T);
      const bool take = x > T || (x == T && seen + __popcll(tie & below) < most);
      const uint64_t taken = __ballot(take);
      if (take) {
        const int t = keys.first + 64 * j + lane, to = pos + __popcll(taken & below);
        idx[to] = t;
        kept[to] = mass[t];
      }
      pos += __popcll(taken);
      seen += __popcll(tie);
    });
  for (int i = K + (int)threadIdx.x; i < want; i += kThreads) idx[i] = -1;
  for (int i = threadIdx.x; i < a.recent; i += kThreads) kept[K + i] = mass[span + i];
  if (layer == 0 && threadIdx.x == 0) {
    a.counts[b] = K;                 // the same in every layer
    a.stay[b] = STARKV_SEQ_OK;
  }
}

__global__ __launch_bounds__(kThreads) void evict_select(PagedView v, Slots s, EvictArgs a) {
  __shared__ int sh[3][kWaves];
  const int b = blockIdx.x % s.n, layer = blockIdx.x / s.n, slot = s.slot[b];
  const int n = seq_len(v, slot);
  const int want = a.sinks + a.keep;
  if (n <= want + a.recent) {
    for (int i = threadIdx.x; i < want; i += kThreads)
      a.idx[((size_t)layer * s.n + b) * want + i] = -1;
    if (layer == 0 && threadIdx.x == 0) {
      a.counts[b] = 0;
      a.stay[b] = STARKV_SEQ_SHORT;
    }
    return;
  }
  const int span = n - a.recent;
  if (span <= 4 * kThreads) select<4>(v, a, b, layer, s.n, slot, n, sh);
  else if (span <= 16 * kThreads) select<16>(v, a, b, layer, s.n, slot, n, sh);
  else if (span <= 32 * kThreads) select<32>(v, a, b, layer, s.n, slot, n, sh);
  else select<0>(v, a, b, layer, s.n, slot, n, sh);
}

// The masses that stay, where the rows were compacted; one (layer, sequence) to
// a row of blocks.
__global__ __launch_bounds__(256) void evict_masses(PagedView v, Slots s, EvictArgs a,
                                                    const int32_t* status) {
  const int b = blockIdx.x % s.n, layer = blockIdx.x / s.n;
  if (status[b] != STARKV_SEQ_OK) return;
  const int n = a.counts[b] + a.recent;
  const float* kept = a.kept + ((size_t)layer * s.n + b) * (a.sinks + a.keep + a.recent);
  float* mass = mass_row(v, a.mass, layer, s.slot[b]);
  for (int i = blockIdx.y * 256 + threadIdx.x; i < n; i += gridDim.y * 256) mass[i] = kept[i];
}

__global__ __launch_bounds__(256) void mass_fork(PagedView v, Slots s, float* mass) {
  const int b = blockIdx.x % s.n, layer = blockIdx.x / s.n;
  const int n = seq_len(v, s.from[b]);
  const float* from = mass_row(v, mass, layer, s.from[b]);
  float* to = mass_row(v, mass, layer, s.slot[b]);
  for (int i = blockIdx.y * 256 + threadIdx.x; i < n; i += gridDim.y * 256) to[i] = from[i];
}

Slots slots_of(const SeqList& s) {
  Slots l;
  l.n = s.n;
  for (int i = 0; i < s.n; ++i) {
    l.slot[i] = s.slot[i];
    l.from[i] = s.num[i];
  }
  return l;
}
EvictArgs args_of(const EvictCall& c) {
  return EvictArgs{c.mass, c.keep, c.sinks, c.recent, c.idx, c.counts, c.stay, c.kept};
}
// Blocks of 256 that share a row of n floats: as many as fill the card, eight
// floats to a thread at least.
unsigned row_blocks(int64_t pairs, int64_t n) {
  return (unsigned)std::max<int64_t>(1, std::min<int64_t>((n + 2047) / 2048, 2048 / pairs));
}

}  // namespace

int launch_evict_select(const PagedView& v, const EvictCall& c, void* stream) {
  evict_select<<<(unsigned)(v.n_layers * c.s.n), kThreads, 0, reinterpret_cast<hipStream_t>(stream)>>>(
      v, slots_of(c.s), args_of(c));
  return (int)hipGetLastError();
}

int launch_evict_masses(const PagedView& v, const EvictCall& c, const int32_t* status,
                        void* stream) {
  const int64_t pairs = (int64_t)v.n_layers * c.s.n;
  const dim3 grid((unsigned)pairs, row_blocks(pairs, (int64_t)c.keep + c.sinks + c.recent));
  evict_masses<<<grid, 256, 0, reinterpret_cast<hipStream_t>(stream)>>>(v, slots_of(c.s), args_of(c),
                                                                        status);
  return (int)hipGetLastError();
}

int launch_mass_fork(const PagedView& v, const SeqList& s, float* mass, void* stream) {
  const int64_t pairs = (int64_t)v.n_layers * s.n;
  mass_fork<<<dim3((unsigned)pairs, row_blocks(pairs, v.cap)), 256, 0,
              reinterpret_cast<hipStream_t>(stream)>>>(v, slots_of(s), mass);
  return (int)hipGetLastError();
}

}  // namespace starkv
