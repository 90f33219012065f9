// Eviction by accumulated attention weight: of a sequence's masses the largest,
// in the order of their tokens.  The compaction moves their rows, and their masses
// from where they are put aside here.
//
// One block of 16 waves works on a (layer, sequence).  The masses become 32-bit
// keys in the order of the numbers, a wave keeps a range of tokens' keys in its
// registers, and the largest threshold that K keys reach is found bit by bit: a round
// is two instructions per 64 keys, a sum and one barrier, whatever the distribution of
// the masses.  What a round costs is what its 16 waves issue, so once few keys agree
// with the threshold so far they go to one wave, which ends the search alone.  It ends
// early where the count is met.
//
// Bound by that chain, not by the bytes: two sequences of 10,956 and 13,711 tokens in
// 28 layers (56 blocks) 21 us, and 34 before one wave took the last rounds and lanes
// counted their own keys; 16 sequences of up to 1,500 in one layer 10.  The rows' moves
// cost 110 and 6.  Above 32,768 tokens half of the keys lie in LDS (40,941 in 28 layers 61
// us, and about 250 with all keys read again each round), above 65,536 they are read
// again for every two bits (131,072 in one layer 322).
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

// The sum over the 16 lanes of a row, in all of them.
__device__ inline int row_sum(int x) {
  x += __builtin_amdgcn_mov_dpp(x, 0x128, 0xF, 0xF, true);     // the row turned by 8, 4, 2, 1
  x += __builtin_amdgcn_mov_dpp(x, 0x124, 0xF, 0xF, true);
  x += __builtin_amdgcn_mov_dpp(x, 0x122, 0xF, 0xF, true);
  return x + __builtin_amdgcn_mov_dpp(x, 0x121, 0xF, 0xF, true);
}
// The sum over the wave.
__device__ inline int wave_sum(int x) {
  x = row_sum(x);
  return __builtin_amdgcn_readlane(x, 0) + __builtin_amdgcn_readlane(x, 16) + __builtin_amdgcn_readlane(x, 32) +
         __builtin_amdgcn_readlane(x, 48);
}

// Sinks above all, then NaN, then the masses; 0: not to be kept.
constexpr uint32_t kSink = ~0u, kNan = ~0u - 1;
__device__ inline uint32_t key_of(const PagedView& v, int page, float m, int t, int span, int sinks) {
  if (t >= span || page < 0 || page >= v.n_pages) return 0;
  return t < sinks ? kSink : m != m ? kNan : fkey(m + 0.f);      // (-0 counts as 0)
}

// The mass that a key below kNan is of (0 for -0).
__device__ inline float mass_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

// The keys of a wave's tokens [first, first + 64 * count): N to a lane, in registers with
// their masses, or the first 32 in registers and the rest in LDS; or (N = 0) read again each time.
constexpr int kRegs = 32;
template <int N>
struct Keys {
  static constexpr int kHere = N > kRegs ? kRegs : N;
  static constexpr int kLoads = N > 0 && N <= kRegs ? N : 16;      // at once
  uint32_t k[N > 0 ? kHere : 1];
  static constexpr bool kMasses = N > 0 && N <= kRegs;
  float m[kMasses ? N : 1];
  uint32_t* more;                  // [N - kRegs][kThreads]
  const PagedView& v;
  const int32_t* table;
  const float* mass;
  int first, count, span, sinks;

  __device__ inline int token(int j) const { return first + 64 * j + (int)(threadIdx.x & 63); }
  // f(key, mass, j) from j0 on, all loads at once: those behind the last token are of the
  // last, and their keys 0
  template <typename F>
  __device__ inline void read(int j0, F f) const {
    int page[kLoads];
    float x[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int t = min(token(j0 + j), span - 1);
      x[j] = mass[t];
      page[j] = table[t >> v.psh];
    }
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
      f(j0 + j < count ? key_of(v, page[j], x[j], token(j0 + j), span, sinks) : 0, x[j], j0 + j);
  }
  __device__ inline void load() {
#pragma unroll
    for (int j0 = 0; j0 < N; j0 += kLoads)
      read(j0, [&](uint32_t key, float x, int j) {
        if (j < kHere) k[j] = key;
        else more[(j - kRegs) * kThreads + threadIdx.x] = key;
        if constexpr (kMasses) m[j] = x;
      });
  }
  __device__ inline float mass_at(uint32_t key, int j) const { return key < kNan ? mass_of(key) : mass[token(j)]; }
  // f(key, mass, j) for each of them, in the order of the tokens
  template <typename F>
  __device__ inline void each(F f) const {
    if constexpr (N > 0) {
#pragma unroll
      for (int j = 0; j < kHere; ++j) f(k[j], kMasses ? m[j] : mass_at(k[j], j), j);   // (those behind the last are 0)
      if constexpr (N > kRegs) {
#pragma unroll 8
        for (int j = kRegs; j < N; ++j) {
          const uint32_t x = more[(j - kRegs) * kThreads + threadIdx.x];
          f(x, mass_at(x, j), j);
        }
      }
    } else {
      for (int j0 = 0; j0 < count; j0 += kLoads) read(j0, f);
    }
  }
  // How many there are of at least `bound`, in all lanes: each lane counts its own
  // (a ballot and a count of its bits for each 64 keys took three times as long).
  __device__ inline int at_least(uint32_t bound) const {
    int c = 0;
    each([&](uint32_t x, float, int) { c += x >= bound; });
    return wave_sum(c);
  }
  // The same for three bounds, in one pass.
  __device__ inline void at_least(const uint32_t (&bound)[3], int (&c)[3]) const {
    c[0] = c[1] = c[2] = 0;
    each([&](uint32_t x, float, int) {
#pragma unroll
      for (int i = 0; i < 3; ++i) c[i] += x >= bound[i];
    });
#pragma unroll
    for (int i = 0; i < 3; ++i) c[i] = wave_sum(c[i]);
  }
};

// The sums over the block of counts that are the same in all lanes of a wave, each wave's
// read by a lane of every row; and (before) over the waves before this one.  Calls in
// a row take the places `sh` by turns.
using Counts = int2[kWaves];
struct Totals {
  int a, b;
  int2 mine;       // of wave lane % 16
  __device__ inline int before(int x) const {
    return __builtin_amdgcn_readfirstlane(row_sum((threadIdx.x & 15) < threadIdx.x >> 6 ? x : 0));
  }
};
static_assert(kWaves == 16, "a lane of a row to each wave");
__device__ inline Totals block_totals(Counts& sh, int a, int b = 0) {
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = int2{a, b};
  __syncthreads();
  const int2 x = sh[threadIdx.x & 15];
  return Totals{__builtin_amdgcn_readfirstlane(row_sum(x.x)), __builtin_amdgcn_readfirstlane(row_sum(x.y)), x};
}

// The search for the largest T that K keys reach: the bits above `bit` are settled, met
// keys are at T or above, over of them behind those that agree with T.
struct Search {
  int K;
  uint32_t T = 0;
  int met, over = 0, bit = 31;
  __device__ inline bool done() const { return bit < 0 || met == K; }
  // The next bit: c keys are at T | 1 << bit or above.
  __device__ inline uint32_t next() const { return T | 1u << bit; }
  __device__ inline void settle(int c) {
    if (c >= K) {
      T = next();
      met = c;
    } else {
      over = c;
    }
    --bit;
  }
};

// The most keys of the last rounds, 16 to a lane of one wave.
constexpr int kCands = 1024;

template <int N>
__device__ __forceinline__ void select(const PagedView& v, const EvictArgs& a, int b, int layer,
                                       int n_seqs, int slot, int n, Counts* sh, uint32_t* cands,
                                       uint32_t* more) {
  const int want = a.sinks + a.keep, span = n - a.recent;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int per = (span + kThreads - 1) / kThreads;          // groups of 64 tokens of a wave
  const float* mass = mass_row(v, a.mass, layer, slot);
  Keys<N> keys{{}, {}, more, v, v.table + (size_t)slot * v.max_pages, mass, w * per * 64, per, span, a.sinks};
  keys.load();
  int turn = 0;
  int some[3];
  keys.at_least({1, kSink, kSink}, some);
  Totals t = block_totals(sh[turn++ & 1], some[0], some[1]);
  const int here = t.a, K = here - t.b <= a.keep ? here : t.b + a.keep;
  Search f{K, 0, here};
  if (K == here) {
    f.T = 1;
  } else {
    while (!f.done() && f.met - f.over > kCands) {
      if constexpr (N > 0) {
        f.settle(block_totals(sh[turn++ & 1], keys.at_least(f.next())).a);
      } else {
        // two bits of a pass over keys that are read again (31 and 30, 29 and 28, ..)
        const uint32_t half = 1u << (f.bit - 1);
        int c[3];
        keys.at_least({f.T | half, f.T | 2 * half, f.T | 3 * half}, c);
        const Totals lo = block_totals(sh[turn++ & 1], c[0], c[1]), hi = block_totals(sh[turn++ & 1], c[2]);
        f.settle(lo.b);
        if (!f.done()) f.settle(lo.b >= K ? hi.a : lo.a);
      }
    }
    if (!f.done()) {
      const uint32_t mask = f.bit == 31 ? 0u : ~0u << (f.bit + 1);
      const auto agrees = [&](uint32_t x) { return x != 0 && (x & mask) == f.T; };
      int mine = 0;
      keys.each([&](uint32_t x, float, int) { mine += __popcll(__ballot(agrees(x))); });
      t = block_totals(sh[turn++ & 1], mine);
      int at = t.before(t.mine.x);
      keys.each([&](uint32_t x, float, int) {
        const uint64_t agree = __ballot(agrees(x));
        if (agrees(x)) cands[at + __popcll(agree & ((1ull << lane) - 1))] = x;
        at += __popcll(agree);
      });
      __syncthreads();
      if (w == 0) {
        uint32_t few[kCands / 64];
#pragma unroll
        for (int i = 0; i < kCands / 64; ++i) few[i] = 64 * i + lane < t.a ? cands[64 * i + lane] : 0;
        const int over = f.over;          // behind all of the few
        while (!f.done()) {
          const uint32_t next = f.next();
          int c = 0;
#pragma unroll
          for (int i = 0; i < kCands / 64; ++i) c += few[i] >= next;
          f.settle(over + wave_sum(c));
        }
        if (lane == 0) cands[0] = f.T;
      }
      __syncthreads();
      f.T = cands[0];
    }
  }
  const uint32_t T = f.T;
  // all above T, and of those at T the first ones
  keys.at_least({T, T + (T != kSink), kSink}, some);
  const int above = T == kSink ? 0 : some[1];
  t = block_totals(sh[turn++ & 1], above, some[0] - above);
  const int most = K - t.a;
  int seen = t.before(t.mine.y), pos = t.before(t.mine.x) + min(seen, most);
  const size_t row = (size_t)layer * n_seqs + b;
  int32_t* idx = a.idx + row * want;
  float* kept = a.kept + row * (want + a.recent);
  if (K > 0)
    keys.each([&](uint32_t x, float m, int j) {
      const uint64_t below = (1ull << lane) - 1;
      const uint64_t tie = __ballot(x == T);
      const bool take = x > T || (x == T && seen + __popcll(tie & below) < most);
      const uint64_t taken = __ballot(take);
      if (take) {
        const int to = pos + __popcll(taken & below);
        idx[to] = keys.token(j);
        kept[to] = m;
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
  __shared__ Counts sh[2];
  __shared__ uint32_t cands[kCands];
  __shared__ uint32_t more[kRegs * kThreads];       // (a CU holds one block, by its registers)
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
  if (span <= 4 * kThreads) select<4>(v, a, b, layer, s.n, slot, n, sh, cands, more);
  else if (span <= 16 * kThreads) select<16>(v, a, b, layer, s.n, slot, n, sh, cands, more);
  else if (span <= 32 * kThreads) select<32>(v, a, b, layer, s.n, slot, n, sh, cands, more);
  else if (span <= 64 * kThreads) select<64>(v, a, b, layer, s.n, slot, n, sh, cands, more);
  else select<0>(v, a, b, layer, s.n, slot, n, sh, cands, more);
}

// Masses of a forked sequence, a row of blocks to a (layer, sequence): 24,667 tokens'
// in 28 layers 6 us, a launch and two dependent loads.
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

int launch_mass_fork(const PagedView& v, const SeqList& s, float* mass, void* stream) {
  const int64_t pairs = (int64_t)v.n_layers * s.n;
  mass_fork<<<dim3((unsigned)pairs, row_blocks(pairs, v.cap)), 256, 0,
              reinterpret_cast<hipStream_t>(stream)>>>(v, slots_of(s), mass);
  return (int)hipGetLastError();
}

}  // namespace starkv
