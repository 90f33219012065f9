// The attention weights of query rows added up per cached token,
//   add[t] = sum_{i, h} 2^(x[h,t] log2(e) - lse[i,h] log2(e)),  x = q . k / sqrt(d),
// over the rows i that see token t.  K is read once and V not at all; a row's sum
// is known (lse), so no running maximum is needed and the order of the rows is
// free.
//
// The rows are on the side of A of the products and the tokens on the side of B,
// so a lane holds rows of one token: the sum over rows stays in the lane until the
// end, and what lies in a token's place that nobody should see (no page, behind
// the last) spoils no other token.
//
// Few rows (a decoded token, a few drafted ones) are bound by HBM: mass_few takes
// tiles of tokens, K straight to registers, and adds up the groups through LDS.
// Many rows are bound by the matrix units and the exponentials: mass_many keeps 64
// tokens' K in a wave's registers and walks the rows, which all waves read from
// LDS, groups one after the other into the same sums.
//
// Measured, few rows: one token of each of 16 sequences of 500 to 2,747 tokens in 28
// layers 137 us (754 MB, 5.5 TB/s; a copy makes 4.9), of 32 sequences of 37 to 40,941
// in one layer 125 in bf16 (5.5), 43 in 4 bits, 242 in float32; one over 13,711 in 28
// layers 74, 26 and 143, four 85, 40 and 201.  4 bits are bound by what the waves issue.
// Many rows, with the join (5 us): 2,755 over 13,711 tokens 264 to 276 us (244 GFLOP, 880 to
// 920 TFLOP/s), in 4 bits 260, in float32 2,284 (107; a library product makes 154); all of
// 8,192 335 (720); 16 tokens' rows over 13,711 in 28 layers 125, 93 and 498.  The matrix units
// are busy in 41% of the SIMDs' cycles, as in the attention of many rows, and for the
// same reason: 8.9 vector instructions to a product, itself among them, which fill the rest.
#include <algorithm>
#include <type_traits>

#include "device_common.h"
#include "evict.h"

namespace starkv {
namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct MassArgs {
  const char* q;
  const float* lse;
  const float* mass;
  float* out;
  float* part;       // the splits' sums
  int window, sinks;
  int n_rows, blocks, tiles, n_split;
  float scale;       // log2(e) / sqrt(d)
};

// A sequence of the call in one layer.
struct Seq {
  int n, T, first;          // length, query tokens, position of the first (may be negative)
  bool kept;                // the grow before the call left it unchanged: it has no query tokens
  int row0, hpg, R;         // its first row of the call; heads, and rows, of a group
  int slot, layer;
};
__device__ inline Seq seq_of(const PagedView& v, const RowList& r, int layer, int b) {
  Seq s;
  s.slot = r.slot[b];
  s.layer = layer;
  s.n = min(max(const_ints(v.len)[s.slot], 0), v.cap);
  s.row0 = r.row0[b];
  s.T = r.row0[b + 1] - s.row0;
  s.kept = s.T > 0 && r.grown && const_ints(r.grown)[b] != STARKV_SEQ_OK;
  if (s.kept) s.T = 0;
  s.first = s.n - s.T;
  s.hpg = v.H / v.G;
  s.R = s.T * s.hpg;
  return s;
}
__device__ inline size_t first_mass(const PagedView& v, const Seq& s) {
  return ((size_t)s.layer * v.n_slots + s.slot) * v.cap;
}
__device__ inline const int32_t* table_of(const PagedView& v, const Seq& s) {
  return v.table + (size_t)s.slot * v.max_pages;
}
__device__ inline bool is_page(const PagedView& v, int p) { return p >= 0 && p < v.n_pages; }

// Token t's mass with what the rows add to it (nothing to a dropped token,
// whatever was computed in its place).
__device__ inline void store_mass(const PagedView& v, const MassArgs& a, const Seq& s, int t,
                                  float add) {
  const size_t at = first_mass(v, s) + t;
  const float old = t < s.first ? a.mass[at] : 0.f;
  a.out[at] = is_page(v, table_of(v, s)[t >> v.psh]) ? old + add : old;
}
// Whether any row sees any of the tokens [t0, t1).
__device__ inline bool any_sees(const MassArgs& a, const Seq& s, int t0, int t1) {
  // the first row has the widest reach back; every token from it on is seen by its own row
  return !s.kept && (t1 - 1 > max(s.first, 0) - a.window || t0 < a.sinks);
}
// Row position p sees token t.
__device__ inline bool sees(const MassArgs& a, int p, int t) {
  return t <= p && (t > p - a.window || t < a.sinks);
}

// ---------------------------------------------------------------- few rows

template <typename T>
struct Frag;
template <>
struct Frag<__bf16> {
  using type = bf16x8;
  static constexpr int kElems = 8;
  __device__ static inline f32x4 mma(type a, type b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Frag<float> {
  using type = f32x4;
  static constexpr int kElems = 4;
  __device__ static inline f32x4 mma(type a, type b, f32x4 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
  }
};

// The sum over the four lanes of the same l16, in all of them.
__device__ inline float quads_sum(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Four elements' pairs of a 4-bit word, times the scale, exactly.
__device__ inline bf16x8 from_fp4(uint32_t w, float s) {
  u32x4 x;
  x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0));
  x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1));
  x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2));
  x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3));
  return __builtin_bit_cast(bf16x8, x);
}

// A lane's part of a K row: the products may take a row's elements in any order
// that Q's take too.  Plain rows: 16 bytes of every 64; 4 bits: the D/4
// neighbouring elements of the lane's quarter, which are of one scale.
template <typename T, int D, bool F4>
struct KRow {
  using frag = typename Frag<T>::type;
  static constexpr int NF = D / (4 * Frag<T>::kElems);
  frag f[NF];
  __device__ inline void load(const PagedView&, const char* block, int in_page, int quad, int64_t ts) {
    const char* row = block + (int64_t)in_page * ts + 16 * quad;
#pragma unroll
    for (int i = 0; i < NF; ++i) f[i] = *reinterpret_cast<const frag*>(row + 64 * i);
  }
  __device__ inline frag get(int i) const { return f[i]; }
  __device__ static inline int q_byte(int i, int quad) { return 64 * i + 16 * quad; }
};
template <int D>
struct KRow<__bf16, D, true> {
  static constexpr int NF = D / 32;
  uint32_t w[NF];
  uint8_t s;
  __device__ inline void load(const PagedView& v, const char* block, int in_page, int quad, int64_t) {
    using Quarter = std::conditional_t<D == 128, u32x4, uint2>;
    const Quarter got = *reinterpret_cast<const Quarter*>(block + in_page * (D / 2) + quad * (D / 8));
    __builtin_memcpy(w, &got, sizeof w);
    s = *reinterpret_cast<const uint8_t*>(block + v.P * (D / 2) + in_page * (D / 32) + quad * (D / 4) / 32);
  }
  __device__ inline bf16x8 get(int i) const { return from_fp4(w[i], __uint_as_float((uint32_t)s << 23)); }
  __device__ static inline int q_byte(int i, int quad) { return quad * (D / 2) + 16 * i; }
};

// What 16 rows of a group are to a lane: its part of row l16 of Q, and of rows 4*quad
// + e the log-sum and the position (-1: sees nothing).
template <typename T, int D, bool F4>
struct Rows16 {
  using K = KRow<T, D, F4>;
  typename Frag<T>::type q[K::NF];
  float l[4];
  int p[4];
  __device__ inline void load(const PagedView& v, const MassArgs& a, const Seq& s, int g, int r0) {
    const int l16 = threadIdx.x & 15, quad = threadIdx.x >> 4 & 3;
    const size_t at = ((size_t)s.layer * a.n_rows + s.row0) * v.H + g * s.hpg;
    const int mine = min(r0 + l16, s.R - 1), i = mine / s.hpg;
    const char* qr = a.q + (at + (size_t)i * v.H + (mine - i * s.hpg)) * D * sizeof(T);
#pragma unroll
    for (int f = 0; f < K::NF; ++f)
      q[f] = *reinterpret_cast<const typename Frag<T>::type*>(qr + K::q_byte(f, quad));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int row = r0 + 4 * quad + e, r = min(row, s.R - 1), qi = r / s.hpg;
      const float lse = a.lse[at + (size_t)qi * v.H + (r - qi * s.hpg)];
      l[e] = lse * kLog2e;
      p[e] = row < s.R && lse > -INFINITY ? s.first + qi : -1;      // (nor NaN)
    }
  }
  // The lane's rows' weights of token t, whose part of K the lane holds.  `whole`:
  // every row but those that see nothing (p < 0) sees it.
  __device__ inline float weigh(const MassArgs& a, const K& k, int t, bool whole) const {
    f32x4 x{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int f = 0; f < K::NF; ++f) x = Frag<T>::mma(q[f], k.get(f), x);
    float w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = __builtin_amdgcn_exp2f(fmaf(x[e], a.scale, -l[e]));
    if (whole) {
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = __uint_as_float(__float_as_uint(w[e]) & ~(p[e] >> 31));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = sees(a, p[e], t) ? w[e] : 0.f;
    }
    return (w[0] + w[1]) + (w[2] + w[3]);
  }
};

// The token tiles of a call, of kTokens each: those of its sequences in order, layer
// by layer; a block takes every gridDim.x-th, so that all have as many whatever the
// lengths are.  The lanes of a wave know how many tiles come before each sequence.
template <int kTokens>
struct Tiles {
  static constexpr int kPer = kMaxSeqs / 64;
  int before[kPer], count[kPer];
  int all;                   // tiles of a layer
  int next = blockIdx.x;     // the block's next one, in layer `layer`
  int layer = 0;

  __device__ inline Tiles(const PagedView& v, const RowList& r) {
    int mine = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = kPer * (threadIdx.x & 63) + j;
      count[j] = 0;
      if (i < r.n && r.row0[i + 1] > r.row0[i])
        count[j] = (min(max(v.len[r.slot[i]], 0), v.cap) + kTokens - 1) / kTokens;
      mine += count[j];
    }
    const int inc = wave_incl_scan(mine);
    all = __builtin_amdgcn_readlane(inc, 63);
    before[0] = inc - mine;
#pragma unroll
    for (int j = 1; j < kPer; ++j) before[j] = before[j - 1] + count[j - 1];
  }
  // The block's next tile that rows see, of sequence s from token t0 on; the others
  // keep their masses.  False when there is none.
  __device__ inline bool take(const PagedView& v, const MassArgs& a, const RowList& r, Seq* s,
                              int* t0) {
    if (all == 0) return false;
    for (;; next += gridDim.x) {
      while (next >= all) {
        next -= all;
        if (++layer >= v.n_layers) return false;
      }
      int b = 0;
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const uint64_t hit = __ballot(before[j] <= next && next < before[j] + count[j]);
        if (hit) {
          const int lane = __ffsll((unsigned long long)hit) - 1;
          b = kPer * lane + j;
          *t0 = (next - __builtin_amdgcn_readlane(before[j], lane)) * kTokens;
        }
      }
      *s = seq_of(v, r, layer, b);
      if (any_sees(a, *s, *t0, min(*t0 + kTokens, s->n))) break;
      const int t = *t0 + threadIdx.x;
      if (a.out != a.mass && threadIdx.x < kTokens && t < s->n) a.out[first_mass(v, *s) + t] = a.mass[first_mass(v, *s) + t];
    }
    next += gridDim.x;
    return true;
  }
};

// A block takes tiles of S parts of a group, and of all groups' parts each wave a
// quarter, whole groups first.  The next part's K is on its way while one is worked on,
// across tiles.  NB: the 16-row blocks of every sequence, which stay in registers while
// the group does.
template <typename T, int D, bool F4, int NB>      // blocks of a CU
constexpr int kResident = sizeof(T) == 4 && D == 128 ? (NB == 2 ? 2 : 3) : (NB == 1 ? 5 : 4) - (F4 && D == 128);
template <typename T, int D, bool F4>
constexpr int kPart = mass_part(F4, F4 ? D / 2 : (int)sizeof(T) * D);
template <typename T, int D, bool F4, int NB, int S>
__global__ __launch_bounds__(kThreads, (kResident<T, D, F4, NB>)) void mass_few(PagedView v, MassArgs a,
                                                                          RowList r) {
  constexpr int kTokens = S * kPart<T, D, F4>, kHalves = kPart<T, D, F4> / 16;
  static_assert(kTokens <= kThreads, "a thread to each token of a tile");
  struct K {
    KRow<T, D, F4> half[kHalves];
  };
  extern __shared__ float sums[];       // [2][G][kTokens]
  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int parts = v.G * S, per = (parts + 3) / 4;
  const int p0 = wave * per, p1 = min(p0 + per, parts);       // of this wave
  Tiles<kTokens> tiles(v, r);
  Seq s, s1;                            // this tile and the next
  int t0, t1, part = p0, buf = 0;
  bool again = false, whole = false;
  const auto load = [&](const Seq& q, int first, int p, K& k) {
    const int g = p / S;
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      const int t = min(first + kPart<T, D, F4> * (p % S) + 16 * h, (q.n - 1) & ~15);
      const int page = const_ints(table_of(v, q))[t >> v.psh];
      // where there is no page the products are of page 0's, and dropped
      k.half[h].load(v, v.k + (int64_t)q.layer * v.ls + (int64_t)(is_page(v, page) ? page : 0) * v.ps +
                            (int64_t)g * v.gs,
                     (t & (v.P - 1)) + l16, quad, v.ts);
    }
  };
  const auto begin = [&]() {
    const int te = min(t0 + kTokens, s.n);
    whole = te - 1 <= s.first && (t0 > s.n - 1 - a.window || te <= a.sinks);
  };
  Rows16<T, D, F4> rows[NB];
  int row_layer = -1, row_slot = -1, row_g = -1;
  // the wave's next part, K of which is in `k`; K of the one behind it comes into
  // `ahead`.  False behind the last
  const auto step = [&](K& k, K& ahead) {
    const int g = part / S;
    const bool last = part + 1 >= p1;
    if (part < p1 && (g != row_g || s.slot != row_slot || s.layer != row_layer)) {
#pragma unroll
      for (int i = 0; i < NB; ++i) rows[i].load(v, a, s, g, 16 * i);
      __builtin_amdgcn_s_waitcnt(0x0F70);   // here, and not behind the next K below
      row_g = g;
      row_slot = s.slot;
      row_layer = s.layer;
    }
    if (last) again = tiles.take(v, a, r, &s1, &t1);
    if (!last) load(s, t0, part + 1, ahead);
    else if (again && p0 < p1) load(s1, t1, p0, ahead);
    float* const mine = sums + buf * v.G * kTokens;
    if (part < p1) {
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        const int in_tile = kPart<T, D, F4> * (part % S) + 16 * h + l16, t = t0 + in_tile;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NB; ++i) sum += rows[i].weigh(a, k.half[h], t, whole);
        sum = quads_sum(sum);
        if (quad == 0) mine[g * kTokens + in_tile] = sum;
      }
    }
    ++part;
    if (!last) return true;
    __syncthreads();
    const int t = t0 + threadIdx.x;
    if (threadIdx.x < kTokens && t < s.n) {
      float add = 0.f;
      for (int i = 0; i < v.G; ++i) add += mine[i * kTokens + threadIdx.x];
      store_mass(v, a, s, t, add);
    }
    s = s1;
    t0 = t1;
    part = p0;
    buf ^= 1;
    begin();
    return again;
  };
  if (!tiles.take(v, a, r, &s, &t0)) return;
  begin();
  K ka, kb;
  if (p0 < p1) load(s, t0, p0, ka);
  while (step(ka, kb) && step(kb, ka)) {
  }
}

// --------------------------------------------------------------- many rows

constexpr int kTile = kMassTile;   // tokens of a block, 64 to a wave
static_assert(kTile == kThreads, "a thread to each token of a tile");
constexpr int kStage = 64;         // rows of a stage
constexpr int kRing = 3;           // stages in LDS: this one, the next, and one that is loading

// Where 16-byte piece c of a row of Q lies in LDS: the lanes of a read, which
// differ in the row, meet different banks.
template <int D>
__device__ constexpr int q_swizzle(int row) {
  return D == 128 ? row & 15 : (row >> 1) & 7;
}

// The masses of a kept sequence, where they are to go elsewhere: one block's tiles.
__device__ inline void keep_masses(const PagedView& v, const MassArgs& a, const Seq& s, int tile, int split) {
  if (!s.kept || a.out == a.mass || split) return;
  const size_t at = first_mass(v, s);
  for (int64_t t = (int64_t)tile * kTile + threadIdx.x; t < s.n; t += (int64_t)a.blocks * kTile)
    a.out[at + t] = a.mass[at + t];
}

// What a block does of a tile: `w0` to `w1` of the products of 32 rows of a group that
// see some of it, group after group.
struct Share {
  int t0;            // the tile's first token
  int p0, p1;        // products of a group
  int64_t w0, w1;
  bool joined;       // its sums are added to other blocks' afterwards

  // False: nothing, others do it.
  __device__ inline bool take(const PagedView& v, const MassArgs& a, const Seq& s, int tile, int split) {
    // tiles behind the bound that the splits' sums were sized by are not split
    joined = a.n_split > 1 && tile < a.tiles;
    if (!joined && split) return false;
    t0 = tile * kTile;
    // from the row at t0 to the last one whose window reaches back to the tile's end
    const int t1 = min(t0 + kTile, s.n), i0 = max(t0 - s.first, 0);
    const int64_t reach = t0 < a.sinks ? s.T - 1 : (int64_t)t1 - 1 + a.window - 1 - s.first;
    const int i1 = (int)min(reach, (int64_t)s.T - 1);
    p0 = i0 * s.hpg / 32;
    p1 = i1 < i0 ? p0 : ((i1 + 1) * s.hpg + 31) / 32;
    const int64_t all = (int64_t)v.G * (p1 - p0);
    w0 = joined ? all * split / a.n_split : 0;
    w1 = joined ? all * (split + 1) / a.n_split : all;
    return true;
  }
  // The products [from, to) of the next group.
  __device__ inline bool next(int* g, int* from, int* to) {
    if (w0 >= w1) return false;
    *g = (int)(w0 / (p1 - p0));
    *from = p0 + (int)(w0 - (int64_t)*g * (p1 - p0));
    *to = (int)min((int64_t)p1, *from + w1 - w0);
    w0 += *to - *from;
    return true;
  }
  __device__ inline void store(const PagedView& v, const MassArgs& a, const Seq& s, int pair, int split,
                               int t, float add) const {
    if (joined)
      a.part[((size_t)pair * a.n_split + split) * a.tiles * kTile + t] = add;
    else if (t < s.n)
      store_mass(v, a, s, t, add);
  }
};

template <int D, bool F4>
__global__ __launch_bounds__(kThreads, 2) void mass_many(PagedView v, MassArgs a, RowList r) {
  constexpr int NF = D / 16, NP = D / 8, kRow = D * 2;
  constexpr int kLoads = kStage * NP / kThreads;          // 16-byte pieces of a thread per stage
  constexpr int kLoadRows = kThreads / NP;
  // (three arrays, so that a read of one need not wait for loads into another)
  __shared__ __align__(1024) char q0[kStage * kRow], q1[kStage * kRow], q2[kStage * kRow];
  __shared__ __align__(16) float ls[kRing][kStage];       // lse log2(e); infinite behind the last row
  __shared__ __align__(16) int ps[kRing][kStage];         // the rows' positions; -1: sees nothing
  __shared__ int span[kRing][2][2];                       // the least (-1: some see nothing) and largest of 32

  const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int split = blockIdx.x % a.n_split, at = blockIdx.x / a.n_split;
  const int pair = at / a.blocks, b = pair % r.n, layer = pair / r.n;
  const Seq s = seq_of(v, r, layer, b);
  if (s.T == 0) {
    keep_masses(v, a, s, at % a.blocks, split);
    return;
  }
  const size_t row_at = ((size_t)layer * a.n_rows + s.row0) * v.H;
  // x / hpg is the upper half of x * per_head for x < 2^20 (hpg is under 2^12)
  const uint32_t per_head = (uint32_t)(((1ull << 32) + s.hpg - 1) / s.hpg);

  // (the first tile moves on with the sequence and the layer: the XCDs take the blocks by
  // turns, and those of the last tiles, which short sequences do not have, are spread over
  // them; 40 rows of 4 sequences in 28 layers 240 -> 207 us)
  for (int tile = (at % a.blocks + b + layer) % a.blocks; (int64_t)tile * kTile < s.n; tile += a.blocks) {
    Share share;
    if (!share.take(v, a, s, tile, split)) continue;
    const int t0 = share.t0;
    float sum[2][2] = {};
    // K of the wave's tokens: a lane holds half a row of tokens l32 and 32 + l32
    const char* rows_of[2];           // in group 0's block
    const char* scales_of[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int t = min(t0 + 64 * wave + 32 * h + l32, s.n - 1);
      const int page = table_of(v, s)[t >> v.psh], in_page = t & (v.P - 1);
      const char* block = v.k + (int64_t)layer * v.ls + (int64_t)(is_page(v, page) ? page : 0) * v.ps;
      rows_of[h] = block + (int64_t)in_page * v.ts + half * (F4 ? D / 4 : kRow / 2);
      scales_of[h] = block + v.P * (D / 2) + in_page * (D / 32) + half * (D / 64);
    }
    int g, from, to;
    while (share.next(&g, &from, &to)) {
      bf16x8 kf[2][NF];
      // Rows 32*from.. in stages of 64, asked for in order: query token i0 and head h0
      // are the stage's first row, and row x behind it is head (h0 + x) % hpg of token
      // i0 + (h0 + x) / hpg; rows behind the last repeat it.  A thread's pieces are of
      // rows kLoadRows apart, whose places in LDS are permuted alike
      const int piece = threadIdx.x % NP, sub = threadIdx.x / NP;
      const size_t group_at = row_at + g * s.hpg;
      const uint32_t at_piece = (piece ^ q_swizzle<D>(sub)) * 16;
      static_assert(q_swizzle<D>(kLoadRows) == 0, "whole turns of the swizzle");
      int first = 32 * from, i0 = first / s.hpg, h0 = first - i0 * s.hpg;
      const int ahead_i = kStage / s.hpg, ahead_h = kStage - ahead_i * s.hpg;
      // of wave 0's lanes: a row's query token, and its log-sum, read a stage ahead
      int lrow = 32 * from + lane, li = lrow / s.hpg, lhead = lrow - li * s.hpg;
      const auto log_sum = [&](int more) {        // of `more` stages behind
        const int row = lrow + more * kStage;
        int i = li + more * ahead_i, head = lhead + more * ahead_h;
        for (int j = 0; j < more; ++j)
          if (head >= s.hpg) {
            head -= s.hpg;
            ++i;
          }
        return row < s.R ? a.lse[group_at + (size_t)i * v.H + head] : -INFINITY;
      };
      const auto put_sums = [&](int buf, float lse) {
        // (also for the rows behind the last, and where the sum is NaN)
        const bool none = !(lse > -INFINITY);
        const float l = none ? INFINITY : lse * kLog2e;
        const int p = none ? -1 : s.first + li;
        ls[buf][lane] = l;
        ps[buf][lane] = p;
        // positions rise with the rows: the first and the last of each 32, or -1
        // where one sees nothing
        const uint64_t dead = __ballot(p < 0);
        if (l32 == 0) span[buf][half][0] = (uint32_t)(dead >> (32 * half)) ? -1 : p;
        if (l32 == 31) span[buf][half][1] = p;
        lrow += kStage;
        li += ahead_i;
        lhead += ahead_h;
        if (lhead >= s.hpg) {
          lhead -= s.hpg;
          ++li;
        }
      };
      const auto load_rows = [&](char* to) {
        const char* const at = a.q + (group_at + (size_t)i0 * v.H) * kRow;
        const int last = h0 + s.R - 1 - first;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          const uint32_t x = min(h0 + sub + j * kLoadRows, last), i = s.hpg == 1 ? x : __umulhi(x, per_head);
          const uint32_t off = (i * (uint32_t)(v.H - s.hpg) + x) * kRow + at_piece;
          __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(at + off),
                                           (__attribute__((address_space(3))) void*)(to + (wave * 64 / NP + j * kLoadRows) * kRow),
                                           16, 0, 0);
        }
        first += kStage;
        i0 += ahead_i;
        h0 += ahead_h;
        if (h0 >= s.hpg) {
          h0 -= s.hpg;
          ++i0;
        }
      };
      // A step takes the weights of one 32-row product while the next runs on the
      // matrix units: x holds product j, y becomes product j + 1
      const int rows = to - from;           // products
      const int tw = t0 + 64 * wave, te = min(tw + 64, s.n);        // the wave's tokens
      using Product = f32x16[2];
      Product x, y;
      const auto q_frag = [&](const char* qs, int u, int f) {
        const int row = 32 * u + l32;
        return *reinterpret_cast<const bf16x8*>(qs + row * kRow + (((half * NP / 2 + f) ^ q_swizzle<D>(row)) * 16));
      };
      // the weights of x, half u of stage `buf`, beside the product y of the rows at
      // qn, half un
      const auto step = [&](Product& x, int buf, int u, Product& y, const char* qn, int un) {
        f32x4 l4[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) l4[e] = *reinterpret_cast<const f32x4*>(&ls[buf][32 * u + 8 * e + 4 * half]);
        // unless all rows see all tokens of the wave that there are
        const int p_first = __builtin_amdgcn_readfirstlane(span[buf][u][0]);
        const int p_last = __builtin_amdgcn_readfirstlane(span[buf][u][1]);
        if (te - 1 > p_first || !(tw > p_last - a.window || te <= a.sinks)) {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int p = ps[buf][32 * u + 8 * (e >> 2) + 4 * half + (e & 3)];
#pragma unroll
            for (int h = 0; h < 2; ++h) x[h][e] = sees(a, p, tw + 32 * h + l32) ? x[h][e] : -INFINITY;
          }
        }
        constexpr int kShare = 32 / NF;
        bf16x8 qf[NF];
        qf[0] = q_frag(qn, un, 0);
        qf[1] = q_frag(qn, un, 1);
#pragma unroll
        for (int f = 0; f < NF; ++f) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
            y[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[f], kf[h][f], f ? y[h] : f32x16{}, 0, 0, 0);
          if (f + 2 < NF) qf[f + 2] = q_frag(qn, un, f + 2);
#pragma unroll
          for (int i = 0; i < kShare; ++i) {
            const int w = kShare * f + i, e = w >> 1, h = w & 1;
            sum[h][e & 1] += __builtin_amdgcn_exp2f(fmaf(x[h][e], a.scale, -l4[e >> 2][e & 3]));
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      const auto landed = [&]() {
        __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
        __syncthreads();
      };
      // (all loads at once: the first two stages' rows and log-sums, and K)
      __syncthreads();                        // the rows before are done with
      load_rows(q0);
      if (rows > 2) load_rows(q1);
      float lse = 0.f, lse0 = 0.f, lse1 = 0.f;
      if (wave == 0) {
        lse0 = log_sum(0);
        lse1 = log_sum(1);
        lse = log_sum(2);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const char* row = rows_of[h] + (int64_t)g * v.gs;
        if constexpr (F4) {
          const char* scales = scales_of[h] + (int64_t)g * v.gs;
#pragma unroll
          for (int f = 0; f < NF; f += 4) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(row + 4 * f);
            const float sc = __uint_as_float((uint32_t)*reinterpret_cast<const uint8_t*>(scales + f / 4) << 23);
#pragma unroll
            for (int e = 0; e < 4; ++e) kf[h][f + e] = from_fp4(w[e], sc);
          }
        } else {
#pragma unroll
          for (int f = 0; f < NF; ++f) kf[h][f] = *reinterpret_cast<const bf16x8*>(row + 16 * f);
        }
      }
      if (wave == 0) {
        put_sums(0, lse0);
        put_sums(1, lse1);
      }
      const auto stage = [&](char* to, int buf) {
        // (before the loads into LDS: what waits for the log-sums waits for all loads before)
        if (wave == 0) {
          put_sums(buf, lse);
          lse = log_sum(0);
        }
        load_rows(to);
      };
      landed();
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          x[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q_frag(q0, 0, f), kf[h][f], f ? x[h] : f32x16{}, 0, 0, 0);
      // stage products j and j + 1; behind the last come products of whatever LDS
      // holds, and nobody reads them
      const auto two = [&](int j, const char* q, int buf, const char* qn, char* free, int free_buf) {
        // the next stage has landed, and every wave is done with the one before
        if (j) landed();
        if (j + 4 < rows) stage(free, free_buf);
        step(x, buf, 0, y, q, 1);
        if (j + 1 < rows) step(y, buf, 1, x, qn, 0);
      };
      for (int j = 0; j < rows; j += 6) {
        two(j, q0, 0, q1, q2, 2);
        if (j + 2 < rows) two(j + 2, q1, 1, q2, q0, 0);
        if (j + 4 < rows) two(j + 4, q2, 2, q0, q1, 1);
      }
    }
    // the two halves' rows; lane l32 of half h writes token 32 h + l32
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      sum[h][0] += sum[h][1];
      sum[h][0] += __shfl_xor(sum[h][0], 32);
    }
    const int t = t0 + 64 * wave + lane;
    share.store(v, a, s, pair, split, t, half ? sum[1][0] : sum[0][0]);
  }
}

// float32: as above, with a wave's 64 tokens as four times 16 and the rows straight to
// registers, 16 at a time: the matrix units take 16 times as long for a row as in bf16,
// and a CU's other waves have them while one waits.
template <int D>
__global__ __launch_bounds__(kThreads, 2) void mass_many_f32(PagedView v, MassArgs a, RowList r) {
  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int split = blockIdx.x % a.n_split, at = blockIdx.x / a.n_split;
  const int pair = at / a.blocks, b = pair % r.n, layer = pair / r.n;
  const Seq s = seq_of(v, r, layer, b);
  if (s.T == 0) {
    keep_masses(v, a, s, at % a.blocks, split);
    return;
  }
  for (int tile = (at % a.blocks + b + layer) % a.blocks; (int64_t)tile * kTile < s.n; tile += a.blocks) {
    Share share;
    if (!share.take(v, a, s, tile, split)) continue;
    const int tw = share.t0 + 64 * wave, te = min(tw + 64, s.n);      // the wave's tokens
    float sum[4] = {};
    int g, from, to;
    while (share.next(&g, &from, &to)) {
      KRow<float, D, false> k[4];
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const int t = min(tw + 16 * h + l16, s.n - 1), page = table_of(v, s)[t >> v.psh];
        k[h].load(v, v.k + (int64_t)layer * v.ls + (int64_t)(is_page(v, page) ? page : 0) * v.ps +
                         (int64_t)g * v.gs,
                  t & (v.P - 1), quad, v.ts);
      }
      const int end = min(32 * to, s.R);
      for (int r0 = 32 * from; r0 < end; r0 += 16) {
        Rows16<float, D, false> rows;
        rows.load(v, a, s, g, r0);
        const int p_first = s.first + r0 / s.hpg, p_last = s.first + min(r0 + 15, s.R - 1) / s.hpg;
        const bool whole = te - 1 <= p_first && (tw > p_last - a.window || te <= a.sinks);
#pragma unroll
        for (int h = 0; h < 4; ++h) sum[h] += rows.weigh(a, k[h], tw + 16 * h + l16, whole);
      }
    }
#pragma unroll
    for (int h = 0; h < 4; ++h) sum[h] = quads_sum(sum[h]);
    // lane l16 of quad h writes token 16 h + l16
    const float lo = quad & 1 ? sum[1] : sum[0], hi = quad & 1 ? sum[3] : sum[2];
    share.store(v, a, s, pair, split, tw + lane, quad & 2 ? hi : lo);
  }
}

// The splits' sums of the tokens within the bound, one after the other.
__global__ __launch_bounds__(kThreads) void mass_join(PagedView v, MassArgs a, RowList r) {
  const int b = blockIdx.x % r.n, layer = blockIdx.x / r.n;
  const Seq s = seq_of(v, r, layer, b);
  if (s.T == 0) return;
  const int bound = a.tiles * kTile;
  const float* part = a.part + (size_t)blockIdx.x * a.n_split * bound;
  for (int t = blockIdx.y * kThreads + threadIdx.x; t < min(s.n, bound); t += gridDim.y * kThreads) {
    float add[4] = {};
    // 16 loads at once: the join waits for little else (four at a time 11 us where
    // 16 take 7, 32 splits of 13,711 tokens)
    for (int i = 0; i < a.n_split; i += 16) {
      float x[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) x[j] = part[(size_t)min(i + j, a.n_split - 1) * bound + t];
#pragma unroll
      for (int j = 0; j < 16; ++j) add[j & 3] += i + j < a.n_split ? x[j] : 0.f;
    }
    store_mass(v, a, s, t, (add[0] + add[1]) + (add[2] + add[3]));
  }
}

template <int I>
using Int = std::integral_constant<int, I>;
template <typename T>
struct Type {
  using type = T;
};

}  // namespace

int launch_mass_add(const PagedView& v, const MassCall& c, void* stream) {
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  MassArgs a;
  a.q = static_cast<const char*>(c.q);
  a.lse = c.lse;
  a.mass = c.mass;
  a.out = c.out;
  a.part = c.part;
  a.window = c.window;
  a.sinks = c.sinks;
  a.n_rows = c.s.n_rows;
  a.blocks = c.s.blocks;
  a.tiles = c.s.tiles;
  a.n_split = c.s.n_split;
  a.scale = kLog2e / sqrtf((float)v.d);
  if (c.s.many) {
    const unsigned pairs = (unsigned)(v.n_layers * c.r.n);
    const unsigned blocks = pairs * c.s.blocks * c.s.n_split;
    const auto go = [&](auto kernel) { kernel<<<blocks, kThreads, 0, st>>>(v, a, c.r); };
    if (v.esz == 4) v.d == 128 ? go(mass_many_f32<128>) : go(mass_many_f32<64>);
    else if (v.d == 128) v.fp4 ? go(mass_many<128, true>) : go(mass_many<128, false>);
    else v.fp4 ? go(mass_many<64, true>) : go(mass_many<64, false>);
    if (c.s.n_split > 1) {
      const unsigned parts = (unsigned)std::min(c.s.tiles, std::max(1, (int)(2048 / pairs)));
      mass_join<<<dim3(pairs, parts), kThreads, 0, st>>>(v, a, c.r);
    }
    return (int)hipGetLastError();
  }
  const size_t lds = (size_t)2 * v.G * c.s.tile * sizeof(float);
  if (c.s.tile < 1 || lds > 64 * 1024 || c.s.row_blocks < 1 || c.s.row_blocks > 2) return (int)hipErrorInvalidValue;
  bool made = true;          // a kernel for the division
  const auto by_tile = [&](auto t, auto d, auto f4, auto nb) {
    using T = typename decltype(t)::type;
    constexpr int D = decltype(d)::value, NB = decltype(nb)::value;
    constexpr bool F4 = decltype(f4)::value;
    const unsigned blocks = (unsigned)std::min<int64_t>(c.s.blocks, 256 * kResident<T, D, F4, NB>);
    const auto go = [&](auto kernel) { kernel<<<blocks, kThreads, lds, st>>>(v, a, c.r); };
    constexpr int kMost = kMassTile / kPart<T, D, F4>;
    if (c.s.tile == kPart<T, D, F4>) go(mass_few<T, D, F4, NB, 1>);
    else if (c.s.tile == 4 * kPart<T, D, F4>) go(mass_few<T, D, F4, NB, 4>);
    else if (c.s.tile == kMassTile) go(mass_few<T, D, F4, NB, kMost>);
    else made = false;
  };
  const auto by_rows = [&](auto t, auto d, auto f4) {
    if (c.s.row_blocks == 1) by_tile(t, d, f4, Int<1>{});
    else by_tile(t, d, f4, Int<2>{});
  };
  const auto by_type = [&](auto d) {
    if (v.fp4) by_rows(Type<__bf16>{}, d, std::true_type{});
    else if (v.esz == 2) by_rows(Type<__bf16>{}, d, std::false_type{});
    else by_rows(Type<float>{}, d, std::false_type{});
  };
  v.d == 128 ? by_type(Int<128>{}) : by_type(Int<64>{});
  return made ? (int)hipGetLastError() : (int)hipErrorInvalidValue;
}

}  // namespace starkv
