// Attention over the pages of a cache: for the query rows of a sequence,
//   o = sum_t softmax_t(q . k_t / sqrt(d)) v_t  over the tokens a row sees
// (a tree's mask, or a sliding window with sinks), in one pass over the
// tokens with a running maximum m and sum l per row:
//   m' = max(m, x), l' = l 2^(m-m') + sum 2^(x-m'), o' = o 2^(m-m') + sum 2^(x-m') v.
//
// Few rows (one token, a small tree) read each K and V row once for all the
// rows of the KV group, so the pass is bound by HBM.  A block takes 16*NB
// rows and one split of the tokens; its four waves take steps of 32 tokens in
// turn and are joined through LDS, and a second kernel joins the splits.
//
// Both products run on 16x16 MFMAs with the tokens on the side of A and the
// rows on the side of B, straight from registers:
//   S^T = K Q^T   lane (quad, l16) gets tokens 4*quad + 0..3 of row l16, so
//                 the softmax of a row stays in four lanes, two shuffles;
//   O^T = V^T P^T the lane's own weights are its part of B as they are, with
//                 k = 8*quad + j standing for token 4*quad + j of the step's
//                 first 16 (j < 4) or of its last (j >= 4).  A needs eight
//                 tokens of one column per lane: the lane reads 16 bytes, eight
//                 columns, of each of its eight tokens and swaps them into eight
//                 fragments with 32 v_perm, so V needs no LDS either.
// float32 caches run the same scheme on the 16x16x4 MFMA, four per 16 bytes,
// and are bound by it from a few tiles of rows on.
//
// Measured, with the join: one token of each of 32 sequences of 37 to 40,941
// tokens under a window of 4,096 and 4 sinks (252 MB) 46 to 55 us, the kernel
// itself 41 to 45 (5.6 to 6.1 TB/s; a copy makes 4.9); one token over 13,711 in
// 28 layers 142 us (5.5 TB/s), a tree of four 150; over 700 in one layer 11 us,
// the two launches and their chains of loads.  float32: one token over 13,711 in
// 28 layers 271 us (5.8 TB/s), one of each of 16 sequences of 3,000 to 12,000 116
// (4.2); 4 trees of up to 13 tokens in 4 layers 35, 8 trees of up to 48 over
// 1,664 to 39,197 tokens 347 (57 TFLOP/s of 154); a chunk of 1,000 tokens behind
// 12,711 2,502 (76).  4 bits: one token over 40,941 in 28 layers 118 us (624 MB, 5.3
// TB/s), over 13,711 40, where bf16 takes 143; one of each of 32 sequences of 37 to
// 40,941 tokens 89 (357 MB, 4.0); over 600 in one layer 11; trees of seven (28 rows
// of 64 elements) of 16 sequences of 500 to 13,711 tokens 24.
#include <algorithm>
#include <type_traits>

#include "attend.h"

namespace starkv {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kStep = 32;         // tokens of a step

// 16-byte fragments of a K or Q row and their product.
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

// A lane's columns of one V row: column C*l16 + e of each of NV loads.
template <typename T, int D>
struct VRow;
template <>
struct VRow<__bf16, 128> {
  typedef uint32_t type __attribute__((ext_vector_type(4)));
  static constexpr int kLoads = 1, kCols = 8;
};
template <>
struct VRow<__bf16, 64> {
  typedef uint32_t type __attribute__((ext_vector_type(2)));
  static constexpr int kLoads = 1, kCols = 4;
};
template <>
struct VRow<float, 128> {
  typedef uint32_t type __attribute__((ext_vector_type(4)));
  static constexpr int kLoads = 2, kCols = 4;
};
template <>
struct VRow<float, 64> {
  typedef uint32_t type __attribute__((ext_vector_type(4)));
  static constexpr int kLoads = 1, kCols = 4;
};

// What a lane loads of a 4-bit step: the row of K of each 16-token half that it
// holds for the products and that row's scale, and its columns of eight rows of
// V and of four rows' scales at a time.
template <int D>
struct Fp4Step {
  using KRow = std::conditional_t<D == 128, i32x4, uint2>;      // D/4 elements
  using VRow = std::conditional_t<D == 128, uint32_t, uint16_t>;  // D/16 elements
  using Scales = std::conditional_t<D == 128, i32x4, uint2>;    // four rows of D/32 bytes
  KRow k[2];
  uint8_t ks[2];
  VRow v[8];
  Scales vs[2];
};
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// Elements 2i and 2i + 1 of w, times 2^(byte - 127) (NaN for 255), exactly.
template <int I>
__device__ inline uint32_t from_fp4(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, I));
}

__device__ inline float max4(f32x4 v) { return fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])); }

// The largest over the four lanes of the same l16, in all of them.
__device__ inline float quads_max(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Any of the lane's V elements an infinity or NaN.
template <typename T, typename R>
__device__ inline bool any_not_finite(const R& r) {
  constexpr int n = sizeof(R) / 4;
  bool bad = false;
#pragma unroll
  for (int w = 0; w < n; ++w) {
    if constexpr (sizeof(T) == 2)
      bad |= (r[w] & 0x7F80u) == 0x7F80u || (r[w] & 0x7F800000u) == 0x7F800000u;
    else
      bad |= (r[w] & 0x7F800000u) == 0x7F800000u;
  }
  return bad;
}
template <typename T, typename R>
__device__ inline void zero_not_finite(R& r) {
  constexpr int n = sizeof(R) / 4;
#pragma unroll
  for (int w = 0; w < n; ++w) {
    if constexpr (sizeof(T) == 2) {
      if ((r[w] & 0x7F80u) == 0x7F80u) r[w] &= 0xFFFF0000u;
      if ((r[w] & 0x7F800000u) == 0x7F800000u) r[w] &= 0xFFFFu;
    } else if ((r[w] & 0x7F800000u) == 0x7F800000u) {
      r[w] = 0;
    }
  }
}

// Two blocks to a CU at least: the registers then all come from one file, none
// is copied, and two or three blocks fit where one or two did (eight trees of
// four tokens 33.2 -> 27.5 us, four layers of 22 sequences 105 -> 86).
//
// F4: a cache of 4 bits.  Its elements become bf16, exactly, by the hardware's
// conversion, two at a time, as the fragments are made, and all else is the
// same.  K's products may take the elements of a row in any order that Q's take
// too: lane quad holds the D/4 neighbouring ones that it reads at once, which are
// of one scale.  A step is a quarter of bf16's bytes for more instructions (201 of
// vectors, 16 products among them, and 97 scalar ones for 32 tokens), so its rows are asked
// for while the step before is worked on.  (Made into bf16 only where they are used, which leaves
// registers for a third block on a CU, they took 95 us of 32 sequences and 129 of 28
// layers, where this takes 93 and 127.)
// kOnePage: pages of 32 tokens or more, so that a step lies in one.
template <typename T, int D, int NB, bool F4 = false, bool kOnePage = false>
__global__ __launch_bounds__(kThreads, 2) void attend_few(PagedView v, AttendArgs a, AttendLists s,
                                                       unsigned run) {
  using F = Frag<T>;
  using frag = typename F::type;
  using VR = VRow<T, D>;
  using vrow = typename VR::type;
  constexpr int kBlk = 4 * F::kElems;           // elements of d per fragment over the quads
  constexpr int NF = D / kBlk;                  // fragments of a row
  constexpr int ND = D / 16;                    // 16-column tiles of the output
  constexpr int kRows = 16 * NB;
  __shared__ __align__(16) float ow[kWaves][16][D + 4];
  __shared__ float2 st[kWaves][16];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, quad = lane >> 4;
  // `run` tiles of one split of a (layer, group) follow each other: they read
  // the same K and V.  All (layer, group)s of a run are together and the
  // splits, of which short sequences have fewer, come last, so that each XCD
  // gets the same share of every sequence.  With the splits first it got every
  // eighth item, of 2, 4 or 8 splits always the same (one token of five
  // sequences of 1,000 to 5,000 tokens in 28 layers 234 us and now 167, of 64
  // sequences in one 94 and 85)
  const unsigned item = xcd_item(blockIdx.x, run);
  const unsigned lgs = v.n_layers * v.G, runs = (a.n_tiles + run - 1) / run, at_run = item / run;
  const int lg = at_run % lgs, split = at_run / lgs / runs;
  const int tile = at_run / lgs % runs * run + item % run;
  if (split >= a.n_split || tile >= a.n_tiles) return;
  const int unit = lg * a.n_tiles + tile;
  const int g = lg % v.G, layer = lg / v.G;
  const int b = tile_owner(s.tile0, s.r.n, tile);
  const TokenSpan ts = token_span<kStep>(v, a, s, b, tile, kRows);
  const int live = (ts.nt + ts.per - 1) / ts.per;     // splits with tokens
  if (split >= max(live, 1)) return;
  const int hpg = v.H / v.G;
  const int r0 = (tile - s.tile0[b]) * kRows;
  const int rows = ts.T * hpg;
  const AllSee all = all_see(a, ts, r0 / hpg, min(r0 + kRows - 1, rows - 1) / hpg);

  // this lane's row of each 16-row block: query token qi (its rows past the
  // last repeat the last, and are not written)
  frag qf[NB][NF];
  int qi[NB];
  const char* qbase = a.q + ((size_t)layer * a.n_rows + ts.row0) * v.H * D * sizeof(T);
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int r = min(r0 + 16 * nb + l16, rows - 1);
    qi[nb] = r / hpg;
    const char* qr = qbase + ((size_t)qi[nb] * v.H + g * hpg + r % hpg) * D * sizeof(T) +
                     (F4 ? D / 2 : 16) * quad;
#pragma unroll
    for (int f = 0; f < NF; ++f) qf[nb][f] = *reinterpret_cast<const frag*>(qr + (F4 ? 16 : 64) * f);
  }

  float m[NB], l[NB];        // maximum; this lane's part of the sum
  f32x4 o[NB][ND];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    m[nb] = -INFINITY;
    l[nb] = 0.f;
#pragma unroll
    for (int t = 0; t < ND; ++t) o[nb][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const const_i32* table = const_ints(v.table + (size_t)s.r.slot[b] * v.max_pages);
  const int64_t base = (int64_t)layer * v.ls + (int64_t)g * v.gs;
  const int u1 = min((split + 1) * ts.per, ts.nt);
  // the page of a step's 16-token half, read a step before its use
  const auto page_of = [&](int u, int h) {
    const int t = step_token<kStep>(ts, min(u, ts.nt - 1)) + 16 * h;
    return table[min(t, ts.n - 1) >> v.psh];
  };
  int u = split * ts.per + wave, next0 = 0, next1 = 0;
  if (u < u1) {
    next0 = page_of(u, 0);
    next1 = page_of(u, 1);
  }
  // 4 bits: a step's rows are read while the step before is worked on
  [[maybe_unused]] Fp4Step<D> ahead;
  // the lane's bytes behind those of a half's first row
  [[maybe_unused]] const uint32_t k_at = l16 * (D / 2) + quad * (D / 8);
  [[maybe_unused]] const uint32_t ks_at = l16 * (D / 32) + quad * (D / 4) / 32;
  [[maybe_unused]] const uint32_t v_at = 4 * quad * (D / 2) + l16 * (D / 32), vs_at = 4 * quad * (D / 32);
  [[maybe_unused]] const auto fetch = [&](int w, int p0, int p1) {
    using S = Fp4Step<D>;
    const int at0 = step_token<kStep>(ts, min(w, ts.nt - 1));
    const char *kr, *vr, *ksr, *vsr;       // a half's first rows and their scales
    const auto rows_at = [&](int page, int in_page) {
      const int64_t at = base + (int64_t)(page >= 0 && page < v.n_pages ? page : 0) * v.ps;
      kr = v.k + at + in_page * (D / 2);
      vr = v.v + at + in_page * (D / 2);
      ksr = v.k + at + v.P * (D / 2) + in_page * (D / 32);
      vsr = v.v + at + v.P * (D / 2) + in_page * (D / 32);
    };
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (h == 0 || !kOnePage) rows_at(h ? p1 : p0, (at0 + 16 * h) & (v.P - 1));
      const uint32_t more = kOnePage ? h : 0;      // 16 rows behind kr and vr
      ahead.k[h] = *reinterpret_cast<const typename S::KRow*>(kr + (k_at + more * 8 * D));
      ahead.ks[h] = *reinterpret_cast<const uint8_t*>(ksr + (ks_at + more * (D / 2)));
#pragma unroll
      for (int j = 0; j < 4; ++j)
        ahead.v[4 * h + j] =
            *reinterpret_cast<const typename S::VRow*>(vr + (v_at + more * 8 * D + j * (D / 2)));
      ahead.vs[h] = *reinterpret_cast<const typename S::Scales*>(vsr + (vs_at + more * (D / 2)));
    }
  };
  int page0 = next0, page1 = next1;     // 4 bits: this step's pages
  if constexpr (F4) {
    if (u < u1) {
      fetch(u, next0, next1);
      next0 = page_of(u + kWaves, 0);
      next1 = kOnePage ? next0 : page_of(u + kWaves, 1);
    }
  }
  for (; u < u1; u += kWaves) {
    const int t0 = step_token<kStep>(ts, u);
    // where there is no page the loads go to page 0 and the tokens are masked
    // below
    int page[2] = {F4 ? page0 : next0, F4 ? page1 : next1};
    bool there[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      there[h] = page[h] >= 0 && page[h] < v.n_pages;
      if (!there[h]) page[h] = 0;
    }
    frag kf[2][NF];
    vrow vv[8][VR::kLoads];
    if constexpr (F4) {
      // (the empty asm: now, or the words are copied out of the way of the next loads, to be
      // made into numbers behind them; one token over 13,711 in 28 layers 43 us and not 40)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float ks = __uint_as_float((uint32_t)ahead.ks[h] << 23);
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          const uint32_t w = reinterpret_cast<const uint32_t(&)[NF]>(ahead.k[h])[f];
          typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
          kf[h][f] = __builtin_bit_cast(frag, u32x4{from_fp4<0>(w, ks), from_fp4<1>(w, ks),
                                                    from_fp4<2>(w, ks), from_fp4<3>(w, ks)});
          asm volatile("" : "+v"(kf[h][f]));
        }
        // the byte of the lane's columns among each row's scales, turned to where a
        // float's exponent lies; the conversion looks at nothing else of it
        constexpr int kPer = D / 32;
        const int byte = l16 * kPer / 16;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t sw = reinterpret_cast<const uint32_t(&)[kPer]>(ahead.vs[h])[j * kPer / 4];
          const float vs = __uint_as_float(__builtin_amdgcn_alignbit(sw, sw, 8 * byte + j * kPer % 4 * 8 + 9));
          const uint32_t w = ahead.v[4 * h + j];
          vv[4 * h + j][0][0] = from_fp4<0>(w, vs);
          vv[4 * h + j][0][1] = from_fp4<1>(w, vs);
          if constexpr (D == 128) {
            vv[4 * h + j][0][2] = from_fp4<2>(w, vs);
            vv[4 * h + j][0][3] = from_fp4<3>(w, vs);
          }
          asm volatile("" : "+v"(vv[4 * h + j][0]));
        }
      }
      page0 = next0;
      page1 = next1;
      if (u + kWaves < u1) fetch(u + kWaves, page0, page1);
      next0 = page_of(u + 2 * kWaves, 0);
      next1 = kOnePage ? next0 : page_of(u + 2 * kWaves, 1);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int in_page = (t0 + 16 * h) & (v.P - 1);
        const int64_t at = base + (int64_t)page[h] * v.ps;
        const char* kr = v.k + at + (int64_t)(in_page + l16) * v.ts + 16 * quad;
#pragma unroll
        for (int f = 0; f < NF; ++f) kf[h][f] = *reinterpret_cast<const frag*>(kr + 64 * f);
        const char* vr = v.v + at + (int64_t)(in_page + 4 * quad) * v.ts + sizeof(vrow) * l16;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int c = 0; c < VR::kLoads; ++c)
            vv[4 * h + j][c] = *reinterpret_cast<const vrow*>(vr + j * v.ts + 16 * sizeof(vrow) * c);
      }
      next0 = page_of(u + kWaves, 0);
      next1 = page_of(u + kWaves, 1);
    }
    const bool whole = there[0] && there[1] && sees_step<kStep>(all, t0);

    f32x4 x[NB][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        x[nb][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int f = 0; f < NF; ++f) x[nb][h] = F::mma(kf[h][f], qf[nb][f], x[nb][h]);
      }
    bool odd = false;     // a masked step whose V holds infinities or NaN
    uint32_t seen[NB];    // the step's tokens that this lane's rows see
    if (!whole) {
      const uint32_t pages = (there[0] ? 0xFFFFu : 0u) | (there[1] ? 0xFFFF0000u : 0u);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        seen[nb] = pages & seen_bits(a, ts, qi[nb], t0);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const bool bit = seen[nb] >> (16 * (j >> 2) + 4 * quad + (j & 3)) & 1;
          x[nb][j >> 2][j & 3] = bit ? x[nb][j >> 2][j & 3] : -INFINITY;
        }
      }
      // what no page of the sequence holds counts as zero
      const uint32_t held = pages & low_bits(ts.n - t0);
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int c = 0; c < VR::kLoads; ++c) {
          if (!(held >> (16 * (j >> 2) + 4 * quad + (j & 3)) & 1)) vv[j][c] = vrow{};
          odd |= any_not_finite<T>(vv[j][c]);
        }
      odd = __any(odd);
    }
    float p[NB][8];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float mt = fmaxf(max4(x[nb][0]), max4(x[nb][1]));
      mt = quads_max(mt);
      const float mn = fmaxf(m[nb], mt);
      const float ms = mn == -INFINITY ? 0.f : mn;     // a row that saw nothing yet
      const float alpha = __builtin_amdgcn_exp2f((m[nb] - ms) * a.scale);
      m[nb] = mn;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        p[nb][j] = __builtin_amdgcn_exp2f((x[nb][j >> 2][j & 3] - ms) * a.scale);
        sum += p[nb][j];
      }
      l[nb] = l[nb] * alpha + sum;
      if (__any(alpha != 1.0f)) {
#pragma unroll
        for (int t = 0; t < ND; ++t) o[nb][t] *= alpha;
      }
    }
    if (odd) {
      // infinities and NaN in places that some rows see and some do not: they
      // are added token by token to the rows that see them, and are zero in
      // the product below
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        for (int k = 0; k < kStep; ++k) {
          const int h = k >> 4, src = ((k & 15) >> 2) * 16 + l16;
          float pk = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float w = __shfl(p[nb][j], src);
            if (j == 4 * h + (k & 3)) pk = w;
          }
          const int t = t0 + k;
          if (!(seen[nb] >> k & 1)) continue;
          const char* block = v.v + base + (int64_t)page[h] * v.ps;
          const char* vr = block + (int64_t)(t & (v.P - 1)) * v.ts;
#pragma unroll
          for (int e = 0; e < ND; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int col = 16 * VR::kCols * (e / VR::kCols) + VR::kCols * (4 * quad + i) +
                              e % VR::kCols;
              float val;
              if constexpr (F4) {    // (scale bytes 253 and 254: some elements of a block are infinite)
                const uint8_t s = block[v.P * (D / 2) + (t & (v.P - 1)) * (D / 32) + col / 32];
                val = 0.f;
                if (s >= 253) {
                  const uint32_t pair = from_fp4<0>((uint8_t)vr[col / 2], __uint_as_float((uint32_t)s << 23));
                  val = __uint_as_float(col & 1 ? pair & 0xFFFF0000u : pair << 16);
                }
              } else {
                val = (float)reinterpret_cast<const T*>(vr)[col];
              }
              if (!(fabsf(val) < INFINITY)) o[nb][e][i] = fmaf(pk, val, o[nb][e][i]);
            }
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int c = 0; c < VR::kLoads; ++c) zero_not_finite<T>(vv[j][c]);
    }
    if constexpr (sizeof(T) == 2) {
      // the weights rounded to bf16, V's type: half a step of 2^-8 each,
      // below the rounding of the output that they are averaged into
      bf16x8 pf[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int j = 0; j < 8; ++j) pf[nb][j] = (__bf16)p[nb][j];
#pragma unroll
      for (int e = 0; e < ND; ++e) {
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
        u32x4 w;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          w[k] = __builtin_amdgcn_perm(vv[2 * k + 1][0][e / 2], vv[2 * k][0][e / 2],
                                       e & 1 ? 0x07060302u : 0x05040100u);
        const bf16x8 vf = __builtin_bit_cast(bf16x8, w);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) o[nb][e] = F::mma(vf, pf[nb], o[nb][e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < ND; ++e)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float vf = __uint_as_float(vv[j][e / VR::kCols][e % VR::kCols]);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            o[nb][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf, p[nb][j], o[nb][e], 0, 0, 0);
        }
    }
  }

  // the four waves joined, 16 rows at a time
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    float lt = l[nb];
    lt += __shfl_xor(lt, 16);
    lt += __shfl_xor(lt, 32);
    __syncthreads();
    if (quad == 0) st[wave][l16] = float2{m[nb], lt};
#pragma unroll
    for (int e = 0; e < ND; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        ow[wave][l16][16 * VR::kCols * (e / VR::kCols) + VR::kCols * (4 * quad + i) +
                      e % VR::kCols] = o[nb][e][i];
    __syncthreads();
    for (int it = threadIdx.x; it < 16 * D / 4; it += kThreads) {
      const int row = it / (D / 4), c = it % (D / 4) * 4;
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) M = fmaxf(M, st[w][row].x);
      float L = 0.f;
      f32x4 O{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((st[w][row].x - M) * a.scale);
        L += st[w][row].y * f;
        O += *reinterpret_cast<const f32x4*>(&ow[w][row][c]) * f;
      }
      const int r = r0 + 16 * nb + row;
      if (r >= rows) continue;
      if (live > 1) {
        const size_t rec = ((size_t)unit * a.n_split + split) * kRows + 16 * nb + row;
        *reinterpret_cast<f32x4*>(a.part + rec * D + c) = O;
        if (c == 0) a.stat[rec] = float2{M, L};
      } else {
        store_row<T>(a, v, layer, g, hpg, ts.row0, r, c, M, L, O);
      }
    }
  }
}

// The splits of a row joined: D/4 threads for four columns each, times
// `groups` that take every groups-th split and are joined through LDS.  The
// order is fixed by the numbers of splits alone.  `parts` blocks share a row
// tile, each with every parts-th handful of its rows.  4 to 5 us where there is
// little to join (a launch and its chain: length, steps, statistics, sums); 54
// us for the 50,176 rows of a tree of 64 tokens in 28 layers, at most 0.2 GB of
// partial sums.
template <typename T, int D, int TT>
__global__ __launch_bounds__(kThreads) void attend_join(PagedView v, AttendArgs a, AttendLists s,
                                                        int row_tile, int groups, int parts) {
  constexpr int kPerRow = D / 4, kSlots = kThreads / kPerRow;
  __shared__ __align__(16) float oo[kSlots][D];
  __shared__ float2 ss[kSlots];
  const int slot = threadIdx.x / kPerRow, c = threadIdx.x % kPerRow * 4;
  const int group = slot & (groups - 1), here = kSlots / groups;
  const int unit = blockIdx.x / parts, part = blockIdx.x % parts;
  const int tile = unit % a.n_tiles, lg = unit / a.n_tiles;
  const int g = lg % v.G, layer = lg / v.G, hpg = v.H / v.G;
  const int b = tile_owner(s.tile0, s.r.n, tile);
  const TokenSpan ts = token_span<TT>(v, a, s, b, tile, row_tile, a.steps ? *a.steps : 0);
  const int live = (ts.nt + ts.per - 1) / ts.per;
  const int r0 = (tile - s.tile0[b]) * row_tile, rows = min(ts.T * hpg - r0, row_tile);
  if (live <= 1) return;
  for (int first = part * here; first < rows; first += parts * here) {
    const int row = first + slot / groups;
    const size_t rec = (size_t)unit * a.n_split * row_tile + row;
    float M = -INFINITY, L = 0.f;
    f32x4 O{0.f, 0.f, 0.f, 0.f};
    if (row < rows)
      for (int u0 = group; u0 < live; u0 += 4 * groups) {
        float2 st[4];
        f32x4 piece[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int u = u0 + j * groups;
          st[j] = float2{-INFINITY, 0.f};
          piece[j] = f32x4{0.f, 0.f, 0.f, 0.f};
          if (u < live) {
            const size_t at = rec + (size_t)u * row_tile;
            st[j] = a.stat[at];
            piece[j] = *reinterpret_cast<const f32x4*>(a.part + at * D + c);
          }
        }
        float top = M;
#pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, st[j].x);
        const float ref = top == -INFINITY ? 0.f : top;
        const float old = __builtin_amdgcn_exp2f((M - ref) * a.scale);
        M = top;
        L *= old;
        O *= old;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float f = __builtin_amdgcn_exp2f((st[j].x - ref) * a.scale);
          L += st[j].y * f;
          O += piece[j] * f;
        }
      }
    if (groups > 1) {
      __syncthreads();   // the rows before are read
      *reinterpret_cast<f32x4*>(&oo[slot][c]) = O;
      if (c == 0) ss[slot] = float2{M, L};
      __syncthreads();
      if (group == 0) {
        float top = M;
        for (int j = 1; j < groups; ++j) top = fmaxf(top, ss[slot + j].x);
        const float ref = top == -INFINITY ? 0.f : top;
        const float mine = __builtin_amdgcn_exp2f((M - ref) * a.scale);
        L *= mine;
        O *= mine;
        for (int j = 1; j < groups; ++j) {
          const float f = __builtin_amdgcn_exp2f((ss[slot + j].x - ref) * a.scale);
          L += ss[slot + j].y * f;
          O += *reinterpret_cast<const f32x4*>(&oo[slot + j][c]) * f;
        }
        M = top;
      }
    }
    if (group == 0 && row < rows) store_row<T>(a, v, layer, g, hpg, ts.row0, r0 + row, c, M, L, O);
  }
}

template <typename T, int D, bool F4 = false>
int launch(const PagedView& v, const AttendArgs& a, const AttendLists& l, const AttendShape& s,
           hipStream_t st) {
  const unsigned run = (unsigned)std::min(s.seq_tiles, 4);
  const unsigned runs = (s.n_tiles + run - 1) / run * v.n_layers * v.G * s.n_split;
  const unsigned blocks = (runs + 7) / 8 * 8 * run;
  if (s.many) {
    const int err = launch_attend_many(v, a, l, s, st);
    if (err) return err;
  } else {
    const auto go = [&](auto kernel) { kernel<<<blocks, kThreads, 0, st>>>(v, a, l, run); };
    const auto by_rows = [&](auto one_page) {
      constexpr bool kOnePage = decltype(one_page)::value;
      if (s.row_tile == 16) go(attend_few<T, D, 1, F4, kOnePage>);
      else if constexpr (sizeof(T) == 2) go(attend_few<T, D, 2, F4, kOnePage>);
    };
    if constexpr (F4) {
      if (v.P >= kStep) by_rows(std::true_type{});
      else by_rows(std::false_type{});
    } else {
      by_rows(std::false_type{});
    }
  }
  if (s.n_split > 1) {
    // up to four splits for each thread
    constexpr int kSlots = kThreads / (D / 4);
    int groups = 1;
    while (groups < kSlots && groups * 4 < s.n_split) groups *= 2;
    const int handfuls = s.row_tile / (kSlots / groups);
    const int parts = (int)std::max<int64_t>(1, std::min<int64_t>(handfuls, 2048 / s.units));
    const unsigned joins = (unsigned)(s.units * parts);
    if (!s.many)
      attend_join<T, D, kStep><<<joins, kThreads, 0, st>>>(v, a, l, s.row_tile, groups, parts);
    else if constexpr (sizeof(T) == 2)
      attend_join<T, D, 64><<<joins, kThreads, 0, st>>>(v, a, l, s.row_tile, groups, parts);
  }
  return (int)hipGetLastError();
}

}  // namespace

int launch_attend(const PagedView& v, const AttendCall& c, void* stream) {
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  AttendArgs a;
  a.q = static_cast<const char*>(c.q);
  a.out = static_cast<char*>(c.out);
  a.lse = c.lse;
  a.part = static_cast<float*>(c.ws);
  a.stat = reinterpret_cast<float2*>(static_cast<char*>(c.ws) + c.s.stat_off);
  a.mask = c.mask;
  a.words = c.words;
  a.window = c.window;
  a.sinks = c.sinks;
  a.n_split = c.s.n_split;
  a.chunk = c.s.chunk;
  a.n_tiles = c.s.n_tiles;
  a.most_steps = c.s.steps;
  a.steps = c.s.balance ? reinterpret_cast<int*>(static_cast<char*>(c.ws) + c.s.steps_off) : nullptr;
  a.n_rows = c.s.n_rows;
  a.scale = 1.4426950408889634f / sqrtf((float)v.d);
  AttendLists l;
  l.r = c.r;
  for (int i = 0; i <= c.r.n; ++i) l.tile0[i] = c.tile0[i];
  if (v.fp4)
    return v.d == 128 ? launch<__bf16, 128, true>(v, a, l, c.s, st)
                      : launch<__bf16, 64, true>(v, a, l, c.s, st);
  if (v.esz == 2)
    return v.d == 128 ? launch<__bf16, 128>(v, a, l, c.s, st) : launch<__bf16, 64>(v, a, l, c.s, st);
  return v.d == 128 ? launch<float, 128>(v, a, l, c.s, st) : launch<float, 64>(v, a, l, c.s, st);
}

}  // namespace starkv
