// Attention over the pages of a cache for many query rows (bf16): a tree of
// several tokens, or a chunk of a prefill.  The rows of a (sequence, group)
// share its K and V, so the pass is bound by the matrix units, or by HBM
// where the rows are few.
//
// A block takes up to 128 rows, 32 for each of its waves, and walks the
// tokens in steps of 64 that all its waves read from LDS, while the next
// step's K and V travel from HBM straight to the other half of LDS, and the
// next step's S runs on the matrix units beside this step's weights.  As in
// the kernel for few rows the tokens are on the A side of both products:
//   S^T = K Q^T   on 32x32x16 MFMAs: a lane gets 16 tokens of each half of the
//                 step for one row, so a row's maximum and sum stay in two lanes;
//   O^T = V^T P^T the lane's weights are its part of B as they are (k = 8*half
//                 + j stands for token 4*half + j or 8 + 4*half + j - 4 of 16),
//                 and A's four tokens of a column come from LDS transposed.
// The running maximum is only moved when a row's grows by more than 2^8: until
// then the weights, up to 2^8, lose nothing, and the output need not be
// rescaled.
//
// Measured, over several cards: the prefill of 8,192 tokens under a window of
// 4,096 388 to 417 us, 870 to 930 TFLOP/s; 2,755 tokens appended to 10,956 under
// a window of 8,192 392 to 400 us, 835 to 850 (25 of them the join); a tree of 64
// tokens over 40,941 in 28 layers 1,266 to 1,306 us, 805 to 830 (448 rows that
// take the place of 512, and 53 us of joining).  A library product of 8192^3
// makes 1,203 to 1,370.  The matrix units are busy in 41 to 43% of the SIMDs'
// cycles, in the library's product in 69%, at 1.9 to 2.1 GHz in both: both lose
// by power (on zeros these calls run 12 to 19% faster), and what lies between
// them is what a wave issues beside its products, five to six vector
// instructions to each against one.  LDS has no bank conflicts.  Short calls are
// bound by their chain of loads (eight tokens over 600: 9 us, and 3 to join).
// 4 bits, which pass through registers on their way to LDS: 2,755 tokens appended to
// 10,956 408 to 418 us (800 to 820 TFLOP/s; matrix units and vector work 35 and 38% of the
// cycles, and a quarter neither); trees of 24 tokens over 13,711 in 28 layers 235 to 238
// (560; 168 rows in the place of 256, as in bf16, which takes 236); of 64 over 40,941 1,213.
#include <algorithm>

#include "attend.h"

namespace starkv {
namespace {

constexpr int kWaves = 4;
constexpr int kStep = 64;
constexpr int kBlocks = 512;             // that the card holds at a time
constexpr int kGroups = kStep / 16;      // 16-token groups of a step: one page each

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

// v, opaque to the compiler: what is computed from it stays where it is
// written.  The loop needs nearly every register, and what its rare branches
// compute from the lane would be hoisted out of it and kept.
__device__ __forceinline__ int here(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

__device__ inline float both_halves_max(float v) {
  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}
__device__ inline float both_halves_sum(float v) {
  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
}

// Where 16-byte piece c of a token's row lies in LDS: the pieces of a row are
// permuted by the token, so that the lanes of a read, which differ in the
// token, meet different banks.  K is read one piece per token, V four
// neighbouring ones of four tokens by half a wave.
template <int D>
__host__ __device__ constexpr int k_swizzle(int token) {
  return D == 128 ? token & 15 : (token >> 1) & 7;
}
template <int D>
__host__ __device__ constexpr int v_swizzle(int token) {
  return D == 128 ? (token & 3) * 4 : ((token >> 1) & 1) * 4;
}

// One 16-token group's K or V rows into LDS, 1 KB per instruction: lane i of
// instruction j fills 16 bytes, piece i % NP of row j*kRows + i / NP, with the
// piece that belongs there.  `row` is the lane's row behind an instruction's
// first, `piece` the byte of its piece in instruction 0, `turn` what each
// further instruction's rows add to the swizzle.
template <int D>
__device__ inline void stage(const char* from, int64_t ts, uint32_t row, uint32_t piece,
                             uint32_t turn, char* to) {
  constexpr int kLoads = 16 * D * 2 / 1024, kRows = 16 / kLoads;
#pragma unroll
  for (int j = 0; j < kLoads; ++j)
    __builtin_amdgcn_global_load_lds(
        (const __attribute__((address_space(1))) void*)(from + j * kRows * ts +
                                                        (row + (piece ^ turn * j))),
        (__attribute__((address_space(3))) void*)(to + j * 1024), 16, 0, 0);
}

// The same of a 4-bit cache, whose elements become bf16 on their way: a lane
// takes the four bytes of a piece, and the byte of its scale, into registers a
// step before they go to LDS.  One conversion of a number for all rows of a block:
// 7.7 vector instructions to each product, itself among them, where bf16 has 6.6, and LDS
// written by them.
template <int D>
struct Fp4Group {
  static constexpr int kLoads = 16 * D * 2 / 1024, kRows = 16 / kLoads, NP = D / 8;
  uint32_t w[kLoads];
  uint8_t s[kLoads];
  // from: the group's first row, scales: its first scale
  __device__ __forceinline__ void fetch(const char* from, const char* scales, int lane) {
    const int at = lane / NP * (D / 32) + lane % NP / 4;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      w[j] = *reinterpret_cast<const uint32_t*>(from + 256 * j + 4 * lane);
      s[j] = *reinterpret_cast<const uint8_t*>(scales + 16 * j + at);
    }
  }
  // as stage(): `piece` is where the lane's piece lies in instruction 0's row
  __device__ __forceinline__ void put(uint32_t piece, uint32_t turn, char* to, int lane) const {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const float f = __uint_as_float((uint32_t)s[j] << 23);
      u32x4 x;
      x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[j], f, 0));
      x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[j], f, 1));
      x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[j], f, 2));
      x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[j], f, 3));
      *reinterpret_cast<u32x4*>(to + j * 1024 + lane / NP * (D * 2) + (piece ^ turn * j)) = x;
    }
  }
};

template <int D, bool F4 = false>
__global__ __launch_bounds__(64 * kWaves, 2) void attend_many(PagedView v, AttendArgs a,
                                                              AttendLists s, unsigned run) {
  constexpr int NF = D / 16;               // k-steps of S
  constexpr int ND = D / 32;               // 32-column tiles of the output
  constexpr int kRow = D * 2;              // bytes of a row
  constexpr int kLoads = 16 * kRow / 1024, kLoadRows = 16 / kLoads, NP = kRow / 16;
  __shared__ __align__(1024) char k0[kStep * kRow], k1[kStep * kRow];
  __shared__ __align__(1024) char v0[kStep * kRow], v1[kStep * kRow];

  const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr int row_tile = kWaves * 32;
  // `run` tiles of one split of a (layer, group) follow each other: they read
  // the same K and V.  Later tiles, which may see more, come first, those of
  // all (layer, group)s together
  const unsigned item = xcd_item(blockIdx.x, run);
  const unsigned lgs = v.n_layers * v.G, runs = (a.n_tiles + run - 1) / run, at_run = item / run;
  const int lg = at_run % lgs, split = at_run / lgs / runs;
  const int tile = a.n_tiles - 1 - (int)(at_run / lgs % runs * run + item % run);
  const int chosen = a.steps ? balanced_steps<kStep>(v, a, s, kBlocks) : 0;
  if (a.steps && blockIdx.x == 0 && threadIdx.x == 0) *a.steps = chosen;   // for the join
  if (split >= a.n_split || tile < 0) return;
  const int g = lg % v.G, layer = lg / v.G;
  const int b = tile_owner(s.tile0, s.r.n, tile);
  const TokenSpan ts = token_span<kStep>(v, a, s, b, tile, row_tile, chosen);
  const int live = (ts.nt + ts.per - 1) / ts.per;
  if (split >= max(live, 1)) return;
  const int hpg = v.H / v.G;
  const int rows = ts.T * hpg;
  const int r0 = (tile - s.tile0[b]) * row_tile + wave * 32;
  // a wave whose rows all lie behind the last only helps to load
  const bool idle = r0 >= rows;
  const auto row_of = [&](int ln) { return min(r0 + (ln & 31), rows - 1); };
  const auto out_row_of = [&](int r) {
    return ((size_t)layer * a.n_rows + ts.row0 + r / hpg) * v.H + g * hpg + r % hpg;
  };
  const AllSee mine = all_see(a, ts, min(r0, rows - 1) / hpg, min(r0 + 31, rows - 1) / hpg);
  const int b0 = r0 - wave * 32;
  const AllSee block = all_see(a, ts, b0 / hpg, min(b0 + row_tile - 1, rows - 1) / hpg);
  bf16x8 qf[NF];
  {
    const char* qr = a.q + out_row_of(row_of(lane)) * kRow + 16 * half;
#pragma unroll
    for (int f = 0; f < NF; ++f) qf[f] = *reinterpret_cast<const bf16x8*>(qr + 32 * f);
  }

  // the lane's row and pieces of a staged group; the swizzles of tokens
  // j*kLoadRows + i are those of j*kLoadRows and i combined by xor
  const int sub = lane / NP;
  const uint32_t row_off = here(sub * (int)v.ts);
  const uint32_t kpiece = here(((lane % NP) ^ k_swizzle<D>(sub)) * 16);
  const uint32_t vpiece = here(((lane % NP) ^ v_swizzle<D>(sub)) * 16);
  constexpr uint32_t kturn = k_swizzle<D>(kLoadRows) * 16, vturn = v_swizzle<D>(kLoadRows) * 16;

  const const_i32* table = const_ints(v.table + (size_t)s.r.slot[b] * v.max_pages);
  const int64_t base = (int64_t)layer * v.ls + (int64_t)g * v.gs;
  const int u0 = split * ts.per, u1 = min(u0 + ts.per, ts.nt);
  // The pages of a step's four groups, and from them which have none (bit by
  // bit) and where the one that this wave stages lies in the pool
  using Pages = i32x4;
  const auto pages_at = [&](int u) {
    const int t = step_token<kStep>(ts, min(u, ts.nt - 1));
    const auto one = [&](int at) {
      const uint32_t off = (uint32_t)min(at, ts.n - 1) >> v.psh << 2;
      return *(const const_i32*)((const __attribute__((address_space(4))) char*)table + off);
    };
    return Pages{one(t), one(t + 16), one(t + 32), one(t + 48)};
  };
  const auto holes_of = [&](const Pages& p) {
    const unsigned n = (unsigned)v.n_pages;
    return ((unsigned)p[0] >= n ? 1u : 0u) | ((unsigned)p[1] >= n ? 2u : 0u) |
           ((unsigned)p[2] >= n ? 4u : 0u) | ((unsigned)p[3] >= n ? 8u : 0u);
  };
  const auto where = [&](int u, const Pages& p) {
    unsigned page = wave < 2 ? (wave < 1 ? p[0] : p[1]) : (wave < 3 ? p[2] : p[3]);
    if (page >= (unsigned)v.n_pages) page = 0;      // masked in the step
    const unsigned row = (unsigned)(step_token<kStep>(ts, min(u, ts.nt - 1)) + 16 * wave) &
                         (unsigned)(v.P - 1);
    return (uint64_t)base + page * (uint64_t)v.ps + row * (uint64_t)v.ts;
  };
  const auto load_k = [&](uint64_t at, char* to) {
    stage<D>(v.k + at, v.ts, row_off, kpiece, kturn, to + wave * 16 * kRow);
  };
  const auto load_v = [&](uint64_t at, char* to) {
    stage<D>(v.v + at, v.ts, row_off, vpiece, vturn, to + wave * 16 * kRow);
  };
  // 4 bits: step u + 1's group of V and u + 2's of K, in registers
  [[maybe_unused]] Fp4Group<D> raw_k, raw_v;
  [[maybe_unused]] const auto fetch = [&](const char* pool, uint64_t at, int u, Fp4Group<D>& raw) {
    const int row = (step_token<kStep>(ts, min(u, ts.nt - 1)) + 16 * wave) & (v.P - 1);
    raw.fetch(pool + at, pool + at + v.P * (D / 2) - row * (D / 2 - D / 32), lane);
  };
  const auto landed = [&]() {
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    __syncthreads();
  };

  float m = -INFINITY, l = 0.f;       // reference of the weights; this lane's part of the sum
  float top = -INFINITY;              // the step's largest logit of the lane
  f32x16 o[ND], x[2];
#pragma unroll
  for (int t = 0; t < ND; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[t][e] = 0.f;

  const auto quarter_max = [](const f32x16 (&z)[2], int q, float best) {
#pragma unroll
    for (int e = 0; e < 8; ++e) best = fmaxf(best, z[q >> 1][8 * (q & 1) + e]);
    return best;
  };
  // LDS offsets of the lane's fragments, the same in every buffer
  uint32_t kat[NF], vat[ND];
#pragma unroll
  for (int f = 0; f < NF; ++f)
    kat[f] = here(l32 * kRow + ((2 * f + half) ^ k_swizzle<D>(l32)) * 16);
#pragma unroll
  for (int t = 0; t < ND; ++t) {
    const int token = 4 * half + (lane >> 2 & 3), piece = 4 * t + 2 * (lane >> 4 & 1) + (lane >> 1 & 1);
    vat[t] = here(token * kRow + (piece ^ v_swizzle<D>(token)) * 16 + (lane & 1) * 8);
  }
  static_assert(k_swizzle<D>(32) == 0 && v_swizzle<D>(8) == 0, "whole turns of the swizzles");
  const auto k_frag = [&](const char* ks, int f, int h) {
    return *reinterpret_cast<const bf16x8*>(ks + kat[f] + 32 * h * kRow);
  };
  const auto v_frag = [&](const char* vs, int k, int t) {
    s16x4 got[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
      got[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(
          vs + vat[t] + (16 * k + 8 * h) * kRow));
    return __builtin_bit_cast(
        bf16x8, __builtin_shufflevector(got[0], got[1], 0, 1, 2, 3, 4, 5, 6, 7));
  };

  // One step: x holds its S.  Its weights are taken while the next step's S
  // runs on the matrix units, so K is a step ahead of V: K of step u + 1 is
  // read from kn, K of u + 2 fills the other half kf, V of u is in vs, V of u +
  // 1 fills vn.
  // The addresses of the next rows to stage are worked out beside the products
  // with V, the part of a step that is poorest in other work.
  uint64_t at1 = 0, at2 = 0;                 // of steps u + 1 and u + 2 (4 bits: u + 2 and u + 3)
  unsigned hole0 = 0, hole1 = 0, hole2 = 0;  // groups without a page, of u and the next two
  [[maybe_unused]] unsigned hole3 = 0;       // (4 bits: three)
  const auto step = [&](int u, const char* kn, char* kf, char* vs, char* vn) {
    // the loads are complete, and every wave is done with what they replace
    landed();
    if constexpr (F4) {
      if (u + 1 < u1) raw_v.put(vpiece, vturn, vn + wave * 16 * kRow, lane);
      if (u + 2 < u1) raw_k.put(kpiece, kturn, kf + wave * 16 * kRow, lane);
      if (u + 2 < u1) fetch(v.v, at1, u + 2, raw_v);
      if (u + 3 < u1) fetch(v.k, at2, u + 3, raw_k);
    } else {
      if (u + 1 < u1) load_v(at1, vn);
      if (u + 2 < u1) load_k(at2, kf);
    }
    const Pages ahead = pages_at(u + (F4 ? 4 : 3));

    const int t0 = step_token<kStep>(ts, u);
    const bool whole = hole0 == 0 && sees_step<kStep>(block, t0);
    uint64_t held = ~0ull;       // the tokens of the step that lie in a page
    bool odd = false;
    if (!whole) {
#pragma unroll
      for (int grp = 0; grp < kGroups; ++grp)
        if (hole0 >> grp & 1) held &= ~((uint64_t)0xFFFF << (16 * grp));
      held &= (uint64_t)low_bits(ts.n - t0) | (uint64_t)low_bits(ts.n - t0 - 32) << 32;
      // some rows do not see all of it.  What no page holds counts as zero;
      // infinities and NaN of V need the way below
      for (int i = here(threadIdx.x); i < kStep * NP; i += 64 * kWaves) {
        const int token = i / NP;
        u32x4* at = reinterpret_cast<u32x4*>(vs + i * 16);
        if (!(held >> token & 1)) {
          *at = u32x4{0, 0, 0, 0};
        } else {
          const u32x4 w = *at;
#pragma unroll
          for (int c = 0; c < 4; ++c)
            odd |= (w[c] & 0x7F80u) == 0x7F80u || (w[c] & 0x7F800000u) == 0x7F800000u;
        }
      }
      odd = __syncthreads_or(odd);
    }
    f32x16 y[2];
    bf16x8 vf0[ND];
    uint32_t seen[2] = {~0u, ~0u};
    if (!idle) {
      if (!whole && (hole0 || !sees_step<kStep>(mine, t0))) {
        const int ln = here(lane), qi = row_of(ln) / hpg;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          seen[h] = (uint32_t)(held >> (32 * h)) & seen_bits(a, ts, qi, t0 + 32 * h);
          const uint32_t bits = seen[h] >> (ln >> 5 << 2);
#pragma unroll
          for (int e = 0; e < 16; ++e)
            x[h][e] = bits >> (8 * (e >> 2) + (e & 3)) & 1 ? x[h][e] : -INFINITY;
        }
        top = -INFINITY;
#pragma unroll
        for (int q = 0; q < 4; ++q) top = quarter_max(x, q, top);
      }
      // the weights, against the row's reference
      const float mt = both_halves_max(top);
      const bool grows = mt > m && (m == -INFINITY || (mt - m) * a.scale > 8.f);
      if (__any(grows)) {
        const float mn = grows ? mt : m;
        const float alpha = mn == m ? 1.f : __builtin_amdgcn_exp2f((m - mn) * a.scale);
        m = mn;
        l *= alpha;
#pragma unroll
        for (int t = 0; t < ND; ++t) o[t] *= alpha;
      }
      float mf = m == -INFINITY ? 0.f : m, ms = mf * a.scale;
      if (__any(!(fabsf(ms) < 1048576.f))) {
        // a reference whose product with the scale has no places left for the
        // differences: they are taken first
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 16; ++e) x[h][e] -= mf;
        ms = 0.f;
      }
      float sum[2] = {0.f, 0.f};
      const auto weight = [&](int e) {
        const float w = __builtin_amdgcn_exp2f(fmaf(x[e >> 4][e & 15], a.scale, -ms));
        x[e >> 4][e & 15] = w;
        sum[e & 1] += w;
      };
      // two products, their share of the weights and the fragments of two
      // products later by turns (behind the last step the products are of
      // whatever K the buffer holds, and nobody reads them)
      bf16x8 kfr[NF][2];
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int h = 0; h < 2; ++h) kfr[f][h] = k_frag(kn, f, h);
#pragma unroll
      for (int f = 0; f < NF; ++f) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          y[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kfr[f][h], qf[f], f ? y[h] : f32x16{}, 0, 0, 0);
        if (f + 2 < NF) {
#pragma unroll
          for (int h = 0; h < 2; ++h) kfr[f + 2][h] = k_frag(kn, f + 2, h);
        } else if (f + 1 == NF) {
#pragma unroll
          for (int t = 0; t < ND; ++t) vf0[t] = v_frag(vs, 0, t);
        }
#pragma unroll
        for (int e = 0; e < 32 / NF; ++e) weight(32 / NF * f + e);
        __builtin_amdgcn_sched_barrier(0);
      }
      l += sum[0] + sum[1];
    }
    if (odd) {
      // infinities and NaN that some rows see and some do not: they are added
      // token by token to the rows that see them, and are zero from then on
      if (!idle) {
        const int ln = here(lane);
        for (int token = 0; token < kStep; ++token) {
          const int want = (token & 31) >> 3 << 2 | (token & 3) | token >> 5 << 4;
          float w = 0.f;
#pragma unroll
          for (int k = 0; k < 32; ++k) w = k == want ? x[k >> 4][k & 15] : w;
          w = __shfl(w, (token >> 2 & 1) * 32 + (ln & 31));
          const bool sees_it = (token < 32 ? seen[0] : seen[1]) >> (token & 31) & 1;
#pragma unroll
          for (int t = 0; t < ND; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int col = 32 * t + 8 * (e >> 2) + 4 * (ln >> 5) + (e & 3);
              const float val = (float)*reinterpret_cast<const __bf16*>(
                  vs + token * kRow + ((col >> 3) ^ v_swizzle<D>(token)) * 16 + (col & 7) * 2);
              if (sees_it && !(fabsf(val) < INFINITY)) o[t][e] = fmaf(w, val, o[t][e]);
              __builtin_amdgcn_sched_barrier(0);   // few registers at a time
            }
        }
      }
      __syncthreads();
      for (int i = here(threadIdx.x); i < kStep * NP; i += 64 * kWaves) {
        u32x4 w = *reinterpret_cast<u32x4*>(vs + i * 16);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          if ((w[c] & 0x7F80u) == 0x7F80u) w[c] &= 0xFFFF0000u;
          if ((w[c] & 0x7F800000u) == 0x7F800000u) w[c] &= 0xFFFFu;
        }
        *reinterpret_cast<u32x4*>(vs + i * 16) = w;
      }
      __syncthreads();
      if (!idle) {
#pragma unroll
        for (int t = 0; t < ND; ++t) vf0[t] = v_frag(vs, 0, t);
      }
    }
    hole0 = hole1;
    hole1 = hole2;
    if constexpr (F4) hole2 = hole3;
    const auto look_ahead = [&]() {
      (F4 ? hole3 : hole2) = holes_of(ahead);
      at1 = at2;
      at2 = where(u + (F4 ? 4 : 3), ahead);
    };
    if (idle) {
      look_ahead();
      return;
    }
    // the products with V go first where two waves of a SIMD want the matrix
    // unit (2 to 3% over equal turns)
    __builtin_amdgcn_s_setprio(1);
    bf16x8 vf[4][ND];
#pragma unroll
    for (int t = 0; t < ND; ++t) vf[0][t] = vf0[t];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      // tokens 16 k.. of the step; the weights rounded to bf16, V's type:
      // half a step of 2^-8 each, below the rounding of the output
      bf16x8 pf;
#pragma unroll
      for (int j = 0; j < 8; ++j) pf[j] = (__bf16)x[k >> 1][8 * (k & 1) + j];
#pragma unroll
      for (int t = 0; t < ND; ++t) {
        if (k < 3) vf[k + 1][t] = v_frag(vs, k + 1, t);
        o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[k][t], pf, o[t], 0, 0, 0);
      }
      if (k == 1) look_ahead();
      // the next step's largest logit, should all of it be seen
      top = quarter_max(y, k, k ? top : -INFINITY);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    x[0] = y[0];
    x[1] = y[1];
  };

  if (u0 < u1) {
    const Pages p0 = pages_at(u0), p1 = pages_at(u0 + 1), p2 = pages_at(u0 + 2);
    hole0 = holes_of(p0);
    hole1 = holes_of(p1);
    hole2 = holes_of(p2);
    const uint64_t at0 = where(u0, p0);
    at1 = where(u0 + 1, p1);
    at2 = where(u0 + 2, p2);
    if constexpr (F4) {
      char* const k_to = k0 + wave * 16 * kRow;
      fetch(v.k, at0, u0, raw_k);
      fetch(v.v, at0, u0, raw_v);
      Fp4Group<D> next;
      if (u0 + 1 < u1) fetch(v.k, at1, u0 + 1, next);
      raw_k.put(kpiece, kturn, k_to, lane);
      raw_v.put(vpiece, vturn, v0 + wave * 16 * kRow, lane);
      if (u0 + 1 < u1) {
        next.put(kpiece, kturn, k1 + wave * 16 * kRow, lane);
        fetch(v.v, at1, u0 + 1, raw_v);
      }
      if (u0 + 2 < u1) fetch(v.k, at2, u0 + 2, raw_k);
      const Pages p3 = pages_at(u0 + 3);
      hole3 = holes_of(p3);
      at1 = at2;
      at2 = where(u0 + 3, p3);
    } else {
      load_k(at0, k0);
      load_v(at0, v0);
      if (u0 + 1 < u1) load_k(at1, k1);
    }
    landed();
    if (!idle) {
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          x[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(k0, f, h), qf[f], f ? x[h] : f32x16{}, 0,
                                                         0, 0);
#pragma unroll
      for (int q = 0; q < 4; ++q) top = quarter_max(x, q, top);
    }
  }
  for (int u = u0; u < u1; u += 2) {
    step(u, k1, k0, v0, v1);
    if (u + 1 < u1) step(u + 1, k0, k1, v1, v0);
  }

  l = both_halves_sum(l);
  if (idle || r0 + l32 >= rows) return;
  const size_t out_row = out_row_of(row_of(here(lane)));
  if (live > 1) {
    const size_t unit = (size_t)lg * a.n_tiles + tile;
    const size_t rec = (unit * a.n_split + split) * row_tile + wave * 32 + l32;
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(a.part + rec * D + 32 * t + 8 * i + 4 * half) =
            f32x4{o[t][4 * i], o[t][4 * i + 1], o[t][4 * i + 2], o[t][4 * i + 3]};
    if (half == 0) a.stat[rec] = float2{m, l};
    return;
  }
#pragma unroll
  for (int t = 0; t < ND; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      store_out<__bf16>(a, v.d, out_row, 32 * t + 8 * i + 4 * half, m, l,
                        f32x4{o[t][4 * i], o[t][4 * i + 1], o[t][4 * i + 2], o[t][4 * i + 3]});
}

}  // namespace

int launch_attend_many(const PagedView& v, const AttendArgs& a, const AttendLists& l,
                       const AttendShape& s, hipStream_t st) {
  // the row tiles of a sequence that one XCD takes at a time
  const unsigned run = (unsigned)std::min(s.seq_tiles, 4);
  const unsigned runs = (unsigned)((s.n_tiles + run - 1) / run) * v.n_layers * v.G * s.n_split;
  const unsigned blocks = (runs + 7) / 8 * 8 * run;
  const auto go = [&](auto kernel) { kernel<<<blocks, 64 * kWaves, 0, st>>>(v, a, l, run); };
  if (v.d == 128) v.fp4 ? go(attend_many<128, true>) : go(attend_many<128>);
  else v.fp4 ? go(attend_many<64, true>) : go(attend_many<64>);
  return (int)hipGetLastError();
}

}  // namespace starkv
