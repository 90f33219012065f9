// Attention over the pages of a cache for many query rows (bf16): a tree of
// several tokens, or a chunk of a prefill.  The rows of a (sequence, group)
// share its K and V, so the pass is bound by the matrix units, or by HBM
// where the rows are few.
//
// A block takes up to 128 rows, 32 for each of its waves, and walks the
// tokens in steps of 64 that all its waves read from LDS, while the next
// step's K and V travel from HBM straight to the other half of LDS.  As in
// the kernel for few rows the tokens are on the A side of both products:
//   S^T = K Q^T   on 32x32x16 MFMAs: a lane gets 16 tokens of each half of the
//                 step for one row, so a row's maximum and sum stay in two lanes;
//   O^T = V^T P^T the lane's weights are its part of B as they are (k = 8*half
//                 + j stands for token 4*half + j or 8 + 4*half + j - 4 of 16),
//                 and A's four tokens of a column come from LDS transposed.
// The running maximum is only moved when a row's grows by more than 2^8: until
// then the weights, up to 2^8, lose nothing, and the output need not be
// rescaled.
#include <algorithm>

#include "attend.h"

namespace starkv {
namespace {

constexpr int kMaxWaves = 4;
constexpr int kStep = 64;
constexpr int kGroups = kStep / 16;      // 16-token groups of a step: one page each

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

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
__device__ inline int k_swizzle(int token) {
  return D == 128 ? token & 15 : (token >> 1) & 7;
}
template <int D>
__device__ inline int v_swizzle(int token) {
  return D == 128 ? (token & 3) * 4 : ((token >> 1) & 1) * 4;
}

// One 16-token group's K or V rows into LDS, 1 KB per instruction: lane i of
// instruction j fills 16 bytes, piece i % NP of row j*kRows + i / NP, with the
// piece that belongs there, off[j] behind the group's first row.
template <int D>
__device__ inline void stage(const char* from, const uint32_t (&off)[16 * D * 2 / 1024], char* to) {
#pragma unroll
  for (int j = 0; j < 16 * D * 2 / 1024; ++j)
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from + off[j]),
                                     (__attribute__((address_space(3))) void*)(to + j * 1024), 16, 0,
                                     0);
}

// Blocks are dealt to the 8 XCDs round-robin by number.  Work items that
// follow each other share K and V: each XCD takes `run` of them in turn, so
// that its L2 holds what they read, and all XCDs move through the items
// together, whose costs differ from end to end.
__device__ inline unsigned xcd_item(unsigned block, unsigned run) {
  const unsigned xcd = block & 7, i = block >> 3;
  return (i / run * 8 + xcd) * run + i % run;
}

template <int D>
__global__ __launch_bounds__(64 * kMaxWaves, 2) void attend_many(PagedView v, AttendArgs a,
                                                                 AttendLists s, unsigned run) {
  constexpr int NF = D / 16;               // k-steps of S
  constexpr int ND = D / 32;               // 32-column tiles of the output
  constexpr int kRow = D * 2;              // bytes of a row
  constexpr int kLoads = 16 * kRow / 1024, kLoadRows = 16 / kLoads, NP = kRow / 16;
  __shared__ __align__(1024) char k0[kStep * kRow], k1[kStep * kRow];
  __shared__ __align__(1024) char v0[kStep * kRow], v1[kStep * kRow];

  const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = blockDim.x >> 6, row_tile = waves * 32;
  // tiles of one split of a (layer, group) follow each other: they read the
  // same K and V.  Later tiles, which may see more, come first
  const unsigned item = xcd_item(blockIdx.x, run);
  const int tile = a.n_tiles - 1 - item % a.n_tiles;
  const int split = item / a.n_tiles % a.n_split;
  const int lg = item / a.n_tiles / a.n_split;
  if (lg >= v.n_layers * v.G) return;
  const int g = lg % v.G, layer = lg / v.G;
  const int b = tile_owner(s.tile0, s.r.n, tile);
  const TokenSpan ts = token_span<kStep>(v, a, s, b, tile, row_tile);
  const int live = (ts.nt + ts.per - 1) / ts.per;
  if (split >= max(live, 1)) return;
  const int hpg = v.H / v.G;
  const int rows = ts.T * hpg;
  const int r0 = (tile - s.tile0[b]) * row_tile + wave * 32;
  // a wave whose rows all lie behind the last only helps to load
  const bool idle = r0 >= rows;
  const int r = min(r0 + l32, rows - 1);
  const int qi = r / hpg;
  const AllSee mine = all_see(a, ts, min(r0, rows - 1) / hpg, min(r0 + 31, rows - 1) / hpg);
  const int b0 = r0 - wave * 32;
  const AllSee block = all_see(a, ts, b0 / hpg, min(b0 + row_tile - 1, rows - 1) / hpg);
  const size_t out_row = ((size_t)layer * a.n_rows + ts.row0 + qi) * v.H + g * hpg + r % hpg;

  bf16x8 qf[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f)
    qf[f] = *reinterpret_cast<const bf16x8*>(a.q + out_row * kRow + 32 * f + 16 * half);

  // where the lane's 16 bytes of a staged group's loads lie
  uint32_t koff[kLoads], voff[kLoads];
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    const int token = j * kLoadRows + lane / NP, piece = lane % NP;
    koff[j] = (uint32_t)token * (uint32_t)v.ts + (piece ^ k_swizzle<D>(token)) * 16;
    voff[j] = (uint32_t)token * (uint32_t)v.ts + (piece ^ v_swizzle<D>(token)) * 16;
  }

  const const_i32* table = const_ints(v.table + (size_t)s.r.slot[b] * v.max_pages);
  const int64_t base = (int64_t)layer * v.ls + (int64_t)g * v.gs;
  const int u0 = split * ts.per, u1 = min(u0 + ts.per, ts.nt);
  // the pages of half a step's two groups, read a step before their use
  static_assert(kGroups == 4, "two words of two pages");
  const auto two_pages = [&](int t) {
    return (uint64_t)(uint32_t)table[min(t, ts.n - 1) >> v.psh] |
           (uint64_t)(uint32_t)table[min(t + 16, ts.n - 1) >> v.psh] << 32;
  };
  // A step's 16-token groups are dealt to the waves
  const auto load_step = [&](int u, uint64_t lo, uint64_t hi, char* kd, char* vd) {
    const int t0 = step_token<kStep>(ts, u);
    for (int grp = wave; grp < kGroups; grp += waves) {
      int page = (int)((grp & 2 ? hi : lo) >> (32 * (grp & 1)));
      if ((unsigned)page >= (unsigned)v.n_pages) page = 0;     // masked in the step
      const int64_t from = base + (int64_t)page * v.ps +
                           (int64_t)((t0 + 16 * grp) & (v.P - 1)) * v.ts;
      stage<D>(v.k + from, koff, kd + grp * 16 * kRow);
      stage<D>(v.v + from, voff, vd + grp * 16 * kRow);
    }
  };

  float m = -INFINITY, l = 0.f;       // reference of the weights; this lane's part of the sum
  f32x16 o[ND];
#pragma unroll
  for (int t = 0; t < ND; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[t][e] = 0.f;

  // One step on one half of LDS, while the next one's rows fill the other.
  uint64_t now_lo = 0, now_hi = 0, next_lo = 0, next_hi = 0;
  const auto step = [&](int u, char* ks, char* vs, char* kn, char* vn) {
    // the step's loads are complete, and every wave is done with the step
    // before, whose half of LDS the next loads fill
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    __syncthreads();
    const int t2 = step_token<kStep>(ts, min(u + 2, ts.nt - 1));
    const uint64_t later_lo = two_pages(t2), later_hi = two_pages(t2 + 32);
    if (u + 1 < u1) load_step(u + 1, next_lo, next_hi, kn, vn);
    // the page numbers are waited for here: scalar loads under way would make
    // every wait for a fragment one for all of them
    asm volatile("" ::"s"(later_lo), "s"(later_hi));

    const int t0 = step_token<kStep>(ts, u);
    const unsigned top_page = max(max((unsigned)now_lo, (unsigned)(now_lo >> 32)),
                                  max((unsigned)now_hi, (unsigned)(now_hi >> 32)));
    const bool all_pages = top_page < (unsigned)v.n_pages;
    uint64_t held = ~0ull;       // the tokens of the step that lie in a page
    bool odd = false;
    if (!all_pages || !sees_step<kStep>(block, t0)) {
#pragma unroll
      for (int grp = 0; grp < kGroups; ++grp) {
        const unsigned page = (unsigned)((grp & 2 ? now_hi : now_lo) >> (32 * (grp & 1)));
        if (page >= (unsigned)v.n_pages) held &= ~((uint64_t)0xFFFF << (16 * grp));
      }
      held &= (uint64_t)low_bits(ts.n - t0) | (uint64_t)low_bits(ts.n - t0 - 32) << 32;
      // some rows do not see all of it.  What no page holds counts as zero;
      // infinities and NaN of V need the way below
      for (int i = threadIdx.x; i < kStep * NP; i += blockDim.x) {
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
    now_lo = next_lo;
    now_hi = next_hi;
    next_lo = later_lo;
    next_hi = later_hi;

    f32x16 x[2];
    uint32_t seen[2] = {~0u, ~0u};
    if (!idle) {
      bf16x8 kf[2][NF];
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int token = 32 * h + l32;
          kf[h][f] = *reinterpret_cast<const bf16x8*>(
              ks + token * kRow + ((2 * f + half) ^ k_swizzle<D>(token)) * 16);
        }
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          x[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[h][f], qf[f], f ? x[h] : f32x16{}, 0, 0, 0);
      // six fragments ahead of the products, then one for one
      __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
      for (int f = 0; f < 2 * NF - 6; ++f) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, 6, 0);
      if (!all_pages || !sees_step<kStep>(mine, t0)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          seen[h] = (uint32_t)(held >> (32 * h)) & seen_bits(a, ts, qi, t0 + 32 * h);
          const uint32_t mine = seen[h] >> (4 * half);
#pragma unroll
          for (int e = 0; e < 16; ++e)
            x[h][e] = mine >> (8 * (e >> 2) + (e & 3)) & 1 ? x[h][e] : -INFINITY;
        }
      }
      // the weights, against the row's reference
      float mt = -INFINITY;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 16; ++e) mt = fmaxf(mt, x[h][e]);
      mt = both_halves_max(mt);
      const bool grows = mt > m && (m == -INFINITY || (mt - m) * a.scale > 8.f);
      if (__any(grows)) {
        const float mn = grows ? mt : m;
        const float alpha = mn == m ? 1.f : __builtin_amdgcn_exp2f((m - mn) * a.scale);
        m = mn;
        l *= alpha;
#pragma unroll
        for (int t = 0; t < ND; ++t) o[t] *= alpha;
      }
      const float mf = m == -INFINITY ? 0.f : m, ms = mf * a.scale;
      if (__any(!(fabsf(ms) < 1048576.f))) {
        // a reference whose product with the scale has no places left for the
        // differences: they are taken first
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 16; ++e) x[h][e] = __builtin_amdgcn_exp2f((x[h][e] - mf) * a.scale);
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            x[h][e] = __builtin_amdgcn_exp2f(fmaf(x[h][e], a.scale, -ms));
      }
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[h] += x[h][e];
      l += sum[0] + sum[1];
    }
    if (odd) {
      // infinities and NaN that some rows see and some do not: they are added
      // token by token to the rows that see them, and are zero from then on
      if (!idle) {
        for (int token = 0; token < kStep; ++token) {
          const int want = (token & 31) >> 3 << 2 | (token & 3) | token >> 5 << 4;
          float w = 0.f;
#pragma unroll
          for (int k = 0; k < 32; ++k) w = k == want ? x[k >> 4][k & 15] : w;
          w = __shfl(w, (token >> 2 & 1) * 32 + l32);
          const bool sees_it = (token < 32 ? seen[0] : seen[1]) >> (token & 31) & 1;
#pragma unroll
          for (int t = 0; t < ND; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int col = 32 * t + 8 * (e >> 2) + 4 * half + (e & 3);
              const float val = (float)*reinterpret_cast<const __bf16*>(
                  vs + token * kRow + ((col >> 3) ^ v_swizzle<D>(token)) * 16 + (col & 7) * 2);
              if (sees_it && !(fabsf(val) < INFINITY)) o[t][e] = fmaf(w, val, o[t][e]);
            }
        }
      }
      __syncthreads();
      for (int i = threadIdx.x; i < kStep * NP; i += blockDim.x) {
        u32x4 w = *reinterpret_cast<u32x4*>(vs + i * 16);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          if ((w[c] & 0x7F80u) == 0x7F80u) w[c] &= 0xFFFF0000u;
          if ((w[c] & 0x7F800000u) == 0x7F800000u) w[c] &= 0xFFFFu;
        }
        *reinterpret_cast<u32x4*>(vs + i * 16) = w;
      }
      __syncthreads();
    }
    if (idle) return;
    const int quad = lane >> 4 & 1, i = lane & 15;
    s16x8 vf[4][ND];
    bf16x8 pf[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      // tokens 16 k.. of the step; the weights rounded to bf16, V's type:
      // half a step of 2^-8 each, below the rounding of the output
#pragma unroll
      for (int j = 0; j < 8; ++j) pf[k][j] = (__bf16)x[k >> 1][8 * (k & 1) + j];
#pragma unroll
      for (int t = 0; t < ND; ++t) {
        s16x4 got[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int token = 16 * k + 8 * h + 4 * half + (i >> 2);
          const int piece = 4 * t + 2 * quad + (i >> 1 & 1);
          got[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) s16x4*)(
                  vs + token * kRow + (piece ^ v_swizzle<D>(token)) * 16 + (i & 1) * 8));
        }
        vf[k][t] = __builtin_shufflevector(got[0], got[1], 0, 1, 2, 3, 4, 5, 6, 7);
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int t = 0; t < ND; ++t)
        o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[k][t]), pf[k], o[t],
                                                       0, 0, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 12, 1);
#pragma unroll
    for (int f = 0; f < 4 * ND - 6; ++f) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, 6, 1);
  };

  if (u0 < u1) {
    const int t0 = step_token<kStep>(ts, u0), t1 = step_token<kStep>(ts, min(u0 + 1, ts.nt - 1));
    now_lo = two_pages(t0);
    now_hi = two_pages(t0 + 32);
    next_lo = two_pages(t1);
    next_hi = two_pages(t1 + 32);
    load_step(u0, now_lo, now_hi, k0, v0);
  }
  for (int u = u0; u < u1; u += 2) {
    step(u, k0, v0, k1, v1);
    if (u + 1 < u1) step(u + 1, k1, v1, k0, v0);
  }

  l = both_halves_sum(l);
  if (idle || r0 + l32 >= rows) return;
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
  // the row tiles of a (layer, group) that one XCD takes at a time
  const unsigned run = (unsigned)std::min(s.n_tiles, 4), items = (unsigned)(s.units * s.n_split);
  const unsigned blocks = (items + 8 * run - 1) / (8 * run) * (8 * run);
  const unsigned threads = (unsigned)(s.row_tile * 2);
  if (v.d == 128) attend_many<128><<<blocks, threads, 0, st>>>(v, a, l, run);
  else attend_many<64><<<blocks, threads, 0, st>>>(v, a, l, run);
  return (int)hipGetLastError();
}

}  // namespace starkv
