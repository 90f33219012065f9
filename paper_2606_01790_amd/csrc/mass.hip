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
// Few rows (a decoded token, a few drafted ones; float32 of any number) are bound
// by HBM: mass_few takes 64 tokens a block, K straight to registers, four items of
// 16 tokens of a group to a wave and a group; the groups are added up through LDS.
// Many rows are bound by the matrix units and the exponentials: mass_many keeps 64
// tokens' K in a wave's registers and walks the rows, which all waves read from
// LDS, groups one after the other into the same sums.
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
  int row0, hpg, R;         // its first row of the call; heads, and rows, of a group
  const int32_t* table;
  const float* mass;
  float* out;
};
__device__ inline Seq seq_of(const PagedView& v, const MassArgs& a, const RowList& r, int layer,
                             int b) {
  Seq s;
  const int slot = r.slot[b];
  s.n = min(max(v.len[slot], 0), v.cap);
  s.row0 = r.row0[b];
  s.T = r.row0[b + 1] - s.row0;
  s.first = s.n - s.T;
  s.hpg = v.H / v.G;
  s.R = s.T * s.hpg;
  s.table = v.table + (size_t)slot * v.max_pages;
  const size_t at = ((size_t)layer * v.n_slots + slot) * v.cap;
  s.mass = a.mass + at;
  s.out = a.out + at;
  return s;
}
__device__ inline bool is_page(const PagedView& v, int p) { return p >= 0 && p < v.n_pages; }

// Token t's mass with what the rows add to it (nothing to a dropped token,
// whatever was computed in its place).
__device__ inline void store_mass(const PagedView& v, const Seq& s, int t, float add) {
  const float old = t < s.first ? s.mass[t] : 0.f;
  s.out[t] = is_page(v, s.table[t >> v.psh]) ? old + add : old;
}
// Whether any row sees any of the tokens [t0, t1).
__device__ inline bool any_sees(const MassArgs& a, const Seq& s, int t0, int t1) {
  // the first row has the widest reach back; every token from it on is seen by its own row
  return t1 - 1 > max(s.first, 0) - a.window || t0 < a.sinks;
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

// 16-token parts of a group: a wave takes G of the tile's 4*G, whole groups where
// there are four or more.
template <typename T, int D, bool F4>
__global__ __launch_bounds__(kThreads) void mass_few(PagedView v, MassArgs a, RowList r) {
  using F = Frag<T>;
  using frag = typename F::type;
  using K = KRow<T, D, F4>;
  extern __shared__ float sums[];       // [G][64]
  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int pair = blockIdx.x / a.blocks, b = pair % r.n, layer = pair / r.n;
  const Seq s = seq_of(v, a, r, layer, b);
  if (s.T == 0) return;
  const int64_t layer_at = (int64_t)layer * v.ls;
  const size_t row_at = ((size_t)layer * a.n_rows + s.row0) * v.H;      // of q and lse
  for (int tile = blockIdx.x % a.blocks; (int64_t)tile * 64 < s.n; tile += a.blocks) {
    const int t0 = tile * 64;
    if (!any_sees(a, s, t0, min(t0 + 64, s.n))) {
      const int t = t0 + threadIdx.x;
      if (threadIdx.x < 64 && t < s.n) s.out[t] = s.mass[t];
      continue;
    }
    const auto load = [&](int it, K& k) {
      const int item = wave * v.G + it, g = item >> 2;
      const int t = min(t0 + 16 * (item & 3), (s.n - 1) & ~15);
      const int page = s.table[t >> v.psh];
      // where there is no page the products are of page 0's, and dropped
      const char* block = v.k + layer_at + (int64_t)(is_page(v, page) ? page : 0) * v.ps + (int64_t)g * v.gs;
      k.load(v, block, (t & (v.P - 1)) + l16, quad, v.ts);
    };
    K k;
    load(0, k);
    for (int it = 0; it < v.G; ++it) {
      K next;
      if (it + 1 < v.G) load(it + 1, next);
      const int item = wave * v.G + it, g = item >> 2, t = t0 + 16 * (item & 3) + l16;
      float sum = 0.f;
      for (int r0 = 0; r0 < s.R; r0 += 16) {
        const int mine = min(r0 + l16, s.R - 1), i = s.T == 1 ? 0 : mine / s.hpg;
        const char* qr = a.q + (row_at + (size_t)i * v.H + g * s.hpg + (mine - i * s.hpg)) * D * sizeof(T);
        f32x4 x{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int f = 0; f < K::NF; ++f)
          x = F::mma(*reinterpret_cast<const frag*>(qr + K::q_byte(f, quad)), k.get(f), x);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = r0 + 4 * quad + e, at = min(row, s.R - 1), qi = s.T == 1 ? 0 : at / s.hpg;
          const float lse = a.lse[row_at + (size_t)qi * v.H + g * s.hpg + (at - qi * s.hpg)];
          const bool see = row < s.R && lse != -INFINITY && sees(a, s.first + qi, t);
          const float w = __builtin_amdgcn_exp2f(fmaf(x[e], a.scale, -lse * kLog2e));
          sum += see ? w : 0.f;
        }
      }
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (quad == 0) sums[g * 64 + 16 * (item & 3) + l16] = sum;
      k = next;
    }
    __syncthreads();
    if (threadIdx.x < 64 && t0 + (int)threadIdx.x < s.n) {
      float add = 0.f;
      for (int g = 0; g < v.G; ++g) add += sums[g * 64 + threadIdx.x];
      store_mass(v, s, t0 + threadIdx.x, add);
    }
    __syncthreads();
  }
}

// --------------------------------------------------------------- many rows

constexpr int kTile = 256;         // tokens of a block, 64 to a wave
constexpr int kStage = 64;         // rows in LDS at a time, twice

// Where 16-byte piece c of a row of Q lies in LDS: the lanes of a read, which
// differ in the row, meet different banks.
template <int D>
__device__ constexpr int q_swizzle(int row) {
  return D == 128 ? row & 15 : (row >> 1) & 7;
}

template <int D, bool F4>
__global__ __launch_bounds__(kThreads, 2) void mass_many(PagedView v, MassArgs a, RowList r) {
  constexpr int NF = D / 16, NP = D / 8, kRow = D * 2;
  constexpr int kLoads = kStage * NP / kThreads;          // 16-byte pieces of a thread per stage
  constexpr int kLoadRows = kThreads / NP;
  __shared__ __align__(1024) char qs[2][kStage * kRow];
  __shared__ __align__(16) float ls[2][kStage];           // lse log2(e); infinite behind the last row
  __shared__ __align__(16) int ps[2][kStage];             // the rows' positions; -1: sees nothing
  __shared__ int odd[2][2];                               // of 32 rows: some see nothing

  const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int split = blockIdx.x % a.n_split, at = blockIdx.x / a.n_split;
  const int pair = at / a.blocks, b = pair % r.n, layer = pair / r.n;
  const Seq s = seq_of(v, a, r, layer, b);
  if (s.T == 0) return;
  const size_t row_at = ((size_t)layer * a.n_rows + s.row0) * v.H;

  for (int tile = at % a.blocks; (int64_t)tile * kTile < s.n; tile += a.blocks) {
    // tiles behind the bound that the splits' sums were sized by are not split
    const bool shared_tile = a.n_split > 1 && tile < a.tiles;
    if (!shared_tile && split) continue;
    const int t0 = tile * kTile, t1 = min(t0 + kTile, s.n);
    // the 32-row products of each group that see some of the tile: from the row
    // at t0 to the last one whose window reaches back to t1 - 1
    const int i0 = max(t0 - s.first, 0);
    const int64_t reach = t0 < a.sinks ? s.T - 1 : (int64_t)t1 - 1 + a.window - 1 - s.first;
    const int i1 = (int)min(reach, (int64_t)s.T - 1);
    const int p0 = i0 * s.hpg / 32, p1 = i1 < i0 ? p0 : ((i1 + 1) * s.hpg + 31) / 32;
    const int64_t all = (int64_t)v.G * (p1 - p0);
    int64_t w0 = shared_tile ? all * split / a.n_split : 0;
    const int64_t w1 = shared_tile ? all * (split + 1) / a.n_split : all;

    float sum[2] = {0.f, 0.f};
    while (w0 < w1) {
      const int g = (int)(w0 / (p1 - p0));
      const int from = p0 + (int)(w0 - (int64_t)g * (p1 - p0));
      const int to = (int)min((int64_t)p1, from + w1 - w0);
      w0 += to - from;
      // K of the wave's tokens: a lane holds half a row of tokens l32 and 32 + l32
      bf16x8 kf[2][NF];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int t = min(t0 + 64 * wave + 32 * h + l32, s.n - 1);
        const int page = s.table[t >> v.psh], in_page = t & (v.P - 1);
        const char* block = v.k + (int64_t)layer * v.ls + (int64_t)(is_page(v, page) ? page : 0) * v.ps +
                            (int64_t)g * v.gs;
        if constexpr (F4) {
          const char* row = block + in_page * (D / 2) + half * (D / 4);
          const char* scales = block + v.P * (D / 2) + in_page * (D / 32) + half * (D / 64);
#pragma unroll
          for (int f = 0; f < NF; f += 4) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(row + 4 * f);
            const float sc = __uint_as_float((uint32_t)*reinterpret_cast<const uint8_t*>(scales + f / 4) << 23);
#pragma unroll
            for (int e = 0; e < 4; ++e) kf[h][f + e] = from_fp4(w[e], sc);
          }
        } else {
          const char* row = block + (int64_t)in_page * v.ts + half * (kRow / 2);
#pragma unroll
          for (int f = 0; f < NF; ++f) kf[h][f] = *reinterpret_cast<const bf16x8*>(row + 16 * f);
        }
      }
      // rows 32*from.. in stages of 64; the thread's rows of a stage are kLoadRows apart
      const int piece = threadIdx.x % NP, sub = threadIdx.x / NP;
      const auto stage = [&](int first, int buf) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          const int in_stage = sub + j * kLoadRows, row = min(first + in_stage, s.R - 1), i = row / s.hpg;
          const char* qr = a.q + (row_at + (size_t)i * v.H + g * s.hpg + (row - i * s.hpg)) * kRow;
          __builtin_amdgcn_global_load_lds(
              (const __attribute__((address_space(1))) void*)(qr + (piece ^ q_swizzle<D>(in_stage)) * 16),
              (__attribute__((address_space(3))) void*)(qs[buf] + (wave * 64 / NP + j * kLoadRows) * kRow),
              16, 0, 0);
        }
        if (threadIdx.x < kStage) {
          const int row = first + threadIdx.x, i = min(row, s.R - 1) / s.hpg;
          float l = INFINITY;
          int p = -1;
          if (row < s.R) {
            const float lse = a.lse[row_at + (size_t)i * v.H + g * s.hpg + (row - i * s.hpg)];
            if (lse != -INFINITY) {
              l = lse * kLog2e;
              p = s.first + i;
            }
          }
          ls[buf][threadIdx.x] = l;
          ps[buf][threadIdx.x] = p;
          const uint64_t dead = __ballot(p < 0);
          if (threadIdx.x < 2) odd[buf][threadIdx.x] = (uint32_t)(dead >> (32 * threadIdx.x)) != 0;
        }
      };
      const int rows = to - from;           // of 32 each
      int buf = 0;
      __syncthreads();                      // the rows before are done with
      stage(32 * from, 0);
      for (int j = 0; j < rows; j += 2, buf ^= 1) {
        __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
        __syncthreads();
        if (j + 2 < rows) stage(32 * (from + j + 2), buf ^ 1);
        const int tw = t0 + 64 * wave;        // the wave's first token
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          if (j + u >= rows) break;
          f32x16 x[2];
#pragma unroll
          for (int f = 0; f < NF; ++f) {
            const int row = 32 * u + l32;
            const bf16x8 qf = *reinterpret_cast<const bf16x8*>(
                qs[buf] + row * kRow + (((half * NP / 2 + f) ^ q_swizzle<D>(row)) * 16));
#pragma unroll
            for (int h = 0; h < 2; ++h)
              x[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf, kf[h][f], f ? x[h] : f32x16{}, 0, 0, 0);
          }
          f32x4 l4[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            l4[e] = *reinterpret_cast<const f32x4*>(&ls[buf][32 * u + 8 * e + 4 * half]);
          // all rows see all tokens of the wave that there are
          const int r_first = 32 * (from + j + u), i_first = r_first / s.hpg;
          const int i_last = min(r_first + 31, s.R - 1) / s.hpg;
          const int te = min(tw + 64, s.n);
          const bool whole = !odd[buf][u] && te - 1 <= s.first + i_first &&
                             (tw > s.first + i_last - a.window || te <= a.sinks);
          if (whole) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int e = 0; e < 16; ++e)
                sum[h] += __builtin_amdgcn_exp2f(fmaf(x[h][e], a.scale, -l4[e >> 2][e & 3]));
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int p = ps[buf][32 * u + 8 * (e >> 2) + 4 * half + (e & 3)];
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const float w = __builtin_amdgcn_exp2f(fmaf(x[h][e], a.scale, -l4[e >> 2][e & 3]));
                sum[h] += sees(a, p, tw + 32 * h + l32) ? w : 0.f;
              }
            }
          }
        }
      }
    }
    // the two halves' rows; lane l32 of half h writes token 32 h + l32
#pragma unroll
    for (int h = 0; h < 2; ++h) sum[h] += __shfl_xor(sum[h], 32);
    const int t = t0 + 64 * wave + lane;
    const float add = half ? sum[1] : sum[0];
    if (shared_tile)
      a.part[((size_t)pair * a.n_split + split) * a.tiles * kTile + t] = add;
    else if (t < s.n)
      store_mass(v, s, t, add);
  }
}

// The splits' sums of the tokens within the bound, one after the other.
__global__ __launch_bounds__(kThreads) void mass_join(PagedView v, MassArgs a, RowList r) {
  const int b = blockIdx.x % r.n, layer = blockIdx.x / r.n;
  const Seq s = seq_of(v, a, r, layer, b);
  if (s.T == 0) return;
  const int bound = a.tiles * kTile;
  const float* part = a.part + (size_t)blockIdx.x * a.n_split * bound;
  for (int t = blockIdx.y * kThreads + threadIdx.x; t < min(s.n, bound); t += gridDim.y * kThreads) {
    float add = 0.f;
    for (int i = 0; i < a.n_split; ++i) add += part[(size_t)i * bound + t];
    store_mass(v, s, t, add);
  }
}

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
  const unsigned pairs = (unsigned)(v.n_layers * c.r.n);
  const unsigned blocks = pairs * c.s.blocks * c.s.n_split;
  if (c.s.many) {
    const auto go = [&](auto kernel) { kernel<<<blocks, kThreads, 0, st>>>(v, a, c.r); };
    if (v.d == 128) v.fp4 ? go(mass_many<128, true>) : go(mass_many<128, false>);
    else v.fp4 ? go(mass_many<64, true>) : go(mass_many<64, false>);
    if (c.s.n_split > 1) {
      const unsigned parts = (unsigned)std::min(c.s.tiles, std::max(1, (int)(2048 / pairs)));
      mass_join<<<dim3(pairs, parts), kThreads, 0, st>>>(v, a, c.r);
    }
    return (int)hipGetLastError();
  }
  const size_t lds = (size_t)v.G * 64 * sizeof(float);
  const auto go = [&](auto kernel) { kernel<<<blocks, kThreads, lds, st>>>(v, a, c.r); };
  if (v.fp4) v.d == 128 ? go(mass_few<__bf16, 128, true>) : go(mass_few<__bf16, 64, true>);
  else if (v.esz == 2) v.d == 128 ? go(mass_few<__bf16, 128, false>) : go(mass_few<__bf16, 64, false>);
  else v.d == 128 ? go(mass_few<float, 128, false>) : go(mass_few<float, 64, false>);
  return (int)hipGetLastError();
}

}  // namespace starkv
