// Attention of packed prompts over their own keys and values, in fp32 and bf16.
//
// A workgroup of four waves has 128, 64 or 32 rows of a key head (a row is a query
// and one of the heads that share the key head), 32 a wave, and walks the keys
// that they see in tiles, whose keys and values go to LDS by DMA as they lie in
// memory, a tile ahead: one barrier a tile.  With fewer than 128 rows the waves
// of a block of 32 share out each tile's keys, and their results meet at the end.
//
// Scores are K q^T in blocks of 32 x 32, so that a lane ends with 16 keys of one
// row, in runs of four, and feeds its weights to the second product, V^T P^T,
// without moving them: in which order a product takes the keys does not matter
// while both operands agree.  V's operand needs four keys of one column a lane,
// which the transposing LDS read gives for bf16 and single words for fp32.
//
// In LDS a row's 16-byte units are permuted so that the rows that are read
// together fall on different banks: unit u of row r lies at u ^ turn(r), where
// turn() takes as many values as rows of U units meet on the same banks.
//
// Softmax in one pass, in powers of two (the scale carries log2 e): running
// maximum m and sum l of a row, weights 2^(s - m).  bf16 calls multiply each
// weight as three bf16 numbers, which hold all of its 24 bits: with two, 16 bits,
// 20 % less time, 0.20 % of the results of 8192 tokens were a neighbour of the
// rounded one, where fp32 steps throughout leave 0.08 and three numbers 0.06.
// fp32 calls use the fp32 matrix instructions.
//
// What bounds it.  Heads of 128 and more, long: the matrix cores (64 % busy at 1.84
// GHz), two thirds of whose work with values is the weights' second and third
// numbers, and the vector unit beside them (50 %): 8192 tokens of 32 heads on 8,
// causal: 917 us, 600 TFLOP/s, 1200 with those numbers (980 on a card of lower
// clock).  Heads of 64: the vector unit (75 % busy; 8192 tokens of 16 on 4: 300 us,
// 458 TFLOP/s); a weight costs a fused product, a transcendental (four slots), an
// addition, seven halves of an operation for its three numbers and half a maximum.
// fp32: the fp32 products (2048 tokens of 12 heads of 128 on 4: 160 us, 81 TFLOP/s).
#include <stdio.h>

#include <type_traits>

#include "igemm_common.hpp"
#include "lm_common.hpp"
#include "lm_kernels.hpp"

namespace convsel {
namespace {

using namespace igemm;
using namespace lm;

constexpr float kInf = __builtin_inff();
constexpr int kWaves = 4;

struct PromptLaunch {
  PromptArgs g;
  int group, y_vec;
  float scale;  // times log2 e
  UnitRow units;
  uint32_t magic, shift;  // row / group = row * magic >> shift

  // magic = ceil(2^shift / group), shift = 31 + ceil(log2 group): exact for rows below 2^31.
  __device__ __forceinline__ int token_of(int row) const {
    return static_cast<int>((static_cast<uint64_t>(static_cast<uint32_t>(row)) * magic) >> shift);
  }
};

typedef __attribute__((address_space(3))) char lds_char_t;
typedef const __attribute__((address_space(3))) u32x4_t lds_u32x4_t;
typedef uint32_t u32x2v_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float low_half(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_half(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// The largest of three, of which the compiler would first quiet signalling NaN, an operation each.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm volatile("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
// w less a number of a pair of bf16, in one operation: the pair's product with (-1, 0) or (0, -1) added to w.
typedef __bf16 bf16x2v_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float less(float w, uint32_t pair, uint32_t which) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2v_t, pair), __builtin_bit_cast(bf16x2v_t, which), w,
                                         false);
}

// Sizes of a tile: T elements, rows of 32 NC columns, R blocks of 32 rows.  The four waves are R blocks of rows times G
// groups of keys.
template <typename T, int NC, int R>
struct Shape {
  static constexpr int ES = elem<T>::bytes, UE = elem<T>::per16;
  static constexpr int G = kWaves / R, ROWS = 32 * R;
  static constexpr int SB = ES == 2 && G == 1 ? 2 : 1;        // blocks of 32 keys of a wave
  static constexpr int KT = 32 * SB * G;                      // keys; prompt_attention_describe() says them too
  static constexpr int RB = 32 * NC * ES, U = RB / 16;        // bytes and units of a row
  static constexpr int QU = U / 2;                            // units of a lane's half of a row
  static constexpr int TILE = KT * RB, NDMA = TILE / 1024 / kWaves;
  static constexpr int BUFS = 4 * TILE <= 144 * 1024 ? 2 : 1;  // tiles in LDS
  // Workgroups that a CU holds.
  static constexpr int PER_CU = ES == 2 && NC <= 4 && TILE <= 20 * 1024 - 16 ? (NC <= 2 && KT == 64 ? 3 : 2) : 1;
  __device__ static __forceinline__ int turn_k(int r) {
    return U % 16 == 0 ? r & 15 : U % 8 == 0 ? (r >> 1) & 7 : (r >> 2) & 3;
  }
  // bf16: four rows, of which 64 bytes are read, meet; fp32: a row and the fourth from it.
  __device__ static __forceinline__ int turn_v(int r) {
    if constexpr (ES == 2) return U % 16 == 0 ? (r & 3) << 2 : U % 8 == 0 ? ((r >> 1) & 1) << 2 : 0;
    return U % 16 == 0 ? ((r >> 2) & 1) << 3 : 0;
  }
};

template <typename T, int NC, int R>
__global__ __launch_bounds__(64 * kWaves, (Shape<T, NC, R>::PER_CU)) void prompt_attention_kernel(PromptLaunch a) {
  typedef Shape<T, NC, R> S;
  constexpr int ES = S::ES, UE = S::UE, KT = S::KT, SB = S::SB, RB = S::RB, U = S::U, QU = S::QU, TILE = S::TILE;
  constexpr int NDMA = S::NDMA, G = S::G, ROWS = S::ROWS, BUFS = S::BUFS;
  constexpr bool PIPED = ES == 2;
  constexpr uint32_t kNowhere = 0xfffffff0u;  // beyond every buffer: zeros
  __shared__ __align__(1024) char lds[2 * BUFS * TILE];  // keys of the tiles, then values
  __shared__ int spoilt[kWaves];
  const PromptArgs& g = a.g;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int head = blockIdx.x;  // heads vary fastest: eight of them have an XCD's L2 each
  const Unit un = find_unit<true>(a.units, g.offsets, g.offsets);
  const Span sp = un.span;
  const int rows = sp.count * a.group;
  const int ntile = (rows + ROWS - 1) / ROWS;
  const int wrow = 32 * (wave % R), wkey = 32 * SB * (wave / R);  // the wave's first row, and key of a tile
  const uint32_t lds0 = lds_address(lds);

  // DMA instruction d of this wave fills units 64 (4 d + wave) .. of a tile, keys and values alike.  Where a row's
  // units divide 256 and rows 16 apart are turned alike, instructions differ by whole rows only.
  constexpr bool EVEN = 256 % U == 0 && 256 / U % 16 == 0;
  constexpr int ND = EVEN ? 1 : NDMA, STEP = EVEN ? 256 / U : 0;
  int drow[ND];
  uint32_t kvo[ND], vvo[ND];
  const uint32_t kstep = static_cast<uint32_t>(g.k_token * ES), vstep = static_cast<uint32_t>(g.v_token * ES);
  const int dim_units = (g.dim + UE - 1) / UE;
#pragma unroll
  for (int d = 0; d < ND; ++d) {
    const int s = (4 * d + wave) * 64 + lane, r = s / U, p = s % U;
    drow[d] = r;
    const int ku = p ^ S::turn_k(r), vu = p ^ S::turn_v(r);
    kvo[d] = ku < dim_units ? r * kstep + ku * 16 : kNowhere;
    vvo[d] = vu < dim_units ? r * vstep + vu * 16 : kNowhere;
  }
  // Tile of keys j0 .. of the sequence; rows behind its last key are zeros, whatever lies there.
  auto issue = [&](int buf, int j0, bool values) {
    const int n = min(KT, sp.count - j0);
    const int64_t tok = sp.first + j0;
    const T* src = values ? reinterpret_cast<const T*>(g.v) + tok * g.v_token + head * g.v_head
                          : reinterpret_cast<const T*>(g.k) + tok * g.k_token + head * g.k_head;
    const uint32_t step = values ? vstep : kstep;
    const u32x4_t r = dma_rsrc(src, (n - 1) * step + dim_units * 16);
#pragma unroll
    for (int d = 0; d < NDMA; ++d) {
      const uint32_t at = lds0 + (buf + (values ? BUFS : 0)) * TILE + (4 * d + wave) * 1024;
      const uint32_t vo = values ? vvo[EVEN ? 0 : d] : kvo[EVEN ? 0 : d];
      if constexpr (EVEN)
        dma16(r, at, drow[0] + d * STEP < n ? vo : kNowhere, d * STEP < n ? d * STEP * step : 0);
      else
        dma16(r, at, drow[d] < n ? vo : kNowhere, 0);
    }
  };

  if (un.index >= ntile) return;  // uniform
  // Every tile of rows has a unit.  Under a causal mask the last rows have the most keys: they start first.
  const int tile = ntile - 1 - un.index;
  const int r0 = tile * ROWS;
  // Keys that tokens t0..t1 see between them, and that every one of them sees.
  auto seen_by = [&](int t0, int t1, int& lo, int& hi, int& in_lo, int& in_hi) {
    hi = g.causal ? t1 + 1 : sp.count;
    in_hi = g.causal ? t0 + 1 : sp.count;
    lo = g.window > 0 ? max(0, t0 - g.window + 1) : 0;
    in_lo = g.window > 0 ? max(0, t1 - g.window + 1) : 0;
  };
  int lo, hi, in_lo, in_hi;
  seen_by(a.token_of(r0), a.token_of(min(r0 + ROWS - 1, rows - 1)), lo, hi, in_lo, in_hi);
  const int kt0 = lo / KT, kt1 = (hi + KT - 1) / KT;
  const int b0 = PIPED ? ((kt1 - kt0) & 1) ^ 1 : 0;  // the first tile's buffer
  issue(b0, kt0 * KT, false);
  issue(b0, kt0 * KT, true);
  if (PIPED && kt0 + 1 < kt1) issue(b0 ^ 1, kt0 * KT + KT, false);
  // This wave's rows and this lane's; rows past the last one work on the last one's values.
  const int w0 = min(r0 + wrow, rows - 1), w1 = min(r0 + wrow + 31, rows - 1);
  int wlo, whi;
  seen_by(a.token_of(w0), a.token_of(w1), wlo, whi, in_lo, in_hi);
  const bool idle = r0 + wrow >= rows;
  const int row = min(r0 + wrow + col, rows - 1);
  const int tok = a.token_of(row), hq = head * a.group + row - tok * a.group;
  const int row_hi = g.causal ? tok + 1 : sp.count;
  const int row_lo = g.window > 0 ? max(0, tok - g.window + 1) : 0;

  // The queries: lane (row, half) holds units half, half + 2 ... of its row.
  vec16 qf[QU];
  {
    const T* src = reinterpret_cast<const T*>(g.q) + (sp.first + tok) * g.q_token + hq * g.q_head;
#pragma unroll
    for (int u = 0; u < QU; ++u) {
      const int d = (2 * u + half) * UE;
      qf[u] = d < g.dim ? load16(src + d) : vec16_zero();
    }
    // The sign of the scale goes with the query: scores then grow with the products.
    if (a.scale < 0.f) {
#pragma unroll
      for (int u = 0; u < QU; ++u)
#pragma unroll
        for (int x = 0; x < 4; ++x) qf[u].d[x] ^= ES == 2 ? 0x80008000u : 0x80000000u;
    }
  }
  // Never zero: a masked score of -inf times it stays -inf.  The largest score times the least number is 2^-21.
  const float cs = fmaxf(fabsf(a.scale), 0x1p-149f);
  const float share = __builtin_amdgcn_ldexpf(1.f, __builtin_clz(sp.count) - 32);
  f32x16_t o[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i) o[i] = zero16();
  float m = -kInf, l = 0.f;

  // Scores of keys j0 .. that the lane's row does not see.
  auto hide = [&](f32x16_t (&sc)[SB], int j0) {
    const int lo_at = row_lo - j0 - 4 * half, hi_at = row_hi - j0 - 4 * half;
#pragma unroll
    for (int b = 0; b < SB; ++b)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int j = 32 * b + 8 * (v >> 2) + (v & 3);
        sc[b][v] = j >= lo_at && j < hi_at ? sc[b][v] : -kInf;
      }
  };
  // Brings the row's results to a new maximum.
  auto rescale = [&](float most) {
    const float mn = fmaxf(m, most);
    const float s = m == mn ? 1.f : __builtin_amdgcn_exp2f(m - mn);
    m = mn;
    l *= s;
#pragma unroll
    for (int i = 0; i < NC; ++i) o[i] *= s;
  };
  auto compute = [&](int buf, int j0, bool masked, auto exact_c) {
    const lds_char_t* kl = (lds_char_t*)lds + buf * TILE + wkey * RB;
    const lds_char_t* vl = (lds_char_t*)lds + (BUFS + buf) * TILE + wkey * RB;
    f32x16_t sc[SB];
#pragma unroll
    for (int b = 0; b < SB; ++b) sc[b] = zero16();
    constexpr int AHEAD = 2;  // operands on their way
    vec16 kf[AHEAD];
    auto key = [&](int n) {
      return __builtin_bit_cast(
          vec16, *(lds_u32x4_t*)(kl + (32 * (n % SB) + col) * RB + (((2 * (n / SB) + half) ^ S::turn_k(col)) << 4)));
    };
    static_for<AHEAD>([&](auto n) { kf[n] = key(n); });
    static_for<SB * QU>([&](auto n) {
      mfma_32x32<T>(sc[n % SB], kf[n % AHEAD], qf[n / SB]);
      if constexpr (n + AHEAD < SB * QU) kf[n % AHEAD] = key(n + AHEAD);
      __builtin_amdgcn_sched_barrier(0);
    });
    if (masked) hide(sc, j0);
    float most = -kInf;
#pragma unroll
    for (int b = 0; b < SB; ++b)
#pragma unroll
      for (int v = 0; v < 16; ++v) most = fmaxf(most, sc[b][v]);
    most = fmaxf(most, __shfl_xor(most, 32)) * cs;
    if (__any(most > m)) rescale(most);
    const float from = m == -kInf ? 0.f : m;  // a row with nothing yet: its weights are 2^-inf
#pragma unroll
    for (int b = 0; b < SB; ++b)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        sc[b][v] = __builtin_amdgcn_exp2f(fmaf(sc[b][v], cs, -from));
        if constexpr (decltype(exact_c)::value) sc[b][v] *= share;
        l += sc[b][v];
      }
    if constexpr (decltype(exact_c)::value) {
#pragma unroll 1
      for (int k = 0; k < 32 * SB; ++k) {
        const int v = 4 * ((k & 31) >> 3) + (k & 3);
        float mine = sc[0][v];
        if constexpr (SB == 2) mine = k < 32 ? mine : sc[1][v];
        const float w = __shfl(mine, col + 8 * (k & 4));
        if (j0 + k < row_lo || j0 + k >= row_hi) continue;
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
          for (int v4 = 0; v4 < 4; ++v4) {
            const int d = 32 * i + 8 * v4 + 4 * half;
            const lds_char_t* at = vl + k * RB + (((d / UE) ^ S::turn_v(k)) << 4) + d % UE * ES;
            float z[4];
            if constexpr (ES == 2) {
              const u32x2v_t t = *(const __attribute__((address_space(3))) u32x2v_t*)at;
              z[0] = low_half(t[0]); z[1] = high_half(t[0]); z[2] = low_half(t[1]); z[3] = high_half(t[1]);
            } else {
              const f32x4_t t = *(const __attribute__((address_space(3))) f32x4_t*)at;
              z[0] = t[0]; z[1] = t[1]; z[2] = t[2]; z[3] = t[3];
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) o[i][4 * v4 + x] = fmaf(w, z[x], o[i][4 * v4 + x]);
          }
      }
      return;
    }
    if constexpr (!PIPED) {
      constexpr int FAR = 8;
      float z[FAR];
      auto value = [&](int n) {  // of key 8 (v / 4) + 4 half + v % 4, v = n / NC, column 32 (n % NC) + col
        const int v = n / NC, k = 8 * (v >> 2) + 4 * half + (v & 3);
        return *(const __attribute__((address_space(3))) float*)(
            vl + k * RB + (((8 * (n % NC) + (col >> 2)) ^ S::turn_v(k)) << 4) + (col & 3) * 4);
      };
      static_for<FAR>([&](auto n) { z[n] = value(n); });
      static_for<16 * NC>([&](auto n) {
        o[n % NC] = __builtin_amdgcn_mfma_f32_32x32x2f32(z[n % FAR], sc[0][n / NC], o[n % NC], 0, 0, 0);
        if constexpr (n + FAR < 16 * NC) z[n % FAR] = value(n + FAR);
        __builtin_amdgcn_sched_barrier(0);
      });
    }
  };

  // Values that are not finite spoil products that they have no part in: a weight of zero, where they are hidden, or
  // the second or third part of one, which may be zero or negative.  Rows that end so go once more, adding up key by
  // key what they see.  So do rows of finite values whose sum leaves fp32, as the weights' sum divides it only at the
  // end: `share` makes the weights so small that all of them together are less than one.
  auto walk = [&](auto exact_c) {
    for (int kt = kt0; kt < kt1; ++kt) {
      const int buf = BUFS == 2 ? (kt - kt0) & 1 : 0, j0 = kt * KT;
      if (BUFS == 1 && kt > kt0) {
        lds_sync();  // all are done with the tile before
        issue(0, j0, false);
        issue(0, j0, true);
      }
      // This tile's DMAs are in; behind the barrier everyone's are, and all are done with the other buffer.
      CONVSEL_WAIT_VMCNT(0);
      lds_sync();
      if (BUFS == 2 && kt + 1 < kt1) {
        issue(buf ^ 1, j0 + KT, false);
        issue(buf ^ 1, j0 + KT, true);
      }
      const int jw = j0 + wkey, je = jw + 32 * SB;
      if (idle || jw >= whi || je <= wlo) continue;
      compute(buf, jw, !(jw >= in_lo && je <= in_hi), exact_c);
    }
  };
  // bf16: the scores of the next tile are formed among the softmax of this one, and its weights, 16 keys ahead, among
  // the products with its values: a wave's vector operations run beside its own matrix ones.
  auto piped = [&] {
    if constexpr (PIPED) {
      const auto fix = [] { __builtin_amdgcn_sched_barrier(0); };
      // Places of the lane's operands that differ by more than a constant.
      constexpr int PK = U % 16 == 0 ? 8 : U % 8 == 0 ? 4 : 2, PV = U % 16 == 0 ? 4 : U % 8 == 0 ? 2 : 1;
      lds_char_t *ka[PK], *va[PV];
#pragma unroll
      for (int j = 0; j < PK; ++j)
        ka[j] = (lds_char_t*)lds + (wkey + col) * RB + (((2 * j + half) ^ S::turn_k(col)) << 4);
      // Lane i16 of sixteen reads 8 bytes of values; their 4 keys x 16 columns come back transposed.
      const int i16 = lane & 15, vkey = 4 * half + (i16 >> 2);
      const int unit = 2 * ((lane >> 4) & 1) + ((i16 >> 1) & 1);
#pragma unroll
      for (int j = 0; j < PV; ++j)
        va[j] = (lds_char_t*)lds + 2 * TILE + (wkey + vkey) * RB + (((4 * j + unit) ^ S::turn_v(vkey)) << 4) +
                (i16 & 1) * 8;
      auto key = [&](int buf, int u, int b) {
        const u32x4_t w = *(lds_u32x4_t*)(ka[u % PK] + (buf * TILE + 32 * b * RB + u / PK * PK * 32));
        return __builtin_bit_cast(vec16, w);
      };
      auto value = [&](int buf, int kb, int i) {  // 16 keys from 16 kb on, columns 32 i ..
        vec16 r;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          lds_char_t* at = va[i % PV] + (buf * TILE + (16 * kb + 8 * p) * RB + i / PV * PV * 64);
          const v4s_t t = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t*)at);
          uint2 w;
          __builtin_memcpy(&w, &t, 8);
          r.d[2 * p] = w.x;
          r.d[2 * p + 1] = w.y;
        }
        return r;
      };
      // Products of a tile's scores, and operands of keys on their way.
      constexpr int NQ = SB * QU, AHEAD = NQ < 4 ? NQ : 4;
      auto scores = [&](auto buf_c, f32x16_t (&sc)[SB], auto between) {
        constexpr int buf = decltype(buf_c)::value;
        vec16 f[AHEAD];
        static_for<AHEAD>([&](auto n) { f[n] = key(buf, n / SB, n % SB); });
        static_for<SB>([&](auto b) { sc[b] = zero16(); });
        static_for<NQ>([&](auto n) {
          mfma_32x32<T>(sc[n % SB], f[n % AHEAD], qf[n / SB]);
          if constexpr (n + AHEAD < NQ) f[n % AHEAD] = key(buf, (n + AHEAD) / SB, (n + AHEAD) % SB);
          between(n);
          fix();
        });
      };
      constexpr int PARTS = 3;
      vec16 part[PARTS];  // of the weights of 16 keys, a lane's eight
      float from = 0.f;
      // Kept from the compiler, which would write (-1, 0) as the fp32 constant -1, which is (0, -1).
      uint32_t low = 0x0000bf80u, high = 0xbf800000u;
      asm volatile("" : "+s"(low), "+s"(high));
      // Weight e of a lane's eight of 16 keys kb, in its score's place.
      auto weigh = [&](f32x16_t (&sc)[SB], auto kb_c, auto e_c) {
        constexpr int kb = decltype(kb_c)::value, v = 8 * (kb & 1) + decltype(e_c)::value;
        const float w = __builtin_amdgcn_exp2f(fmaf(sc[kb >> 1][v], cs, -from));
        l += w;
        sc[kb >> 1][v] = w;
      };
      // Part p of weights 2 e and 2 e + 1: what the part before leaves of them, rounded.  Of 24 bits it leaves 16 at
      // most, and the next one 8: three parts hold all.
      auto split = [&](f32x16_t (&sc)[SB], auto kb_c, auto p_c, auto e_c) {
        constexpr int kb = decltype(kb_c)::value, p = decltype(p_c)::value, e = decltype(e_c)::value;
        constexpr int b = kb >> 1, v = 8 * (kb & 1) + 2 * e;
        if constexpr (p > 0) {
          sc[b][v] = less(sc[b][v], part[p - 1].d[e], low);
          sc[b][v + 1] = less(sc[b][v + 1], part[p - 1].d[e], high);
        }
        part[p].d[e] = f32x2_to_bf16x2(sc[b][v], sc[b][v + 1]);
      };
      const std::integral_constant<int, 0> zero{};
      // Tile it of the walk, whose scores are sc; the next one's go to nx.
      auto step = [&](int it, auto p_c, f32x16_t (&sc)[SB], f32x16_t (&nx)[SB], auto last_c) {
        constexpr int P = decltype(p_c)::value;
        constexpr bool LAST = decltype(last_c)::value;
        const int j0 = (kt0 + it) * KT, jw = j0 + wkey;
        // Formed before the barrier, whatever the compiler moves: max3() reads them without its knowledge.
#pragma unroll
        for (int b = 0; b < SB; ++b) asm volatile("" : "+v"(sc[b]));
        CONVSEL_WAIT_VMCNT(0);
        lds_sync();
        if (kt0 + it + 2 < kt1) issue(P, j0 + 2 * KT, false);
        if constexpr (!LAST) issue(P ^ 1, j0 + KT, true);
        if (!(jw >= in_lo && jw + 32 * SB <= in_hi)) hide(sc, jw);
        float most = -kInf;
        vec16 fv[NC];
        auto top = [&](auto n) {  // an eighth of the scores
          static_for<SB>([&](auto b) { most = max3(most, sc[b][2 * n], sc[b][2 * n + 1]); });
        };
        auto settle = [&] {
          const uint32_t mine = __float_as_uint(most);
          const auto both = __builtin_amdgcn_permlane32_swap(mine, mine, false, false);
          most = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * cs;
          // Weights may grow to 2^8 before the results are brought to a new maximum.
          if (__any(most > m + 8.f)) rescale(most);
          from = m == -kInf ? 0.f : m;  // a row with nothing yet: its weights are 2^-inf
        };
        auto first_values = [&] { static_for<NC>([&](auto i) { fv[i] = value(P, 0, i); }); };
        if constexpr (LAST) {
          first_values();
          static_for<8>(top);
          settle();
          static_for<8>([&](auto e) { weigh(sc, zero, e); });
          static_for<4>([&](auto e) { split(sc, zero, zero, e); });
        } else {
          constexpr int M = NQ >= 16 ? 4 : NQ >= 4 ? 2 : 1;  // products beside the maximum; 8 weights beside the others
          scores(std::integral_constant<int, P ^ 1>{}, nx, [&](auto n) {
            if constexpr (n < M)
              static_for<8 / M>([&](auto x) {
                  top(std::integral_constant<int, decltype(n)::value * (8 / M) + decltype(x)::value>{});
                });
            if constexpr (n == M - 1) {
              fix();
              settle();
            }
            constexpr int rest = NQ - M, i0 = n < M ? 0 : (n - M) * 8 / rest, i1 = n < M ? 0 : (n - M + 1) * 8 / rest;
            static_for<i1 - i0>(
                [&](auto e) { weigh(sc, zero, std::integral_constant<int, i0 + decltype(e)::value>{}); });
            if constexpr (n == (NQ > 4 ? NQ - 4 : 0)) first_values();
            if constexpr (n == NQ - 1) static_for<4>([&](auto e) { split(sc, zero, zero, e); });
          });
        }
        static_for<2 * SB>([&](auto kb) {
          static_for<PARTS * NC>([&](auto n) {
            constexpr int i = n % NC, p = n / NC;
            mfma_32x32<T>(o[i], fv[i], part[p]);
            // Beside the products with a part the next one, and the next 16 keys' weights and first part.
            constexpr bool next = kb + 1 < 2 * SB;
            const std::integral_constant<int, decltype(kb)::value + 1> kb1{};
            if constexpr (next && p == PARTS - 1) fv[i] = value(P, kb + 1, i);
            constexpr int s0 = i * 4 / NC, s1 = (i + 1) * 4 / NC;
            constexpr int i0 = n * 8 / (PARTS * NC), i1 = (n + 1) * 8 / (PARTS * NC);
            static_assert(p + 1 < PARTS || 2 * s1 <= i1, "split after they are weighed");
            if constexpr (p + 1 < PARTS)
              static_for<s1 - s0>([&](auto e) {
                split(sc, kb, std::integral_constant<int, p + 1>{},
                      std::integral_constant<int, s0 + decltype(e)::value>{});
              });
            if constexpr (next) {
              static_for<i1 - i0>([&](auto e) {
                weigh(sc, kb1, std::integral_constant<int, i0 + decltype(e)::value>{});
              });
              if constexpr (p == PARTS - 1)
                static_for<s1 - s0>([&](auto e) {
                  split(sc, kb1, zero, std::integral_constant<int, s0 + decltype(e)::value>{});
                });
            }
            fix();
          });
        });
      };
      const int count = kt1 - kt0;
      const std::integral_constant<int, 1> one{};
      f32x16_t sa[SB];
      // The first keys are in; behind the barrier everyone's are.
      if (count > 1) CONVSEL_WAIT_VMCNT(2 * NDMA);
      else CONVSEL_WAIT_VMCNT(NDMA);
      lds_sync();
      int it = 0;
      if (idle) {
        for (; it < count; ++it) {
          CONVSEL_WAIT_VMCNT(0);
          lds_sync();
          if (it + 2 < count) issue((it + b0) & 1, (kt0 + it + 2) * KT, false);
          if (it + 1 < count) issue(((it + b0) & 1) ^ 1, (kt0 + it + 1) * KT, true);
        }
        return;
      }
      // The last tile's scores are sa, so the first one's are sb if there is an even number: one copy of the last step.
      if (b0 != 0) {
        f32x16_t sb[SB];
        scores(one, sb, [](auto) {});
        asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");
        step(it++, one, sb, sa, std::false_type{});
      } else {
        scores(zero, sa, [](auto) {});
      }
      asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");  // max3() reads products' results unseen by the compiler
      for (; it + 1 < count; it += 2) {
        f32x16_t sb[SB];
        step(it, zero, sa, sb, std::false_type{});
        step(it + 1, one, sb, sa, std::false_type{});
      }
      step(it, zero, sa, sa, std::true_type{});
    }
  };
  if constexpr (PIPED)
    piped();
  else
    walk(std::false_type{});
  float odd = 0.f;  // NaN if a result is not finite
#pragma unroll
  for (int i = 0; i < NC; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) odd = fmaf(o[i][v], 0.f, odd);
  const int again = __any(odd != 0.f);
  if (lane == 0) spoilt[wave] = again;
  lds_sync();  // also before another tile is fetched
  if (spoilt[0] | spoilt[1] | spoilt[2] | spoilt[3]) {
#pragma unroll
    for (int i = 0; i < NC; ++i) o[i] = zero16();
    m = -kInf;
    l = 0.f;
    issue(0, kt0 * KT, false);
    issue(0, kt0 * KT, true);
    walk(std::true_type{});
    lds_sync();
  }

  l += __shfl_xor(l, 32);
  if constexpr (G > 1) {
    // The groups' results meet in the first one's waves, brought to the largest of their maxima.
    typedef __attribute__((address_space(3))) float lds_float_t;
    typedef __attribute__((address_space(3))) f32x4_t lds_f32x4_t;
    lds_float_t* stat = (lds_float_t*)(lds_char_t*)lds;
    lds_f32x4_t* part = (lds_f32x4_t*)((lds_char_t*)lds + 1024);
    if (half == 0) {
      stat[2 * (wave * 32 + col)] = m;
      stat[2 * (wave * 32 + col) + 1] = l;
    }
    lds_sync();
    float most = m, sum = 0.f;
#pragma unroll
    for (int x = 0; x < G; ++x) most = fmaxf(most, stat[2 * ((x * R + wave % R) * 32 + col)]);
#pragma unroll
    for (int x = 0; x < G; ++x) {
      const lds_float_t* at = stat + 2 * ((x * R + wave % R) * 32 + col);
      sum += at[1] * __builtin_amdgcn_exp2f(at[0] - most);
    }
    const float s = __builtin_amdgcn_exp2f(m - most);
    l = sum;
#pragma unroll
    for (int i = 0; i < NC; ++i) o[i] *= s;
    if (wave >= R) {
#pragma unroll
      for (int i = 0; i < NC; ++i)
#pragma unroll
        for (int v4 = 0; v4 < 4; ++v4)
          part[((wave - R) * NC * 4 + i * 4 + v4) * 64 + lane] =
              f32x4_t{o[i][4 * v4], o[i][4 * v4 + 1], o[i][4 * v4 + 2], o[i][4 * v4 + 3]};
    }
    lds_sync();
    if (wave >= R) return;
#pragma unroll
    for (int x = 1; x < G; ++x)
#pragma unroll
      for (int i = 0; i < NC; ++i)
#pragma unroll
        for (int v4 = 0; v4 < 4; ++v4) {
          const f32x4_t t = part[(((x - 1) * R + wave) * NC * 4 + i * 4 + v4) * 64 + lane];
#pragma unroll
          for (int e = 0; e < 4; ++e) o[i][4 * v4 + e] += t[e];
        }
  }
  // Lane (row, half) holds columns 32 i + 8 (v / 4) + 4 half + v % 4.
  if (r0 + wrow + col < rows) {
    const float inv = 1.f / l;
    T* dst = reinterpret_cast<T*>(g.y) + (sp.first + tok) * g.y_token + hq * g.y_head;
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int v4 = 0; v4 < 4; ++v4) {
        const int d = 32 * i + 8 * v4 + 4 * half;
        float v[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) v[x] = o[i][4 * v4 + x] * inv;
        if (a.y_vec) {
          if (d < g.dim) {
            if constexpr (ES == 4)
              *reinterpret_cast<float4*>(dst + d) = make_float4(v[0], v[1], v[2], v[3]);
            else
              *reinterpret_cast<uint2*>(dst + d) = make_uint2(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]));
          }
        } else {
#pragma unroll
          for (int x = 0; x < 4; ++x)
            if (d + x < g.dim) elem<T>::store(dst + d + x, v[x]);
        }
      }
  }
}

// Rows that cannot be read in 16-byte units where they lie, copied to [token][head] rows of whole ones.
template <typename T>
__global__ __launch_bounds__(256) void prompt_pack_kernel(const T* src, int64_t token, int64_t head, int64_t tokens,
                                                          int heads, int dim, int units, T* dst) {
  constexpr int UE = elem<T>::per16;
  const int64_t all = tokens * heads * units;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < all;
       i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t r = i / units, t = r / heads, h = r - t * heads;
    const int d = static_cast<int>(i - r * units) * UE;
    const T* row = src + t * token + h * head;
    uint32_t e[UE];
#pragma unroll
    for (int x = 0; x < UE; ++x) {
      const uint32_t bits = load_bits(row + min(d + x, dim - 1));
      e[x] = d + x < dim ? bits : 0u;
    }
    vec16 v;
    pack16<T>(v, e);
    store16(dst + i * UE, v);
  }
}

int64_t elem_bytes(const PromptArgs& a) { return a.dtype == CONV_F32 ? 4 : 2; }
int64_t row_units(const PromptArgs& a) { return (a.dim * elem_bytes(a) + 15) / 16; }

// Whether rows are no whole 16-byte units, or so far apart that a tile of 128 of them does not fit a buffer.
bool needs_pack(const PromptArgs& a, const void* p, int64_t token, int64_t head) {
  const int64_t es = elem_bytes(a), per = 16 / es, far = ((int64_t)1 << 31) / 128 / es - 256;
  return a.dim % per != 0 || token % per != 0 || head % per != 0 || (uintptr_t)p % 16 != 0 || token > far;
}

// Bytes of the copies of q, k and v.
struct Packs {
  size_t q, k, v;
};
Packs packs_of(const PromptArgs& a) {
  auto bytes = [&](int heads) { return ((size_t)(a.tokens * heads * row_units(a) * 16) + 255) / 256 * 256; };
  Packs p;
  p.q = needs_pack(a, a.q, a.q_token, a.q_head) ? bytes(a.q_heads) : 0;
  p.k = needs_pack(a, a.k, a.k_token, a.k_head) ? bytes(a.kv_heads) : 0;
  p.v = needs_pack(a, a.v, a.v_token, a.v_head) ? bytes(a.kv_heads) : 0;
  return p;
}

template <typename T>
void pack(const PromptArgs& g, const void*& src, int64_t& token, int64_t& head, int heads, size_t bytes, char*& ws,
          hipStream_t st) {
  if (bytes == 0) return;
  const int64_t units = row_units(g), blocks = (g.tokens * heads * units + 255) / 256;
  hipLaunchKernelGGL(prompt_pack_kernel<T>, dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, st,
                     (const T*)src, token, head, g.tokens, heads, g.dim, (int)units, (T*)ws);
  src = ws;
  head = units * elem<T>::per16;
  token = heads * head;
  ws += bytes;
}

template <typename T, int NC, int R>
hipError_t launch_rows(PromptLaunch a, hipStream_t st) {
  each_grid(a.units, [&](const UnitRow& r, unsigned n) {
    a.units = r;
    const dim3 grid((unsigned)a.g.kv_heads, 1, n);
    hipLaunchKernelGGL((prompt_attention_kernel<T, NC, R>), grid, dim3(64 * kWaves), 0, st, a);
  });
  return hipGetLastError();
}

// Whether tiles of so many blocks of rows fit in LDS: two of them in bf16, one at least in fp32.
constexpr bool fits(int blocks, int es, int nc) {
  return blocks == 4 || (es == 2 ? 4 : 2) * (blocks == 2 ? 64 : 128) * 32 * nc * es <= 144 * 1024;
}

UnitRow units_for(const PromptArgs& g, int blocks) {
  convsel_kv_batch_t b = {};
  b.seqs = g.seqs;
  b.tokens = g.tokens;
  return unit_row(b, g.q_heads / g.kv_heads, blocks == 4 ? 7 : blocks == 2 ? 6 : 5);
}

// Blocks of 32 rows a workgroup: four, or, where that gives few workgroups, two or one, whose keys the waves share out.
// us of the kernel with four, two and one:
//   bf16, 32/8 heads of 128, 512, 700, 1024, 2048 tokens   21 16 20 | 28 21 32 | 37 29 49 | 82 78 141
//         8/8 heads of 128, 400, 1024, 2048, 4096          18 13 12 | 36 24 19 | 64 43 38 | 122 91 115
//         16/4 heads of 64, 400, 1024, 2048, 4096          13 10 8 | 25 17 13 | 44 31 31 | 94 82 95
//         8/2 heads of 256, 4096, 8192                     211 154 | 478 546
//   fp32, 8/8 heads of 64, 300, 1024, 2048                 29 18 13 | 85 47 29 | 165 88 58
//         12/4 heads of 80, 300, 1024, 2048                40 24 18 | 118 64 40 | 230 123 129
//         32/8 heads of 128, 300, 701                      50 31 25 | 106 61 72
// One block has most to join, so sequences are to be long enough for it:
//   bf16, 8/8 heads of 128, 64, 200 tokens                 6.8 6.9 8.3 | 12.5 9.8 9.4
//         16/4 heads of 64, 64, 200                        6.0 5.3 5.6 | 9.0 7.3 6.4
//   fp32, 12/4 heads of 80, 37, 100                        11.7 8.8 9.7 | 18.5 12.4 9.7
// Every sequence counts as a workgroup of each head at least, so many short ones beside a long one lead to four blocks
// too early (2048 tokens of 8/8 heads of 128 and 60 prompts of one token: 65, 42 with two).
int blocks_for(const PromptArgs& g) {
  const bool f32 = g.dtype == CONV_F32;
  // Workgroups that are enough, of four blocks and of two.
  const int64_t enough[2] = {!f32 && (g.dim > 128 || !g.causal) ? 400 : 560, f32 && g.dim <= 64 ? 512 : 256};
  int best = 4;
  for (int blocks = 2; blocks > 0; blocks /= 2) {
    if ((int64_t)units_of(units_for(g, best)) * g.kv_heads >= enough[best == 2]) break;
    if (blocks == 1 && g.tokens < g.seqs * (f32 ? 64 : 3 * (int64_t)g.dim)) break;
    if (fits(blocks, (int)elem_bytes(g), (g.dim + 31) / 32)) best = blocks;
  }
  return best;
}

template <typename T, int NC>
hipError_t launch_nc(PromptLaunch a, hipStream_t st) {
  const int blocks = blocks_for(a.g);
  a.units = units_for(a.g, blocks);
  if constexpr (fits(1, sizeof(T), NC)) {
    if (blocks == 1) return launch_rows<T, NC, 1>(a, st);
  }
  if constexpr (fits(2, sizeof(T), NC)) {
    if (blocks == 2) return launch_rows<T, NC, 2>(a, st);
  }
  return launch_rows<T, NC, 4>(a, st);
}

template <typename T>
hipError_t launch(const PromptArgs& g, void* workspace, hipStream_t st) {
  PromptLaunch a;
  a.g = g;
  const Packs p = packs_of(g);
  char* ws = (char*)workspace;
  pack<T>(g, a.g.q, a.g.q_token, a.g.q_head, g.q_heads, p.q, ws, st);
  pack<T>(g, a.g.k, a.g.k_token, a.g.k_head, g.kv_heads, p.k, ws, st);
  pack<T>(g, a.g.v, a.g.v_token, a.g.v_head, g.kv_heads, p.v, ws, st);
  a.group = g.q_heads / g.kv_heads;
  a.scale = g.scale * 1.4426950408889634f;
  a.shift = 31;
  while (((int64_t)1 << (a.shift - 31)) < a.group) ++a.shift;
  a.magic = (uint32_t)((((uint64_t)1 << a.shift) + a.group - 1) / a.group);
  a.y_vec = g.dim % 4 == 0 && g.y_token % 4 == 0 && g.y_head % 4 == 0 && (uintptr_t)g.y % (4 * sizeof(T)) == 0;
  switch ((g.dim + 31) / 32) {
    case 1: return launch_nc<T, 1>(a, st);
    case 2: return launch_nc<T, 2>(a, st);
    case 3: return launch_nc<T, 3>(a, st);
    case 4: return launch_nc<T, 4>(a, st);
    case 5: return launch_nc<T, 5>(a, st);
    case 6: return launch_nc<T, 6>(a, st);
    case 7: return launch_nc<T, 7>(a, st);
    default: return launch_nc<T, 8>(a, st);
  }
}

}  // namespace

size_t prompt_attention_workspace(const PromptArgs& a) {
  const Packs p = packs_of(a);
  return p.q + p.k + p.v;
}

hipError_t launch_prompt_attention(const PromptArgs& a, void* workspace, hipStream_t stream) {
  return a.dtype == CONV_F32 ? launch<float>(a, workspace, stream) : launch<bf16_t>(a, workspace, stream);
}

void prompt_attention_describe(const PromptArgs& a, char* buf, size_t len) {
  const int blocks = blocks_for(a);
  const int keys = blocks == 4 ? (a.dtype == CONV_F32 ? 32 : 64) : 128 / blocks;  // Shape::KT
  const size_t workspace = prompt_attention_workspace(a);
  snprintf(buf, len, "prompt_attention kernels=%sprompt_attention_kernel rows=%d keys=%d workspace=%zu",
           workspace ? "prompt_pack_kernel;" : "", 32 * blocks, keys, workspace);
}

}  // namespace convsel
