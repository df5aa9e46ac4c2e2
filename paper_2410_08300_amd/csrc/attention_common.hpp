// What the attention kernels share.
//
// Mathematics.  With codes K, V and one scale a block of tokens, a query's score
// is s_j = scale * ks * (q . K_j) and its result sum_j e^(s_j) vs V_j / sum_j
// e^(s_j).  Everything runs in powers of two (scale carries log2 e).  vs = vf *
// 2^ve; the running maximum M is a whole number of at least s_j + ve (so that
// M - ve is exact), and
//   u_j = 2^(s_j + ve - M)
//   result = sum_j (u_j vf) V_j / sum_j u_j 2^-ve
// holds the largest weight times its value scale near one: a page of small
// values may hold the weight, and no scale overflows.  Scales reach from 2^-100
// to 2^121, so a change of M is an exponent added, and where u would leave fp32
// (scales 2^100 apart within a row) the sum's terms are formed without it.
// Weights go to the matrix cores as two 16-bit floats, 22 bits, 2^15 times as
// large (their steps are then 2^-39 of the largest); codes are exact in one.
// One number, 11 bits, turns 7 % of bf16 results into a neighbour of the rounded
// one, though it saves a fifth of a long prompt (4096 tokens of 32 heads of 128
// on 8: 194 us, 241 with two).  fp32 calls hold queries as two such numbers;
// bf16 queries are exact in one, brought to [2^14, 2^15) by a power of two, but
// for elements below 2^-32 of a head's largest.  Sums and statistics are fp32.
#pragma once

#include "lm_common.hpp"
#include "lm_kernels.hpp"

namespace convsel {
namespace lm {

// A call as the kernels take it.  `part` and `stat` hold the parts of a split
// axis: for each (token, head) nsplit rows of results before the division, of
// whole 16-byte units, and (maximum, sum) pairs.
struct AttnArgs {
  int64_t pages, table_width;
  int64_t q_token, q_head, y_token, y_head;
  int tokens, kv_heads, group, dim, ps_shift, causal, window, nsplit, q_vec, y_vec;
  float scale;  // times log2 e
  UnitRow units;  // tiles of rows, of all sequences in one row
};

struct AttnPointers {
  const void* q;
  const uint8_t* k_codes;
  const uint8_t* v_codes;
  const float* k_scales;
  const float* v_scales;
  const int32_t* table;
  const int32_t* lengths;
  const int32_t* offsets;
  void* y;
  float* part;
  float* stat;
};

// Four codes as 16-bit floats, exactly.
template <int FMT>
__device__ __forceinline__ void widen4(uint32_t w, f16x2_t& lo, f16x2_t& hi) {
  if constexpr (FMT == CONVSEL_KV_INT8) {
    // 1024 + (code + 128) has the code's byte as its lowest bits.
    const uint32_t u = w ^ 0x80808080u;
    const f16x2_t off = {static_cast<_Float16>(-1152.f), static_cast<_Float16>(-1152.f)};
    lo = __builtin_bit_cast(f16x2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) + off;
    hi = __builtin_bit_cast(f16x2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) + off;
  } else {
    lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false);
    hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true);
  }
}

template <int FMT>
__device__ __forceinline__ f16x8_t widen8(uint32_t a, uint32_t b) {
  f16x2_t p[4];
  widen4<FMT>(a, p[0], p[1]);
  widen4<FMT>(b, p[2], p[3]);
  f16x8_t r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[2 * i] = p[i][0];
    r[2 * i + 1] = p[i][1];
  }
  return r;
}

constexpr float kWeight = 0x1p15f;  // weights as the matrix cores take them, and back
constexpr float kResult = 0x1p-15f;
constexpr float kFar = -100.f;      // exponents of u below this are near the end of fp32

// A value scale as mantissa and exponent.  Zero, which a page has that nothing was written to yet, takes the exponent of
// the least scale that a write gives: its values are zeros, and must not raise the maximum above what others need.
__device__ __forceinline__ float split_scale(float s, int& e) {
  const float f = frexpf(s, &e);
  if (s == 0.f) e = -99;
  return f;
}

// Exponent to add to what was kept at maximum `from`, now at `to` >= from.
__device__ __forceinline__ int shift_of(float from, float to) {
  return from == to ? 0 : static_cast<int>(fmaxf(from - to, -300.f));
}

// Power of two that brings magnitudes up to amax under 2^15.
__device__ __forceinline__ int query_exponent(float amax) {
  int e = 0;
  if (amax > 0.f && amax < __builtin_inff()) frexpf(amax, &e);
  return e - 15;
}

}  // namespace lm

// Many query rows (attention_tiles.hip): 128 of them a workgroup, or 256 where
// attention_tiles_wide() has them.
bool attention_tiles_wide(int dtype, int head_dim);
hipError_t launch_attention_tiles(const lm::AttnPointers& p, const lm::AttnArgs& a, int dtype, int format, int rows,
                                  hipStream_t stream);

}  // namespace convsel
