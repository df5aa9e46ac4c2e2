// Device-side helpers of the decoder operators: 8-bit codes, the sequences of
// a call and cache addresses.
#pragma once

#include "../../include/convsel_lm.h"
#include "common.hpp"

namespace convsel {
namespace lm {

typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

constexpr float kMinScale = 7.888609052210118e-31f;  // 2^-100

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }

// A sequence's packed tokens, bounded by the call's.
struct Span {
  int first, count;
};
__device__ __forceinline__ Span span_of(const int32_t* offsets, int64_t b, int tokens) {
  const int lo = clampi(offsets[b], 0, tokens);
  const int hi = clampi(offsets[b + 1], lo, tokens);
  return {lo, hi - lo};
}

// How a call's sequences are dealt to workgroups, whose third axis it is.
//
// In one row: the work of sequence b, in units, starts at base(b) = offsets[b] *
// num / 2^shift + b, and it has one unit at least; num over 2^shift are the units
// of a token, and what they round off is less than the one more.  (Units behind
// offsets[seqs] are the last sequence's too, beyond what it needs.)  So a long
// sequence among short ones has its share of workgroups, which a plan by the
// average denies it (a prompt of 4096 tokens beside 127 single ones: attention
// 7.0 ms, where apart they take 0.3 and 0.1).  Each unit searches its sequence,
// first where it stands if all are alike, then ever further from there, at last
// by halves.
//
// By sequence (num 0): the first axis is for a sequence's units, which it strides
// by.  Nothing is searched, which a workgroup of a microsecond would feel.
struct UnitRow {
  uint32_t first, seqs, num;  // first: the unit or sequence at which the launch starts
  int32_t tokens, shift;
  float per;                  // sequences a unit
};
struct Unit {
  int64_t seq;
  int index, count;  // its place among its sequence's units, and their number
  Span span;         // the sequence's tokens
  int length;        // and lengths[seq]
};
inline uint32_t units_of(const UnitRow& r) {  // below 2^32: no call has 2^31 tokens times num, nor sequences
  return r.num ? (static_cast<uint32_t>(r.tokens) * r.num >> r.shift) + r.seqs : r.seqs;
}
inline UnitRow unit_row(const convsel_kv_batch_t& b, int64_t num, int shift) {
  UnitRow r = {0, static_cast<uint32_t>(b.seqs), static_cast<uint32_t>(num), static_cast<int32_t>(b.tokens), shift, 0.f};
  r.per = static_cast<float>(b.seqs) / static_cast<float>(units_of(r));
  return r;
}
// launch(row, units) for all of them, as many at once as a grid's third axis holds.
template <typename F>
void each_grid(UnitRow r, const F& launch) {
  for (uint32_t left = units_of(r); left > 0;) {
    const uint32_t n = left < 65535 ? left : 65535;
    launch(r, n);
    left -= n;
    r.first += n;
  }
}
template <bool ROW>
__device__ __forceinline__ Unit find_unit(const UnitRow& r, const int32_t* offsets, const int32_t* lengths) {
  const uint32_t unit = r.first + blockIdx.z;
  if constexpr (!ROW)
    return {unit, static_cast<int>(blockIdx.x), static_cast<int>(gridDim.x), span_of(offsets, unit, r.tokens),
            lengths[unit]};
  uint32_t lo = 0, hi = r.seqs;  // base(lo) <= unit < base(hi)
  uint32_t b = min(static_cast<uint32_t>((static_cast<float>(unit) + 0.5f) * r.per), hi - 1), step = 1;
  for (;;) {
    const Span span = span_of(offsets, b, r.tokens);
    const int length = lengths[b];
    const uint32_t base = (span.first * r.num >> r.shift) + b;
    const uint32_t next = ((span.first + span.count) * r.num >> r.shift) + b + 1;
    // Offsets that do not rise are nobody's; the search still ends, and what it gives stays within bounds.
    const bool low = base > unit && b > lo, high = next <= unit && b + 1 < hi;
    if (!low && !high)
      return {b, static_cast<int>(unit > base ? min(unit - base, 0x7fffffffu) : 0u), static_cast<int>(next - base), span,
              length};
    (low ? hi : lo) = low ? b : b + 1;
    b = hi - lo <= 2 * step ? lo + ((hi - lo) >> 1) : low ? hi - step : lo + step - 1;
    step = min(2 * step, 1u << 30);
  }
}

// Value that a code stands for, before its scale.
__device__ __forceinline__ float decode(uint32_t byte, int format) {
  if (format == CONVSEL_KV_INT8) return static_cast<float>(static_cast<int8_t>(byte));
  return __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(byte), 0);
}

// Code of x in a block of scale s: the fp32 quotient, rounded to nearest even.
__device__ __forceinline__ uint32_t encode(float x, float s, int format) {
  float t = x / s;
  t = t != t ? 0.f : t;
  if (format == CONVSEL_KV_INT8) {
    t = fminf(fmaxf(t, -127.f), 127.f);
    return static_cast<uint32_t>(static_cast<int>(rintf(t))) & 0xffu;
  }
  t = fminf(fmaxf(t, -448.f), 448.f);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(t, t, 0, false)) & 0xffu;
}

__device__ __forceinline__ float qmax_of(int format) { return format == CONVSEL_KV_INT8 ? 127.f : 448.f; }

// Byte of value code (t, d) within a page and head.
__device__ __forceinline__ int v_byte(int t, int d, int dp) {
  return (t & ~15) * dp + (((t & 15) >> 2) * 16 + (d & 15)) * (dp >> 2) + (d >> 4) * 4 + (t & 3);
}

template <typename T, int ACT>
__device__ __forceinline__ float activate(float z) {
  constexpr bool exact = sizeof(T) == 4;  // fp32 outputs show the last bits of exp and the quotient
  if constexpr (ACT == CONVSEL_ACT_RELU) return z < 0.f ? 0.f : z;  // NaN stays
  if constexpr (ACT == CONVSEL_ACT_GELU) {
    // Phi(-a) = e^(-a^2 / 2) R(a), where R falls slowly from 1/2: t P(t) with t = 1 / (1 + 0.21 a) and P of degree 8,
    // fitted for its relative error, 7e-8 at most on 0 .. 14, where Phi leaves fp32.  Left of zero gelu is far smaller
    // than z, and 1 + erf would cancel (a wrong first digit at -6).
    const float a = fminf(fabsf(z), 64.f);  // a^2 stays finite
    const float t = exact ? 1.f / (1.f + 0.21f * a) : __builtin_amdgcn_rcpf(1.f + 0.21f * a);
    float p = -0.0716561838f;
    p = fmaf(p, t, 0.283587965f);
    p = fmaf(p, t, -0.330252068f);
    p = fmaf(p, t, 0.349399428f);
    p = fmaf(p, t, -0.0939240670f);
    p = fmaf(p, t, 0.124872222f);
    p = fmaf(p, t, 0.0691923046f);
    p = fmaf(p, t, 0.0850688382f);
    p = fmaf(p, t, 0.0837115769f);
    const float sq = a * a;
    // fp32 outputs show what the square rounds off, half of it in the exponent; bf16 ones do not (within 2^-17).
    const float e = exact ? expf(-0.5f * sq) * (1.f - 0.5f * fmaf(a, a, -sq)) : __expf(-0.5f * sq);
    const float tail = p * t * e;
    return z < 0.f ? z * tail : z * (1.f - tail);
  }
  if constexpr (ACT == CONVSEL_ACT_GELU_TANH) {
    // (1 + tanh u) / 2 = 1 / (1 + exp(-2u))
    const float u2 = -1.5957691216057308f * (z + 0.044715f * z * z * z);
    return exact ? z / (1.f + expf(u2)) : z * __builtin_amdgcn_rcpf(1.f + __expf(u2));
  }
  if constexpr (ACT == CONVSEL_ACT_SILU)
    return exact ? z / (1.f + expf(-z)) : z * __builtin_amdgcn_rcpf(1.f + __expf(-z));
  return z;
}

template <typename T, int ACT, int N>
__device__ __forceinline__ void activate_all(float (&z)[N][4]) {
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) z[n][i] = activate<T, ACT>(z[n][i]);
}

// One choice for all of the values.
template <typename T, int N>
__device__ __forceinline__ void activate_all(float (&z)[N][4], int act) {
  switch (act) {
    case CONVSEL_ACT_RELU: return activate_all<T, CONVSEL_ACT_RELU>(z);
    case CONVSEL_ACT_GELU: return activate_all<T, CONVSEL_ACT_GELU>(z);
    case CONVSEL_ACT_GELU_TANH: return activate_all<T, CONVSEL_ACT_GELU_TANH>(z);
    case CONVSEL_ACT_SILU: return activate_all<T, CONVSEL_ACT_SILU>(z);
    default: return;
  }
}

}  // namespace lm
}  // namespace convsel
