// What the linear-layer kernels share.
#pragma once

#include "lm_common.hpp"
#include "lm_kernels.hpp"

namespace convsel {
namespace lm {

typedef float f32x4v_t __attribute__((ext_vector_type(4)));

// One 16-byte unit of a 16 x 16 product's operands: 8 bf16 or 4 fp32 of a lane.
__device__ __forceinline__ f32x4v_t mac16(bf16_t, const vec16& a, const vec16& b, f32x4v_t c) {
  bf16x8_t av, bv;
  __builtin_memcpy(&av, &a, 16);
  __builtin_memcpy(&bv, &b, 16);
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, bv, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4v_t mac16(float, const vec16& a, const vec16& b, f32x4v_t c) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.d[i]), __uint_as_float(b.d[i]), c, 0, 0, 0);
  return c;
}

// The biases of outputs o .. o + 3.
template <typename T>
__device__ __forceinline__ void load_bias4(const LinearArgs& g, int64_t o, float (&b)[4]) {
  const T* B = reinterpret_cast<const T*>(g.b);
#pragma unroll
  for (int i = 0; i < 4; ++i) b[i] = B && o + i < g.out ? elem<T>::load(B + o + i) : 0.f;
}

// Outputs o .. o + 3 of N rows m, m + step ... from their sums z: bias,
// activation, residual, one rounding.  `vec`: every row of y and r starts on a
// whole unit of four.
template <typename T, int N>
__device__ __forceinline__ void finish4(const LinearArgs& g, int64_t m, int step, int64_t o, float (&z)[N][4],
                                        const float (&bias)[4], bool vec) {
  const T* R = reinterpret_cast<const T*>(g.r);
  T* Y = reinterpret_cast<T*>(g.y) + m * g.ldy + o;
  const int64_t left = g.m - m, ldy = step * g.ldy, ldr = step * g.ldr;
  const bool whole = vec && o + 4 <= g.out;
  float r[N][4];
  if (R) {
    R += m * g.ldr + o;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const T* p = n * step < left ? R + n * ldr : R;
      if (whole) {
        if constexpr (sizeof(T) == 4) {
          const float4 v = *reinterpret_cast<const float4*>(p);
          r[n][0] = v.x; r[n][1] = v.y; r[n][2] = v.z; r[n][3] = v.w;
        } else {
          const uint2 v = *reinterpret_cast<const uint2*>(p);
          r[n][0] = bf16_to_f32(v.x & 0xffffu); r[n][1] = bf16_to_f32(v.x >> 16);
          r[n][2] = bf16_to_f32(v.y & 0xffffu); r[n][3] = bf16_to_f32(v.y >> 16);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) r[n][i] = elem<T>::load(p + (o + i < g.out ? i : 0));
      }
    }
  }
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) z[n][i] += bias[i];
  activate_all<T, N>(z, g.act);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (n * step >= left) break;
    if (R) {
#pragma unroll
      for (int i = 0; i < 4; ++i) z[n][i] += r[n][i];
    }
    T* p = Y + n * ldy;
    if (whole) {
      if constexpr (sizeof(T) == 4)
        *reinterpret_cast<float4*>(p) = make_float4(z[n][0], z[n][1], z[n][2], z[n][3]);
      else
        *reinterpret_cast<uint2*>(p) = make_uint2(f32x2_to_bf16x2(z[n][0], z[n][1]), f32x2_to_bf16x2(z[n][2], z[n][3]));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (o + i < g.out) elem<T>::store(p + i, z[n][i]);
    }
  }
}

}  // namespace lm

// Tiles of 64 to 256 rows and outputs (linear_tiles.hip).
struct LinearTiles {
  int config;  // -1: operands out of the kernel's reach
  int splits;
  bool pack;   // operands are copied to rows of whole 16-byte units first
  size_t part_bytes, pack_bytes;
  double us;   // what it should take
};
LinearTiles linear_tiles_plan(const LinearArgs& a);
hipError_t launch_linear_tiles(const LinearArgs& a, const LinearTiles& p, void* workspace, hipStream_t stream);
const char* linear_tiles_name(int config);

}  // namespace convsel
