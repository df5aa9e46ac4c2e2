// What the linear-layer kernels share.
#pragma once

#include "lm_common.hpp"
#include "lm_kernels.hpp"

namespace convsel {
namespace lm {

// Four neighbouring outputs o .. o + 3 of row m from their sums: bias,
// activation, residual, one rounding.  `vec`: every row of y and r starts on a
// whole unit of four.
template <typename T>
__device__ __forceinline__ void finish4(const LinearArgs& g, int64_t m, int64_t o, const float (&sum)[4], bool vec) {
  const T* B = reinterpret_cast<const T*>(g.b);
  const T* R = reinterpret_cast<const T*>(g.r);
  T* Y = reinterpret_cast<T*>(g.y) + m * g.ldy + o;
  if (R) R += m * g.ldr + o;
  const bool whole = o + 4 <= g.out;
  float z[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    z[i] = sum[i];
    if (B) z[i] += elem<T>::load(B + (whole || o + i < g.out ? o + i : o));
    z[i] = activate<T>(z[i], g.act);
  }
  if (vec && whole) {
    if constexpr (sizeof(T) == 4) {
      float4 v = make_float4(z[0], z[1], z[2], z[3]);
      if (R) {
        const float4 r = *reinterpret_cast<const float4*>(R);
        v.x += r.x; v.y += r.y; v.z += r.z; v.w += r.w;
      }
      *reinterpret_cast<float4*>(Y) = v;
    } else {
      if (R) {
        const uint2 r = *reinterpret_cast<const uint2*>(R);
        z[0] += bf16_to_f32(r.x & 0xffffu); z[1] += bf16_to_f32(r.x >> 16);
        z[2] += bf16_to_f32(r.y & 0xffffu); z[3] += bf16_to_f32(r.y >> 16);
      }
      *reinterpret_cast<uint2*>(Y) = make_uint2(f32x2_to_bf16x2(z[0], z[1]), f32x2_to_bf16x2(z[2], z[3]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (o + i < g.out) elem<T>::store(Y + i, R ? z[i] + elem<T>::load(R + i) : z[i]);
  }
}

}  // namespace lm

// Tiles of 64 to 256 rows and outputs (linear_tiles.hip).
struct LinearTiles {
  int config;  // -1: operands out of the kernel's reach
  int splits;
  bool pack;   // operands are copied to rows of whole 16-byte units first
  size_t part_bytes, pack_bytes;
};
LinearTiles linear_tiles_plan(const LinearArgs& a);
hipError_t launch_linear_tiles(const LinearArgs& a, const LinearTiles& p, void* workspace, hipStream_t stream);
const char* linear_tiles_name(int config);

}  // namespace convsel
