// Linear layers: y = act(x W^T + b) + r.
#include <stdio.h>

#include "lm_common.hpp"
#include "lm_kernels.hpp"

namespace convsel {
namespace {

using namespace lm;

// Any sizes, strides and alignment.  256 threads = 4 waves in a 2 x 2 grid
// own a 64 x 64 tile of y; rows of x and w are staged in LDS in k-tiles of
// 64 bytes, element by element where a 16-byte load could be misaligned or
// leave the row.  The matrix product's rows are w's and its columns x's, so a
// lane ends with four consecutive outputs of one token.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void linear_tile_kernel(LinearArgs g, int tiles_o) {
  constexpr int UE = elem<T>::per16;
  constexpr int BK = 4 * UE, KP = BK + UE;
  __shared__ __align__(16) T Ws[64 * KP];
  __shared__ __align__(16) T Xs[64 * KP];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wo = wave >> 1, wx = wave & 1;
  const int64_t o0 = static_cast<int64_t>(blockIdx.x % tiles_o) * 64, m0 = static_cast<int64_t>(blockIdx.x / tiles_o) * 64;
  const int row = tid >> 2, kc = (tid & 3) * UE;
  const T* X = reinterpret_cast<const T*>(g.x) + (m0 + row) * g.ldx;
  const T* W = reinterpret_cast<const T*>(g.w) + (o0 + row) * g.in;
  const bool xok = m0 + row < g.m, wok = o0 + row < g.out;
  auto fetch = [&](const T* base, bool ok, int64_t k) -> vec16 {
    if (VEC) return ok && k < g.in ? load16(base + k) : vec16_zero();
    uint32_t e[UE];
#pragma unroll
    for (int i = 0; i < UE; ++i) e[i] = ok && k + i < g.in ? load_bits(base + k + i) : 0u;
    vec16 r;
    pack16<T>(r, e);
    return r;
  };
  f32x16_t acc = zero16();
  vec16 rx = fetch(X, xok, kc), rw = fetch(W, wok, kc);
  const int half = lane >> 5, l32 = lane & 31;
  for (int64_t k0 = 0; k0 < g.in; k0 += BK) {
    store16(&Xs[row * KP + kc], rx);
    store16(&Ws[row * KP + kc], rw);
    lds_sync();
    rx = fetch(X, xok, k0 + BK + kc);
    rw = fetch(W, wok, k0 + BK + kc);
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      const int kofs = st * 2 * UE + half * UE;
      mfma_32x32<T>(acc, load16(&Ws[(wo * 32 + l32) * KP + kofs]), load16(&Xs[(wx * 32 + l32) * KP + kofs]));
    }
    lds_sync();
  }
  const int64_t m = m0 + wx * 32 + l32;
  if (m >= g.m) return;
  const T* B = reinterpret_cast<const T*>(g.b);
  const T* R = reinterpret_cast<const T*>(g.r);
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const int64_t o = o0 + wo * 32 + mfma_row(v, lane);
    if (o >= g.out) continue;
    float z = acc[v];
    if (B) z += elem<T>::load(B + o);
    z = activate<T>(z, g.act);
    if (R) z += elem<T>::load(R + m * g.ldr + o);
    elem<T>::store(reinterpret_cast<T*>(g.y) + m * g.ldy + o, z);
  }
}

}  // namespace

size_t linear_workspace(const LinearArgs&) { return 0; }

hipError_t launch_linear(const LinearArgs& a, void*, hipStream_t stream) {
  const int64_t per = a.dtype == CONV_F32 ? 4 : 8;
  const bool vec = a.in % per == 0 && a.ldx % per == 0 && (uintptr_t)a.x % 16 == 0 && (uintptr_t)a.w % 16 == 0;
  const int64_t to = (a.out + 63) / 64, tm = (a.m + 63) / 64;
  const dim3 grid((unsigned)(to * tm));
  if (a.dtype == CONV_F32) {
    if (vec)
      hipLaunchKernelGGL((linear_tile_kernel<float, true>), grid, dim3(256), 0, stream, a, (int)to);
    else
      hipLaunchKernelGGL((linear_tile_kernel<float, false>), grid, dim3(256), 0, stream, a, (int)to);
  } else {
    if (vec)
      hipLaunchKernelGGL((linear_tile_kernel<bf16_t, true>), grid, dim3(256), 0, stream, a, (int)to);
    else
      hipLaunchKernelGGL((linear_tile_kernel<bf16_t, false>), grid, dim3(256), 0, stream, a, (int)to);
  }
  return hipGetLastError();
}

void linear_describe(const LinearArgs&, char* buf, size_t len) {
  snprintf(buf, len, "linear kernels=linear_tile_kernel tile=64x64 workspace=0");
}

}  // namespace convsel
