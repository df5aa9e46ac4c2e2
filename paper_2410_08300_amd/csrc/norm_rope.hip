// Norm and position rotation of query and key heads, in one pass over both.
#include "lm_common.hpp"
#include "lm_kernels.hpp"

namespace convsel {
namespace {

constexpr int kMaxDim = 1024;

// One wave per (token, head): the head is read once, its sum of squares joined
// across the wave, and the scaled values pass through LDS so that every lane
// finds its rotation partner.
template <typename T>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(QkArgs a, int64_t items) {
  __shared__ float buf[4][kMaxDim];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int all = a.heads[0] + a.heads[1];
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * 4; base < items; base += static_cast<int64_t>(gridDim.x) * 4) {
    const int64_t it = base + wave;
    const bool live = it < items;
    const int64_t t = live ? it / all : 0;
    int h = live ? static_cast<int>(it - t * all) : 0;
    const int which = h >= a.heads[0];
    if (which) h -= a.heads[0];
    const T* src = reinterpret_cast<const T*>(a.in[which]) + t * a.in_token[which] + h * a.in_head[which];
    T* dst = reinterpret_cast<T*>(a.out[which]) + t * a.out_token[which] + h * a.out_head[which];
    const T* wt = reinterpret_cast<const T*>(a.weight[which]);
    float sum = 0.f;
    if (live)
      for (int d = lane; d < a.dim; d += 64) {
        const float v = elem<T>::load(src + d);
        buf[wave][d] = v;
        sum += v * v;
      }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    const float inv = a.norm ? 1.f / sqrtf(sum / a.dim + a.eps) : 1.f;
    if (live)
      for (int d = lane; d < a.dim; d += 64) buf[wave][d] = buf[wave][d] * inv * (wt ? elem<T>::load(wt + d) : 1.f);
    lds_sync();
    if (live) {
      const int half = a.rotary / 2;
      const int64_t p = half ? a.positions[t] : 0;
      const bool bad = half && (p < 0 || p >= a.max_position);
      for (int d = lane; d < a.dim; d += 64) {
        float z = buf[wave][d];
        if (d < a.rotary && !bad) {
          const int i = a.interleaved ? d >> 1 : (d < half ? d : d - half);
          const bool second = a.interleaved ? (d & 1) : d >= half;
          const float other = buf[wave][a.interleaved ? d ^ 1 : (second ? d - half : d + half)];
          const float c = a.cos[p * half + i], s = a.sin[p * half + i];
          z = second ? z * c + other * s : z * c - other * s;
        }
        elem<T>::store(dst + d, bad ? __builtin_nanf("") : z);
      }
    }
    lds_sync();
  }
}

}  // namespace

hipError_t launch_qk_norm_rope(const QkArgs& a, hipStream_t stream) {
  const int64_t items = a.tokens * (a.heads[0] + a.heads[1]);
  int64_t blocks = (items + 3) / 4;
  if (blocks > 65536) blocks = 65536;
  if (a.dtype == CONV_F32)
    hipLaunchKernelGGL(qk_norm_rope_kernel<float>, dim3((unsigned)blocks), dim3(256), 0, stream, a, items);
  else
    hipLaunchKernelGGL(qk_norm_rope_kernel<bf16_t>, dim3((unsigned)blocks), dim3(256), 0, stream, a, items);
  return hipGetLastError();
}

}  // namespace convsel
