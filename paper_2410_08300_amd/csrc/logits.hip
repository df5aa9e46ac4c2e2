// Penalties of repeated tokens, biases and masks on the logits of a batch.
//
// A workgroup owns kChunk neighbouring tokens of a row.  It counts in LDS how
// often its row's history holds each of them (whole numbers, in any order), then
// passes once over its logits.  What bounds it: traffic, and the history, which
// every workgroup of a row reads from the caches.
#include "lm_common.hpp"
#include "lm_kernels.hpp"

namespace convsel {
namespace {

using namespace lm;

constexpr int kThreads = 256, kChunk = 8192;
constexpr uint32_t kSeen = 0x80000000u;  // the prompt holds it; the bits below count generated ones

template <typename T>
__global__ __launch_bounds__(kThreads) void adjust_logits_kernel(LogitsArgs a, int64_t chunks, int vec) {
  constexpr int N = 8;  // tokens of a step of a thread
  __shared__ uint32_t count[kChunk];
  for (int64_t unit = blockIdx.x; unit < chunks * a.rows; unit += gridDim.x) {
    const int64_t row = unit / chunks, c0 = (unit - row * chunks) * kChunk;
    const int width = static_cast<int>(min(a.vocab - c0, static_cast<int64_t>(kChunk)));
    int first = 0, end = 0;
    if (a.history) {
      const int limit = static_cast<int>(a.tokens);
      first = clampi(a.offsets[row], 0, limit);
      end = clampi(a.offsets[row + 1], first, limit);
    }
    const bool counted = end > first;  // uniform
    if (counted) {
      const int prompt = a.prompt_lengths ? clampi(a.prompt_lengths[row], 0, end - first) : 0;
      for (int i = threadIdx.x; i < width; i += kThreads) count[i] = 0;
      __syncthreads();
      for (int i = first + static_cast<int>(threadIdx.x); i < end; i += kThreads) {
        const int64_t at = a.history[i] - c0;
        if (at >= 0 && at < width) {
          if (i - first < prompt)
            atomicOr(&count[at], kSeen);
          else
            atomicAdd(&count[at], 1u);
        }
      }
      __syncthreads();
    }
    const float r = a.repetition ? a.repetition[row] : 1.f;
    const float p = a.presence ? a.presence[row] : 0.f, f = a.frequency ? a.frequency[row] : 0.f;
    const T* x = reinterpret_cast<const T*>(a.x) + row * a.ldx + c0;
    T* y = reinterpret_cast<T*>(a.y) + row * a.ldy + c0;
    const float* bias = a.bias ? a.bias + row * a.ldbias + c0 : nullptr;
    const uint32_t* mask = a.mask ? a.mask + row * a.ldmask + c0 / 32 : nullptr;
    for (int i = threadIdx.x * N; i < width; i += kThreads * N) {
      const int n = min(N, width - i);
      const bool whole = vec && n == N;
      float z[N];
      if (whole) {
        constexpr int UE = elem<T>::per16;
#pragma unroll
        for (int u = 0; u < N / UE; ++u) {
          const vec16 v = load16(x + i + u * UE);
#pragma unroll
          for (int e = 0; e < UE; ++e) z[u * UE + e] = elem<T>::to_f32(vec16_get<T>(v, e));
        }
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = elem<T>::load(x + i + min(e, n - 1));
      }
      if (counted) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const uint32_t c = count[i + min(e, n - 1)];
          if (c != 0) {
            if (a.repetition) z[e] = z[e] > 0.f ? z[e] / r : z[e] * r;
            const uint32_t made = c & ~kSeen;
            if (made != 0) z[e] -= fmaf(f, static_cast<float>(made), p);
          }
        }
      }
      if (bias) {
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] += bias[i + min(e, n - 1)];
      }
      if (mask) {
        const uint32_t bits = mask[i >> 5] >> (i & 31);
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = (bits >> e) & 1u ? z[e] : -__builtin_inff();
      }
      if (whole) {
        if constexpr (sizeof(T) == 4) {
          *reinterpret_cast<float4*>(y + i) = make_float4(z[0], z[1], z[2], z[3]);
          *reinterpret_cast<float4*>(y + i + 4) = make_float4(z[4], z[5], z[6], z[7]);
        } else {
          vec16 v;
#pragma unroll
          for (int w = 0; w < 4; ++w) v.d[w] = f32x2_to_bf16x2(z[2 * w], z[2 * w + 1]);
          store16(y + i, v);
        }
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (e < n) elem<T>::store(y + i + e, z[e]);
      }
    }
    __syncthreads();  // before the next row's counts
  }
}

}  // namespace

hipError_t launch_adjust_logits(const LogitsArgs& a, hipStream_t stream) {
  const int64_t chunks = (a.vocab + kChunk - 1) / kChunk, units = chunks * a.rows;
  const dim3 grid((unsigned)(units < (1 << 20) ? units : 1 << 20));
  const int64_t per = a.dtype == CONV_F32 ? 4 : 8;
  const int vec = a.ldx % per == 0 && a.ldy % per == 0 && (uintptr_t)a.x % 16 == 0 && (uintptr_t)a.y % 16 == 0;
  if (a.dtype == CONV_F32)
    hipLaunchKernelGGL(adjust_logits_kernel<float>, grid, dim3(kThreads), 0, stream, a, chunks, vec);
  else
    hipLaunchKernelGGL(adjust_logits_kernel<bf16_t>, grid, dim3(kThreads), 0, stream, a, chunks, vec);
  return hipGetLastError();
}

}  // namespace convsel
