// Penalties of repeated tokens, biases and masks on the logits of a batch.
//
// A workgroup owns 8 THREADS STEPS neighbouring tokens of a row, eight at a time
// a thread, whose logits are on their way while it counts in LDS how often its row's
// history holds each of them (whole numbers, in any order).  What bounds it:
// traffic (256 rows of 128000 in fp32 without a history: 51 us, 5.1 TB/s, a copy's
// rate; in bf16, whose results stay in the caches, 28 us, 4.7 TB/s), and the
// history, which every workgroup of a row reads from the caches (in bf16 with
// histories of 2000: 44 us, 3.0 TB/s).
#include "lm_common.hpp"
#include "lm_kernels.hpp"

namespace convsel {
namespace {

using namespace lm;

constexpr int kEach = 8;  // tokens of a step of a thread
constexpr uint32_t kSeen = 0x80000000u;  // the prompt holds it; the bits below count generated ones

// Eight values; rows lie on any alignment of elements, which wide loads and stores of global memory may too.
template <typename T>
__device__ __forceinline__ void get8(const T* p, float (&z)[8]) {
  constexpr int UE = elem<T>::per16;
#pragma unroll
  for (int u = 0; u < 8 / UE; ++u) {
    vec16 v;
    __builtin_memcpy(&v, p + u * UE, 16);
#pragma unroll
    for (int e = 0; e < UE; ++e) z[u * UE + e] = elem<T>::to_f32(vec16_get<T>(v, e));
  }
}
// Stored past the caches where they would not keep it: what a call reads then stays in them, and what it wrote does not.
// us of the call and an argmax of its results, past the caches and not, histories of 600: bf16, 16 MB 61.8 and 52.0, 66
// MB 89.5 and 79.9, 98 MB 110.5 and 110.8, 131 MB 127.7 and 129.7; fp32, 16 MB 60.8 and 49.2, 98 MB 93.8 and 95.3, 131
// MB 105.7 and 109.9, 164 MB 121.2 and 124.9.
typedef uint32_t words_t __attribute__((ext_vector_type(4), aligned(2)));
template <bool PAST>
__device__ __forceinline__ void put16(void* p, const words_t& w) {
  if constexpr (PAST)
    __builtin_nontemporal_store(w, reinterpret_cast<words_t*>(p));
  else
    *reinterpret_cast<words_t*>(p) = w;
}
template <bool PAST>
__device__ __forceinline__ void put8(float* p, const float (&z)[8]) {
#pragma unroll
  for (int u = 0; u < 8; u += 4)
    put16<PAST>(p + u, words_t{__float_as_uint(z[u]), __float_as_uint(z[u + 1]), __float_as_uint(z[u + 2]),
                               __float_as_uint(z[u + 3])});
}
template <bool PAST>
__device__ __forceinline__ void put8(bf16_t* p, const float (&z)[8]) {
  put16<PAST>(p, words_t{f32x2_to_bf16x2(z[0], z[1]), f32x2_to_bf16x2(z[2], z[3]), f32x2_to_bf16x2(z[4], z[5]),
                         f32x2_to_bf16x2(z[6], z[7])});
}

template <typename T, int THREADS, int STEPS, bool PAST>
__global__ __launch_bounds__(THREADS) void adjust_logits_kernel(LogitsArgs a, int64_t chunks) {
  constexpr int CHUNK = THREADS * kEach * STEPS;
  extern __shared__ __align__(16) uint32_t count[];  // CHUNK of them, with a history
  for (int64_t unit = blockIdx.x; unit < chunks * a.rows; unit += gridDim.x) {
    const int64_t row = unit / chunks, c0 = (unit - row * chunks) * CHUNK;
    const int width = static_cast<int>(min(a.vocab - c0, static_cast<int64_t>(CHUNK)));
    const T* x = reinterpret_cast<const T*>(a.x) + row * a.ldx + c0;
    T* y = reinterpret_cast<T*>(a.y) + row * a.ldy + c0;
    float z[STEPS][kEach];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int i = (s * THREADS + threadIdx.x) * kEach;
      if (i + kEach <= width) {
        get8(x + i, z[s]);
      } else {
#pragma unroll
        for (int e = 0; e < kEach; ++e) z[s][e] = i + e < width ? elem<T>::load(x + i + e) : 0.f;
      }
    }
    int first = 0, end = 0;
    if (a.history) {
      const int limit = static_cast<int>(a.tokens);
      first = clampi(a.offsets[row], 0, limit);
      end = clampi(a.offsets[row + 1], first, limit);
    }
    const bool counted = end > first;  // uniform
    if (counted) {
      const int generated = first + (a.prompt_lengths ? clampi(a.prompt_lengths[row], 0, end - first) : 0);
#pragma unroll
      for (int s = 0; s < 2 * STEPS; ++s)
        *reinterpret_cast<uint4*>(count + (s * THREADS + threadIdx.x) * 4) = make_uint4(0, 0, 0, 0);
      lds_sync();
      for (int64_t i0 = static_cast<int64_t>(first) + threadIdx.x; i0 < end; i0 += 4 * THREADS) {
        int64_t at[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) at[n] = a.history[min(i0 + n * THREADS, static_cast<int64_t>(end) - 1)] - c0;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const int64_t i = i0 + n * THREADS;
          if (i < end && at[n] >= 0 && at[n] < width) {
            if (i < generated)
              atomicOr(&count[at[n]], kSeen);
            else
              atomicAdd(&count[at[n]], 1u);
          }
        }
      }
      lds_sync();
    }
    const float r = a.repetition ? a.repetition[row] : 1.f;
    const float p = a.presence ? a.presence[row] : 0.f, f = a.frequency ? a.frequency[row] : 0.f;
    const float* bias = a.bias ? a.bias + row * a.ldbias + c0 : nullptr;
    const uint32_t* mask = a.mask ? a.mask + row * a.ldmask + c0 / 32 : nullptr;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int i = (s * THREADS + threadIdx.x) * kEach;
      if (i >= width) break;
      float(&v)[kEach] = z[s];
      if (counted) {
        uint32_t c[kEach];
        *reinterpret_cast<uint4*>(c) = *reinterpret_cast<const uint4*>(count + i);
        *reinterpret_cast<uint4*>(c + 4) = *reinterpret_cast<const uint4*>(count + i + 4);
        if ((c[0] | c[1] | c[2] | c[3] | c[4] | c[5] | c[6] | c[7]) != 0) {
#pragma unroll
          for (int e = 0; e < kEach; ++e) {
            if (c[e] == 0) continue;
            if (a.repetition) v[e] = v[e] > 0.f ? v[e] / r : v[e] * r;
            const uint32_t made = c[e] & ~kSeen;
            if (made != 0) v[e] -= fmaf(f, static_cast<float>(made), p);
          }
        }
      }
      const bool whole = i + kEach <= width;
      if (bias) {
        float b[kEach];
        if (whole) {
          get8(bias + i, b);
        } else {
#pragma unroll
          for (int e = 0; e < kEach; ++e) b[e] = i + e < width ? bias[i + e] : 0.f;
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) v[e] += b[e];
      }
      if (mask) {
        const uint32_t bits = mask[i >> 5] >> (i & 31);
#pragma unroll
        for (int e = 0; e < kEach; ++e) v[e] = (bits >> e) & 1u ? v[e] : -__builtin_inff();
      }
      if (whole) {
        put8<PAST>(y + i, v);
      } else {
#pragma unroll
        for (int e = 0; e < kEach; ++e)
          if (i + e < width) elem<T>::store(y + i + e, v[e]);
      }
    }
    if (counted) lds_sync();  // before the next row's counts
  }
}

// More bytes of results than the caches keep for who reads them next.
template <typename T>
bool past_caches(const LogitsArgs& a) {
  return a.rows * a.vocab * (int64_t)sizeof(T) > (int64_t)96 << 20;
}

template <typename T, int THREADS, int STEPS, bool PAST>
hipError_t launch(const LogitsArgs& a, hipStream_t st) {
  constexpr int chunk = THREADS * kEach * STEPS;
  const int64_t chunks = (a.vocab + chunk - 1) / chunk, units = chunks * a.rows;
  const dim3 grid((unsigned)(units < (1 << 20) ? units : 1 << 20));
  hipLaunchKernelGGL((adjust_logits_kernel<T, THREADS, STEPS, PAST>), grid, dim3(THREADS),
                     a.history ? chunk * 4 : 0, st, a, chunks);
  return hipGetLastError();
}
template <typename T, int THREADS, int STEPS>
hipError_t launch(const LogitsArgs& a, hipStream_t st) {
  return past_caches<T>(a) ? launch<T, THREADS, STEPS, true>(a, st) : launch<T, THREADS, STEPS, false>(a, st);
}

template <typename T>
hipError_t launch_steps(const LogitsArgs& a, hipStream_t st) {
  // Threads and steps, in us of the call alone with 256 x 1, 512 x 2 and 1024 x 4:
  //   bf16, 512 rows of 500, 8 of 128000, histories of 200, 2000    4.9 5.2 9.6 | 5.3 5.8 9.2
  //         32, 64 and 256 of 128000, 2000                          9.9 8.0 10.5 | 14.2 12.7 11.9 | 47.2 43.8 44.9
  //         1, 64 and 256 of 128000, 8000                           7.2 6.8 10.1 | 24.4 16.6 13.9 | 82.6 54.3 51.5
  //   fp32, 64 and 256 of 128000, 1000 (the last past the caches)   16.2 16.8 15.7 | 53.0 58.7 67.2
  //         256 of 128000, 600, bias and mask; 8000                 57.9 60.0 63.8 | 88.2 70.9 70.9
  //         16 of 200000, 8000                                      14.0 11.1 12.8
  // Few logits need many workgroups, long histories few readers of them.
  const int64_t logits = a.rows * a.vocab;
  const bool few = logits < 256 * 8192, longs = a.tokens / a.rows >= 4000;
  if constexpr (sizeof(T) == 4) {
    if (!longs) return launch<T, 256, 1>(a, st);
  } else {
    if (few && !longs) return launch<T, 256, 1, false>(a, st);
  }
  if (few) return launch<T, 512, 2, false>(a, st);
  return longs && logits >= 6000000 ? launch<T, 1024, 4>(a, st) : launch<T, 512, 2>(a, st);
}

}  // namespace

hipError_t launch_adjust_logits(const LogitsArgs& a, hipStream_t stream) {
  return a.dtype == CONV_F32 ? launch_steps<float>(a, stream) : launch_steps<bf16_t>(a, stream);
}

}  // namespace convsel
