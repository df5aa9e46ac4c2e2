// Norm and position rotation of query and key heads, in one pass over both.
#include "lm_common.hpp"
#include "lm_kernels.hpp"

namespace convsel {
namespace {

constexpr int kMaxDim = 1024;

// Whole 16-byte units: one wave per token.  A lane holds the two units of a head
// whose values turn together (i and i + R/2, or two neighbours where pairs lie
// side by side), so that no value crosses lanes but the sum of squares; as many
// heads as fit stand side by side in the wave, ROUNDS rounds of them on their
// way at once, and a lane's cosines and sines are read once for all its heads.
//
// What bounds it: traffic, each value read and written once (16384 tokens of 40
// heads of 128 in bf16: 71 us, 4.8 TB/s, where a copy of 1 GiB reaches 5.0); for
// few tokens, the way from the position to the angles, which starts with the
// heads' own.
template <typename T, bool INTER, int ROUNDS>
__global__ __launch_bounds__(256) void qk_units_kernel(QkArgs a, int lanes, int shift) {
  constexpr int UE = elem<T>::per16;
  constexpr int NC = INTER ? UE / 2 : UE;  // angles of a unit
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int j = lane & ((1 << shift) - 1), side = lane >> shift, abreast = 64 >> shift;
  const int units = a.dim / UE, turned = a.rotary / UE;
  const int pairs = INTER ? 0 : turned / 2;  // units that turn with another
  int ua, ub;
  if (j < pairs) {
    ua = j; ub = j + pairs;
  } else {
    ua = 2 * j; ub = ua + 1;  // behind the pairs (2 pairs + 2 (j - pairs)), or neighbours
  }
  const bool has_a = j < lanes && ua < units, has_b = j < lanes && ub < units;
  const int ca = has_a ? ua * UE : 0, cb = has_b ? ub * UE : 0;  // an idle lane reads the head's first unit
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * 4 + wave; t < a.tokens; t += static_cast<int64_t>(gridDim.x) * 4) {
    float cosv[2][NC], sinv[2][NC];  // [1]: the second unit's, interleaved only
    bool bad = false, turn[2] = {false, false};  // units that do not turn are left alone: 0 times infinity is not 0
    const int64_t p = a.rotary > 0 ? a.positions[t] : 0;
    bool have = false;
    // The token's heads in pieces of ROUNDS rounds, those of q before those of k, dealt to the grid's second axis.
    const int piece = ROUNDS * abreast;
    const int qp = (a.heads[0] + piece - 1) / piece, all = qp + (a.heads[1] + piece - 1) / piece;
    for (int c = blockIdx.y; c < all; c += gridDim.y) {
      const int which = c >= qp;
      const int heads = a.heads[which];
      const T* src = reinterpret_cast<const T*>(a.in[which]) + t * a.in_token[which];
      T* dst = reinterpret_cast<T*>(a.out[which]) + t * a.out_token[which];
      const T* wt = reinterpret_cast<const T*>(a.weight[which]);
      const int h0 = (which ? c - qp : c) * piece + side;
      vec16 va[ROUNDS], vb[ROUNDS], wa = vec16_zero(), wb = vec16_zero();
#pragma unroll
      for (int r = 0; r < ROUNDS; ++r) {
        const T* x = src + min(h0 + r * abreast, heads - 1) * a.in_head[which];
        va[r] = load16(x + ca);
        vb[r] = load16(x + cb);
      }
      if (wt) {
        wa = load16(wt + ca);
        wb = load16(wt + cb);
      }
      if (!have && a.rotary > 0) {  // behind the first heads' loads: the angles wait for the position
        have = true;
        bad = p < 0 || p >= a.max_position;
        const int64_t row = (bad ? 0 : p) * (a.rotary / 2);
#pragma unroll
        for (int u = 0; u < (INTER ? 2 : 1); ++u) {
          const int first = INTER ? (u ? cb : ca) / 2 : ca;
          const bool on = INTER ? (u ? has_b && ub < turned : has_a && ua < turned) : j < pairs;
          const int64_t at = row + (on ? first : 0);
          turn[u] = on;
#pragma unroll
          for (int i = 0; i < NC; i += 2) {
            const float2 cv = *reinterpret_cast<const float2*>(a.cos + at + i);
            const float2 sv = *reinterpret_cast<const float2*>(a.sin + at + i);
            cosv[u][i] = cv.x; cosv[u][i + 1] = cv.y;
            sinv[u][i] = sv.x; sinv[u][i + 1] = sv.y;
          }
        }
      }
#pragma unroll
      for (int r = 0; r < ROUNDS; ++r) {
        float za[UE], zb[UE], sum = 0.f;
#pragma unroll
        for (int i = 0; i < UE; ++i) {
          za[i] = elem<T>::to_f32(vec16_get<T>(va[r], i));
          zb[i] = elem<T>::to_f32(vec16_get<T>(vb[r], i));
          sum += (has_a ? za[i] * za[i] : 0.f) + (has_b ? zb[i] * zb[i] : 0.f);
        }
        if (a.norm) {
          for (int o = 1 << shift >> 1; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
          const float inv = 1.f / sqrtf(sum / a.dim + a.eps);
#pragma unroll
          for (int i = 0; i < UE; ++i) {
            za[i] *= inv;
            zb[i] *= inv;
          }
        }
        if (wt) {
#pragma unroll
          for (int i = 0; i < UE; ++i) {
            za[i] *= elem<T>::to_f32(vec16_get<T>(wa, i));
            zb[i] *= elem<T>::to_f32(vec16_get<T>(wb, i));
          }
        }
        if (a.rotary > 0) {
          if constexpr (INTER) {
#pragma unroll
            for (int i = 0; i < NC; ++i) {
              const float x = za[2 * i], y = za[2 * i + 1];
              za[2 * i] = turn[0] ? x * cosv[0][i] - y * sinv[0][i] : x;
              za[2 * i + 1] = turn[0] ? y * cosv[0][i] + x * sinv[0][i] : y;
              const float u = zb[2 * i], v = zb[2 * i + 1];
              zb[2 * i] = turn[1] ? u * cosv[1][i] - v * sinv[1][i] : u;
              zb[2 * i + 1] = turn[1] ? v * cosv[1][i] + u * sinv[1][i] : v;
            }
          } else {
#pragma unroll
            for (int i = 0; i < UE; ++i) {
              const float x = za[i], y = zb[i];
              za[i] = turn[0] ? x * cosv[0][i] - y * sinv[0][i] : x;
              zb[i] = turn[0] ? y * cosv[0][i] + x * sinv[0][i] : y;
            }
          }
        }
        const int h = h0 + r * abreast;
        if (h < heads) {
          T* y = dst + h * a.out_head[which];
          vec16 oa, ob;
#pragma unroll
          for (int i = 0; i < UE; ++i) {
            vec16_set<T>(oa, i, elem<T>::from_f32(bad ? __builtin_nanf("") : za[i]));
            vec16_set<T>(ob, i, elem<T>::from_f32(bad ? __builtin_nanf("") : zb[i]));
          }
          if (has_a) store16(y + ca, oa);
          if (has_b) store16(y + cb, ob);
        }
      }
    }
  }
}

// Any widths, strides and alignment, among them ordinary heads whose rotated part
// is no whole units: one wave per (token, head).  The head is
// read once, its sum of squares joined across the wave, and the scaled values
// pass through LDS so that every lane finds its rotation partner.  What bounds it:
// instructions, one element a lane at a time (16384 tokens of 40 heads in bf16:
// of 80, 40 turned, 273 us, of 96, 24 turned, 284, where their bytes take 42 and
// 50).
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

namespace {

template <typename T>
hipError_t launch(const QkArgs& a, hipStream_t stream) {
  const int64_t ue = elem<T>::per16;
  // Whole units that start on 16 bytes everywhere, and pairs that turn are whole units too.
  bool whole = a.dim % ue == 0 && a.dim <= 128 * ue && a.rotary % (a.interleaved ? ue : 2 * ue) == 0 &&
               (uintptr_t)a.cos % 16 == 0 && (uintptr_t)a.sin % 16 == 0;
  for (int i = 0; i < 2; ++i)
    if (a.heads[i] > 0)
      whole = whole && a.in_token[i] % ue == 0 && a.in_head[i] % ue == 0 && a.out_token[i] % ue == 0 &&
              a.out_head[i] % ue == 0 && (uintptr_t)a.in[i] % 16 == 0 && (uintptr_t)a.out[i] % 16 == 0 &&
              (uintptr_t)a.weight[i] % 16 == 0;
  if (whole) {
    const int lanes = (int)(a.dim / ue + 1) / 2;
    int shift = 0;
    while (1 << shift < lanes) ++shift;
    const int64_t blocks = (a.tokens + 3) / 4;
    // Many tokens: a wave takes a token's heads in fours of rounds.  Few: a wave takes one round, and the heads of a
    // token go to as many waves as that gives (one token of 40 heads of 128: 3.6 us for 7.6).
    const int abreast = 64 >> shift;
    const int64_t pieces = (a.heads[0] + abreast - 1) / abreast + (a.heads[1] + abreast - 1) / abreast;
    const unsigned bx = (unsigned)(blocks < 65536 ? blocks : 65536), by = (unsigned)(pieces < 64 ? pieces : 64);
    if (blocks >= 512) {
      if (a.interleaved)
        hipLaunchKernelGGL((qk_units_kernel<T, true, 4>), dim3(bx), dim3(256), 0, stream, a, lanes, shift);
      else
        hipLaunchKernelGGL((qk_units_kernel<T, false, 4>), dim3(bx), dim3(256), 0, stream, a, lanes, shift);
    } else {
      if (a.interleaved)
        hipLaunchKernelGGL((qk_units_kernel<T, true, 1>), dim3(bx, by), dim3(256), 0, stream, a, lanes, shift);
      else
        hipLaunchKernelGGL((qk_units_kernel<T, false, 1>), dim3(bx, by), dim3(256), 0, stream, a, lanes, shift);
    }
    return hipGetLastError();
  }
  const int64_t items = a.tokens * (a.heads[0] + a.heads[1]);
  const int64_t blocks = (items + 3) / 4;
  hipLaunchKernelGGL(qk_norm_rope_kernel<T>, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, stream, a,
                     items);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_qk_norm_rope(const QkArgs& a, hipStream_t stream) {
  return a.dtype == CONV_F32 ? launch<float>(a, stream) : launch<bf16_t>(a, stream);
}

}  // namespace convsel
