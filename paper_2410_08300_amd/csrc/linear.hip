// Linear layers: y = act(x W^T + b) + r.  Few rows stream the weights through
// registers (here); more rows go in tiles (linear_tiles.hip).
#include <stdio.h>

#include <type_traits>

#include "linear_common.hpp"

namespace convsel {
namespace {

using namespace lm;

// Few rows: a workgroup owns 16 outputs and 16 rows of x, and its waves share
// out the reduction, whose sums meet in LDS.  A lane holds 32
// neighbouring bytes of one weight row (four lanes read a whole 128-byte line)
// and the same columns of one row of x; which column a product takes at which
// step does not matter while both operands agree.
//
// What bounds it: the weights' way from memory.  A step of a wave is 2 KiB of
// them; steps are fetched kDepth ahead, and as many waves as leave each of them
// a few steps keep a CU's share of the weights on their way at once.  One row of
// 4096 on 4096 x 4096 in bf16: 9.1 us, 3.7 TB/s where a large copy reaches 5.05
// (weights larger than the caches come nearer; here launch and the first loads'
// latency are a third).
constexpr int kDepth = 4;

template <typename T, bool VEC>
__global__ __launch_bounds__(1024) void linear_rows_kernel(LinearArgs g, int waves, int vec_out) {
  constexpr int UE = elem<T>::per16;
  constexpr int SK = 8 * UE;  // columns of a step: two units of each of four lanes
  __shared__ f32x4v_t part[16][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r16 = lane & 15, q = lane >> 4;
  const int64_t o0 = static_cast<int64_t>(blockIdx.x) * 16, m0 = static_cast<int64_t>(blockIdx.y) * 16;
  // Rows past the last one read the last one's values; their results go nowhere.
  const T* W = reinterpret_cast<const T*>(g.w) + min(o0 + r16, g.out - 1) * g.in;
  const T* X = reinterpret_cast<const T*>(g.x) + min(m0 + r16, g.m - 1) * g.ldx;
  auto unit = [&](const T* row, int64_t k) -> vec16 {
    if constexpr (VEC) {
      // Whole units: none straddles the end of the reduction.
      const vec16 v = load16(row + (k < g.in ? k : 0));
      vec16 r;
#pragma unroll
      for (int i = 0; i < 4; ++i) r.d[i] = k < g.in ? v.d[i] : 0u;
      return r;
    } else {
      uint32_t e[UE];
#pragma unroll
      for (int i = 0; i < UE; ++i) {
        const uint32_t bits = load_bits(row + (k + i < g.in ? k + i : 0));
        e[i] = k + i < g.in ? bits : 0u;
      }
      vec16 r;
      pack16<T>(r, e);
      return r;
    }
  };
  const int64_t steps = (g.in + SK - 1) / SK;
  f32x4v_t acc = {0.f, 0.f, 0.f, 0.f};
  vec16 wv[kDepth][2], xv[kDepth][2];
  auto walk = [&](int64_t s0, auto depth_c, const auto& get) {
    constexpr int DEPTH = decltype(depth_c)::value;
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      const int64_t k = (s0 + static_cast<int64_t>(d) * waves) * SK + q * 2 * UE;
#pragma unroll
      for (int u = 0; u < 2; ++u) wv[d][u] = get(W, k + u * UE);
#pragma unroll
      for (int u = 0; u < 2; ++u) xv[d][u] = get(X, k + u * UE);
    }
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
#pragma unroll
      for (int u = 0; u < 2; ++u) acc = mac16(T{}, wv[d][u], xv[d][u], acc);
  };
  const std::integral_constant<int, kDepth> deep{};
  int64_t s0 = wave;
  const int64_t stride = static_cast<int64_t>(waves) * kDepth;
  if constexpr (!VEC) {
    // Away from the rows' ends 16 bytes are read at once from where they lie, on no 16 bytes (15 rows, 2041 -> 2752 in
    // fp32: 10.6 us; 24.3 value by value).
    const auto near = [](const T* row, int64_t k) -> vec16 {
      vec16 v;
      __builtin_memcpy(&v, row + k, 16);
      return v;
    };
    const std::integral_constant<int, 1> one{};
    for (; (s0 + (kDepth - 1) * static_cast<int64_t>(waves) + 1) * SK <= g.in; s0 += stride) walk(s0, deep, near);
    for (; (s0 + 1) * SK <= g.in; s0 += waves) walk(s0, one, near);
    for (; s0 < steps; s0 += waves) walk(s0, one, unit);
  } else {
    for (; s0 < steps; s0 += stride) walk(s0, deep, unit);
  }
  part[wave][lane] = acc;
  __syncthreads();
  // Lane (row of x, q) holds outputs 4 q .. 4 q + 3: the first wave finishes them.
  const int64_t m = m0 + r16, o = o0 + 4 * q;
  if (wave != 0 || m >= g.m || o >= g.out) return;
  float sum[1][4] = {}, bias[4];
  load_bias4<T>(g, o, bias);
  for (int w = 0; w < waves; ++w) {
    const f32x4v_t v = part[w][lane];
#pragma unroll
    for (int x = 0; x < 4; ++x) sum[0][x] += v[x];
  }
  finish4<T, 1>(g, m, 0, o, sum, bias, vec_out);
}

// Up to so many rows are few.
constexpr int64_t kFewRows = 16;

struct RowsPlan {
  int waves;
  bool vec;
};

RowsPlan rows_plan(const LinearArgs& a) {
  const int64_t per = a.dtype == CONV_F32 ? 4 : 8;
  RowsPlan p;
  p.vec = a.in % per == 0 && a.ldx % per == 0 && (uintptr_t)a.x % 16 == 0 && (uintptr_t)a.w % 16 == 0;
  // Each wave has kDepth steps at least where the reduction is that long.
  const int64_t steps = (a.in + 8 * per - 1) / (8 * per);
  int64_t w = steps / kDepth;
  p.waves = (int)(w < 1 ? 1 : w > 16 ? 16 : w);
  return p;
}

template <typename T, bool VEC>
hipError_t launch_rows(const LinearArgs& a, const RowsPlan& p, int vec_out, hipStream_t st) {
  const int64_t groups = (a.m + 15) / 16;
  for (int64_t g0 = 0; g0 < groups; g0 += 65535) {
    LinearArgs b = a;
    const int64_t es = sizeof(T), m0 = g0 * 16;
    b.x = (const char*)a.x + m0 * a.ldx * es;
    b.y = (char*)a.y + m0 * a.ldy * es;
    if (a.r) b.r = (const char*)a.r + m0 * a.ldr * es;
    b.m = a.m - m0;
    const int64_t n = groups - g0 < 65535 ? groups - g0 : 65535;
    if (n * 16 < b.m) b.m = n * 16;
    hipLaunchKernelGGL((linear_rows_kernel<T, VEC>), dim3((unsigned)((a.out + 15) / 16), (unsigned)n),
                       dim3(64 * p.waves), 0, st, b, p.waves, vec_out);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t launch_rows_t(const LinearArgs& a, const RowsPlan& p, int vec_out, hipStream_t st) {
  return p.vec ? launch_rows<T, true>(a, p, vec_out, st) : launch_rows<T, false>(a, p, vec_out, st);
}

// Whether outputs may be read and written four at a time.
int outputs_vec(const LinearArgs& a) {
  const uintptr_t unit = a.dtype == CONV_F32 ? 16 : 8;
  return a.ldy % 4 == 0 && (uintptr_t)a.y % unit == 0 && (!a.r || (a.ldr % 4 == 0 && (uintptr_t)a.r % unit == 0));
}

// A workgroup of rows brings its weights in at some 22 GB/s; 16 rows of x take 0.4 as long again.  With few outputs
// there are few workgroups, and the tiles, which cut the reduction into parts, are through sooner (7 rows, 14088 -> 541 in
// fp32: 44 us by rows, 26 in tiles; 5 rows, 11648 -> 68 in bf16: 17 and 10; 16 rows, 11008 -> 4100: 38 and 27; but 1 row,
// 4096 -> 1024: 7.5 and 8.5, 5000 -> 5120: 17 and 20).  Rows that would be copied for the tiles are read as they lie
// where they are few, 1.3 times as slowly in fp32 and 2.5 times in bf16 (24 rows, 2611 -> 7680 in fp32: 61 us in tiles,
// 51 by rows; 29, 2282 -> 1496: 24 and 12; but 50, 3897 -> 7064 in bf16: 47 and 131).
bool in_rows(const LinearArgs& a, LinearTiles* t) {
  *t = linear_tiles_plan(a);
  if (t->config < 0) return true;
  const double bytes = 16. * a.in * (a.dtype == CONV_F32 ? 4 : 2);
  const double groups = (double)((a.out + 15) / 16) * ((a.m + 15) / 16);
  const double us = bytes / 22e3 * (groups > 256 ? groups / 256 : 1.) * (1 + 0.4 * (a.m < 16 ? a.m : 16) / 16);
  if (a.m <= kFewRows) return us <= 3 + 1.15 * t->us;
  return a.m <= 4 * kFewRows && t->pack && us * (a.dtype == CONV_F32 ? 1.3 : 2.5) <= t->us;
}

}  // namespace

size_t linear_workspace(const LinearArgs& a) {
  LinearTiles t;
  if (in_rows(a, &t)) return 0;
  return t.pack_bytes + t.part_bytes;
}

hipError_t launch_linear(const LinearArgs& a, void* workspace, hipStream_t stream) {
  LinearTiles t;
  if (!in_rows(a, &t)) return launch_linear_tiles(a, t, workspace, stream);
  const RowsPlan p = rows_plan(a);
  return a.dtype == CONV_F32 ? launch_rows_t<float>(a, p, outputs_vec(a), stream)
                             : launch_rows_t<bf16_t>(a, p, outputs_vec(a), stream);
}

void linear_describe(const LinearArgs& a, char* buf, size_t len) {
  LinearTiles t;
  if (in_rows(a, &t)) {
    const RowsPlan p = rows_plan(a);
    snprintf(buf, len, "linear kernels=linear_rows_kernel tile=16x16 waves=%d workspace=0", p.waves);
    return;
  }
  snprintf(buf, len, "linear kernels=%slinear_tiles%s_kernel%s tile=%s split=%d workspace=%zu",
           t.pack ? "linear_pack_kernel;" : "", t.config == 0 && a.dtype != CONV_F32 ? "256" : "", t.splits > 1 ? ";linear_join_kernel" : "",
           linear_tiles_name(t.config), t.splits, linear_workspace(a));
}

}  // namespace convsel
