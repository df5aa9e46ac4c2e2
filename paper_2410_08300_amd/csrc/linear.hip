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
// 4096 on 4096 x 4096 in bf16: 9.0 us, 3.7 TB/s where a large copy reaches 5.05
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

// Few rows.  By rows: 3 us, and the longer of the weights' way from memory (5.3 TB/s; 4.8 in fp32) and the way of one
// CU's share of them, whole workgroups (25 GB/s; 24 in fp32); 16 rows of x add 0.4 of that, and rows of an odd number of
// bf16 take 2.2 times as long.  In tiles: by their plan, which counts no bytes, but at least 7.5 us, all bytes at a
// copy's rate and the copies of rows of no whole 16 bytes.  So wide layers of a row go by rows, and few outputs, which
// give few workgroups, in tiles, which cut the reduction into parts.  Of 368 sizes, random ones among them, the choice
// was more than a tenth behind the other in 8.  us by rows and in tiles, weights from memory:
//   bf16, from 4096   -> 1024      5120      11008     16384     32000   |  8192 -> 8192  11008 -> 4100  14088 -> 541
//     1 row           7.4  8.9  13.5 17.6  20.9 24.1  27.8 38.1  50.7 59.1 |  28.0 37.2      27.6 25.2      18.6 12.4
//     4 rows          8.1  9.1  14.9 17.6  22.5 23.5  29.6 37.9  55.0 61.7 |  28.3 36.2      29.9 25.5      20.9 12.8
//     16 rows        10.1  9.4  18.7 14.8  27.8 24.2  39.0 37.7  71.8 59.4 |  37.4 36.7      38.1 26.3      32.2 13.3
//   fp32, 1 row      14.3 12.6  27.3 32.6  42.7 61.4  58.3 83.0   107  152 |  63.1 83.4      65.6 62.0      44.2 24.9
//     16 rows        19.2 13.4  37.5 34.3  57.3 63.8  79.5 85.2   150  157 |  76.7 85.9      85.4 65.1      67.2 25.5
// More rows.  Those that would be copied for the tiles are read as they lie where they are few, 1.3 times as slowly in
// fp32 and 2.5 times in bf16 (24 rows, 2611 -> 7680 in fp32: 61 us in tiles, 51 by rows; 29, 2282 -> 1496: 24 and 12; but
// 50, 3897 -> 7064 in bf16: 47 and 131).
bool in_rows(const LinearArgs& a, LinearTiles* t) {
  *t = linear_tiles_plan(a);
  if (t->config < 0) return true;
  const bool f32 = a.dtype == CONV_F32;
  const double es = f32 ? 4 : 2, strip = 16. * a.in * es;  // bytes of a workgroup's weights
  const int64_t groups = ((a.out + 15) / 16) * ((a.m + 15) / 16);
  if (a.m <= kFewRows) {
    const bool odd = !f32 && (a.in % 2 != 0 || a.ldx % 2 != 0);
    const double memory = (double)a.out * a.in * es / (f32 ? 4.8e6 : 5.3e6);
    const double cu = (double)((groups + 255) / 256) * strip / (f32 ? 24e3 : 25e3);
    const double rows = 3 + (memory > cu ? memory : cu) * (1 + 0.4 * a.m / 16) * (odd ? 2.2 : 1.);
    const double copy = t->pack ? 2.5 + (double)(a.m + a.out) * a.in * es * 2 / 4e6 : 0.;
    const double least = 7.5 + ((double)a.out * a.in + (double)a.m * (a.in + a.out)) * es / 5.05e6 + copy;
    const double tiles = 1.05 * t->us;
    return rows <= (tiles > least ? tiles : least);
  }
  const double us = strip / 22e3 * (groups > 256 ? groups / 256. : 1.) * 1.4;
  return a.m <= 4 * kFewRows && t->pack && us * (f32 ? 1.3 : 2.5) <= t->us;
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
