// Linear layers on 8-bit codes: y = act((X W^T) sx sw + b) + r, with a scale for
// each row of x and each output.
//
// Sums of codes are 32-bit whole numbers, exact up to 131071 input features.
// Many rows go in the tiles of linear_tiles.hip, whose walk of 16-byte units is
// the same for codes, sixteen a unit; few stream the weights through registers
// (here).  Rows of x that come as numbers are coded by a kernel before the
// product.
#include <stdio.h>

#include <type_traits>

#include "linear_common.hpp"

namespace convsel {
namespace {

using namespace lm;

constexpr int64_t kUnit = 16;
constexpr size_t kAlign = 256;
size_t align_up(int64_t bytes) { return ((size_t)bytes + kAlign - 1) / kAlign * kAlign; }

// ---- codes ----

// One workgroup a row: its largest finite magnitude, then codes, from the CU's own cache.
//   scale = max(largest / 127, 2^-100), code = round(x / scale), both quotients in fp32
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(CodeArgs a, int vec) {
  constexpr int UE = 8;  // numbers of a step of a thread
  __shared__ float red[4];
  const int64_t row = blockIdx.x + static_cast<int64_t>(blockIdx.y) * gridDim.x;
  if (row >= a.m) return;
  const T* x = reinterpret_cast<const T*>(a.x) + row * a.ldx;
  int8_t* codes = a.codes + row * a.ldc;
  auto get = [&](int64_t k, float (&z)[UE]) {
    if (vec && k + UE <= a.in) {
      if constexpr (sizeof(T) == 2) {
        const vec16 v = load16(x + k);
#pragma unroll
        for (int i = 0; i < UE; ++i) z[i] = elem<T>::to_f32(vec16_get<T>(v, i));
      } else {
        const vec16 v = load16(x + k), w = load16(x + k + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          z[i] = vec16_get<T>(v, i);
          z[i + 4] = vec16_get<T>(w, i);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < UE; ++i) {
        const float v = elem<T>::load(x + min(k + i, a.in - 1));
        z[i] = k + i < a.in ? v : 0.f;
      }
    }
  };
  float top = 0.f;
  for (int64_t k = threadIdx.x * UE; k < a.in; k += 256 * UE) {
    float z[UE];
    get(k, z);
#pragma unroll
    for (int i = 0; i < UE; ++i) top = fmaxf(top, fabsf(z[i]) < __builtin_inff() ? fabsf(z[i]) : 0.f);
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const float scale = fmaxf(top / 127.f, kMinScale), inverse = 1.f / scale;
  const float end = fmaxf(top, fminf(127.f * scale, 0x1.fffffep127f));  // what infinities count as
  if (threadIdx.x == 0) a.scales[row] = scale;
  for (int64_t k = threadIdx.x * UE; k < a.ldc; k += 256 * UE) {
    float z[UE];
    if (k < a.in) {
      get(k, z);
    } else {
#pragma unroll
      for (int i = 0; i < UE; ++i) z[i] = 0.f;
    }
    // Infinities take the largest code of their sign, NaN zero.
#pragma unroll
    for (int i = 0; i < UE; ++i) z[i] = z[i] != z[i] ? 0.f : fminf(fmaxf(z[i], -end), end);
    uint2 c;
    c.x = four_codes<CONVSEL_KV_INT8>(z[0], z[1], z[2], z[3], scale, inverse);
    c.y = four_codes<CONVSEL_KV_INT8>(z[4], z[5], z[6], z[7], scale, inverse);
    if (k + UE <= a.ldc && a.ldc % UE == 0 && reinterpret_cast<uintptr_t>(a.codes) % UE == 0) {
      *reinterpret_cast<uint2*>(codes + k) = c;
    } else {
#pragma unroll
      for (int i = 0; i < UE; ++i)
        if (k + i < a.ldc) codes[k + i] = static_cast<int8_t>((i < 4 ? c.x : c.y) >> (8 * (i & 3)));
    }
  }
}

// Rows of codes copied to rows of whole 16-byte units, zeros behind them.
__global__ __launch_bounds__(256) void pack_codes_kernel(const int8_t* src, int64_t rows, int64_t in, int64_t ld,
                                                         int8_t* dst, int64_t padded) {
  const int64_t per = padded / kUnit;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < rows * per;
       i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t row = i / per, k = (i - row * per) * kUnit;
    const int8_t* p = src + row * ld;
    vec16 v;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      v.d[w] = 0;
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int64_t at = k + 4 * w + b;
        const uint32_t c = static_cast<uint8_t>(p[at < in ? at : 0]);
        v.d[w] |= (at < in ? c : 0u) << (8 * b);
      }
    }
    store16(dst + i * kUnit, v);
  }
}

// ---- few rows ----

// A workgroup owns 16 outputs and 16 rows of x, and its waves share out the reduction, whose sums meet in LDS.  A lane
// holds 32 neighbouring codes of one weight row (four lanes read a whole 128-byte line) and the same of one row of x.
// What bounds it is the weights' way from memory; steps are fetched kDepth ahead.
constexpr int kDepth = 4;

template <typename Y>
__global__ __launch_bounds__(1024) void linear_int8_rows_kernel(LinearArgs g, int waves, int vec_out) {
  constexpr int SK = 128;  // codes of a step: two units of each of four lanes
  __shared__ i32x4v_t part[16][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r16 = lane & 15, q = lane >> 4;
  const int64_t o0 = static_cast<int64_t>(blockIdx.x) * 16, m0 = static_cast<int64_t>(blockIdx.y) * 16;
  // Rows past the last one read the last one's values; their results go nowhere.
  const int8_t* W = reinterpret_cast<const int8_t*>(g.w) + min(o0 + r16, g.out - 1) * g.ldw;
  const int8_t* X = reinterpret_cast<const int8_t*>(g.x) + min(m0 + r16, g.m - 1) * g.ldx;
  auto unit = [&](const int8_t* row, int64_t k) -> vec16 {
    const vec16 v = load16(row + (k < g.in ? k : 0));
    vec16 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.d[i] = k < g.in ? v.d[i] : 0u;
    return r;
  };
  const int64_t steps = (g.in + SK - 1) / SK;
  i32x4v_t acc = {0, 0, 0, 0};
  vec16 wv[kDepth][2], xv[kDepth][2];
  for (int64_t s0 = wave; s0 < steps; s0 += static_cast<int64_t>(waves) * kDepth) {
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
      const int64_t k = (s0 + static_cast<int64_t>(d) * waves) * SK + q * 32;
#pragma unroll
      for (int u = 0; u < 2; ++u) wv[d][u] = unit(W, k + u * 16);
#pragma unroll
      for (int u = 0; u < 2; ++u) xv[d][u] = unit(X, k + u * 16);
    }
#pragma unroll
    for (int d = 0; d < kDepth; ++d)
#pragma unroll
      for (int u = 0; u < 2; ++u) acc = mac16(code_t{}, wv[d][u], xv[d][u], acc);
  }
  part[wave][lane] = acc;
  __syncthreads();
  // Lane (row of x, q) holds outputs 4 q .. 4 q + 3: the first wave finishes them.
  const int64_t m = m0 + r16, o = o0 + 4 * q;
  if (wave != 0 || m >= g.m || o >= g.out) return;
  float z[1][4], bias[4], scale[4];
  load_bias4<Y>(g, o, bias);
  load_scale4(g, o, scale);
  i32x4v_t sum = {0, 0, 0, 0};
  for (int w = 0; w < waves; ++w) sum += part[w][lane];
  sums4<true>(__builtin_bit_cast(float4, sum), g.x_scale[m], scale, z[0]);
  finish4<Y, 1>(g, m, 0, o, z, bias, vec_out);
}

template <typename Y>
hipError_t launch_rows(const LinearArgs& a, hipStream_t st) {
  const int64_t steps = (a.in + 127) / 128, w = steps / kDepth;
  const int waves = (int)(w < 1 ? 1 : w > 16 ? 16 : w);
  const uintptr_t unit = 4 * sizeof(Y);
  const int vec_out = a.ldy % 4 == 0 && (uintptr_t)a.y % unit == 0 &&
                      (!a.r || (a.ldr % 4 == 0 && (uintptr_t)a.r % unit == 0));
  const int64_t groups = (a.m + 15) / 16;
  for (int64_t g0 = 0; g0 < groups; g0 += 65535) {
    LinearArgs b = a;
    const int64_t es = sizeof(Y), m0 = g0 * 16;
    b.x = (const char*)a.x + m0 * a.ldx;
    b.x_scale = a.x_scale + m0;
    b.y = (char*)a.y + m0 * a.ldy * es;
    if (a.r) b.r = (const char*)a.r + m0 * a.ldr * es;
    b.m = a.m - m0;
    const int64_t n = groups - g0 < 65535 ? groups - g0 : 65535;
    if (n * 16 < b.m) b.m = n * 16;
    hipLaunchKernelGGL(linear_int8_rows_kernel<Y>, dim3((unsigned)((a.out + 15) / 16), (unsigned)n), dim3(64 * waves), 0,
                       st, b, waves, vec_out);
  }
  return hipGetLastError();
}

// ---- plan ----

constexpr int64_t kFewRows = 16;

struct Plan {
  bool code_x, pack_x, pack_w, rows;
  size_t x_bytes, scale_bytes, w_bytes;
  LinearTiles tiles;
  LinearArgs a;  // the product, with the strides that its operands have then
};

int64_t padded(int64_t in) { return (in + kUnit - 1) / kUnit * kUnit; }

// Rows of whole 16-byte units, so that no unit of one holds what is not its: w's codes behind `in` meet zeros, which
// only rows that are no whole units need of x.
Plan plan_of(const LinearArgs& a, int x_dtype) {
  Plan p;
  p.a = a;
  p.code_x = x_dtype >= 0;
  p.pack_x = !p.code_x && (a.in % kUnit != 0 || a.ldx % kUnit != 0 || (uintptr_t)a.x % kUnit != 0);
  p.pack_w = a.ldw % kUnit != 0 || (uintptr_t)a.w % kUnit != 0;
  const int64_t wide = padded(a.in);
  p.x_bytes = p.code_x || p.pack_x ? align_up(a.m * wide) : 0;
  p.scale_bytes = p.code_x ? align_up(a.m * 4) : 0;
  p.w_bytes = p.pack_w ? align_up(a.out * wide) : 0;
  p.a.in = wide;
  if (p.code_x || p.pack_x) p.a.ldx = wide;
  if (p.pack_w) p.a.ldw = wide;
  if (p.code_x || p.pack_x) p.a.x = nullptr;  // in the workspace, on 256 bytes
  if (p.pack_w) p.a.w = nullptr;
  p.tiles = linear_tiles_plan(p.a);
  p.rows = p.tiles.config < 0 || a.m <= kFewRows;
  return p;
}

}  // namespace

hipError_t launch_quantize_rows(const CodeArgs& a, hipStream_t stream) {
  const int64_t per = a.dtype == CONV_F32 ? 4 : 8;
  const int vec = a.ldx % per == 0 && (uintptr_t)a.x % 16 == 0;
  const int64_t x = a.m < 65535 * (int64_t)256 ? (a.m < 65535 ? a.m : 65535) : 1 << 24;
  const dim3 grid((unsigned)x, (unsigned)((a.m + x - 1) / x));
  if (a.dtype == CONV_F32)
    hipLaunchKernelGGL(quantize_rows_kernel<float>, grid, dim3(256), 0, stream, a, vec);
  else
    hipLaunchKernelGGL(quantize_rows_kernel<bf16_t>, grid, dim3(256), 0, stream, a, vec);
  return hipGetLastError();
}

size_t linear_int8_workspace(const LinearArgs& a, int x_dtype) {
  const Plan p = plan_of(a, x_dtype);
  return p.x_bytes + p.scale_bytes + p.w_bytes + (p.rows ? 0 : p.tiles.part_bytes);
}

hipError_t launch_linear_int8(const LinearArgs& a, int x_dtype, void* workspace, hipStream_t stream) {
  Plan p = plan_of(a, x_dtype);
  char* ws = (char*)workspace;
  const int64_t wide = padded(a.in);
  if (p.code_x) {
    const CodeArgs c = {a.x, (int8_t*)ws, (float*)(ws + p.x_bytes), a.m, a.in, a.ldx, wide, x_dtype};
    const hipError_t e = launch_quantize_rows(c, stream);
    if (e != hipSuccess) return e;
    p.a.x = c.codes;
    p.a.x_scale = c.scales;
  }
  auto copy = [&](const void* src, int64_t rows, int64_t ld, char* dst) {
    const int64_t blocks = (rows * (wide / kUnit) + 255) / 256;
    hipLaunchKernelGGL(pack_codes_kernel, dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, stream,
                       (const int8_t*)src, rows, a.in, ld, (int8_t*)dst, wide);
  };
  if (p.pack_x) {
    copy(a.x, a.m, a.ldx, ws);
    p.a.x = ws;
  }
  ws += p.x_bytes + p.scale_bytes;
  if (p.pack_w) {
    copy(a.w, a.out, a.ldw, ws);
    p.a.w = ws;
    ws += p.w_bytes;
  }
  if (!p.rows) return launch_linear_tiles(p.a, p.tiles, ws, stream);
  return a.dtype == CONV_F32 ? launch_rows<float>(p.a, stream) : launch_rows<bf16_t>(p.a, stream);
}

void linear_int8_describe(const LinearArgs& a, int x_dtype, char* buf, size_t len) {
  const Plan p = plan_of(a, x_dtype);
  char product[96];
  if (p.rows)
    snprintf(product, sizeof product, "linear_int8_rows_kernel tile=16x16 split=1");
  else
    snprintf(product, sizeof product, "linear_tiles%s_kernel%s tile=%s split=%d", p.tiles.config == 0 ? "256" : "",
             p.tiles.splits > 1 ? ";linear_join_kernel" : "", linear_tiles_name(p.tiles.config), p.tiles.splits);
  snprintf(buf, len, "linear_int8 kernels=%s%s%s workspace=%zu", p.code_x ? "quantize_rows_kernel;" : "",
           p.pack_x || p.pack_w ? "pack_codes_kernel;" : "", product, linear_int8_workspace(a, x_dtype));
}

}  // namespace convsel
