// Linear layers on 8-bit codes: y = act((X W^T) sx sw + b) + r, with a scale for
// each row of x and each output.
//
// Sums of codes are 32-bit whole numbers, exact up to 131071 input features.
// Many rows go in the tiles of linear_tiles.hip, whose walk of 16-byte units is
// the same for codes, sixteen a unit; few stream the weights through registers
// (here).  Rows of x that come as numbers are coded by a kernel before the
// product (4096 rows of 4096 in bf16: 13.6 us, 3.7 TB/s), one or two of them by the
// product's own.
//
// What bounds it: few rows, the weights' way from memory (1 row, 4096 -> 4096:
// 6.5 us in the kernel, 2.6 TB/s, of which launch and first loads are half); many,
// the matrix cores at the clock that the card's power leaves (4096 rows, 4096 ->
// 16384: 231 us, 2380 TOP/s, 251 on a card of lower clock; a large library product
// reaches 2130).
#include <stdio.h>

#include <type_traits>

#include "linear_common.hpp"

namespace convsel {
namespace {

using namespace lm;

constexpr int64_t kUnit = 16;
constexpr size_t kAlign = 256;
size_t align_up(int64_t bytes) { return ((size_t)bytes + kAlign - 1) / kAlign * kAlign; }

int64_t padded(int64_t in) { return (in + kUnit - 1) / kUnit * kUnit; }

// ---- codes ----

//   scale = max(largest / 127, 2^-100), code = round(x / scale), both quotients in fp32
constexpr int kCoded = 8;  // numbers of a step of a thread

// Numbers k .. of a row of n, zeros behind it; `vec`: rows start on 16 bytes.
template <typename T>
__device__ __forceinline__ void numbers(const T* x, int64_t k, int64_t n, int vec, float (&z)[kCoded]) {
  if (vec && k + kCoded <= n) {
    constexpr int UE = elem<T>::per16;
#pragma unroll
    for (int u = 0; u < kCoded / UE; ++u) {
      const vec16 v = load16(x + k + u * UE);
#pragma unroll
      for (int e = 0; e < UE; ++e) z[u * UE + e] = elem<T>::to_f32(vec16_get<T>(v, e));
    }
  } else {
#pragma unroll
    for (int i = 0; i < kCoded; ++i) {
      const float v = elem<T>::load(x + min(k + i, n - 1));
      z[i] = k + i < n ? v : 0.f;
    }
  }
}
__device__ __forceinline__ float largest(const float (&z)[kCoded], float top) {
#pragma unroll
  for (int i = 0; i < kCoded; ++i) top = fmaxf(top, fabsf(z[i]) < __builtin_inff() ? fabsf(z[i]) : 0.f);
  return top;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
// A row's scale, its reciprocal, and what infinities count as.
struct RowScale {
  float scale, inverse, end;
  __device__ __forceinline__ explicit RowScale(float top) {
    scale = fmaxf(top / 127.f, kMinScale);
    inverse = 1.f / scale;
    end = fmaxf(top, fminf(127.f * scale, 0x1.fffffep127f));
  }
  // Infinities take the largest code of their sign, NaN zero.
  __device__ __forceinline__ uint2 code(float (&z)[kCoded]) const {
#pragma unroll
    for (int i = 0; i < kCoded; ++i) z[i] = z[i] != z[i] ? 0.f : fminf(fmaxf(z[i], -end), end);
    return make_uint2(four_codes<CONVSEL_KV_INT8>(z[0], z[1], z[2], z[3], scale, inverse),
                      four_codes<CONVSEL_KV_INT8>(z[4], z[5], z[6], z[7], scale, inverse));
  }
};

// One workgroup a row: its largest finite magnitude, then codes, from the CU's own cache.
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(CodeArgs a, int vec) {
  __shared__ float red[4];
  const int64_t row = blockIdx.x + static_cast<int64_t>(blockIdx.y) * gridDim.x;
  if (row >= a.m) return;
  const T* x = reinterpret_cast<const T*>(a.x) + row * a.ldx;
  int8_t* codes = a.codes + row * a.ldc;
  const bool whole = a.ldc % kCoded == 0 && reinterpret_cast<uintptr_t>(a.codes) % kCoded == 0;
  // The first 8192 numbers of a row stay in registers (4096 rows of 4096 in bf16: 13.6 us, 4 more when they are read again).
  constexpr int HELD = 4, STEP = 256 * kCoded;
  const int64_t k0 = threadIdx.x * kCoded;
  float top = 0.f, held[HELD][kCoded], z[kCoded];
#pragma unroll
  for (int h = 0; h < HELD; ++h)
    if (k0 + h * STEP < a.in) numbers<T>(x, k0 + h * STEP, a.in, vec, held[h]);
#pragma unroll
  for (int h = 0; h < HELD; ++h)
    if (k0 + h * STEP < a.in) top = largest(held[h], top);
  for (int64_t k = k0 + HELD * STEP; k < a.in; k += STEP) {
    numbers<T>(x, k, a.in, vec, z);
    top = largest(z, top);
  }
  top = wave_max(top);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
  __syncthreads();
  const RowScale s(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
  if (threadIdx.x == 0) a.scales[row] = s.scale;
  auto put = [&](int64_t k, const uint2& c) {
    if (whole) {
      *reinterpret_cast<uint2*>(codes + k) = c;
    } else {
#pragma unroll
      for (int i = 0; i < kCoded; ++i)
        if (k + i < a.ldc) codes[k + i] = static_cast<int8_t>((i < 4 ? c.x : c.y) >> (8 * (i & 3)));
    }
  };
#pragma unroll
  for (int h = 0; h < HELD; ++h) {
    const int64_t k = k0 + h * STEP;
    if (k < a.in) put(k, s.code(held[h]));
    else if (k < a.ldc) put(k, make_uint2(0u, 0u));
  }
  for (int64_t k = k0 + HELD * STEP; k < a.ldc; k += STEP) {
    numbers<T>(x, k, a.in, vec, z);
    put(k, s.code(z));
  }
}

// Rows of codes copied to rows of whole 16-byte units, zeros behind them.
__global__ __launch_bounds__(256) void pack_codes_kernel(const int8_t* src, int64_t rows, int64_t in, int64_t ld,
                                                         int8_t* dst, int64_t padded) {
  const int64_t per = padded / kUnit;
  const bool vec = ld % kUnit == 0 && reinterpret_cast<uintptr_t>(src) % kUnit == 0;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < rows * per;
       i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t row = i / per, k = (i - row * per) * kUnit;
    const int8_t* p = src + row * ld;
    vec16 v;
    if (vec && k + kUnit <= in) {
      store16(dst + i * kUnit, load16(p + k));
      continue;
    }
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
// What bounds it is the weights' way from memory; steps are fetched kDepth ahead.  X numbers: every workgroup codes its
// rows itself, to LDS, while its first weights are on their way, which costs less than a kernel before it as long as
// the rows are short.
constexpr int kDepth = 4;

template <typename Y, typename X>
__global__ __launch_bounds__(1024) void linear_int8_rows_kernel(LinearArgs g, int waves, int vec_out, int vec_in) {
  constexpr int SK = 128;  // codes of a step: two units of each of four lanes
  constexpr bool CODES = operand<X>::codes;
  __shared__ i32x4v_t part[16][64];
  __shared__ float red[CODES ? 1 : 16][16], row_scale[16];
  extern __shared__ __align__(16) int8_t coded[];  // rows of g.in + 16
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r16 = lane & 15, q = lane >> 4;
  const int64_t o0 = static_cast<int64_t>(blockIdx.x) * 16, m0 = static_cast<int64_t>(blockIdx.y) * 16;
  const int rows = static_cast<int>(min(g.m - m0, static_cast<int64_t>(16)));
  // Rows past the last one read the last one's values; their results go nowhere.
  const int8_t* W = reinterpret_cast<const int8_t*>(g.w) + min(o0 + r16, g.out - 1) * g.ldw;
  const int8_t* codes = CODES ? reinterpret_cast<const int8_t*>(g.x) + (m0 + min(r16, rows - 1)) * g.ldx
                              : coded + min(r16, rows - 1) * (g.in + 16);
  auto unit = [&](const int8_t* row, int64_t k) -> vec16 {
    const vec16 v = load16(row + (k < g.in ? k : 0));
    vec16 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.d[i] = k < g.in ? v.d[i] : 0u;
    return r;
  };
  const int64_t steps = (g.in + SK - 1) / SK, stride = static_cast<int64_t>(waves) * kDepth;
  i32x4v_t acc = {0, 0, 0, 0};
  vec16 wv[kDepth][2], xv[kDepth][2];
  auto column = [&](int64_t s0, int d) { return (s0 + static_cast<int64_t>(d) * waves) * SK + q * 32; };
  auto weights = [&](int64_t s0) {
#pragma unroll
    for (int d = 0; d < kDepth; ++d)
#pragma unroll
      for (int u = 0; u < 2; ++u) wv[d][u] = unit(W, column(s0, d) + u * 16);
  };
  int64_t s0 = wave;
  weights(s0);
  if constexpr (!CODES) {
    const int64_t n = g.numbers, per = static_cast<int64_t>(waves) * 64 * kCoded;
    float z[kCoded];
    for (int r = 0; r < rows; ++r) {
      const X* x = reinterpret_cast<const X*>(g.x) + (m0 + r) * g.ldx;
      float top = 0.f;
      for (int64_t k = threadIdx.x * kCoded; k < n; k += per) {
        numbers<X>(x, k, n, vec_in, z);
        top = largest(z, top);
      }
      top = wave_max(top);
      if (lane == 0) red[r][wave] = top;
    }
    lds_sync();
    for (int r = 0; r < rows; ++r) {
      const X* x = reinterpret_cast<const X*>(g.x) + (m0 + r) * g.ldx;
      float top = 0.f;
      for (int w = 0; w < waves; ++w) top = fmaxf(top, red[r][w]);
      const RowScale s(top);
      if (threadIdx.x == 0) row_scale[r] = s.scale;
      for (int64_t k = threadIdx.x * kCoded; k < g.in; k += per) {
        numbers<X>(x, k, n, vec_in, z);
        *reinterpret_cast<uint2*>(coded + r * (g.in + 16) + k) = s.code(z);
      }
    }
    lds_sync();
  }
  for (;;) {
#pragma unroll
    for (int d = 0; d < kDepth; ++d)
#pragma unroll
      for (int u = 0; u < 2; ++u) xv[d][u] = unit(codes, column(s0, d) + u * 16);
#pragma unroll
    for (int d = 0; d < kDepth; ++d)
#pragma unroll
      for (int u = 0; u < 2; ++u) acc = mac16(code_t{}, wv[d][u], xv[d][u], acc);
    s0 += stride;
    if (s0 >= steps) break;
    weights(s0);
  }
  part[wave][lane] = acc;
  __syncthreads();
  // Lane (row of x, q) holds outputs 4 q .. 4 q + 3: the first wave finishes them.
  const int64_t m = m0 + r16, o = o0 + 4 * q;
  if (wave != 0 || m >= g.m || o >= g.out) return;
  float z[1][4], bias[4];
  Scale scale[4];
  load_bias4<Y>(g, o, bias);
  load_scale4(g, o, scale);
  i32x4v_t sum = {0, 0, 0, 0};
  for (int w = 0; w < waves; ++w) sum += part[w][lane];
  sums4<true>(__builtin_bit_cast(float4, sum), CODES ? g.x_scale[m] : row_scale[r16], scale, z[0]);
  finish4<Y, 1>(g, m, 0, o, z, bias, vec_out);
}

template <typename Y, typename X>
hipError_t launch_rows(const LinearArgs& a, hipStream_t st) {
  const int64_t steps = (a.in + 127) / 128, w = steps / kDepth;
  const int waves = (int)(w < 1 ? 1 : w > 16 ? 16 : w);
  const uintptr_t unit = 4 * sizeof(Y);
  const int vec_out = a.ldy % 4 == 0 && (uintptr_t)a.y % unit == 0 &&
                      (!a.r || (a.ldr % 4 == 0 && (uintptr_t)a.r % unit == 0));
  const int vec_in = a.ldx % operand<X>::per16 == 0 && (uintptr_t)a.x % 16 == 0;
  const int64_t groups = (a.m + 15) / 16;
  const size_t lds = operand<X>::codes ? 0 : (size_t)((a.m < 16 ? a.m : 16) * (a.in + 16));
  for (int64_t g0 = 0; g0 < groups; g0 += 65535) {
    LinearArgs b = a;
    const int64_t es = sizeof(Y), m0 = g0 * 16;
    b.x = (const char*)a.x + m0 * a.ldx * operand<X>::bytes;
    if (operand<X>::codes) b.x_scale = a.x_scale + m0;
    b.y = (char*)a.y + m0 * a.ldy * es;
    if (a.r) b.r = (const char*)a.r + m0 * a.ldr * es;
    b.m = a.m - m0;
    const int64_t n = groups - g0 < 65535 ? groups - g0 : 65535;
    if (n * 16 < b.m) b.m = n * 16;
    const dim3 grid((unsigned)((a.out + 15) / 16), (unsigned)n);
    hipLaunchKernelGGL((linear_int8_rows_kernel<Y, X>), grid, dim3(64 * waves), lds, st, b, waves, vec_out, vec_in);
  }
  return hipGetLastError();
}

template <typename Y>
hipError_t launch_rows_of(const LinearArgs& a, int x_dtype, hipStream_t st) {
  return x_dtype < 0 ? launch_rows<Y, code_t>(a, st)
                     : x_dtype == CONV_F32 ? launch_rows<Y, float>(a, st) : launch_rows<Y, bf16_t>(a, st);
}

// ---- plan ----

struct Plan {
  bool code_x, pack_x, pack_w, rows;  // code_x: by a kernel before the product
  size_t x_bytes, scale_bytes, w_bytes;
  LinearTiles tiles;
  LinearArgs a;  // the product, with the strides that its operands have then
};

// Few rows, in us.  By rows: 2.3 and the way of a CU's share of the weights, 16.8 GB/s, a quarter longer with 16 rows.
// In tiles: by their plan, which counts no bytes, but at least 7 and all bytes at a copy's rate.  us by rows and in
// tiles, rows coded before, weights from memory:
//   from 4096 -> 4096     4096 -> 12288   11008 -> 4096    2048 -> 1024
//     1 row    6.3  9.3    14.1 16.1       13.6 15.1        4.1 6.9
//     16       7.2  9.9    17.7 16.6       15.6 15.2        4.7 7.1
//     32      10.7 10.4    27.6 17.4       25.7 15.9        4.7 7.2
//     64      17.9 11.7    50.8 18.8       46.0 17.7        4.8 7.5
constexpr int64_t kFewRows = 64;

bool in_rows(const LinearArgs& a, const LinearTiles& t) {
  if (t.config < 0) return true;
  if (a.m > kFewRows) return false;
  const double groups = (double)((a.out + 15) / 16 * ((a.m + 15) / 16));
  const double share = (groups > 256 ? groups / 256 : 1.) * 16. * a.in;
  const double rows = 2.3 + share / 16.8e3 * (1 + 0.25 * (a.m < 16 ? a.m : 16) / 16);
  const double least = 7 + ((double)a.out * a.in + (double)a.m * (a.in + 4 * a.out)) / 5.05e6;
  return rows <= (t.us + 1.7 > least ? t.us + 1.7 : least);
}

// Whether the kernel for few rows codes them itself: every workgroup does, one row after the other.  us of both ways,
// 4096 -> 4096 in bf16: 1 row 7.8 and 9.9, 2 rows 9.0 and 10.2, 4 rows 11.7 and 10.4; 1 row, 16384 -> 4096: 19 and 24.
bool coded_inside(const LinearArgs& a) { return a.m <= 2 && a.m * (padded(a.in) + 16) <= 40 * 1024; }

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
  p.rows = in_rows(p.a, p.tiles);
  if (p.rows && p.code_x && coded_inside(a)) {
    p.code_x = false;
    p.x_bytes = p.scale_bytes = 0;
    p.a.x = a.x;
    p.a.ldx = a.ldx;
    p.a.numbers = a.in;
  }
  return p;
}

}  // namespace

hipError_t launch_quantize_rows(const CodeArgs& a, hipStream_t stream) {
  const int64_t per = a.dtype == CONV_F32 ? 4 : 8;
  const int vec = a.ldx % per == 0 && (uintptr_t)a.x % 16 == 0;
  const int64_t x = a.m < 65535 * (int64_t)256 ? (a.m < 65535 ? a.m : 65535) : 1 << 23;
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
  const int kind = x_dtype >= 0 && !p.code_x ? x_dtype : CONVSEL_CODES;
  return a.dtype == CONV_F32 ? launch_rows_of<float>(p.a, kind, stream) : launch_rows_of<bf16_t>(p.a, kind, stream);
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
