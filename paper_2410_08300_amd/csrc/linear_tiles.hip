// Linear layers in tiles: both operands through LDS DMA.
//
// A workgroup owns TM rows of x and TO outputs and walks the reduction in
// k-tiles of 128 bytes (64 bf16, 32 fp32), so that every DMA instruction reads
// whole cache lines: eight operand rows of 128 bytes.  In LDS two rows share a
// 256-byte line, with the 16-byte unit u of row r at place 8 (r % 2) + (u ^ (r /
// 2 % 8)): the 16 rows that a quarter wave reads of one unit lie on different
// banks.  Rows past the operand and columns past the reduction read zeros
// through the buffer's range.  The products' rows are w's and their columns x's.
// Sums leave through LDS, each wave in a place of its own, so that every row of
// y is read (residual) and written along its outputs.
//
// Tiles of 64 and 128 (linear_tiles_kernel): NST stages form a ring; a stage is
// filled again as soon as its last unit is read.  A wave multiplies FO x FM
// blocks of 32 x 32 in four steps a k-tile; the operands of a step are read
// while the step before it multiplies, those of the next k-tile's first step
// behind the tile's one barrier.  Two or three workgroups share a CU and fill
// each other's waits.  Tiles of 256 in bf16: linear_tiles256_kernel.
//
// What bounds them: few tiles, the way of a k-tile from memory, once a k-tile;
// many, the matrix cores at the clock that the card's power leaves them (bf16
// 4096 rows, 4096 -> 16384: 416 us, 1320 TFLOP/s; fp32 4096 rows, 2048 -> 4096:
// 494 us, 139 TFLOP/s).
#include <stdio.h>

#include <type_traits>
#include <utility>

#include "igemm_common.hpp"
#include "linear_common.hpp"

namespace convsel {
namespace {

using namespace igemm;
using namespace lm;

template <int FO_, int FM_, int WO_, int WM_, int NST_>
struct Tile {
  static constexpr int PER_CU = FO_ * WO_ == 8 ? 1 : FO_ * WO_ == 4 ? 2 : 3;  // workgroups that a CU holds
  static constexpr int FO = FO_, FM = FM_, WO = WO_, WM = WM_, NST = NST_;
  static constexpr int TO = FO * 32 * WO, TM = FM * 32 * WM, WAVES = WO * WM;
  static constexpr int STAGE = (TO + TM) * 128;
  static constexpr int NDMA = (TO + TM) / 8 / WAVES;  // DMA instructions of a wave and stage
  static constexpr int OUT_ROW = FO * 32 + 4;         // floats: rows 16 bytes apart in the banks
  static constexpr int OUT = WAVES * 32 * OUT_ROW * 4;
  static constexpr int LDS = NST * STAGE > OUT ? NST * STAGE : OUT;
  static_assert((TO + TM) % (8 * WAVES) == 0 && LDS <= 160 * 1024 && NST >= 2 && NST <= 4 && NDMA * (NST - 1) <= 63,
                "tile");
};

struct TileArgs {
  LinearArgs g;
  int to, tm;          // tiles of outputs and of rows
  int splits, per;     // k-tiles of a part
  int vec_out;
  float* part;         // [split][m][out rounded up to 4]
};

// The workgroup's part of the reduction and tile.  Workgroup w runs on XCD w % 8: each XCD has a contiguous run of
// tiles, eight rows of tiles deep before the next outputs, so that the workgroups of one L2 share both operands.  False
// for a workgroup without work.
__device__ __forceinline__ bool place(const TileArgs& a, int& split, int& tm, int& to) {
  const int units = a.to * a.tm * a.splits;
  const int per_xcd = (units + 7) >> 3;
  const int unit = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= per_xcd || unit >= units) return false;
  const int tile = unit / a.splits;
  split = unit % a.splits;
  const int band = tile / (8 * a.to), in_band = tile - band * 8 * a.to;
  const int deep = min(8, a.tm - band * 8);
  tm = band * 8 + in_band % deep;
  to = in_band / deep;
  return true;
}

// f(0), f(1) ... with constants.
template <int... I, typename F>
__device__ __forceinline__ void times(std::integer_sequence<int, I...>, F f) {
  (f(std::integral_constant<int, I>{}), ...);
}

// Four neighbouring values of y's type.
template <typename T> struct Quad;
template <> struct Quad<float> {
  float4 v;
  __device__ __forceinline__ void to(float (&z)[4]) const { z[0] += v.x; z[1] += v.y; z[2] += v.z; z[3] += v.w; }
  __device__ __forceinline__ static Quad from(const float (&z)[4]) { return {make_float4(z[0], z[1], z[2], z[3])}; }
};
template <> struct Quad<bf16_t> {
  uint2 v;
  __device__ __forceinline__ void to(float (&z)[4]) const {
    z[0] += bf16_to_f32(v.x & 0xffffu); z[1] += bf16_to_f32(v.x >> 16);
    z[2] += bf16_to_f32(v.y & 0xffffu); z[3] += bf16_to_f32(v.y >> 16);
  }
  __device__ __forceinline__ static Quad from(const float (&z)[4]) {
    return {make_uint2(f32x2_to_bf16x2(z[0], z[1]), f32x2_to_bf16x2(z[2], z[3]))};
  }
};

// What store_blocks does, of a wave whose rows and outputs all exist, in whole units: eight rows of a lane at most at a
// time, without a test, and the residual's next ones on their way while these are written.  (4096 rows, 512 -> 16384 in
// bf16: 110 us by the general way, 91 by this; with a residual 217 and 120.)
template <typename T, typename S, typename Put>
__device__ __forceinline__ void store_whole(const TileArgs& a, const Put& put, float* mine, int lane, int64_t m0,
                                            int64_t o0) {
  constexpr int FM = S::FM, PER = S::FO * 8, STEP = 64 / PER, PARTS = S::FO == 4 ? 2 : 1, G = 32 / STEP / PARTS;
  const LinearArgs& g = a.g;
  const int row = lane / PER, col = 4 * (lane % PER);
  T* y = reinterpret_cast<T*>(g.y) + (m0 + row) * g.ldy + o0 + col;
  const T* r = reinterpret_cast<const T*>(g.r) + (m0 + row) * g.ldr + o0 + col;
  const std::make_integer_sequence<int, G> all{};
  Quad<T> rest[G];
  auto fetch = [&] {
    times(all, [&](auto n_c) {
      rest[decltype(n_c)::value] = *reinterpret_cast<const Quad<T>*>(r + decltype(n_c)::value * STEP * g.ldr);
    });
    r += G * STEP * g.ldr;
  };
  if (g.r) fetch();
  float bias[4];
  load_bias4<T>(g, o0 + col, bias);
#pragma unroll 1
  for (int k = 0; k < FM * PARTS; ++k) {
    times(std::make_integer_sequence<int, FM>{}, [&](auto j_c) {
      if (decltype(j_c)::value * PARTS == k) put(j_c, mine);
    });
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    const float* from = mine + ((k % PARTS) * G * STEP + row) * S::OUT_ROW + col;
    float z[G][4];
    times(all, [&](auto n_c) {
      constexpr int n = decltype(n_c)::value;
      const float4 v = *reinterpret_cast<const float4*>(from + n * STEP * S::OUT_ROW);
      z[n][0] = v.x + bias[0]; z[n][1] = v.y + bias[1]; z[n][2] = v.z + bias[2]; z[n][3] = v.w + bias[3];
    });
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    activate_all<T, G>(z, g.act);
    if (g.r) {
      times(all, [&](auto n_c) { rest[decltype(n_c)::value].to(z[decltype(n_c)::value]); });
      if (k + 1 < FM * PARTS) fetch();
    }
    times(all, [&](auto n_c) {
      *reinterpret_cast<Quad<T>*>(y + decltype(n_c)::value * STEP * g.ldy) = Quad<T>::from(z[decltype(n_c)::value]);
    });
    y += G * STEP * g.ldy;
  }
}

// Writes a wave's results, whose first row and output are m0 and o0: through its own place in LDS, where put(j, place)
// lays rows 32 j .. of them, so that every row of y is read (residual) and written along its outputs.
template <typename T, typename S, typename Put>
__device__ __forceinline__ void store_blocks(const TileArgs& a, const Put& put, char* lds, int wave, int lane, int64_t m0,
                                             int64_t o0, int split) {
  constexpr int FO = S::FO, FM = S::FM;
  const LinearArgs& g = a.g;
  float* mine = reinterpret_cast<float*>(lds) + wave * 32 * S::OUT_ROW;
  if (a.splits == 1 && a.vec_out && m0 + 32 * FM <= g.m && o0 + 32 * FO <= g.out)  // uniform in a wave
    return store_whole<T, S>(a, put, mine, lane, m0, o0);
  const int64_t opad = (g.out + 3) & ~static_cast<int64_t>(3);
  // A lane has the same four outputs of all its rows.  Rows go in fours, so that what they read is on its way together;
  // one copy of the code for all, as five activations unrolled over a tile do not stay in the instruction cache (37 us
  // of a tile of 256, where this takes 13).
  constexpr int PER = FO * 8, STEP = 64 / PER, N = 4;
  const int row = lane / PER, col = 4 * (lane % PER);
  const int64_t o = o0 + col;
  const bool there = o < g.out;
  float bias[4];
  load_bias4<T>(g, o, bias);
#pragma unroll 1
  for (int j = 0; j < FM; ++j) {
    times(std::make_integer_sequence<int, FM>{}, [&](auto j_c) {
      if (decltype(j_c)::value == j) put(j_c, mine);
    });
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int r0 = 0; r0 < 32; r0 += N * STEP) {
      float z[N][4];
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const float4 v = *reinterpret_cast<const float4*>(mine + (r0 + n * STEP + row) * S::OUT_ROW + col);
        z[n][0] = v.x; z[n][1] = v.y; z[n][2] = v.z; z[n][3] = v.w;
      }
      const int64_t m = m0 + j * 32 + r0 + row;
      if (!there || m >= g.m) continue;
      if (a.splits > 1) {
        float* dst = a.part + (split * g.m + m) * opad + o;
#pragma unroll
        for (int n = 0; n < N; ++n)
          if (m + n * STEP < g.m)
            *reinterpret_cast<float4*>(dst + n * STEP * opad) = make_float4(z[n][0], z[n][1], z[n][2], z[n][3]);
      } else {
        finish4<T, N>(g, m, STEP, o, z, bias, a.vec_out);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
  }
}

template <typename T, typename S>
__global__ __launch_bounds__(S::WAVES * 64, S::PER_CU) void linear_tiles_kernel(TileArgs a) {
  constexpr int FO = S::FO, FM = S::FM, NDMA = S::NDMA, STAGE = S::STAGE;
  constexpr int NST = S::NST, ES = elem<T>::bytes, UE = elem<T>::per16, BK = 128 / ES;
  __shared__ __align__(16) char lds[S::LDS];
  const LinearArgs& g = a.g;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wo = wave % S::WO, wm = wave / S::WO;
  int split, tm, to;
  if (!place(a, split, tm, to)) return;  // uniform
  const int64_t m0 = static_cast<int64_t>(tm) * S::TM, o0 = static_cast<int64_t>(to) * S::TO;

  const int64_t wrows = min(g.out - o0, static_cast<int64_t>(S::TO)), xrows = min(g.m - m0, static_cast<int64_t>(S::TM));
  const uint32_t wbytes = static_cast<uint32_t>(((wrows - 1) * g.in + g.in) * ES);
  const uint32_t xbytes = static_cast<uint32_t>(((xrows - 1) * g.ldx + g.in) * ES);
  const u32x4_t wr = dma_rsrc(reinterpret_cast<const T*>(g.w) + o0 * g.in, wbytes);
  const u32x4_t xr = dma_rsrc(reinterpret_cast<const T*>(g.x) + m0 * g.ldx, xbytes);
  const uint32_t lds0 = lds_address(lds);

  // Instruction J = wave * NDMA + d of a stage fills rows 8 J .. 8 J + 7: w's rows first, then x's.
  uint32_t dvo[NDMA];
  int dku[NDMA];  // this lane's column within a k-tile
#pragma unroll
  for (int d = 0; d < NDMA; ++d) {
    const int U = (wave * NDMA + d) * 64 + lane;
    const int line = U >> 4, pos = U & 15;
    const int row = 2 * line + (pos >> 3);
    dku[d] = ((pos & 7) ^ (line & 7)) * UE;
    const bool isw = row < S::TO;
    const int64_t r = isw ? row : row - S::TO;
    const bool ok = r < (isw ? wrows : xrows);
    dvo[d] = ok ? static_cast<uint32_t>((r * (isw ? g.in : g.ldx) + dku[d]) * ES) : (isw ? wbytes : xbytes);
  }
  const int k0 = split * a.per, all = static_cast<int>((g.in + BK - 1) / BK);
  const int nk = min(all, k0 + a.per) - k0;
  // DMA instruction d of stage kt.  Past the last k-tile it fills the stage with zeros that nobody reads: the loop
  // below has no branch, and the same number is always on its way.
  auto issue = [&](int kt, int d) {
    const uint32_t st = lds0 + (kt % NST) * STAGE;
    const int at = k0 + min(kt, nk - 1);
    const int64_t left = kt < nk ? g.in - static_cast<int64_t>(at) * BK : 0;
    const int J = wave * NDMA + d;
    const bool isw = J < S::TO / 8;
    dma16(isw ? wr : xr, st + J * 1024, dku[d] < left ? dvo[d] : (isw ? wbytes : xbytes),
          static_cast<uint32_t>(at) * 128);
  };

  // Unit 2 t + half of row l32 of a block of 32 rows.
  const int half = lane >> 5, l32 = lane & 31;
  int off[4];
#pragma unroll
  for (int t = 0; t < 4; ++t)
    off[t] = (l32 >> 1) * 256 + ((8 * (l32 & 1) + ((2 * t + half) ^ ((l32 >> 1) & 7))) << 4);

  f32x16_t acc[FO][FM];
#pragma unroll
  for (int i = 0; i < FO; ++i)
#pragma unroll
    for (int j = 0; j < FM; ++j) acc[i][j] = zero16();
  vec16 fw[2][FO], fx[2][FM];
  auto read = [&](int kt, auto t_c) {
    constexpr int t = decltype(t_c)::value;
    const char* st = lds + (kt % NST) * STAGE + off[t];
#pragma unroll
    for (int i = 0; i < FM; ++i) fx[t & 1][i] = *reinterpret_cast<const vec16*>(st + S::TO * 128 + (wm * FM + i) * 4096);
#pragma unroll
    for (int i = 0; i < FO; ++i) fw[t & 1][i] = *reinterpret_cast<const vec16*>(st + (wo * FO + i) * 4096);
  };
  auto multiply = [&](auto t_c) {
    constexpr int t = decltype(t_c)::value;
#pragma unroll
    for (int i = 0; i < FO; ++i)
#pragma unroll
      for (int j = 0; j < FM; ++j) mfma_32x32<T>(acc[i][j], fw[t & 1][i], fx[t & 1][j]);
  };
  // One step: the reads of the next one between the products of this.
  auto interleave = [&]() {
    constexpr int M = FO * FM * (ES == 4 ? 4 : 1), R = FO + FM;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, M >= 2 * R ? 2 : 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // A stage is in once no DMAs but those of the `later` stages issued after it are pending.  This wave's reads of the
  // stage before it have arrived too, so behind the barrier that stage may be filled again.
  auto arrive = [&](auto later_c) {
    CONVSEL_WAIT_VMCNT(decltype(later_c)::value * NDMA);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  const std::integral_constant<int, 0> t0{};
  const std::integral_constant<int, 1> t1{};
  const std::integral_constant<int, 2> t2{};
  const std::integral_constant<int, 3> t3{};
#pragma unroll
  for (int p = 0; p < NST; ++p)
#pragma unroll
    for (int d = 0; d < NDMA; ++d) issue(p, d);
  arrive(std::integral_constant<int, NST - 1>{});
  read(0, t0);
  __builtin_amdgcn_sched_barrier(0);
  for (int kt = 0; kt < nk; ++kt) {
    read(kt, t1);
    multiply(t0);
    interleave();
    read(kt, t2);
    multiply(t1);
    interleave();
    read(kt, t3);
    multiply(t2);
    interleave();
    arrive(std::integral_constant<int, NST - 2>{});
    read(kt + 1, t0);
    __builtin_amdgcn_sched_barrier(0);
    // The stage just read is filled again, an instruction behind each product: a burst of them would leave the matrix
    // cores idle.
#pragma unroll
    for (int q = 0; q < FO * FM || q < NDMA; ++q) {
      if (q < FO * FM) mfma_32x32<T>(acc[q / FM][q % FM], fw[1][q / FM], fx[1][q % FM]);
      __builtin_amdgcn_sched_barrier(0);
      if (q < NDMA) issue(kt + NST, q);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  CONVSEL_WAIT_VMCNT(0);  // the zeros behind the last k-tile too
  lds_sync();             // every wave is done with the stages
  const auto put = [&](auto j_c, float* mine) {
    times(std::make_integer_sequence<int, 4 * FO>{}, [&](auto n_c) {
      constexpr int i = decltype(n_c)::value / 4, v = decltype(n_c)::value % 4;
      const f32x16_t& z = acc[i][decltype(j_c)::value];
      *reinterpret_cast<float4*>(mine + l32 * S::OUT_ROW + 32 * i + 8 * v + 4 * half) =
          make_float4(z[4 * v], z[4 * v + 1], z[4 * v + 2], z[4 * v + 3]);
    });
  };
  store_blocks<T, S>(a, put, lds, wave, lane, m0 + wm * FM * 32, o0 + wo * FO * 32, split);
}

struct Place {
  int i, j;
};
constexpr Place place_of(int n) {
  int r = 0;
  while ((r + 1) * (r + 1) <= n) ++r;
  const int k = n - r * r;
  return k <= r ? Place{r, k} : Place{k - r - 1, r};
}

// Tiles of 256 in bf16: four waves, one to each SIMD, of 128 x 128.  (Eight waves of 128 x 64 read half as much again
// from LDS, which took a quarter longer.)  Products of 16 x 16 x 32: alone, on random operands, they reach 2065
// TFLOP/s, those of 32 x 32 x 16 1810, because the card's power bounds both (5 % less time here).  The ring holds five
// units of one operand's 256 rows and one k-tile, in the order w, x, w, x ...; a wave reads all of a k-tile's operands
// in its first half, so that a unit is on its way for three quarters of a k-tile at least.
typedef Tile<4, 4, 2, 2, 2> Tile256;

__global__ __launch_bounds__(256, 1) void linear_tiles256_kernel(TileArgs a) {
  typedef bf16_t T;
  typedef Tile256 S;
  constexpr int ES = elem<T>::bytes, UE = elem<T>::per16, BK = 128 / ES, UNIT = 256 * 128, RING = 5;
  static_assert(S::OUT <= RING * UNIT, "epilogue");
  __shared__ __align__(16) char lds[RING * UNIT];
  const LinearArgs& g = a.g;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wo = wave & 1, wm = wave >> 1;
  int split, tm, to;
  if (!place(a, split, tm, to)) return;  // uniform
  const int64_t m0 = static_cast<int64_t>(tm) * 256, o0 = static_cast<int64_t>(to) * 256;
  const int wrows = static_cast<int>(min(g.out - o0, static_cast<int64_t>(256)));
  const int xrows = static_cast<int>(min(g.m - m0, static_cast<int64_t>(256)));
  const uint32_t wbytes = static_cast<uint32_t>(wrows * g.in * ES);
  const uint32_t xbytes = static_cast<uint32_t>(((xrows - 1) * g.ldx + g.in) * ES);
  u32x4_t wr = dma_rsrc(reinterpret_cast<const T*>(g.w) + o0 * g.in, wbytes);
  u32x4_t xr = dma_rsrc(reinterpret_cast<const T*>(g.x) + m0 * g.ldx, xbytes);
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(lds) + wave * 8192);
  const int all = static_cast<int>((g.in + BK - 1) / BK);
  const int k0 = __builtin_amdgcn_readfirstlane(split * a.per);
  const int nk = __builtin_amdgcn_readfirstlane(min(all, k0 + a.per) - k0);
  // Columns of the last k-tile, where it is cut off.
  const int ragged = k0 + nk == all ? static_cast<int>(g.in - static_cast<int64_t>(all - 1) * BK) : BK;

  // Instruction d of this wave fills rows 8 (8 wave + d) .. of a unit; the unit of a row that a lane fetches depends on
  // d's parity only.
  uint32_t wvo[8], xvo[8];
  int col[2];
#pragma unroll
  for (int d = 0; d < 8; ++d) {
    const int U = (wave * 8 + d) * 64 + lane;
    const int line = U >> 4, pos = U & 15;
    const int row = 2 * line + (pos >> 3), c = ((pos & 7) ^ (line & 7)) * UE;
    if (d < 2) col[d] = c;
    wvo[d] = row < wrows ? static_cast<uint32_t>((row * g.in + c) * ES) : wbytes;
    xvo[d] = row < xrows ? static_cast<uint32_t>((row * g.ldx + c) * ES) : xbytes;
  }
  // Before k-tile kt is fetched: columns past the reduction, in its last k-tile, and k-tiles past the last lie beyond
  // the buffers and read zeros (which nobody reads, in the latter), so that the loop has no branch around its products
  // and the same number of DMAs is always on its way.
  uint32_t at = 0;
  auto next = [&](int kt) {
    at = static_cast<uint32_t>(k0 + kt) * 128;
    if (kt == nk - 1 && ragged < BK) {
#pragma unroll
      for (int d = 0; d < 8; ++d) {
        wvo[d] = col[d & 1] < ragged ? wvo[d] : wbytes;
        xvo[d] = col[d & 1] < ragged ? xvo[d] : xbytes;
      }
    }
    wr[2] = __builtin_amdgcn_readfirstlane(kt < nk ? wr[2] : 0u);
    xr[2] = __builtin_amdgcn_readfirstlane(kt < nk ? xr[2] : 0u);
  };
  // Few instructions between two products: the address goes straight into m0.
  auto issue = [&](const u32x4_t& r, int slot, uint32_t vo, auto d_c) {
    const uint32_t st = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(lds0 + slot * UNIT)));
    const uint32_t so = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(at)));
    asm volatile("s_add_u32 m0, %0, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :
                 : "s"(st), "v"(vo), "s"(r), "s"(so), "n"(decltype(d_c)::value * 1024)
                 : "memory", "scc");
  };
  auto issue_w = [&](int slot, auto d_c) { issue(wr, slot, wvo[decltype(d_c)::value], d_c); };
  auto issue_x = [&](int slot, auto d_c) { issue(xr, slot, xvo[decltype(d_c)::value], d_c); };

  // Unit 4 t + quarter of row r16 of a block of 16 rows.
  const int quarter = lane >> 4, r16 = lane & 15;
  int off[2];
#pragma unroll
  for (int t = 0; t < 2; ++t)
    off[t] = (r16 >> 1) * 256 + ((8 * (r16 & 1) + ((4 * t + quarter) ^ (r16 >> 1))) << 4);
  f32x4v_t acc[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = f32x4v_t{0.f, 0.f, 0.f, 0.f};
  vec16 f[2][16];  // half of the k-tile, w's blocks and x's
  // Operand n of a half: w's and x's blocks in turn.
  auto read = [&](int sw, int sx, int t, int n) {
    const int i = n >> 1;
    const char* st = lds + ((n & 1) ? sx * UNIT + wm * 16384 : sw * UNIT + wo * 16384) + off[t] + i * 2048;
    f[t][(n & 1) * 8 + i] = *reinterpret_cast<const vec16*>(st);
  };
  auto fix = [] { __builtin_amdgcn_sched_barrier(0); };
  // Product q of a half, in the order in which their operands come: those of the first r blocks of either are the first
  // r^2.
  auto multiply = [&](int t, auto q_c) {
    constexpr Place p = place_of(decltype(q_c)::value);
    acc[p.i][p.j] = mac16(T{}, f[t][p.i], f[t][8 + p.j], acc[p.i][p.j]);
  };

  const std::make_integer_sequence<int, 8> eight{};
  const std::make_integer_sequence<int, 32> pairs{};

  for (int kt = 0; kt < 2; ++kt) {
    next(kt);
    times(eight, [&](auto d) { issue_w(2 * kt, d); });
    times(eight, [&](auto d) { issue_x(2 * kt + 1, d); });
  }
  CONVSEL_WAIT_VMCNT(16);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int n = 0; n < 16; ++n) read(0, 1, 0, n);
  fix();
  // A CU takes 64 bytes of a DMA a cycle, and a wave that finds it busy stops, its products too: behind every product
  // just one of the four waves issues, so each has code of its own.
  auto walk = [&](auto role_c) {
    int sw = 0;  // the slot of w's unit of k-tile kt; x's is the next one
    for (int kt = 0; kt < nk; ++kt) {
      const int sx = sw == 4 ? 0 : sw + 1, before = sw == 0 ? 4 : sw - 1;
      const int nw = sw >= 3 ? sw - 3 : sw + 2, nx = nw == 4 ? 0 : nw + 1;
      next(kt + 2);
      auto refill = [&](auto q_c) {
        constexpr int q = decltype(q_c)::value, d = q / 4;
        if constexpr (q % 4 == decltype(role_c)::value) {
          if constexpr (d < 8) issue_w(before, std::integral_constant<int, d>{});
          else issue_x(sw, std::integral_constant<int, d - 8>{});
        }
        fix();
      };
      times(pairs, [&](auto q_c) {
        constexpr int q = decltype(q_c)::value;
        multiply(0, std::integral_constant<int, 2 * q>{});
        if constexpr (q < 16) read(sw, sx, 1, q);
        multiply(0, std::integral_constant<int, 2 * q + 1>{});
        fix();
        refill(q_c);
      });
      // All of the k-tile's operands are in registers: behind the barrier its two units may be filled again.
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      times(pairs, [&](auto q_c) {
        constexpr int q = decltype(q_c)::value;
        multiply(1, std::integral_constant<int, 2 * q>{});
        if constexpr (q >= 16) read(nw, nx, 0, q - 16);
        multiply(1, std::integral_constant<int, 2 * q + 1>{});
        fix();
        refill(std::integral_constant<int, 32 + q>{});
        if constexpr (q == 15) {
          // The next k-tile's units are in once no DMAs but those issued after them are on their way: all of w's in
          // this k-tile, and half of x's.
          CONVSEL_WAIT_VMCNT(12);
          __builtin_amdgcn_s_barrier();
          asm volatile("" ::: "memory");
        }
        fix();
      });
      sw = nw;
    }
  };
  switch (wave) {
    case 0: walk(std::integral_constant<int, 0>{}); break;
    case 1: walk(std::integral_constant<int, 1>{}); break;
    case 2: walk(std::integral_constant<int, 2>{}); break;
    default: walk(std::integral_constant<int, 3>{}); break;
  }
  CONVSEL_WAIT_VMCNT(0);  // the zeros behind the last k-tile too
  lds_sync();             // every wave is done with the ring
  const auto put = [&](auto j_c, float* mine) {
    times(std::make_integer_sequence<int, 16>{}, [&](auto n_c) {
      constexpr int i = decltype(n_c)::value / 2, h = decltype(n_c)::value % 2;
      const f32x4v_t& z = acc[i][2 * decltype(j_c)::value + h];
      *reinterpret_cast<float4*>(mine + (16 * h + r16) * S::OUT_ROW + 16 * i + 4 * quarter) =
          make_float4(z[0], z[1], z[2], z[3]);
    });
  };
  store_blocks<T, S>(a, put, lds, wave, lane, m0 + wm * 128, o0 + wo * 128, split);
}
// Sums the parts of a split reduction, in their order, four outputs a thread.
template <typename T>
__global__ __launch_bounds__(256) void linear_join_kernel(TileArgs a) {
  const int64_t quads = (a.g.out + 3) / 4;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= quads * a.g.m) return;
  const int64_t m = i / quads, o = (i - m * quads) * 4;
  float s[1][4] = {}, bias[4];
  load_bias4<T>(a.g, o, bias);
#pragma unroll 4
  for (int p = 0; p < a.splits; ++p) {
    const float4 z = reinterpret_cast<const float4*>(a.part)[p * quads * a.g.m + i];
    s[0][0] += z.x; s[0][1] += z.y; s[0][2] += z.z; s[0][3] += z.w;
  }
  finish4<T, 1>(a.g, m, 0, o, s, bias, a.vec_out);
}

// Rows of x and w, one after the other, copied to rows of whole 16-byte units.
template <typename T>
__global__ __launch_bounds__(256) void linear_pack_kernel(LinearArgs g, T* dst, int64_t padded) {
  constexpr int UE = elem<T>::per16;
  const int64_t per = padded / UE;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < (g.m + g.out) * per;
       i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t row = i / per, k = (i - row * per) * UE;
    const T* src = row < g.m ? reinterpret_cast<const T*>(g.x) + row * g.ldx
                             : reinterpret_cast<const T*>(g.w) + (row - g.m) * g.in;
    uint32_t e[UE];
#pragma unroll
    for (int x = 0; x < UE; ++x) {
      const uint32_t bits = load_bits(src + (k + x < g.in ? k + x : 0));
      e[x] = k + x < g.in ? bits : 0u;
    }
    vec16 v;
    pack16<T>(v, e);
    store16(dst + i * UE, v);
  }
}

// A wave's block is 128 x 64, 64 x 64 and 32 x 32 (outputs x rows).
typedef Tile<2, 2, 2, 2, 2> Tile128;
// Three stages: three workgroups fit on a CU (four stages, two: 700 rows, 4096 -> 4096 in bf16, 55 us, not 48).
typedef Tile<1, 1, 2, 2, 3> Tile64;
constexpr int kSide[3] = {256, 128, 64};

template <typename T, typename S>
hipError_t launch(const TileArgs& a, hipStream_t st) {
  const int units = a.to * a.tm * a.splits;
  hipLaunchKernelGGL((linear_tiles_kernel<T, S>), dim3((unsigned)(8 * ((units + 7) / 8))), dim3(S::WAVES * 64), 0, st,
                     a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_all(const LinearArgs& a0, const LinearTiles& p, void* workspace, hipStream_t st) {
  TileArgs a;
  a.g = a0;
  char* ws = (char*)workspace;
  if (p.pack) {
    const int64_t per = elem<T>::per16, padded = (a0.in + per - 1) / per * per;
    const int64_t units = (a0.m + a0.out) * (padded / per);
    const int64_t blocks = (units + 255) / 256;
    hipLaunchKernelGGL(linear_pack_kernel<T>, dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, st, a0,
                       (T*)ws, padded);
    a.g.x = ws;
    a.g.w = ws + a0.m * padded * sizeof(T);
    a.g.in = a.g.ldx = padded;
    ws += p.pack_bytes;
  }
  const int side = kSide[p.config];
  a.to = (int)((a0.out + side - 1) / side);
  a.tm = (int)((a0.m + side - 1) / side);
  const int64_t bk = 128 / sizeof(T), all = (a.g.in + bk - 1) / bk;
  a.splits = p.splits;
  a.per = (int)((all + p.splits - 1) / p.splits);
  a.part = (float*)ws;
  const uintptr_t unit = 4 * sizeof(T);
  a.vec_out = a0.ldy % 4 == 0 && (uintptr_t)a0.y % unit == 0 &&
              (!a0.r || (a0.ldr % 4 == 0 && (uintptr_t)a0.r % unit == 0));
  hipError_t e = hipSuccess;
  if (p.config == 0) {
    if constexpr (sizeof(T) == 4) {
      e = launch<T, Tile256>(a, st);
    } else {
      const int units = a.to * a.tm * a.splits;
      hipLaunchKernelGGL(linear_tiles256_kernel, dim3((unsigned)(8 * ((units + 7) / 8))), dim3(256), 0, st, a);
      e = hipGetLastError();
    }
  } else {
    e = p.config == 1 ? launch<T, Tile128>(a, st) : launch<T, Tile64>(a, st);
  }
  if (e != hipSuccess || p.splits == 1) return e;
  const int64_t quads = (a0.out + 3) / 4 * a0.m;
  hipLaunchKernelGGL(linear_join_kernel<T>, dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

// A launch's limit; the grid is rounded up to 8 workgroups.
constexpr int64_t kThreadsMax = ((int64_t)1 << 32) - 8 * 256;

LinearTiles linear_tiles_plan(const LinearArgs& a) {
  const int64_t es = a.dtype == CONV_F32 ? 4 : 2, per = 16 / es;
  LinearTiles p;
  // By sizes alone: the workspace is asked for before the addresses are known.
  p.pack = a.in % per != 0 || a.ldx % per != 0;
  const int64_t padded = (a.in + per - 1) / per * per;
  p.pack_bytes = p.pack ? align256((size_t)(a.m + a.out) * padded * es) : 0;
  p.part_bytes = 0;
  p.config = 0;
  p.splits = 1;
  // A tile's rows are addressed in 32 bits from its first one.
  const int64_t ld = p.pack || a.in > a.ldx ? padded : a.ldx;
  if (ld * es >= ((int64_t)1 << 31) / 256 || (!p.pack && ((uintptr_t)a.x % 16 != 0 || (uintptr_t)a.w % 16 != 0))) {
    p.config = -1;
    p.us = 0.;
    return p;
  }
  auto tiles = [&](int c) { return ((a.out + kSide[c] - 1) / kSide[c]) * ((a.m + kSide[c] - 1) / kSide[c]); };
  const int64_t all = (a.in + 128 / es - 1) / (128 / es);
  // The tile and the parts that take the least time by what was measured, in us.  A k-tile takes a CU with one workgroup
  // `one`, and with k of them k * `each`, or `one` for the last of an odd number of 128s, which two share a CU; tiles of
  // 256, one a CU, add `alone` for their first loads and last stores.  Joining parts adds 2.5 and their way through the
  // caches at 8 TB/s.  At 4096 -> 4096 in bf16: 4096 rows 125 us in 256s, 171 in 128s, 271 in 64s; 2048 rows 81 (2
  // parts), 80, 138; 700 rows 46 (5), 56 (4), 48; 256 rows 32 (11), 27 (4), 25 (2).
  static const double kOne[2][3] = {{8.3, 2.35, 0.7}, {1.67, 0.83, 0.36}};
  static const double kEach[2][3] = {{8.3, 2.15, 0.61}, {1.67, 0.61, 0.25}};
  static const double kAlone[3] = {6., 0., 0.};
  const int ty = a.dtype == CONV_F32 ? 0 : 1;
  double best = 0.;
  for (int c = 0; c < 3; ++c) {
    const int64_t n = tiles(c);
    for (int64_t s = 1; s <= 16; ++s) {
      if (s > 1 && (s > all / 4 || n * s > 2048)) break;
      if (n * 256 > kThreadsMax) break;  // 2^30 rows of few outputs: tiles of 256 hold 2^31 of them
      const int64_t per_part = (all + s - 1) / s, parts = (all + per_part - 1) / per_part;
      if (parts != s) continue;
      const int64_t k = (n * s + 255) / 256;
      double step = k * kEach[ty][c];
      if (k == 1 || (c == 1 && k % 2)) step += kOne[ty][c] - kEach[ty][c];
      double t = per_part * step + k * kAlone[c];
      if (s > 1) t += 2.5 + (double)s * a.m * a.out * 8 / 8e6;
      if ((c == 0 && s == 1) || t < best) {
        best = t;
        p.config = c;
        p.splits = (int)s;
      }
    }
  }
  // Copying both operands first: a launch, and their way there and back.
  p.us = best + (p.pack ? 2.5 + (double)(a.m + a.out) * a.in * es * 2 / 4e6 : 0.);
  if (p.splits > 1) p.part_bytes = (size_t)p.splits * a.m * ((a.out + 3) / 4 * 4) * 4;
  return p;
}

hipError_t launch_linear_tiles(const LinearArgs& a, const LinearTiles& p, void* workspace, hipStream_t stream) {
  return a.dtype == CONV_F32 ? launch_all<float>(a, p, workspace, stream)
                             : launch_all<bf16_t>(a, p, workspace, stream);
}

const char* linear_tiles_name(int config) {
  static const char* const names[3] = {"256x256", "128x128", "64x64"};
  return names[config];
}

}  // namespace convsel
