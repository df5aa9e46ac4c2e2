// Linear layers in tiles: both operands through LDS DMA.
//
// A workgroup owns TM rows of x and TO outputs and walks the reduction in
// k-tiles of 64 bytes (32 bf16, 16 fp32).  A k-tile of 16 operand rows is 1 KiB
// of LDS, one DMA instruction: its 16-byte units lie unit by unit, 16 rows of
// each in a row, so the 16 rows that a quarter wave reads of one unit are 256
// consecutive bytes.  Rows past the operand and columns past the reduction read
// zeros through the buffer's range.  Four stages form a ring with three k-tiles
// on their way.  A wave multiplies FO x FM blocks of 32 x 32; the operands of a
// k-tile's second half are read while its first half multiplies, and the next
// k-tile's first half (behind the tile's one barrier) while the second does.
//
// The products' rows are w's and their columns x's.  Sums leave through LDS,
// each wave in a place of its own, so that every row of y is read (residual)
// and written along its outputs.
#include <stdio.h>
#include <stdlib.h>

#include <type_traits>

#include "igemm_common.hpp"
#include "linear_common.hpp"

namespace convsel {
namespace {

using namespace igemm;
using namespace lm;

constexpr int kStages = 4;

template <int FO_, int FM_, int WO_, int WM_>
struct Tile {
  static constexpr int FO = FO_, FM = FM_, WO = WO_, WM = WM_;
  static constexpr int TO = FO * 32 * WO, TM = FM * 32 * WM, WAVES = WO * WM;
  static constexpr int STAGE = (TO + TM) * 64;
  static constexpr int NDMA = (TO + TM) / 16 / WAVES;  // DMA instructions of a wave and stage
  static constexpr int OUT_ROW = FO * 32 + 4;          // floats: rows 16 bytes apart in the banks
  static constexpr int OUT = WAVES * 32 * OUT_ROW * 4;
  static constexpr int LDS = kStages * STAGE > OUT ? kStages * STAGE : OUT;
  static_assert((TO + TM) % (16 * WAVES) == 0 && LDS <= 160 * 1024 && NDMA * (kStages - 1) <= 63, "tile");
};

struct TileArgs {
  LinearArgs g;
  int to, tm;          // tiles of outputs and of rows
  int splits, per;     // k-tiles of a part
  int vec_out;
  float* part;         // [split][m][out rounded up to 4]
};

template <typename T, typename S>
__global__ __launch_bounds__(S::WAVES * 64, S::WAVES == 8 ? 2 : 1) void linear_tiles_kernel(TileArgs a) {
  constexpr int FO = S::FO, FM = S::FM, NDMA = S::NDMA, STAGE = S::STAGE;
  constexpr int ES = elem<T>::bytes, UE = elem<T>::per16, BK = 64 / ES;
  __shared__ __align__(16) char lds[S::LDS];
  const LinearArgs& g = a.g;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wo = wave % S::WO, wm = wave / S::WO;
  // Workgroup w runs on XCD w % 8: each XCD has a contiguous run of tiles, eight rows of tiles deep before the next
  // outputs, so that the workgroups of one L2 share both operands.
  const int units = a.to * a.tm * a.splits;
  const int per_xcd = (units + 7) >> 3;
  const int unit = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= per_xcd || unit >= units) return;  // uniform
  const int split = unit % a.splits, tile = unit / a.splits;
  const int band = tile / (8 * a.to), in_band = tile - band * 8 * a.to;
  const int deep = min(8, a.tm - band * 8);
  const int64_t m0 = static_cast<int64_t>(band * 8 + in_band % deep) * S::TM;
  const int64_t o0 = static_cast<int64_t>(in_band / deep) * S::TO;

  const int64_t wrows = min(g.out - o0, static_cast<int64_t>(S::TO)), xrows = min(g.m - m0, static_cast<int64_t>(S::TM));
  const uint32_t wbytes = static_cast<uint32_t>(((wrows - 1) * g.in + g.in) * ES);
  const uint32_t xbytes = static_cast<uint32_t>(((xrows - 1) * g.ldx + g.in) * ES);
  const u32x4_t wr = dma_rsrc(reinterpret_cast<const T*>(g.w) + o0 * g.in, wbytes);
  const u32x4_t xr = dma_rsrc(reinterpret_cast<const T*>(g.x) + m0 * g.ldx, xbytes);
  const uint32_t lds0 = lds_address(lds);

  // Instruction J = wave * NDMA + d of a stage fills rows 16 J .. 16 J + 15: w's rows first, then x's.
  uint32_t dvo[NDMA];
  const int dku = (lane >> 4) * UE;  // this lane's column within a k-tile
#pragma unroll
  for (int d = 0; d < NDMA; ++d) {
    const int row = (wave * NDMA + d) * 16 + (lane & 15);
    const bool isw = row < S::TO;
    const int64_t r = isw ? row : row - S::TO;
    const bool ok = r < (isw ? wrows : xrows);
    dvo[d] = ok ? static_cast<uint32_t>((r * (isw ? g.in : g.ldx) + dku) * ES) : (isw ? wbytes : xbytes);
  }
  const int k0 = split * a.per, all = static_cast<int>((g.in + BK - 1) / BK);
  const int nk = min(all, k0 + a.per) - k0;
  auto issue = [&](int kt) {
    const uint32_t st = lds0 + (kt % kStages) * STAGE;
    const uint32_t so = static_cast<uint32_t>(k0 + kt) * 64;
    const bool past = static_cast<int64_t>(k0 + kt) * BK + dku >= g.in;
#pragma unroll
    for (int d = 0; d < NDMA; ++d) {
      const int J = wave * NDMA + d;
      const bool isw = J < S::TO / 16;
      dma16(isw ? wr : xr, st + J * 1024, past ? (isw ? wbytes : xbytes) : dvo[d], so);
    }
  };

  const int half = lane >> 5, l32 = lane & 31;
  // Unit 2 t + half of row r of a stage.
  auto place = [&](int r, int t) { return (r >> 4) * 1024 + (2 * t + half) * 256 + (r & 15) * 16; };
  int woff[FO], xoff[FM];
#pragma unroll
  for (int i = 0; i < FO; ++i) woff[i] = place((wo * FO + i) * 32 + l32, 0);
#pragma unroll
  for (int i = 0; i < FM; ++i) xoff[i] = place(S::TO + (wm * FM + i) * 32 + l32, 0);

  f32x16_t acc[FO][FM];
#pragma unroll
  for (int i = 0; i < FO; ++i)
#pragma unroll
    for (int j = 0; j < FM; ++j) acc[i][j] = zero16();
  vec16 fw[2][FO], fx[2][FM];
  auto read = [&](int kt, auto t_c) {
    constexpr int t = decltype(t_c)::value;
    const char* st = lds + (kt % kStages) * STAGE + t * 512;
#pragma unroll
    for (int i = 0; i < FO; ++i) fw[t][i] = *reinterpret_cast<const vec16*>(st + woff[i]);
#pragma unroll
    for (int i = 0; i < FM; ++i) fx[t][i] = *reinterpret_cast<const vec16*>(st + xoff[i]);
    __builtin_amdgcn_sched_barrier(0);
  };
  auto multiply = [&](auto t_c) {
    constexpr int t = decltype(t_c)::value;
#pragma unroll
    for (int i = 0; i < FO; ++i)
#pragma unroll
      for (int j = 0; j < FM; ++j) mfma_32x32<T>(acc[i][j], fw[t][i], fx[t][j]);
    __builtin_amdgcn_sched_barrier(0);
  };
  // Stage kt is in once no DMAs but those of later stages are pending: two of them at the start, one from then on
  // (the third is issued behind the barrier).  Behind it every wave is also done with stage kt - 2.
  auto arrive = [&](int kt) {
    const int later = min(nk - 1, kt == 0 ? kStages - 2 : kt + 1) - kt;
    if (later >= 2) CONVSEL_WAIT_VMCNT(2 * NDMA);
    else if (later == 1) CONVSEL_WAIT_VMCNT(NDMA);
    else CONVSEL_WAIT_VMCNT(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  const std::integral_constant<int, 0> first{};
  const std::integral_constant<int, 1> second{};
#pragma unroll
  for (int p = 0; p < kStages - 1; ++p)
    if (p < nk) issue(p);
  arrive(0);
  read(0, first);
  for (int kt = 0; kt < nk; ++kt) {
    read(kt, second);
    multiply(first);
    if (kt + 1 < nk) {
      arrive(kt + 1);
      if (kt + kStages - 1 < nk) issue(kt + kStages - 1);
      read(kt + 1, first);
    }
    multiply(second);
  }

  lds_sync();  // every wave is done with the stages
  float* mine = reinterpret_cast<float*>(lds) + wave * 32 * S::OUT_ROW;
  const int64_t opad = (g.out + 3) & ~static_cast<int64_t>(3);
#pragma unroll
  for (int j = 0; j < FM; ++j) {
#pragma unroll
    for (int i = 0; i < FO; ++i)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        *reinterpret_cast<float4*>(mine + l32 * S::OUT_ROW + 32 * i + 8 * v + 4 * half) =
            make_float4(acc[i][j][4 * v], acc[i][j][4 * v + 1], acc[i][j][4 * v + 2], acc[i][j][4 * v + 3]);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    constexpr int PER = FO * 8;  // units of four of a row
#pragma unroll 4
    for (int u = lane; u < 32 * PER; u += 64) {
      const int r = u / PER, c = u % PER;
      const int64_t m = m0 + (wm * FM + j) * 32 + r, o = o0 + wo * FO * 32 + 4 * c;
      const float4 z = *reinterpret_cast<const float4*>(mine + r * S::OUT_ROW + 4 * c);
      if (m >= g.m || o >= g.out) continue;
      if (a.splits > 1) {
        *reinterpret_cast<float4*>(a.part + (split * g.m + m) * opad + o) = z;
      } else {
        const float s[4] = {z.x, z.y, z.z, z.w};
        finish4<T>(g, m, o, s, a.vec_out);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
  }
}

// Sums the parts of a split reduction, in their order, four outputs a thread.
template <typename T>
__global__ __launch_bounds__(256) void linear_join_kernel(TileArgs a) {
  const int64_t quads = (a.g.out + 3) / 4;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= quads * a.g.m) return;
  const int64_t m = i / quads, o = (i - m * quads) * 4;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int p = 0; p < a.splits; ++p) {
    const float4 z = reinterpret_cast<const float4*>(a.part)[p * quads * a.g.m + i];
    s[0] += z.x; s[1] += z.y; s[2] += z.z; s[3] += z.w;
  }
  finish4<T>(a.g, m, o, s, a.vec_out);
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

typedef Tile<4, 2, 2, 4> Tile256;
typedef Tile<2, 2, 2, 2> Tile128;
typedef Tile<1, 1, 2, 2> Tile64;
constexpr int kTileSide[3] = {256, 128, 64};

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
  const int side = kTileSide[p.config];
  a.to = (int)((a0.out + side - 1) / side);
  a.tm = (int)((a0.m + side - 1) / side);
  const int64_t bk = 64 / sizeof(T), all = (a.g.in + bk - 1) / bk;
  a.splits = p.splits;
  a.per = (int)((all + p.splits - 1) / p.splits);
  a.part = (float*)ws;
  const uintptr_t unit = 4 * sizeof(T);
  a.vec_out = a0.ldy % 4 == 0 && (uintptr_t)a0.y % unit == 0 &&
              (!a0.r || (a0.ldr % 4 == 0 && (uintptr_t)a0.r % unit == 0));
  hipError_t e = hipSuccess;
  if (p.config == 0) e = launch<T, Tile256>(a, st);
  else if (p.config == 1) e = launch<T, Tile128>(a, st);
  else e = launch<T, Tile64>(a, st);
  if (e != hipSuccess || p.splits == 1) return e;
  const int64_t quads = (a0.out + 3) / 4 * a0.m;
  hipLaunchKernelGGL(linear_join_kernel<T>, dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

LinearTiles linear_tiles_plan(const LinearArgs& a) {
  const int64_t es = a.dtype == CONV_F32 ? 4 : 2, per = 16 / es;
  LinearTiles p;
  // By sizes alone: the workspace is asked for before the addresses are known.
  p.pack = a.in % per != 0 || a.ldx % per != 0;
  const int64_t padded = (a.in + per - 1) / per * per;
  p.pack_bytes = p.pack ? align256((size_t)(a.m + a.out) * padded * es) : 0;
  p.part_bytes = 0;
  p.splits = 1;
  // A tile's rows are addressed in 32 bits from its first one.
  const int64_t ld = p.pack || a.in > a.ldx ? padded : a.ldx;
  if (ld * es >= ((int64_t)1 << 31) / 256 || (!p.pack && ((uintptr_t)a.x % 16 != 0 || (uintptr_t)a.w % 16 != 0))) {
    p.config = -1;
    return p;
  }
  auto tiles = [&](int side) { return ((a.out + side - 1) / side) * ((a.m + side - 1) / side); };
  const int64_t all = (a.in + 64 / es - 1) / (64 / es);
  const char* force = getenv("LCFG");
  if (force) { p.config = atoi(force); } else {
  p.config = tiles(256) >= 256 ? 0 : tiles(128) >= 256 ? 1 : 2; }
  const int64_t n = tiles(kTileSide[p.config]);
  int64_t want = getenv("LWANT") ? atoi(getenv("LWANT")) : 512;
  int64_t s = want / n;
  int64_t least = getenv("LLEAST") ? atoi(getenv("LLEAST")) : 16;
  if (s > all / least) s = all / least;
  if (s > 16) s = 16;
  if (s < 1) s = 1;
  if (n * s >= ((int64_t)1 << 22)) { /* grids stay in range: one part */ s = 1; }
  p.splits = (int)((all + (all + s - 1) / s - 1) / ((all + s - 1) / s));
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
