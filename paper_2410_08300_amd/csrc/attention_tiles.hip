// Attention over the 8-bit paged cache for many query rows.
//
// One workgroup of W = 4 or 8 waves per 32 W rows of a key head (a row is a query
// of the sequence and one of the heads that share the key head), 32 rows a wave.
// Keys pass in tiles of W 16-token blocks: wave w loads block w's codes one tile
// ahead, widens them to 16-bit floats once for all rows, and stores them in LDS
// in the order in which lanes read them back: every read of an operand is 1 KiB
// in a row.  Two tiles fit in LDS, so there is one barrier a tile; up to head
// widths of 128 in bf16 a CU has eight waves, of two workgroups or one.
//
// Scores are K q^T in 32 x 32 x 16 products: a lane ends with 16 tokens of one
// query, in runs of four as the cache's blocks hold them, and feeds its weights
// to the second product, V^T P^T, without moving them.  A row's statistics need
// one exchange, with the lane that holds the other tokens.
//
// What bounds it: the vector unit and the matrix cores in turn, with the waits
// between.  A weight costs a fused product, a transcendental (four slots), an
// addition to the sum, a product with its scale, a conversion to each of two
// halves with a subtraction between, and half a maximum; 16 of them a lane and 32 keys stand beside 24
// products of 32 cycles each.  4096 new tokens of 32 heads of 128 on 8, causal,
// int8: 249 us, 550 TFLOP/s, the vector unit 53 % busy and the matrix cores 32 %,
// where the products alone would take 90 us, with each weight in one number, at
// the rate of a large product.
#include "attention_common.hpp"
#include "lm_common.hpp"

namespace convsel {
namespace {

using namespace lm;

constexpr float kInf = __builtin_inff();

__device__ __forceinline__ f32x16_t mfma32(const f16x8_t& a, const f16x8_t& b, const f32x16_t& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// What a tile's block of 16 tokens comes with.  (With the value scale's mantissa
// as a summand of the weights' exponent they would take an operation less, 4096
// tokens 4 % less time, but be off by up to 2^-20 between blocks, and a scale of
// zero has no such summand.)
struct BlockMeta {
  float ks;     // key scale, -1 where there is no page
  float ve;     // exponent of the value scale
  float scale;  // 2^15 times its mantissa
};

__device__ __forceinline__ float uniform(float v) {
  return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v)));
}

// Runs use(i, operand) for N operands that load(i) reads from LDS, four reads
// ahead of the four in use.  The barriers keep the compiler, which would rather
// read one operand at a time into the same registers, to that order.
constexpr int kAhead = 4;

template <int N, typename Load>
__device__ __forceinline__ void read_group(f16x8_t* buf, int g, const Load& load) {
#pragma unroll
  for (int i = 0; i < kAhead; ++i)
    if (g * kAhead + i < N) buf[i] = load(g * kAhead + i);
  __builtin_amdgcn_sched_barrier(0);
}

template <int N, typename Load, typename Use>
__device__ __forceinline__ void use_groups(f16x8_t (&first)[kAhead], const Load& load, const Use& use) {
  constexpr int G = (N + kAhead - 1) / kAhead;
  f16x8_t second[kAhead];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    f16x8_t* cur = g & 1 ? second : first;
    if (g + 1 < G) read_group<N>(g & 1 ? first : second, g + 1, load);
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (g * kAhead + i < N) use(g * kAhead + i, cur[i]);
    __builtin_amdgcn_sched_barrier(0);
  }
}

template <typename T, int FMT, int NC, int W>
__global__ __launch_bounds__(64 * W, (NC <= 4 && sizeof(T) == 2) ? 2 : 1) void attention_tiles_kernel(
    const T* __restrict__ q, const uint8_t* __restrict__ kc, const uint8_t* __restrict__ vc,
    const float* __restrict__ ks, const float* __restrict__ vs, const int32_t* __restrict__ table,
    const int32_t* __restrict__ lengths, const int32_t* __restrict__ offsets, T* __restrict__ y,
    float* __restrict__ part, float* __restrict__ stat, AttnArgs a) {
  constexpr bool TWO = sizeof(T) == 4;
  constexpr int DP = 32 * NC, QC = 2 * NC;  // row bytes, 16-column chunks
  constexpr int ROWS = 32 * W;  // a wave has 32 query rows and stages one block of keys
  constexpr int KB = W / 2 * QC * 1024, VB = W * NC * 1024;  // bytes of a tile's keys and values in LDS
  __shared__ __align__(16) char lds[2 * (KB + VB)];
  char(*const kt_lds)[KB] = reinterpret_cast<char(*)[KB]>(lds);
  char(*const vt_lds)[VB] = reinterpret_cast<char(*)[VB]>(lds + 2 * KB);
  __shared__ BlockMeta meta[2][W];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  // Heads vary fastest: with eight of them, one head's keys stay in one XCD's L2.
  const int head = blockIdx.x % a.kv_heads, split = blockIdx.x / a.kv_heads;
  const Unit un = find_unit<true>(a.units, offsets, lengths);
  const Span sp = un.span;
  const int rows = sp.count * a.group;
  const int64_t len = un.length;
  const int limit = static_cast<int>(max((int64_t)0, min(len, a.table_width << a.ps_shift)));
  const int64_t first = len - sp.count;  // position of the sequence's first query
  const int32_t* my_table = table + un.seq * a.table_width;
  const int ntile = (rows + ROWS - 1) / ROWS;

  for (int nt = un.index; nt < ntile; nt += un.count) {
    const int tile = ntile - 1 - nt;  // under a causal mask the last rows have the most keys: they start first
    const int r0 = tile * ROWS;
    // Keys that tokens t0..t1 see between them, and that every one of them sees.
    auto seen_by = [&](int t0, int t1, int& lo, int& hi, int& in_lo, int& in_hi) {
      lo = 0; hi = limit; in_lo = 0; in_hi = limit;
      if (a.causal) {
        hi = static_cast<int>(max((int64_t)0, min((int64_t)limit, first + t1 + 1)));
        in_hi = static_cast<int>(max((int64_t)0, min((int64_t)limit, first + t0 + 1)));
      }
      if (a.window > 0) {
        lo = static_cast<int>(max((int64_t)0, min((int64_t)limit, first + t0 - a.window + 1)));
        in_lo = static_cast<int>(max((int64_t)0, min((int64_t)limit, first + t1 - a.window + 1)));
      }
    };
    int lo, hi, in_lo, in_hi;
    seen_by(r0 / a.group, min(r0 + ROWS - 1, rows - 1) / a.group, lo, hi, in_lo, in_hi);
    const int b0 = lo >> 4, b1 = hi > lo ? (hi + 15) >> 4 : b0;
    const int steps = (b1 - b0 + W - 1) / W;
    const int per = (steps + a.nsplit - 1) / a.nsplit;
    const int k0 = split * per, k1 = min(steps, k0 + per);
    // This wave's rows and this lane's.
    const int w0 = min(r0 + wave * 32, rows - 1), w1 = min(r0 + wave * 32 + 31, rows - 1);
    int wlo, whi;
    seen_by(w0 / a.group, w1 / a.group, wlo, whi, in_lo, in_hi);
    const bool idle = r0 + wave * 32 >= rows;
    const int row = min(r0 + wave * 32 + col, rows - 1);
    const int tok = row / a.group, hq = head * a.group + row % a.group;
    const int64_t p = first + tok;
    const int row_hi = a.causal ? static_cast<int>(max((int64_t)0, min((int64_t)limit, p + 1))) : limit;
    const int row_lo = a.window > 0 ? static_cast<int>(max((int64_t)0, min((int64_t)limit, p - a.window + 1))) : 0;

    // ---- staging: this wave's block of the next tile ----
    uint2 kr[NC], vr[NC];
    float ksr = 0.f, vsr = 1.f;
    int pg = -1, blk = 0;
    // The page of a tile's block is looked up a tile before its codes are.
    auto look = [&](int kt) {
      const int b = b0 + W * kt + wave;
      return b < b1 ? my_table[b >> (a.ps_shift - 4)] : -1;
    };
    int entry = -1;
    auto fetch = [&](int kt) {
      blk = b0 + W * kt + wave;
      pg = entry >= 0 && entry < a.pages ? entry : -1;
      const int64_t ph = static_cast<int64_t>(pg < 0 ? 0 : pg) * a.kv_heads + head;
      const int t0 = (blk & ((1 << (a.ps_shift - 4)) - 1)) << 4;
      const int64_t at = ((ph << a.ps_shift) + t0) * DP;
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        kr[j] = *reinterpret_cast<const uint2*>(kc + at + (lane + 64 * j) * 8);
        vr[j] = *reinterpret_cast<const uint2*>(vc + at + (lane + 64 * j) * 8);
      }
      ksr = ks[ph];
      vsr = vs[ph];
      entry = look(kt + 1);
    };
    auto stash = [&](int buf) {
      // Keys: unit e of a token's row holds columns 8 e .. 8 e + 7, chunk e / 2, half e % 2.  Slots are permuted
      // within eights so that one token's units fall on different banks.
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const int i = lane + 64 * j, token = i / (4 * NC), e = i % (4 * NC);
        const int slot = ((e & 1) * 32 + (wave & 1) * 16 + token) ^ (e & 7);
        *reinterpret_cast<f16x8_t*>(&kt_lds[buf][(((wave >> 1) * QC + (e >> 1)) * 64 + slot) * 16]) =
            widen8<FMT>(kr[j].x, kr[j].y);
      }
      // Values: a unit is four tokens of two columns 16 apart; rows never written are silenced.
      if (pg < 0 || blk * 16 + 16 > limit) {
#pragma unroll
        for (int j = 0; j < NC; ++j) {
          const int g = (lane + 64 * j) / NC >> 4;
          const int n = pg < 0 ? 0 : clampi(limit - blk * 16 - 4 * g, 0, 4);
          const uint32_t keep = n >= 4 ? 0xffffffffu : (1u << (8 * n)) - 1u;
          vr[j].x &= keep;
          vr[j].y &= keep;
        }
      }
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const int i = lane + 64 * j, L = i / NC, d32 = i % NC, g = L >> 4, dl = L & 15;
        const f16x8_t w = widen8<FMT>(vr[j].x, vr[j].y);
        char* at = &vt_lds[buf][((wave * NC + d32) * 64 + (g & 1) * 32 + dl) * 16 + (g >> 1) * 8];
        uint4 u;
        __builtin_memcpy(&u, &w, 16);
        *reinterpret_cast<uint2*>(at) = make_uint2(u.x, u.y);
        *reinterpret_cast<uint2*>(at + 256) = make_uint2(u.z, u.w);
      }
      if (lane == 0) {
        int e;
        const float f = split_scale(pg < 0 ? 1.f : vsr, e);
        BlockMeta m;
        m.ks = pg < 0 ? -1.f : ksr;
        m.ve = e;
        m.scale = kWeight * f;
        meta[buf][wave] = m;
      }
    };

    if (k0 < k1) {
      entry = look(k0);
      fetch(k0);
    }

    // ---- the queries: lane (row, half) holds columns 16 c + 8 half + 0..7 ----
    f16x8_t qh[QC], ql[TWO ? QC : 1];
    float cs;
    {
      const T* src = q + (sp.first + tok) * a.q_token + static_cast<int64_t>(hq) * a.q_head + 8 * half;
      constexpr int UE = elem<T>::per16, UC = 8 / UE;  // 16-byte units of a chunk
      vec16 raw[QC * UC];
      float amax = 0.f;
      if (a.q_vec) {
#pragma unroll
        for (int u = 0; u < QC * UC; ++u) raw[u] = load16(src + 16 * (u / UC) + UE * (u % UC));
      } else {
        // Element by element, a unit at a time through this lane's own places in LDS: unrolled, the bounds and
        // addresses of so many loads would not fit in registers.
        vec16* mine = reinterpret_cast<vec16*>(lds) + wave * (QC * UC * 64) + lane;
#pragma unroll 1
        for (int u = 0; u < QC * UC; ++u) {
          uint32_t e[UE];
          vec16 v;
#pragma unroll
          for (int x = 0; x < UE; ++x) {
            const int d = 16 * (u / UC) + UE * (u % UC) + x;
            const uint32_t bits = load_bits(src + min(d, a.dim - 1 - 8 * half));  // within the row
            e[x] = d + 8 * half < a.dim ? bits : 0u;
          }
          pack16<T>(v, e);
          mine[u * 64] = v;
        }
#pragma unroll
        for (int u = 0; u < QC * UC; ++u) raw[u] = mine[u * 64];
        lds_sync();  // before a wave stores codes there
      }
#pragma unroll
      for (int u = 0; u < QC * UC; ++u)
#pragma unroll
        for (int x = 0; x < UE; ++x) amax = fmaxf(amax, fabsf(elem<T>::to_f32(vec16_get<T>(raw[u], x))));
      amax = fmaxf(amax, __shfl_xor(amax, 32));
      const int e = query_exponent(amax);
      cs = ldexpf(fabsf(a.scale), e);
#pragma unroll
      for (int c = 0; c < QC; ++c) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          // The sign of the scale goes with the query: scores then grow with the products.
          const float z = elem<T>::to_f32(vec16_get<T>(raw[c * UC + j / UE], j % UE));
          const float v = ldexpf(a.scale < 0.f ? -z : z, -e);
          qh[c][j] = static_cast<_Float16>(v);
          if constexpr (TWO) ql[c][j] = static_cast<_Float16>(v - static_cast<float>(qh[c][j]));
        }
      }
    }

    f32x16_t o[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) o[i] = zero16();
    float m = -kInf, l = 0.f;

    // 32 of the tile's tokens, from position j1 on: their scores and weights fit beside the results without spilling.
    auto compute = [&](int buf, int tt, int j1, bool masked) {
      BlockMeta bm[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const BlockMeta& mb = meta[buf][2 * tt + b];
        bm[b].ks = uniform(mb.ks); bm[b].ve = uniform(mb.ve); bm[b].scale = uniform(mb.scale);
      }
      f32x16_t sc = zero16();
      f16x8_t frag[kAhead];
      const auto key = [&](int c) {
        const int slot = lane ^ ((2 * c + half) & 7);
        return *reinterpret_cast<const f16x8_t*>(&kt_lds[buf][((tt * QC + c) * 64 + slot) * 16]);
      };
      read_group<QC>(frag, 0, key);
      use_groups<QC>(frag, key, [&](int c, const f16x8_t& kf) {
        sc = mfma32(kf, qh[c], sc);
        if constexpr (TWO) sc = mfma32(kf, ql[c], sc);
      });
      const auto value = [&](int i) {  // operand i: block i / NC, columns 32 (i % NC) ..
        return *reinterpret_cast<const f16x8_t*>(&vt_lds[buf][((2 * tt * NC + i) * 64 + lane) * 16]);
      };
      read_group<2 * NC>(frag, 0, value);  // they arrive while the weights are formed
      // Never zero: a masked score of -inf times it stays -inf (and what it rounds off of a score is nothing).
      const float f[2] = {fmaxf(bm[0].ks * cs, 0x1p-126f), fmaxf(bm[1].ks * cs, 0x1p-126f)};
      if (masked) {
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int j = j1 + 8 * (v >> 2) + 4 * half + (v & 3);
          if (!(bm[v >> 3].ks >= 0.f && j >= row_lo && j < row_hi)) sc[v] = -kInf;
        }
      }
      float top[2], most = -kInf;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        float t = -kInf;
#pragma unroll
        for (int x = 0; x < 8; ++x) t = fmaxf(t, sc[b * 8 + x]);
        top[b] = t * f[b];
        most = fmaxf(most, ceilf(top[b]) + bm[b].ve);
      }
      most = fmaxf(most, __shfl_xor(most, 32));
      if (__any(most > m)) {
        const float mn = fmaxf(m, most);
        const int dm = shift_of(m, mn);
        m = mn;
        l = ldexpf(l, dm);
        const float s = ldexpf(1.f, dm);
#pragma unroll
        for (int i = 0; i < NC; ++i) o[i] *= s;
      }
      f16x8_t wh[2], wl[2];
      float add = 0.f;
      bool far = false;
      const float from = m == -kInf ? 0.f : m;  // a row with nothing yet: its weights are 2^-inf
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const float up = bm[b].ve - from;
        float sum = 0.f;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          float w = __builtin_amdgcn_exp2f(fmaf(sc[b * 8 + x], f[b], up));
          sum += w;
          w *= bm[b].scale;
          asm volatile("" : "+v"(w));  // one rounded weight for both halves
          wh[b][x] = static_cast<_Float16>(w);
          wl[b][x] = static_cast<_Float16>(w - static_cast<float>(wh[b][x]));
        }
        far |= top[b] + up < kFar && top[b] > -kInf;
        add += ldexpf(sum, -static_cast<int>(bm[b].ve));
      }
      if (__any(far)) {
        add = 0.f;
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const float z = sc[x] * f[x >> 3], n = rintf(z);
          const float u = ldexpf(__builtin_amdgcn_exp2f(z - n), static_cast<int>(fmaxf(n - m, -300.f)));
          add += sc[x] == -kInf ? 0.f : u;
        }
      }
      l += add;
      use_groups<2 * NC>(frag, value, [&](int i, const f16x8_t& vf) {
        o[i % NC] = mfma32(vf, wh[i / NC], o[i % NC]);
        o[i % NC] = mfma32(vf, wl[i / NC], o[i % NC]);
      });
    };

    if (k0 < k1) {
      stash(0);
      lds_sync();
      for (int kt = k0; kt < k1; ++kt) {
        const int buf = (kt - k0) & 1;
        if (kt + 1 < k1) fetch(kt + 1);
        const int j0 = (b0 + W * kt) * 16;
        if (!idle) {
#pragma unroll 1
          for (int tt = 0; tt < W / 2; ++tt) {
            const int j1 = j0 + 32 * tt;
            if (j1 >= whi || j1 + 32 <= wlo) continue;
            const float worst = fminf(meta[buf][2 * tt].ks, meta[buf][2 * tt + 1].ks);
            compute(buf, tt, j1, !(uniform(worst) >= 0.f && j1 >= in_lo && j1 + 32 <= in_hi));
          }
        }
        if (kt + 1 < k1) stash(buf ^ 1);
        lds_sync();
      }
    }

    // ---- results: lane (row, half) holds columns 32 i + 8 (v / 4) + 4 half + v % 4 ----
    l += __shfl_xor(l, 32);
    if (r0 + wave * 32 + col < rows) {
      if (a.nsplit == 1) {
        const float inv = l == 0.f ? 0.f : kResult / l;
        T* dst = y + (sp.first + tok) * a.y_token + static_cast<int64_t>(hq) * a.y_head;
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
          for (int v4 = 0; v4 < 4; ++v4) {
            const int d = 32 * i + 8 * v4 + 4 * half;
            float v[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) v[x] = o[i][4 * v4 + x] * inv;
            if (a.y_vec) {
              if (d < a.dim) {
                if constexpr (TWO)
                  *reinterpret_cast<float4*>(dst + d) = make_float4(v[0], v[1], v[2], v[3]);
                else
                  *reinterpret_cast<uint2*>(dst + d) =
                      make_uint2(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]));
              }
            } else {
#pragma unroll
              for (int x = 0; x < 4; ++x)
                if (d + x < a.dim) elem<T>::store(dst + d + x, v[x]);
            }
          }
      } else {
        const int pd = (a.dim + 3) & ~3;
        const int64_t at = ((sp.first + tok) * static_cast<int64_t>(a.kv_heads) * a.group + hq) * a.nsplit + split;
        float* dst = part + at * pd;
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
          for (int v4 = 0; v4 < 4; ++v4) {
            const int d = 32 * i + 8 * v4 + 4 * half;
            if (d < pd)
              *reinterpret_cast<float4*>(dst + d) =
                  make_float4(o[i][4 * v4], o[i][4 * v4 + 1], o[i][4 * v4 + 2], o[i][4 * v4 + 3]);
          }
        if (half == 0) {
          stat[2 * at] = m;
          stat[2 * at + 1] = l;
        }
      }
    }
  }
}

// Eight waves' tiles of 128 keys fit in LDS, twice, up to head widths of 128,
// and their registers do in bf16.
template <typename T, int NC>
constexpr bool kWide = sizeof(T) == 2 && NC <= 4;

template <typename T, int FMT, int NC, int W>
hipError_t launch_waves(const AttnPointers& p, AttnArgs a, hipStream_t st) {
  each_grid(a.units, [&](const UnitRow& r, unsigned n) {
    a.units = r;
    const dim3 grid((unsigned)(a.kv_heads * a.nsplit), 1, n);
    hipLaunchKernelGGL((attention_tiles_kernel<T, FMT, NC, W>), grid, dim3(64 * W), 0, st, (const T*)p.q, p.k_codes,
                       p.v_codes, p.k_scales, p.v_scales, p.table, p.lengths, p.offsets, (T*)p.y, p.part, p.stat, a);
  });
  return hipGetLastError();
}

template <typename T, int FMT, int NC>
hipError_t launch(const AttnPointers& p, const AttnArgs& a, int rows, hipStream_t st) {
  if constexpr (kWide<T, NC>) {
    if (rows == 256) return launch_waves<T, FMT, NC, 8>(p, a, st);
  }
  return launch_waves<T, FMT, NC, 4>(p, a, st);
}

template <typename T, int FMT>
hipError_t launch_nc(const AttnPointers& p, const AttnArgs& a, int rows, hipStream_t st) {
  switch ((a.dim + 31) / 32) {
    case 1: return launch<T, FMT, 1>(p, a, rows, st);
    case 2: return launch<T, FMT, 2>(p, a, rows, st);
    case 3: return launch<T, FMT, 3>(p, a, rows, st);
    case 4: return launch<T, FMT, 4>(p, a, rows, st);
    case 5: return launch<T, FMT, 5>(p, a, rows, st);
    case 6: return launch<T, FMT, 6>(p, a, rows, st);
    case 7: return launch<T, FMT, 7>(p, a, rows, st);
    default: return launch<T, FMT, 8>(p, a, rows, st);
  }
}

}  // namespace

bool attention_tiles_wide(int dtype, int head_dim) { return dtype == CONV_BF16 && head_dim <= 128; }

hipError_t launch_attention_tiles(const AttnPointers& p, const AttnArgs& a, int dtype, int format, int rows,
                                  hipStream_t st) {
  if (dtype == CONV_F32)
    return format == CONVSEL_KV_INT8 ? launch_nc<float, CONVSEL_KV_INT8>(p, a, rows, st)
                                     : launch_nc<float, CONVSEL_KV_FP8>(p, a, rows, st);
  return format == CONVSEL_KV_INT8 ? launch_nc<bf16_t, CONVSEL_KV_INT8>(p, a, rows, st)
                                   : launch_nc<bf16_t, CONVSEL_KV_FP8>(p, a, rows, st);
}

}  // namespace convsel
