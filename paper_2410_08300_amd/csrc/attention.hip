// Attention of new queries over the 8-bit paged cache.
#include <math.h>
#include <stdio.h>

#include "attention_common.hpp"

namespace convsel {
namespace {

using namespace lm;

typedef float f32x4v_t __attribute__((ext_vector_type(4)));

// Sixteen tokens of one page: a lane's part of their key and value codes.
template <int NC>
struct Block {
  uint32_t k[2 * NC], v[2 * NC];
  float ks, vs;
};

template <int NC>
__device__ __forceinline__ void load_codes(uint32_t* dst, const uint8_t* src) {
  if constexpr (NC % 2 == 0) {
#pragma unroll
    for (int i = 0; i < NC / 2; ++i) {
      const uint4 u = reinterpret_cast<const uint4*>(src)[i];
      dst[4 * i] = u.x; dst[4 * i + 1] = u.y; dst[4 * i + 2] = u.z; dst[4 * i + 3] = u.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const uint2 u = reinterpret_cast<const uint2*>(src)[i];
      dst[2 * i] = u.x; dst[2 * i + 1] = u.y;
    }
  }
}

__device__ __forceinline__ f32x4v_t mfma16(const f16x8_t& a, const f16x8_t& b, const f32x4v_t& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// ---------------------------------------------------------------------------
// Few query rows: one workgroup of four waves per (16 rows, key head, part of
// the keys).  A row is a query of the sequence and one of the heads that share
// the key head.  Wave w takes every fourth pair of 16-token blocks, keeps its
// own maximum, sums and result, and the four are joined in LDS at the end; the
// parts of a split axis are joined by attention_join_kernel.
//
// Scores are computed as K q^T: a lane of the 16 x 16 x 32 product then holds
// four neighbouring tokens of one query, and in the order in which V lies in
// the cache those are the weights that the second product wants from it: no
// value is moved between lanes, and codes go from memory to the matrix cores
// through registers alone.
//
// What bounds it: the codes' way from memory.  64 sequences of one query on 2048
// .. 8192 tokens, 32 heads of 128 on 8, fp8: 142 us, 4.7 TB/s; one on 32768 in
// 64 parts, int8: 20 us, 3.4 TB/s, and 4 us for the join.
// ---------------------------------------------------------------------------
template <typename T, int FMT, int NC>
__global__ __launch_bounds__(256) void attention_rows_kernel(
    const T* __restrict__ q, const uint8_t* __restrict__ kc, const uint8_t* __restrict__ vc,
    const float* __restrict__ ks, const float* __restrict__ vs, const int32_t* __restrict__ table,
    const int32_t* __restrict__ lengths, const int32_t* __restrict__ offsets, T* __restrict__ y,
    float* __restrict__ part, float* __restrict__ stat, AttnArgs a) {
  constexpr bool TWO = sizeof(T) == 4;
  constexpr int DP = 32 * NC, DT = 2 * NC, LB = DP / 4;  // row bytes, 16-column tiles, bytes of a lane
  __shared__ float so[4][16][DP + 4];
  __shared__ float sm[4][16], sl[4][16];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int head = blockIdx.y, split = blockIdx.x;
  const Unit un = find_unit<true>(a.units, offsets, lengths);
  const Span sp = un.span;
  const int rows = sp.count * a.group;
  const int64_t len = un.length;
  const int limit = static_cast<int>(max((int64_t)0, min(len, a.table_width << a.ps_shift)));
  const int32_t* my_table = table + un.seq * a.table_width;

  const int ntile = (rows + 15) >> 4;

  for (int tile = un.index; tile < ntile; tile += un.count) {
    // This lane's query row, and what the tile's rows see between them.
    const int row = min(tile * 16 + col, rows - 1);
    const int tok = row / a.group;
    const int64_t first = len - sp.count;  // position of the sequence's first query
    int lo = 0, hi = limit;
    {
      const int tok0 = tile * 16 / a.group, tok1 = min(tile * 16 + 15, rows - 1) / a.group;
      if (a.causal) hi = static_cast<int>(max((int64_t)0, min((int64_t)hi, first + tok1 + 1)));
      if (a.window > 0) lo = static_cast<int>(max((int64_t)0, first + tok0 - a.window + 1));
    }
    const int64_t p = first + tok;
    const int row_hi = a.causal ? static_cast<int>(max((int64_t)0, min((int64_t)hi, p + 1))) : hi;
    const int row_lo = a.window > 0 ? static_cast<int>(max((int64_t)0, min((int64_t)hi, p - a.window + 1))) : 0;
    const int b0 = lo >> 4, b1 = hi > lo ? (hi + 15) >> 4 : b0;
    const int pairs = (b1 - b0 + 1) >> 1;
    const int per = (pairs + a.nsplit - 1) / a.nsplit;
    const int pair0 = split * per, pair1 = min(pairs, pair0 + per);

    // The query row, as the second operand: lane (row, g) holds columns
    // g * LB + 8 c + 0..7, the columns that lane (token, g) loads of a key.
    float qv[NC][8];
    {
      const T* src = q + (sp.first + tok) * a.q_token +
                     (static_cast<int64_t>(head) * a.group + row % a.group) * a.q_head + g * LB;
      if (a.q_vec) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int j = 0; j < 8; j += elem<T>::per16) {
            const vec16 v = load16(src + 8 * c + j);
#pragma unroll
            for (int x = 0; x < elem<T>::per16; ++x) qv[c][j + x] = elem<T>::to_f32(vec16_get<T>(v, x));
          }
      } else {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int d = g * LB + 8 * c + j;
            qv[c][j] = d < a.dim ? elem<T>::load(src + 8 * c + j) : 0.f;
          }
      }
    }

    f32x4v_t o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = f32x4v_t{0.f, 0.f, 0.f, 0.f};
    float m = -__builtin_inff(), l = 0.f;

    // Page of block b, -1 where there is none.
    auto page_of = [&](int b) -> int {
      if (b >= b1) return -1;
      const int pg = my_table[b >> (a.ps_shift - 4)];
      return pg >= 0 && pg < a.pages ? pg : -1;
    };
    auto load = [&](Block<NC>& r, int b, int pg) {
      const int64_t ph = static_cast<int64_t>(pg < 0 ? 0 : pg) * a.kv_heads + head;
      const int t0 = (b & ((1 << (a.ps_shift - 4)) - 1)) << 4;
      const int64_t at = ((ph << a.ps_shift) + t0) * DP;
      load_codes<NC>(r.k, kc + at + col * DP + g * LB);
      load_codes<NC>(r.v, vc + at + lane * LB);
      r.ks = ks[ph];
      r.vs = vs[ph];
    };
    f16x8_t qh[NC], ql[TWO ? NC : 1];
    float cs = 0.f;
    auto prepare_query = [&]() {
      float amax = 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fabsf(qv[c][j]));
      amax = fmaxf(amax, __shfl_xor(amax, 16));
      amax = fmaxf(amax, __shfl_xor(amax, 32));
      const int e = query_exponent(amax);
      cs = ldexpf(a.scale, e);
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float v = ldexpf(qv[c][j], -e);
          qh[c][j] = static_cast<_Float16>(v);
          if constexpr (TWO) ql[c][j] = static_cast<_Float16>(v - static_cast<float>(qh[c][j]));
        }
    };
    auto compute = [&](Block<NC> (&r)[2], int pair, int pg0, int pg1) {
      const int pgs[2] = {pg0, pg1};
      float sc[2][4];
      float top = -__builtin_inff();
      int ve[2];
      float vf[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int j0 = (b0 + 2 * pair + i) << 4;
        const bool there = pgs[i] >= 0;
        f32x4v_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const f16x8_t kf = widen8<FMT>(r[i].k[2 * c], r[i].k[2 * c + 1]);
          acc = mfma16(kf, qh[c], acc);
          if constexpr (TWO) acc = mfma16(kf, ql[c], acc);
        }
        vf[i] = split_scale(there ? r[i].vs : 1.f, ve[i]);
        const float f = (there ? r[i].ks : 0.f) * cs;
        const bool whole = there && j0 >= lo && j0 + 16 <= hi && (!a.causal || j0 + 15 <= first + tile * 16 / a.group) &&
                           a.window == 0;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int j = j0 + 4 * g + x;
          const float s = acc[x] * f;
          sc[i][x] = whole || (there && j >= row_lo && j < row_hi) ? s : -__builtin_inff();
          top = fmaxf(top, ceilf(sc[i][x]) + ve[i]);
        }
        // Rows never written may hold any bits; a weight of zero does not silence a NaN code.
        if (!there || j0 + 16 > limit) {
          const int n = there ? clampi(limit - j0 - 4 * g, 0, 4) : 0;
          const uint32_t keep = n >= 4 ? 0xffffffffu : (1u << (8 * n)) - 1u;
#pragma unroll
          for (int d = 0; d < DT; ++d) r[i].v[d] &= keep;
        }
      }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      if (__any(top > m)) {
        const float mn = fmaxf(m, top);
        const int dm = shift_of(m, mn);
        m = mn;
        l = ldexpf(l, dm);
        const float f = ldexpf(1.f, dm);
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] *= f;
      }
      f16x8_t wh, wl;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float sum = 0.f;
        const float vd = vf[i] * kWeight, up = ve[i] - m;
        float tmax = -__builtin_inff();
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          // Scores are finite or -inf here (or NaN, which stays); m is finite once any score is.
          const float t = sc[i][x] == -__builtin_inff() ? -__builtin_inff() : sc[i][x] + up;
          tmax = fmaxf(tmax, t);
          const float u = __builtin_amdgcn_exp2f(t);
          sum += u;
          float w = u * vd;
          // One rounded w: the compiler would fuse the product into one of the two conversions below only, and
          // the second would then miss by a step where the first fell the other way.
          asm volatile("" : "+v"(w));
          wh[4 * i + x] = static_cast<_Float16>(w);
          wl[4 * i + x] = static_cast<_Float16>(w - static_cast<float>(wh[4 * i + x]));
        }
        if (__any(tmax < kFar && tmax > -__builtin_inff())) {
          sum = 0.f;
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const float n = rintf(sc[i][x]);
            if (sc[i][x] > -__builtin_inff())
              sum += ldexpf(__builtin_amdgcn_exp2f(sc[i][x] - n), static_cast<int>(fmaxf(n - m, -300.f)));
          }
          l += sum;
        } else {
          l += ldexpf(sum, -ve[i]);
        }
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const f16x8_t vf8 = widen8<FMT>(r[0].v[d], r[1].v[d]);
        o[d] = mfma16(vf8, wh, o[d]);
        o[d] = mfma16(vf8, wl, o[d]);
      }
    };

    {
      Block<NC> ra[2], rb[2];
      int pa[2], pb[2];
      auto fetch = [&](Block<NC> (&r)[2], int (&pg)[2], int pair) {
#pragma unroll
        for (int i = 0; i < 2; ++i) load(r[i], b0 + 2 * pair + i, pg[i]);
      };
      auto look = [&](int (&pg)[2], int pair) {
#pragma unroll
        for (int i = 0; i < 2; ++i) pg[i] = pair < pair1 ? page_of(b0 + 2 * pair + i) : -1;
      };
      int pair = pair0 + wave;
      if (pair < pair1) {
        look(pa, pair);
        look(pb, pair + 4);
        fetch(ra, pa, pair);
        prepare_query();  // the first codes are on their way
        for (; pair < pair1; pair += 8) {
          int pn[2];
          if (pair + 4 < pair1) fetch(rb, pb, pair + 4);
          look(pn, pair + 8);
          compute(ra, pair, pa[0], pa[1]);
          pa[0] = pn[0]; pa[1] = pn[1];
          if (pair + 4 >= pair1) break;
          if (pair + 8 < pair1) fetch(ra, pa, pair + 8);
          look(pn, pair + 12);
          compute(rb, pair + 4, pb[0], pb[1]);
          pb[0] = pn[0]; pb[1] = pn[1];
        }
      }
    }

    // Join the four waves.
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) {
      sm[wave][col] = m;
      sl[wave][col] = l;
    }
#pragma unroll
    for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4v_t*>(&so[wave][col][16 * d + 4 * g]) = o[d];
    __syncthreads();
    const int r = threadIdx.x >> 4, d0 = threadIdx.x & 15;  // 16 threads a row
    float mt = sm[0][r];
#pragma unroll
    for (int w = 1; w < 4; ++w) mt = fmaxf(mt, sm[w][r]);
    float f[4], lt = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int dm = shift_of(sm[w][r], mt);
      f[w] = ldexpf(1.f, dm);
      lt += ldexpf(sl[w][r], dm);
    }
    if (tile * 16 + r < rows) {
      const int rt = (tile * 16 + r) / a.group, rh = (tile * 16 + r) % a.group;
      const int64_t h = static_cast<int64_t>(head) * a.group + rh;
      if (a.nsplit == 1) {
        T* dst = y + (sp.first + rt) * a.y_token + h * a.y_head;
        const float inv = lt == 0.f ? 0.f : kResult / lt;
        for (int d = d0; d < a.dim; d += 16) {
          float v = 0.f;
#pragma unroll
          for (int w = 0; w < 4; ++w) v += so[w][r][d] * f[w];
          elem<T>::store(dst + d, v * inv);
        }
      } else {
        const int64_t at = ((sp.first + rt) * static_cast<int64_t>(a.kv_heads) * a.group + h) * a.nsplit + split;
        for (int d = d0; d < a.dim; d += 16) {
          float v = 0.f;
#pragma unroll
          for (int w = 0; w < 4; ++w) v += so[w][r][d] * f[w];
          part[at * ((a.dim + 3) & ~3) + d] = v;
        }
        if (d0 == 0) {
          stat[2 * at] = mt;
          stat[2 * at + 1] = lt;
        }
      }
    }
    __syncthreads();
  }
}

// Joins the parts of a split axis: one workgroup per (token, head) that a
// sequence owns.  Partial results are rows of whole 16-byte units.
constexpr int kMaxSplit = 128;

template <typename T>
__global__ __launch_bounds__(256) void attention_join_kernel(const float* __restrict__ part,
                                                             const float* __restrict__ stat,
                                                             const int32_t* __restrict__ offsets, int seqs,
                                                             T* __restrict__ y, AttnArgs a) {
  __shared__ float sf[kMaxSplit];
  __shared__ float4 sv[256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t heads = static_cast<int64_t>(a.kv_heads) * a.group;
  const int64_t it = blockIdx.x, t = it / heads, h = it - t * heads;
  const int owned = clampi(offsets[seqs], 0, a.tokens);
  const int n = a.nsplit;
  // Offsets rise from 0: the tokens behind the last one belong to nobody.
  if (t >= owned) return;
  // Each wave reads all statistics; lane s holds those of parts s and s + 64.
  float ms[2], ls[2], m = -__builtin_inff(), l = 0.f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int s = lane + 64 * i;
    const float2 v = s < n ? reinterpret_cast<const float2*>(stat)[it * n + s] : make_float2(-__builtin_inff(), 0.f);
    ms[i] = v.x;
    ls[i] = v.y;
    m = fmaxf(m, v.x);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int dm = shift_of(ms[i], m);
    if (wave == 0) sf[lane + 64 * i] = ldexpf(1.f, dm);
    l += ldexpf(ls[i], dm);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o);
  __syncthreads();
  // Four columns a thread, the parts dealt to as many groups as the workgroup holds.
  const int c4 = (a.dim + 3) / 4, groups = 256 / c4;
  const int col = threadIdx.x % c4, group = threadIdx.x / c4;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (group < groups) {
    const float4* src = reinterpret_cast<const float4*>(part) + it * n * c4 + col;
#pragma unroll 4
    for (int s = group; s < n; s += groups) {
      const float4 p = src[s * c4];
      const float f = sf[s];
      v.x += p.x * f; v.y += p.y * f; v.z += p.z * f; v.w += p.w * f;
    }
  }
  sv[threadIdx.x] = v;
  __syncthreads();
  const int d = threadIdx.x;
  if (d < a.dim) {
    float r = 0.f;
    for (int i = 0; i < groups; ++i) r += reinterpret_cast<const float*>(&sv[i * c4])[d];
    const float inv = l == 0.f ? 0.f : kResult / l;
    elem<T>::store(y + t * a.y_token + h * a.y_head + d, r * inv);
  }
}

// The same for few parts: four columns of a row a thread, whole rows a workgroup.
// (32768 rows of 128 columns in 2 parts: a workgroup a row took 43 us.)
constexpr int kFewParts = 16;

template <typename T>
__global__ __launch_bounds__(256) void attention_join_few_kernel(const float* __restrict__ part,
                                                                 const float* __restrict__ stat,
                                                                 const int32_t* __restrict__ offsets, int seqs,
                                                                 T* __restrict__ y, AttnArgs a) {
  const int64_t heads = static_cast<int64_t>(a.kv_heads) * a.group;
  const int c4 = (a.dim + 3) / 4, n = a.nsplit;
  const int in_wg = threadIdx.x / c4, col = threadIdx.x % c4;
  const int64_t it = static_cast<int64_t>(blockIdx.x) * (256 / c4) + in_wg, t = it / heads, h = it - t * heads;
  if (in_wg >= 256 / c4 || t >= clampi(offsets[seqs], 0, a.tokens)) return;
  const float2* st = reinterpret_cast<const float2*>(stat) + it * n;
  const float4* src = reinterpret_cast<const float4*>(part) + it * n * c4 + col;
  float m = -__builtin_inff(), l = 0.f;
  for (int s = 0; s < n; ++s) m = fmaxf(m, st[s].x);
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s = 0; s < n; ++s) {
    const float2 ms = st[s];
    const float4 p = src[s * c4];
    const int dm = shift_of(ms.x, m);
    const float f = ldexpf(1.f, dm);
    l += ldexpf(ms.y, dm);
    v.x += p.x * f; v.y += p.y * f; v.z += p.z * f; v.w += p.w * f;
  }
  const float inv = l == 0.f ? 0.f : kResult / l;
  T* dst = y + t * a.y_token + h * a.y_head + 4 * col;
  const float r[4] = {v.x * inv, v.y * inv, v.z * inv, v.w * inv};
#pragma unroll
  for (int x = 0; x < 4; ++x)
    if (4 * col + x < a.dim) elem<T>::store(dst + x, r[x]);
}

// How a call is cut: rows, in 16s, 128s or 256s, and parts of the keys.  The host
// knows how many tokens the call has and how many a sequence may hold, not how
// they are spread: kernel and parts go by the average, tiles of rows by what each
// sequence has.
struct Plan {
  int rows;  // of a workgroup: 16, 128 or 256
  int tiles;  // of a sequence of the average length
  int nsplit;
};

Plan plan(const convsel_kv_cache_t& c, const convsel_kv_batch_t& b, const convsel_attention_desc_t& d) {
  const int64_t group = d.q_heads / c.kv_heads;
  const int64_t avg = (b.tokens + b.seqs - 1) / b.seqs;
  int64_t keys = b.table_width * c.page_size;
  if (d.window > 0 && d.window + avg < keys) keys = d.window + avg;
  Plan p;
  // The 128-row kernel widens codes once for 128 rows but takes some 15 us for
  // its first keys; the 16-row kernel is through them in 8.  Measured with
  // heads of 128 and 64, they cross where rows x keys x width reach 1.6e9 in
  // bf16 and 4e9 in fp32 (one sequence, 32 query heads of 128 on 8, bf16: 128
  // new tokens on 4000, 46 against 48 us; 64 on 1000, 27 against 18; 2048 on
  // none 99 against 177), provided that its tiles are at least half full.
  const double work = (double)avg * d.q_heads * b.seqs * keys * kv_row_bytes(c.head_dim);
  const bool many = avg * group >= 64 && work >= (d.dtype == CONV_F32 ? 4e9 : 1.6e9);
  auto cut = [&](int rows) {
    const int64_t tiles = (avg * group + rows - 1) / rows;
    p.rows = rows;
    p.tiles = (int)(tiles < 32768 ? tiles : 32768);
    const int64_t groups = p.tiles * c.kv_heads * b.seqs;
    // Two workgroups a CU (one of 256 rows), with 256 keys at least in each part.
    const int64_t want = rows == 256 ? 256 : 512;
    int64_t n = rows > 16 ? (want + groups - 1) / groups : want / groups;
    if (n > keys / 256) n = keys / 256;
    if (rows > 16) {
      // 64 keys take 2.3 us where nothing else runs on the CU, a part's results 2e-6 us a value to write and join: the
      // sum is least at the root of their ratio.
      const double walk = keys / 64 * 2.3, join = (double)b.tokens * d.q_heads * c.head_dim * 2e-6;
      const int64_t best = (int64_t)sqrt(walk / join);
      if (n > best) n = best;
    } else {
      // The join's launch costs what 400 keys do (8 key heads of 128: 4 sequences of 20 queries on 500, 14.6 us in one
      // part and 17.2 in two; 16 of one on 1000, 23.2 and 20.8 in three), and a few workgroups more than run at once
      // as much again (24 of one on 1000: 24.4, and 28.9 in three parts).
      if (n > 1 && keys * (n - 1) / n < 400) n = 1;
      // Sequences of unlike lengths end together where each is cut (64 of 2048 .. 8192 tokens: 163 -> 146 us).
      const int64_t even = groups >= 4096 ? 1 : keys / 2048 < 4 ? keys / 2048 : 4;
      if (n < even) n = even;
    }
    if (n > kMaxSplit) n = kMaxSplit;
    p.nsplit = (int)(n < 1 ? 1 : n);
    return groups * p.nsplit;
  };
  // 256 rows share codes and barriers among twice as many, and pay where every CU has work for long: long sequences,
  // and either a second workgroup a CU to even out what a causal mask leaves, or a prefix that makes all alike (32 query
  // heads of 128 on 8: 4096 new tokens 280 -> 250 us, 512 on 8000 152 -> 138; but 2048 new ones 99 -> 116).
  if (many && attention_tiles_wide(d.dtype, c.head_dim) && keys >= 2048) {
    const int64_t wgs = cut(256);
    if (wgs >= 512 || (wgs >= 256 && keys >= 4 * avg)) return p;
  }
  cut(many ? 128 : 16);
  return p;
}

UnitRow tiles_of(const convsel_kv_batch_t& b, int64_t group, int rows) {
  return unit_row(b, group, __builtin_ctz(rows));
}

size_t part_floats(const convsel_kv_cache_t& c, const convsel_kv_batch_t& b, const convsel_attention_desc_t& d,
                   const Plan& p) {
  const size_t n = (size_t)b.tokens * d.q_heads * p.nsplit * ((c.head_dim + 3) / 4 * 4);
  return (n + 63) / 64 * 64;
}

template <typename T, int FMT, int NC>
void launch_rows(dim3 grid, const AttnPointers& p, const AttnArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((attention_rows_kernel<T, FMT, NC>), grid, dim3(256), 0, st, (const T*)p.q, p.k_codes, p.v_codes,
                     p.k_scales, p.v_scales, p.table, p.lengths, p.offsets, (T*)p.y, p.part, p.stat, a);
}

template <typename T, int FMT>
void launch_rows_nc(dim3 grid, const AttnPointers& p, const AttnArgs& a, hipStream_t st) {
  switch ((a.dim + 31) / 32) {
    case 1: return launch_rows<T, FMT, 1>(grid, p, a, st);
    case 2: return launch_rows<T, FMT, 2>(grid, p, a, st);
    case 3: return launch_rows<T, FMT, 3>(grid, p, a, st);
    case 4: return launch_rows<T, FMT, 4>(grid, p, a, st);
    case 5: return launch_rows<T, FMT, 5>(grid, p, a, st);
    case 6: return launch_rows<T, FMT, 6>(grid, p, a, st);
    case 7: return launch_rows<T, FMT, 7>(grid, p, a, st);
    default: return launch_rows<T, FMT, 8>(grid, p, a, st);
  }
}

}  // namespace

size_t attention_workspace(const convsel_kv_cache_t& c, const convsel_kv_batch_t& b,
                           const convsel_attention_desc_t& d) {
  const Plan p = plan(c, b, d);
  if (p.nsplit == 1) return 0;
  return (part_floats(c, b, d, p) + (size_t)b.tokens * d.q_heads * p.nsplit * 2) * 4;
}

hipError_t launch_attention(const void* q, const convsel_kv_cache_t& c, const convsel_kv_batch_t& b, void* y,
                            const convsel_attention_desc_t& d, void* workspace, hipStream_t stream) {
  const Plan p = plan(c, b, d);
  AttnArgs a;
  a.pages = c.pages;
  a.table_width = b.table_width;
  a.q_token = d.q_token_stride; a.q_head = d.q_head_stride;
  a.y_token = d.y_token_stride; a.y_head = d.y_head_stride;
  a.tokens = (int)b.tokens; a.kv_heads = c.kv_heads; a.group = d.q_heads / c.kv_heads; a.dim = c.head_dim;
  a.ps_shift = c.page_size == 16 ? 4 : c.page_size == 32 ? 5 : c.page_size == 64 ? 6 : 7;
  a.causal = d.causal; a.window = d.window; a.nsplit = p.nsplit;
  a.scale = d.scale * 1.4426950408889634f;
  // Queries are read and results written in 16-byte (results: four-value) units where every row starts on one and
  // has no padding.
  const int64_t unit = d.dtype == CONV_F32 ? 4 : 8, es = 16 / unit;
  a.q_vec = c.head_dim % 32 == 0 && a.q_token % unit == 0 && a.q_head % unit == 0 && (uintptr_t)q % 16 == 0;
  a.y_vec = c.head_dim % 4 == 0 && a.y_token % 4 == 0 && a.y_head % 4 == 0 && (uintptr_t)y % (4 * es) == 0;
  AttnPointers ptr;
  ptr.q = q;
  ptr.k_codes = (const uint8_t*)c.k_codes; ptr.v_codes = (const uint8_t*)c.v_codes;
  ptr.k_scales = c.k_scales; ptr.v_scales = c.v_scales;
  ptr.y = y;
  ptr.part = (float*)workspace;
  ptr.stat = p.nsplit > 1 ? ptr.part + part_floats(c, b, d, p) : nullptr;
  ptr.table = b.table; ptr.lengths = b.lengths; ptr.offsets = b.offsets;
  a.units = tiles_of(b, a.group, p.rows);
  if (p.rows > 16) {
    const hipError_t e = launch_attention_tiles(ptr, a, d.dtype, c.format, p.rows, stream);
    if (e != hipSuccess) return e;
  } else {
    each_grid(a.units, [&](const UnitRow& r, unsigned n) {
      a.units = r;
      const dim3 grid(p.nsplit, c.kv_heads, n);
      if (d.dtype == CONV_F32) {
        if (c.format == CONVSEL_KV_INT8) launch_rows_nc<float, CONVSEL_KV_INT8>(grid, ptr, a, stream);
        else launch_rows_nc<float, CONVSEL_KV_FP8>(grid, ptr, a, stream);
      } else {
        if (c.format == CONVSEL_KV_INT8) launch_rows_nc<bf16_t, CONVSEL_KV_INT8>(grid, ptr, a, stream);
        else launch_rows_nc<bf16_t, CONVSEL_KV_FP8>(grid, ptr, a, stream);
      }
    });
  }
  if (p.nsplit > 1) {
    const int64_t rows = b.tokens * d.q_heads, in_wg = p.nsplit <= kFewParts ? 256 / ((c.head_dim + 3) / 4) : 1;
    const dim3 grid((unsigned)((rows + in_wg - 1) / in_wg));
    const int seqs = (int)b.seqs;
    if (p.nsplit <= kFewParts) {
      if (d.dtype == CONV_F32)
        hipLaunchKernelGGL(attention_join_few_kernel<float>, grid, dim3(256), 0, stream, ptr.part, ptr.stat, b.offsets,
                           seqs, (float*)y, a);
      else
        hipLaunchKernelGGL(attention_join_few_kernel<bf16_t>, grid, dim3(256), 0, stream, ptr.part, ptr.stat, b.offsets,
                           seqs, (bf16_t*)y, a);
    } else {
      if (d.dtype == CONV_F32)
        hipLaunchKernelGGL(attention_join_kernel<float>, grid, dim3(256), 0, stream, ptr.part, ptr.stat, b.offsets, seqs,
                           (float*)y, a);
      else
        hipLaunchKernelGGL(attention_join_kernel<bf16_t>, grid, dim3(256), 0, stream, ptr.part, ptr.stat, b.offsets,
                           seqs, (bf16_t*)y, a);
    }
  }
  return hipGetLastError();
}

void attention_describe(const convsel_kv_cache_t& c, const convsel_kv_batch_t& b, const convsel_attention_desc_t& d,
                        char* buf, size_t len) {
  const Plan p = plan(c, b, d);
  snprintf(buf, len, "attention kernels=attention_%s_kernel%s rows=%d tiles=%u split=%d workspace=%zu",
           p.rows > 16 ? "tiles" : "rows",
           p.nsplit <= 1 ? "" : p.nsplit <= kFewParts ? ";attention_join_few_kernel" : ";attention_join_kernel", p.rows,
           units_of(tiles_of(b, d.q_heads / c.kv_heads, p.rows)), p.nsplit, attention_workspace(c, b, d));
}

}  // namespace convsel
