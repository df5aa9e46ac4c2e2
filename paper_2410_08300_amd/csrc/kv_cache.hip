// Writing tokens into the 8-bit paged cache and reading them back.
#include "lm_common.hpp"
#include "lm_kernels.hpp"

namespace convsel {
namespace {

using namespace lm;

// Writing: one workgroup per (page of a sequence, head, keys or values).  The
// page's new tokens are read twice, 16 bytes a lane: for the largest magnitude,
// and, from the CU's own cache now, for the codes.  Keys leave as they lie;
// values, whose layout puts four tokens of a column side by side, are taken four
// tokens at a time and change places in LDS.  A page that already holds tokens,
// or ends inside a block, goes the general way: every 4-byte word of codes
// belongs to one thread, which keeps the bytes that the call does not write.
//
// What bounds it: traffic, two or four bytes in and one out for each value, at
// 3.6 to 4.3 TB/s for prompts in bf16, and for a few tokens (64 sequences of one:
// 6.3 us) the way from the lengths to the table to the page; heads that are no
// multiple of 32 go word by word (16 prompts of 2048 tokens of 8 heads of 80: 101
// us, of 96 41).

// The fp32 quotient x / s of finite numbers, correctly rounded, from r = 1 / s
// (correctly rounded): x r is within two units of it, one step with the exact
// remainder brings that within one, and from there a second step rounds right
// (Markstein 1990).  Five operations; the general quotient takes some twelve.
__device__ __forceinline__ float quotient(float x, float s, float r) {
  float q = x * r;
  q = fmaf(fmaf(-q, s, x), r, q);
  return fmaf(fmaf(-q, s, x), r, q);
}

// Codes of four finite numbers of magnitudes up to the block's largest: no
// quotient is more than a rounding beyond the largest code.
template <int FMT>
__device__ __forceinline__ uint32_t four_codes(float x0, float x1, float x2, float x3, float s, float r) {
  const float q0 = quotient(x0, s, r), q1 = quotient(x1, s, r), q2 = quotient(x2, s, r), q3 = quotient(x3, s, r);
  if constexpr (FMT == CONVSEL_KV_INT8) {
    // 1.5 * 2^23 + q holds q, rounded to nearest even, in its lowest byte.
    const uint32_t a = __float_as_uint(q0 + 12582912.f), b = __float_as_uint(q1 + 12582912.f);
    const uint32_t c = __float_as_uint(q2 + 12582912.f), d = __float_as_uint(q3 + 12582912.f);
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u),
                                 0x05040100u);
  } else {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(q0, q1, 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(q2, q3, lo, true));
  }
}

template <typename T, int FMT, int NT, bool ROW>
__global__ __launch_bounds__(NT) void kv_write_kernel(convsel_kv_cache_t c, convsel_kv_batch_t b, KvTokens in,
                                                       UnitRow row, int vec) {
  constexpr int UE = elem<T>::per16;
  extern __shared__ __align__(16) uint8_t turn[];  // a page's value codes
  __shared__ float red[NT / 64];
  const bool values = blockIdx.y >= static_cast<unsigned>(c.kv_heads);
  const int head = values ? blockIdx.y - c.kv_heads : blockIdx.y;
  const int ps = c.page_size, D = c.head_dim, dp = kv_row_bytes(D);
  const int64_t token = values ? in.v_token : in.k_token;
  const Unit un = find_unit<ROW>(row, b.offsets, b.lengths);
  const int64_t from = un.length < 0 ? 0 : un.length, to = min(from + un.span.count, b.table_width * ps);
  if (from >= to || from / ps + un.index >= (to + ps - 1) / ps) return;
  const int start = static_cast<int>(from), end = static_cast<int>(to);  // within a table: below 2^30
  const int32_t* table = b.table + un.seq * b.table_width;
  const T* src0 = reinterpret_cast<const T*>(values ? in.v : in.k) +
                  head * (values ? in.v_head : in.k_head) + un.span.first * token;
  // Tokens that start within a page may reach one more than their sequence has units: somebody walks two.
  const int pages = (end + ps - 1) / ps;
  for (int pg = start / ps + un.index; pg < pages; pg += un.count) {
    const int64_t page = table[pg];
    if (page < 0 || page >= c.pages) continue;
    const int r0 = max(start - pg * ps, 0), r1 = min(end - pg * ps, ps);
    const T* src = src0 + (pg * ps - start) * token;  // row r of the page is src + r * token
    const int64_t ph = page * c.kv_heads + head;
    float* scale_at = (values ? c.v_scales : c.k_scales) + ph;
    const float old = *scale_at;
    float amax = 0.f;
    bool wild = false;  // infinities or NaN among them
    auto see = [&](float x) {
      const float v = fabsf(x);
      const bool finite = v < __builtin_inff();
      wild |= !finite;
      amax = fmaxf(amax, finite ? v : 0.f);
    };
    const int upr = vec ? D / UE : 0;  // units of a token's row, where rows are whole units
    if (vec) {
#pragma unroll 4
      for (int u = threadIdx.x; u < (r1 - r0) * upr; u += NT) {
        const vec16 v = load16(src + (r0 + u / upr) * token + u % upr * UE);
#pragma unroll
        for (int x = 0; x < UE; ++x) see(elem<T>::to_f32(vec16_get<T>(v, x)));
      }
    } else {
      for (int i = threadIdx.x; i < (r1 - r0) * D; i += NT) see(elem<T>::load(src + (r0 + i / D) * token + i % D));
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = amax;
    wild = __syncthreads_or(wild);
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) amax = fmaxf(amax, red[w]);
    __syncthreads();  // every thread has `old` and red before either is written again
    float scale = fmaxf(amax / qmax_of(FMT), kMinScale);
    if (r0 > 0) scale = fmaxf(scale, old);
    const bool grown = r0 > 0 && scale != old;
    if (threadIdx.x == 0) *scale_at = scale;
    uint8_t* codes = reinterpret_cast<uint8_t*>(values ? c.v_codes : c.k_codes) + ph * static_cast<int64_t>(ps * dp);
    const float inv = 1.f / scale;
    const bool whole = vec && D == dp && r0 == 0 && !wild && (!values || (r1 & 15) == 0);
    if (whole && !values) {
#pragma unroll 2
      for (int u = threadIdx.x; u < r1 * upr; u += NT) {
        const vec16 v = load16(src + (u / upr) * token + u % upr * UE);
        uint32_t w[UE / 4];
#pragma unroll
        for (int x = 0; x < UE; x += 4)
          w[x / 4] = four_codes<FMT>(elem<T>::to_f32(vec16_get<T>(v, x)), elem<T>::to_f32(vec16_get<T>(v, x + 1)),
                                     elem<T>::to_f32(vec16_get<T>(v, x + 2)), elem<T>::to_f32(vec16_get<T>(v, x + 3)),
                                     scale, inv);
        uint8_t* at = codes + u * UE;  // rows lie one behind the other
        if constexpr (UE == 8) *reinterpret_cast<uint2*>(at) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(at) = w[0];
      }
    } else if (whole) {
      for (int u = threadIdx.x; u < (r1 >> 2) * upr; u += NT) {
        const int t = u / upr * 4, d = u % upr * UE;
        vec16 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = load16(src + (t + j) * token + d);
#pragma unroll
        for (int x = 0; x < UE; ++x)
          *reinterpret_cast<uint32_t*>(turn + v_byte(t, d + x, dp)) =
              four_codes<FMT>(elem<T>::to_f32(vec16_get<T>(v[0], x)), elem<T>::to_f32(vec16_get<T>(v[1], x)),
                              elem<T>::to_f32(vec16_get<T>(v[2], x)), elem<T>::to_f32(vec16_get<T>(v[3], x)), scale,
                              inv);
      }
      __syncthreads();
      for (int i = threadIdx.x; i < r1 * dp / 16; i += NT) store16(codes + i * 16, load16(turn + i * 16));
      __syncthreads();
    } else {
      auto code_at = [&](int t, int d, uint32_t was) -> uint32_t {
        if (t >= r1 || (t < r0 && !grown)) return was;
        if (t >= r0 && d >= D) return 0u;
        return encode(t < r0 ? decode(was, FMT) * old : elem<T>::load(src + t * token + d), scale, FMT);
      };
      // Keys: a word is four columns of a token.  Values: four tokens of a column.
      const int from = grown ? 0 : r0;
      const int i0 = values ? (from >> 2) * dp : from * (dp / 4), i1 = values ? ((r1 + 3) >> 2) * dp : r1 * (dp / 4);
#pragma unroll 2
      for (int i = i0 + threadIdx.x; i < i1; i += NT) {
        const int t = values ? i / dp * 4 : i / (dp / 4), d = values ? i % dp : i % (dp / 4) * 4;
        uint32_t* at = reinterpret_cast<uint32_t*>(codes + (values ? v_byte(t, d, dp) : t * dp + d));
        const uint32_t was = t < r0 || (values && t + 4 > r1) ? *at : 0u;
        uint32_t w = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w |= code_at(values ? t + j : t, values ? d : d + j, (was >> (8 * j)) & 0xffu) << (8 * j);
        *at = w;
      }
    }
  }
}

// Reading: one workgroup per (16 positions of a sequence, head), positions
// aligned to the cache's 16-token blocks.  A thread takes four codes at a time,
// neighbours in the cache: four columns of a key, four tokens of a value, whose
// codes reach their rows through LDS.  What bounds it: traffic, 4.1 to 5.1 TB/s
// for prompts in bf16.
template <typename T, bool ROW>
__global__ __launch_bounds__(256) void kv_read_kernel(convsel_kv_cache_t c, convsel_kv_batch_t b, KvTokens to,
                                                      UnitRow units, int vec) {
  T* k = reinterpret_cast<T*>(const_cast<void*>(to.k));
  T* v = reinterpret_cast<T*>(const_cast<void*>(to.v));
  constexpr int UE = elem<T>::per16;
  const int head = blockIdx.y;
  const int ps = c.page_size, D = c.head_dim, dp = kv_row_bytes(D);
  const int64_t row = static_cast<int64_t>(c.kv_heads) * D;
  __shared__ __align__(16) uint8_t turn[16 * 256];
  const Unit un = find_unit<ROW>(units, b.offsets, b.lengths);
  const Span sp = un.span;
  const int64_t start = un.length, end = start + sp.count;  // 64-bit: bounded below
  // Floor division: a negative start names positions before the sequence.
  const int64_t first = start >= 0 ? start / 16 : -((-start + 15) / 16);
  for (int64_t blk = first + un.index; blk * 16 < end; blk += un.count) {
    const int64_t p0 = blk * 16;
    int64_t page = -1;
    if (p0 >= 0 && p0 / ps < b.table_width) page = b.table[un.seq * b.table_width + p0 / ps];
    const bool there = page >= 0 && page < c.pages;
    const int t0 = static_cast<int>(there ? p0 % ps : 0);
    const int64_t ph = there ? page * c.kv_heads + head : 0;
    const uint8_t* kc = reinterpret_cast<const uint8_t*>(c.k_codes) + ph * (ps * dp) + t0 * dp;
    const uint8_t* vc = reinterpret_cast<const uint8_t*>(c.v_codes) + ph * (ps * dp) + t0 * dp;
    const float ks = there ? c.k_scales[ph] : 0.f, vs = there ? c.v_scales[ph] : 0.f;
    // Value codes to token rows: word (g, column) holds tokens 4 g .. 4 g + 3.
    __syncthreads();
    for (int i = threadIdx.x; i < 4 * dp; i += 256) {
      const uint32_t w = reinterpret_cast<const uint32_t*>(vc)[i];
      const int unit = i / (dp / 16), dt = i % (dp / 16);
      const int d = dt * 16 + (unit & 15), t = unit / 16 * 4;
#pragma unroll
      for (int x = 0; x < 4; ++x) turn[(t + x) * dp + d] = static_cast<uint8_t>(w >> (8 * x));
    }
    __syncthreads();
    auto one = [&](uint32_t code, float s) { return there ? decode(code, c.format) * s : 0.f; };
    if (vec) {
      const int upr = D / UE;
      for (int i = threadIdx.x; i < 16 * upr; i += 256) {
        const int t = i / upr, d = i % upr * UE;
        const int64_t p = p0 + t;
        if (p < start || p >= end) continue;
        const int64_t at = (sp.first + (p - start)) * row + static_cast<int64_t>(head) * D + d;
        uint32_t kw[UE / 4], vw[UE / 4];
#pragma unroll
        for (int x = 0; x < UE / 4; ++x) {
          kw[x] = *reinterpret_cast<const uint32_t*>(kc + t * dp + d + 4 * x);
          vw[x] = *reinterpret_cast<const uint32_t*>(turn + t * dp + d + 4 * x);
        }
        vec16 ko, vo;
#pragma unroll
        for (int x = 0; x < UE; ++x) {
          vec16_set<T>(ko, x, elem<T>::from_f32(one(kw[x / 4] >> (8 * (x % 4)) & 0xffu, ks)));
          vec16_set<T>(vo, x, elem<T>::from_f32(one(vw[x / 4] >> (8 * (x % 4)) & 0xffu, vs)));
        }
        store16(k + at, ko);
        store16(v + at, vo);
      }
    } else {
      for (int i = threadIdx.x; i < 16 * D; i += 256) {
        const int t = i / D, d = i % D;
        const int64_t p = p0 + t;
        if (p < start || p >= end) continue;
        const int64_t at = (sp.first + (p - start)) * row + static_cast<int64_t>(head) * D + d;
        elem<T>::store(k + at, one(kc[t * dp + d], ks));
        elem<T>::store(v + at, one(turn[t * dp + d], vs));
      }
    }
  }
}

// Units of 2^shift tokens.  By sequence, with the units that one of the average number of tokens reaches from anywhere,
// where the longest sequence that there can be walks eight of them at most, or sixteen where all may be single tokens, or
// fills the card by itself (64 sequences of one token: 6.4 and 5.1 us to write and read, 7.5 and 6.4 in a row; 16 prompts
// of 2048 in pages of 16: 53 and 41, 58 and 44 in a row).  In a row otherwise: a prompt of 4096 beside 127 single tokens
// takes 24 and 20 us, by sequence 97 and 155; one of 1000 beside 1023 sequences of nothing 18 and 31, 161 and 106; 1024
// single tokens 27 and 21, 25 and 18.  A workgroup more for nothing costs: one for each of 64 sequences, keys and values
// of 8 heads, 3 us.
struct Deal {
  UnitRow row;
  unsigned across;
};
Deal deal(const convsel_kv_batch_t& b, int shift, int heads) {
  const int64_t unit = (int64_t)1 << shift, avg = (b.tokens + b.seqs - 1) / b.seqs;
  int64_t across = (avg + 2 * unit - 2) >> shift;
  if (across > 65536) across = 65536;
  const int64_t longest = (b.tokens >> shift) + 1;
  if (longest <= 8 * across || (b.tokens <= b.seqs && longest <= 17) || across * heads >= 1024)
    return {unit_row(b, 0, shift), (unsigned)across};
  return {unit_row(b, 1, shift), 1};
}

typedef void (*WriteKernel)(convsel_kv_cache_t, convsel_kv_batch_t, KvTokens, UnitRow, int);

template <typename T, int NT, bool ROW>
WriteKernel write_kernel(int format) {
  return format == CONVSEL_KV_INT8 ? kv_write_kernel<T, CONVSEL_KV_INT8, NT, ROW>
                                   : kv_write_kernel<T, CONVSEL_KV_FP8, NT, ROW>;
}

template <typename T, bool ROW>
WriteKernel write_kernel(int format, int threads) {
  return threads == 64    ? write_kernel<T, 64, ROW>(format)
         : threads == 128 ? write_kernel<T, 128, ROW>(format)
                          : write_kernel<T, 256, ROW>(format);
}

template <typename T>
WriteKernel write_kernel(int format, int threads, bool row) {
  return row ? write_kernel<T, true>(format, threads) : write_kernel<T, false>(format, threads);
}

typedef void (*ReadKernel)(convsel_kv_cache_t, convsel_kv_batch_t, KvTokens, UnitRow, int);

}  // namespace

hipError_t launch_kv_write(const convsel_kv_cache_t& c, const convsel_kv_batch_t& b, const KvTokens& t,
                           hipStream_t stream) {
  // Rows of whole 16-byte units that start on one.
  const int64_t ue = t.dtype == CONV_F32 ? 4 : 8;
  const int vec = c.head_dim % ue == 0 && t.k_token % ue == 0 && t.k_head % ue == 0 && t.v_token % ue == 0 &&
                  t.v_head % ue == 0 && (uintptr_t)t.k % 16 == 0 && (uintptr_t)t.v % 16 == 0;
  const size_t lds = (size_t)c.page_size * kv_row_bytes(c.head_dim);  // at most 32 KiB
  // Small pages in few threads: a workgroup's start costs as much as a page of 16 tokens.  (16 prompts of 2048 tokens
  // of 8 heads of 128 in bf16: pages of 16 tokens, 53, 78 and 117 us in 64, 128 and 256 threads; of 32, 47, 54, 81; of
  // 128, 65, 54, 48; of 16 in fp32, 97, 83, 116; six prompts of unlike lengths in pages of 64, 37 in 128, 34 in 256.)
  const int64_t size = c.page_size * c.head_dim * (t.dtype == CONV_F32 ? 3 : 1);
  const int threads = size <= 4096 ? 64 : size <= 6144 ? 128 : 256;
  const Deal g = deal(b, __builtin_ctz(c.page_size), 2 * c.kv_heads);
  const bool row = g.row.num > 0;
  const WriteKernel f =
      t.dtype == CONV_F32 ? write_kernel<float>(c.format, threads, row) : write_kernel<bf16_t>(c.format, threads, row);
  each_grid(g.row, [&](const UnitRow& r, unsigned n) {
    hipLaunchKernelGGL(f, dim3(g.across, 2 * c.kv_heads, n), dim3(threads), lds, stream, c, b, t, r, vec);
  });
  return hipGetLastError();
}

hipError_t launch_kv_read(const convsel_kv_cache_t& c, const convsel_kv_batch_t& b, const KvTokens& t,
                          hipStream_t stream) {
  const int64_t ue = t.dtype == CONV_F32 ? 4 : 8;
  const int vec = c.head_dim % ue == 0 && (uintptr_t)t.k % 16 == 0 && (uintptr_t)t.v % 16 == 0;
  const Deal g = deal(b, 4, c.kv_heads);
  const bool row = g.row.num > 0;
  const ReadKernel f = t.dtype == CONV_F32 ? (row ? kv_read_kernel<float, true> : kv_read_kernel<float, false>)
                                           : (row ? kv_read_kernel<bf16_t, true> : kv_read_kernel<bf16_t, false>);
  each_grid(g.row, [&](const UnitRow& r, unsigned n) {
    hipLaunchKernelGGL(f, dim3(g.across, c.kv_heads, n), dim3(256), 0, stream, c, b, t, r, vec);
  });
  return hipGetLastError();
}

}  // namespace convsel
