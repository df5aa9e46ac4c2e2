// Writing tokens into the 8-bit paged cache and reading them back.
#include "lm_common.hpp"
#include "lm_kernels.hpp"

namespace convsel {
namespace {

using namespace lm;

// One workgroup per (page of a sequence, head, keys or values): the largest
// magnitude of the page's new tokens, the scale, then the codes.  Every
// 4-byte word of codes belongs to one thread, which keeps the bytes that the
// call does not write.
template <typename T>
__global__ __launch_bounds__(256) void kv_write_kernel(convsel_kv_cache_t c, convsel_kv_batch_t b, KvTokens in) {
  const int seq = blockIdx.z;
  const bool values = blockIdx.y >= static_cast<unsigned>(c.kv_heads);
  const int head = values ? blockIdx.y - c.kv_heads : blockIdx.y;
  const Span sp = span_of(b.offsets, seq, static_cast<int>(b.tokens));
  const int ps = c.page_size, D = c.head_dim, dp = kv_row_bytes(D);
  const int64_t start = b.lengths[seq] < 0 ? 0 : b.lengths[seq];
  const int64_t end = min(start + sp.count, b.table_width * ps);
  if (start >= end) return;
  const int64_t token = values ? in.v_token : in.k_token;
  const T* src0 = reinterpret_cast<const T*>(values ? in.v : in.k) +
                  head * (values ? in.v_head : in.k_head) + sp.first * token;
  __shared__ float red[4];
  for (int64_t pg = start / ps + blockIdx.x; pg * ps < end; pg += gridDim.x) {
    const int64_t page = b.table[seq * b.table_width + pg];
    if (page < 0 || page >= c.pages) continue;
    const int r0 = static_cast<int>(max(start - pg * ps, (int64_t)0));
    const int r1 = static_cast<int>(min(end - pg * ps, (int64_t)ps));
    const T* src = src0 + (pg * ps - start) * token;  // row r of the page is src + r * token
    float amax = 0.f;
    for (int i = threadIdx.x; i < (r1 - r0) * D; i += 256) {
      const float v = fabsf(elem<T>::load(src + (r0 + i / D) * token + i % D));
      if (v < __builtin_inff()) amax = fmaxf(amax, v);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = amax;
    __syncthreads();
    amax = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    float* scale_at = (values ? c.v_scales : c.k_scales) + page * c.kv_heads + head;
    const float old = *scale_at;
    float scale = fmaxf(amax / qmax_of(c.format), kMinScale);
    if (r0 > 0) scale = fmaxf(scale, old);
    const bool grown = r0 > 0 && scale != old;
    __syncthreads();
    if (threadIdx.x == 0) *scale_at = scale;
    uint8_t* codes = reinterpret_cast<uint8_t*>(values ? c.v_codes : c.k_codes) +
                     (page * c.kv_heads + head) * static_cast<int64_t>(ps * dp);
    auto code_at = [&](int t, int d, uint32_t held) -> uint32_t {
      if (t >= r1 || (t < r0 && !grown)) return held;
      if (t < r0) return encode(decode(held, c.format) * old, scale, c.format);
      return d < D ? encode(elem<T>::load(src + t * token + d), scale, c.format) : 0u;
    };
    const int from = grown ? 0 : r0;
    if (!values) {
      const int words = dp / 4;
      for (int i = threadIdx.x; i < (r1 - from) * words; i += 256) {
        const int t = from + i / words, d = i % words * 4;
        uint32_t* at = reinterpret_cast<uint32_t*>(codes + t * dp + d);
        const uint32_t held = t < r0 ? *at : 0u;
        uint32_t w = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) w |= code_at(t, d + j, (held >> (8 * j)) & 0xffu) << (8 * j);
        *at = w;
      }
    } else {
      const int t4 = from >> 2;
      for (int i = threadIdx.x; i < ((r1 + 3) / 4 - t4) * dp; i += 256) {
        const int t = (t4 + i / dp) * 4, d = i % dp;
        uint32_t* at = reinterpret_cast<uint32_t*>(codes + v_byte(t, d, dp));
        const uint32_t held = t < r0 || t + 4 > r1 ? *at : 0u;
        uint32_t w = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) w |= code_at(t + j, d, (held >> (8 * j)) & 0xffu) << (8 * j);
        *at = w;
      }
    }
  }
}

// One workgroup per (16 positions of a sequence, head), positions aligned to
// the cache's 16-token blocks.
template <typename T>
__global__ __launch_bounds__(256) void kv_read_kernel(convsel_kv_cache_t c, convsel_kv_batch_t b, T* k, T* v) {
  const int seq = blockIdx.z, head = blockIdx.y;
  const Span sp = span_of(b.offsets, seq, static_cast<int>(b.tokens));
  const int ps = c.page_size, D = c.head_dim, dp = kv_row_bytes(D);
  const int64_t start = b.lengths[seq], end = start + sp.count;  // 64-bit: bounded below
  const int64_t row = static_cast<int64_t>(c.kv_heads) * D;
  // Floor division: a negative start names positions before the sequence.
  const int64_t first = start >= 0 ? start / 16 : -((-start + 15) / 16);
  for (int64_t blk = first + blockIdx.x; blk * 16 < end; blk += gridDim.x) {
    const int64_t p0 = blk * 16;
    int64_t page = -1;
    if (p0 >= 0 && p0 / ps < b.table_width) page = b.table[seq * b.table_width + p0 / ps];
    const bool there = page >= 0 && page < c.pages;
    const int t0 = static_cast<int>(there ? p0 % ps : 0);
    const int64_t ph = there ? page * c.kv_heads + head : 0;
    const uint8_t* kc = reinterpret_cast<const uint8_t*>(c.k_codes) + ph * (ps * dp) + t0 * dp;
    const uint8_t* vc = reinterpret_cast<const uint8_t*>(c.v_codes) + ph * (ps * dp) + t0 * dp;
    const float ks = there ? c.k_scales[ph] : 0.f, vs = there ? c.v_scales[ph] : 0.f;
    for (int i = threadIdx.x; i < 16 * D; i += 256) {
      const int t = i / D, d = i % D;
      const int64_t p = p0 + t;
      if (p < start || p >= end) continue;
      const int64_t at = (sp.first + (p - start)) * row + static_cast<int64_t>(head) * D + d;
      elem<T>::store(k + at, there ? decode(kc[t * dp + d], c.format) * ks : 0.f);
      elem<T>::store(v + at, there ? decode(vc[v_byte(t, d, dp)], c.format) * vs : 0.f);
    }
  }
}

}  // namespace

hipError_t launch_kv_write(const convsel_kv_cache_t& c, const convsel_kv_batch_t& b, const KvTokens& t,
                           hipStream_t stream) {
  // Sequences past the grid's 65535 go in further launches.
  for (int64_t s0 = 0; s0 < b.seqs; s0 += 65535) {
    convsel_kv_batch_t p = b;
    p.seqs = b.seqs - s0 < 65535 ? b.seqs - s0 : 65535;
    p.table += s0 * b.table_width;
    p.lengths += s0;
    p.offsets += s0;
    const int64_t pages = (b.tokens + b.seqs - 1) / b.seqs / c.page_size + 2;
    const dim3 grid((unsigned)(pages < 65536 ? pages : 65536), 2 * c.kv_heads, (unsigned)p.seqs);
    if (t.dtype == CONV_F32)
      hipLaunchKernelGGL(kv_write_kernel<float>, grid, dim3(256), 0, stream, c, p, t);
    else
      hipLaunchKernelGGL(kv_write_kernel<bf16_t>, grid, dim3(256), 0, stream, c, p, t);
  }
  return hipGetLastError();
}

hipError_t launch_kv_read(const convsel_kv_cache_t& c, const convsel_kv_batch_t& b, const KvTokens& t,
                          hipStream_t stream) {
  for (int64_t s0 = 0; s0 < b.seqs; s0 += 65535) {
    convsel_kv_batch_t p = b;
    p.seqs = b.seqs - s0 < 65535 ? b.seqs - s0 : 65535;
    p.table += s0 * b.table_width;
    p.lengths += s0;
    p.offsets += s0;
    const int64_t blocks = (b.tokens + b.seqs - 1) / b.seqs / 16 + 2;
    const dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536), c.kv_heads, (unsigned)p.seqs);
    if (t.dtype == CONV_F32)
      hipLaunchKernelGGL(kv_read_kernel<float>, grid, dim3(256), 0, stream, c, p, (float*)t.k, (float*)t.v);
    else
      hipLaunchKernelGGL(kv_read_kernel<bf16_t>, grid, dim3(256), 0, stream, c, p, (bf16_t*)t.k, (bf16_t*)t.v);
  }
  return hipGetLastError();
}

}  // namespace convsel
