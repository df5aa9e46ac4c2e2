// Attention of new queries over the 8-bit paged cache.
#include <stdio.h>

#include "lm_common.hpp"
#include "lm_kernels.hpp"

namespace convsel {
namespace {

using namespace lm;

// One wave per (query, head): the running maximum and sum of the softmax over
// the keys one by one, four head columns a lane.
template <typename T>
__global__ __launch_bounds__(64) void attention_row_kernel(const T* q, convsel_kv_cache_t c, convsel_kv_batch_t b,
                                                           T* y, convsel_attention_desc_t a) {
  const int lane = threadIdx.x, seq = blockIdx.z, hq = blockIdx.y;
  const int head = hq / (a.q_heads / c.kv_heads);
  const Span sp = span_of(b.offsets, seq, static_cast<int>(b.tokens));
  const int ps = c.page_size, D = c.head_dim, dp = kv_row_bytes(D);
  const int64_t len = b.lengths[seq];
  const int64_t limit = min(len, b.table_width * ps);
  for (int i = blockIdx.x; i < sp.count; i += gridDim.x) {
    const int64_t p = len - sp.count + i;
    int64_t lo = 0, hi = limit;
    if (a.causal) hi = min(hi, p + 1);
    if (a.window > 0) lo = max(lo, p - a.window + 1);
    float qv[4], o[4] = {0.f, 0.f, 0.f, 0.f};
    const T* qr = q + static_cast<int64_t>(sp.first + i) * a.q_token_stride + hq * a.q_head_stride;
    for (int u = 0; u < 4; ++u) qv[u] = lane + 64 * u < D ? elem<T>::load(qr + lane + 64 * u) : 0.f;
    float m = -__builtin_inff(), l = 0.f;
    for (int64_t j = lo; j < hi; ++j) {
      const int64_t page = b.table[seq * b.table_width + j / ps];
      if (page < 0 || page >= c.pages) continue;
      const int t = static_cast<int>(j % ps);
      const int64_t ph = page * c.kv_heads + head;
      const uint8_t* kc = reinterpret_cast<const uint8_t*>(c.k_codes) + ph * (ps * dp);
      const uint8_t* vc = reinterpret_cast<const uint8_t*>(c.v_codes) + ph * (ps * dp);
      float s = 0.f;
      for (int u = 0; u < 4; ++u)
        if (lane + 64 * u < D) s += qv[u] * decode(kc[t * dp + lane + 64 * u], c.format);
#pragma unroll
      for (int x = 32; x > 0; x >>= 1) s += __shfl_xor(s, x);
      // The maximum runs over weight times value scale, so that a page of small values may hold the weight.  It and
      // the scale's exponent are whole numbers: their difference is exact, and the fused product rounds once.
      int ve;
      const float vf = frexpf(c.v_scales[ph], &ve);
      const float sk = s * c.k_scales[ph], c2 = a.scale * 1.4426950408889634f;
      const float mn = fmaxf(m, ceilf(sk * c2) + ve);
      const float f = exp2f(m - mn), u2 = exp2f(fmaf(sk, c2, ve - mn)), ev = u2 * vf;
      l = l * f + ldexpf(u2, -ve);
      m = mn;
      for (int u = 0; u < 4; ++u)
        if (lane + 64 * u < D) o[u] = o[u] * f + ev * decode(vc[v_byte(t, lane + 64 * u, dp)], c.format);
    }
    T* yr = y + static_cast<int64_t>(sp.first + i) * a.y_token_stride + hq * a.y_head_stride;
    const float inv = l != 0.f ? 1.f / l : 0.f;
    for (int u = 0; u < 4; ++u)
      if (lane + 64 * u < D) elem<T>::store(yr + lane + 64 * u, o[u] * inv);
  }
}

}  // namespace

size_t attention_workspace(const convsel_kv_cache_t&, const convsel_kv_batch_t&, const convsel_attention_desc_t&) {
  return 0;
}

hipError_t launch_attention(const void* q, const convsel_kv_cache_t& c, const convsel_kv_batch_t& b, void* y,
                            const convsel_attention_desc_t& d, void*, hipStream_t stream) {
  for (int64_t s0 = 0; s0 < b.seqs; s0 += 65535) {
    convsel_kv_batch_t p = b;
    p.seqs = b.seqs - s0 < 65535 ? b.seqs - s0 : 65535;
    p.table += s0 * b.table_width;
    p.lengths += s0;
    p.offsets += s0;
    const int64_t rows = (b.tokens + b.seqs - 1) / b.seqs;
    const dim3 grid((unsigned)(rows < 65536 ? rows : 65536), d.q_heads, (unsigned)p.seqs);
    if (d.dtype == CONV_F32)
      hipLaunchKernelGGL(attention_row_kernel<float>, grid, dim3(64), 0, stream, (const float*)q, c, p, (float*)y, d);
    else
      hipLaunchKernelGGL(attention_row_kernel<bf16_t>, grid, dim3(64), 0, stream, (const bf16_t*)q, c, p, (bf16_t*)y,
                         d);
  }
  return hipGetLastError();
}

void attention_describe(const convsel_kv_cache_t&, const convsel_kv_batch_t&, const convsel_attention_desc_t&,
                        char* buf, size_t len) {
  snprintf(buf, len, "attention kernels=attention_row_kernel workspace=0");
}

}  // namespace convsel
