// Entry points of the decoder operators (declared in include/convsel_lm.h):
// every check of descriptors, pointers, strides, overlaps and workspace runs on
// the host before the first HIP call, then the kernel launchers run.
#include <math.h>
#include <string.h>

#include "lm_kernels.hpp"

namespace convsel {
conv_status_t device_ready();  // api.hip
}

namespace {

constexpr int64_t kInt31 = ((int64_t)1 << 31) - 1;
constexpr int64_t kStrideMax = (int64_t)1 << 40;
constexpr int64_t kReachMax = (int64_t)1 << 45;  // of n rows, in elements: no memory holds it, and bytes stay below 2^63
constexpr int64_t kOutputsMax = (int64_t)1 << 35;
constexpr int64_t kAttentionRowsMax = ((int64_t)1 << 31) - ((int64_t)1 << 20);

conv_status_t from_hip(hipError_t e) {
  if (e == hipSuccess) return CONV_OK;
  (void)hipGetLastError();
  return CONV_ERR_DEVICE;
}

bool dtype_ok(int32_t t) { return t == CONV_F32 || t == CONV_BF16; }
int64_t esize(int32_t t) { return t == CONV_F32 ? 4 : 2; }
bool flag_ok(int32_t f) { return f == 0 || f == 1; }

bool aligned(const void* p, int64_t a) { return (uintptr_t)p % (uintptr_t)a == 0; }

bool overlaps(const void* a, int64_t na, const void* b, int64_t nb) {
  if (!a || !b || na <= 0 || nb <= 0) return false;
  const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
  return a0 < b0 + (uintptr_t)nb && b0 < a0 + (uintptr_t)na;
}

// Bytes from the first element to behind the last of n0 x n1 rows of `inner`.
int64_t span(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t inner, int64_t es) {
  return ((n0 - 1) * s0 + (n1 - 1) * s1 + inner) * es;
}

// A stride of n rows.
bool stride_ok(int64_t s, int64_t n) { return s >= 0 && s <= kStrideMax && (n < 2 || s <= kReachMax / (n - 1)); }

// No two of the n0 x n1 rows of `inner` elements share an element.
bool rows_apart(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t inner) {
  if (n0 == 1) return n1 == 1 || s1 >= inner;
  if (n1 == 1) return s0 >= inner;
  if (s0 < s1) return s0 >= inner && s1 >= (n0 - 1) * s0 + inner;
  return s1 >= inner && s0 >= (n1 - 1) * s1 + inner;
}

// n0 x n1 rows of `inner` bytes, strides in bytes.
struct Rows {
  const void* base;
  int64_t n0, s0, n1, s1, inner;
};
Rows run_of(const void* p, int64_t bytes) { return {p, 1, 0, 1, 0, bytes}; }

bool same_rows(const Rows& a, const Rows& b) {
  return a.base == b.base && (a.n0 == 1 || a.s0 == b.s0) && (a.n1 == 1 || a.s1 == b.s1);
}

// Whether rows of a and b have a byte in common; rows that only interleave (slices of one projection) have none.  The
// distance of two rows is the bases' plus a whole multiple, within bounds, of each stride; equal strides of a and b make
// one such term.  All terms but the one of most multiples are gone through, that one is solved for.
bool share_bytes(const Rows& a, const Rows& b) {
  if (!a.base || !b.base) return false;
  if (!overlaps(a.base, span(a.n0, a.s0, a.n1, a.s1, a.inner, 1), b.base, span(b.n0, b.s0, b.n1, b.s1, b.inner, 1)))
    return false;
  struct Term {
    int64_t stride, lo, hi;
  } t[4];
  int n = 0;
  auto add = [&](int64_t count, int64_t stride, int sign) {
    if (count == 1 || stride == 0) return;
    int i = 0;
    while (i < n && t[i].stride != stride) ++i;
    if (i == n) t[n++] = {stride, 0, 0};
    (sign > 0 ? t[i].hi : t[i].lo) += sign * (count - 1);
  };
  add(a.n0, a.s0, 1);
  add(a.n1, a.s1, 1);
  add(b.n0, b.s0, -1);
  add(b.n1, b.s1, -1);
  const int64_t d0 = (int64_t)((uintptr_t)a.base - (uintptr_t)b.base);
  // Rows meet where -a.inner < distance < b.inner.
  if (n == 0) return d0 > -a.inner && d0 < b.inner;
  int last = 0;
  for (int i = 1; i < n; ++i)
    if (t[i].hi - t[i].lo > t[last].hi - t[last].lo) last = i;
  const Term most = t[last];
  t[last] = t[--n];
  double walks = 1;
  for (int i = 0; i < n; ++i) walks *= (double)(t[i].hi - t[i].lo + 1);
  if (walks > 1 << 20) return true;  // three strides of many rows each, within one another's span: taken to meet
  int64_t k[3] = {};
  for (int i = 0; i < n; ++i) k[i] = t[i].lo;
  for (;;) {
    int64_t d = d0 + most.lo * most.stride;
    for (int i = 0; i < n; ++i) d += k[i] * t[i].stride;
    // The first multiple that brings the distance above -a.inner.
    const int64_t up = -a.inner + 1 - d, m = up <= 0 ? 0 : (up + most.stride - 1) / most.stride;
    if (m <= most.hi - most.lo && d + m * most.stride < b.inner) return true;
    int i = 0;
    for (; i < n && k[i] == t[i].hi; ++i) k[i] = t[i].lo;
    if (i == n) return false;
    ++k[i];
  }
}

// ---- linear ----

conv_status_t linear_sizes(const convsel_linear_desc_t* d) {
  if (!d || d->m < 0 || d->in_features < 1 || d->out_features < 1) return CONV_ERR_INVALID_ARG;
  if (d->m > kInt31 || d->in_features > kInt31 || d->out_features >= ((int64_t)1 << 26)) return CONV_ERR_INVALID_ARG;
  if (d->m > 0 && d->out_features > kOutputsMax / d->m) return CONV_ERR_INVALID_ARG;
  if (!dtype_ok(d->dtype) || d->act < CONVSEL_ACT_NONE || d->act > CONVSEL_ACT_SILU) return CONV_ERR_INVALID_ARG;
  if (!flag_ok(d->has_bias) || !flag_ok(d->has_residual)) return CONV_ERR_INVALID_ARG;
  if (d->ldx < d->in_features || !stride_ok(d->ldx, d->m) || d->ldy < d->out_features || !stride_ok(d->ldy, d->m))
    return CONV_ERR_INVALID_ARG;
  if (d->has_residual && (d->ldr < d->out_features || !stride_ok(d->ldr, d->m))) return CONV_ERR_INVALID_ARG;
  return CONV_OK;
}

convsel::LinearArgs linear_args(const convsel_linear_desc_t* d, const void* x, const void* w, const void* b,
                                const void* r, void* y) {
  convsel::LinearArgs a;
  a.x = x; a.w = w; a.b = b; a.r = r; a.y = y;
  a.m = d->m; a.in = d->in_features; a.out = d->out_features;
  a.ldx = d->ldx; a.ldr = d->ldr; a.ldy = d->ldy;
  a.dtype = d->dtype; a.act = d->act;
  return a;
}

// ---- cache ----

conv_status_t cache_sizes(const convsel_kv_cache_t* c) {
  if (!c || c->pages < 1 || c->pages > kInt31 || c->kv_heads < 1 || c->kv_heads > 32767) return CONV_ERR_INVALID_ARG;
  if (c->head_dim < 1 || c->head_dim > 256) return CONV_ERR_INVALID_ARG;
  if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128)
    return CONV_ERR_INVALID_ARG;
  if (c->format != CONVSEL_KV_INT8 && c->format != CONVSEL_KV_FP8) return CONV_ERR_INVALID_ARG;
  return CONV_OK;
}

int64_t code_bytes(const convsel_kv_cache_t* c) {
  return c->pages * c->kv_heads * c->page_size * convsel::kv_row_bytes(c->head_dim);
}

conv_status_t cache_pointers(const convsel_kv_cache_t* c) {
  if (!c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales) return CONV_ERR_INVALID_ARG;
  if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_scales, 4) || !aligned(c->v_scales, 4))
    return CONV_ERR_INVALID_ARG;
  return CONV_OK;
}

conv_status_t batch_sizes(const convsel_kv_cache_t* c, const convsel_kv_batch_t* b) {
  if (!b || b->seqs < 0 || b->seqs > kInt31 || b->tokens < 0 || b->tokens > kInt31) return CONV_ERR_INVALID_ARG;
  if (b->table_width < 0 || b->table_width > ((int64_t)1 << 30) / c->page_size) return CONV_ERR_INVALID_ARG;
  return CONV_OK;
}

conv_status_t batch_pointers(const convsel_kv_batch_t* b) {
  if ((!b->table && b->table_width > 0) || !b->lengths || !b->offsets) return CONV_ERR_INVALID_ARG;
  if (!aligned(b->table, 4) || !aligned(b->lengths, 4) || !aligned(b->offsets, 4)) return CONV_ERR_INVALID_ARG;
  return CONV_OK;
}

bool hits_cache(const void* p, int64_t bytes, const convsel_kv_cache_t* c) {
  const int64_t codes = code_bytes(c), scales = c->pages * c->kv_heads * 4;
  return overlaps(p, bytes, c->k_codes, codes) || overlaps(p, bytes, c->v_codes, codes) ||
         overlaps(p, bytes, c->k_scales, scales) || overlaps(p, bytes, c->v_scales, scales);
}

bool hits_batch(const void* p, int64_t bytes, const convsel_kv_batch_t* b) {
  return overlaps(p, bytes, b->table, b->seqs * b->table_width * 4) || overlaps(p, bytes, b->lengths, b->seqs * 4) ||
         overlaps(p, bytes, b->offsets, (b->seqs + 1) * 4);
}

conv_status_t attention_sizes(const convsel_kv_cache_t* c, const convsel_kv_batch_t* b,
                              const convsel_attention_desc_t* d) {
  conv_status_t st = cache_sizes(c);
  if (st == CONV_OK) st = batch_sizes(c, b);
  if (st != CONV_OK) return st;
  if (!d || d->q_heads < 1 || d->q_heads > 65535 || d->q_heads % c->kv_heads != 0) return CONV_ERR_INVALID_ARG;
  // Rows are counted in 32 bits, and rounded up to tiles of them.
  if (b->tokens > kAttentionRowsMax / d->q_heads) return CONV_ERR_INVALID_ARG;
  if (!dtype_ok(d->dtype) || !flag_ok(d->causal) || d->window < 0 || !isfinite(d->scale)) return CONV_ERR_INVALID_ARG;
  if (!stride_ok(d->q_token_stride, b->tokens) || !stride_ok(d->q_head_stride, d->q_heads) ||
      !stride_ok(d->y_token_stride, b->tokens) || !stride_ok(d->y_head_stride, d->q_heads))
    return CONV_ERR_INVALID_ARG;
  return CONV_OK;
}

}  // namespace

extern "C" {

conv_status_t convsel_linear_workspace_bytes(const convsel_linear_desc_t* desc, size_t* bytes) {
  const conv_status_t st = linear_sizes(desc);
  if (st != CONV_OK) return st;
  if (!bytes) return CONV_ERR_INVALID_ARG;
  *bytes = desc->m == 0 ? 0 : convsel::linear_workspace(linear_args(desc, nullptr, nullptr, nullptr, nullptr, nullptr));
  return CONV_OK;
}

conv_status_t convsel_linear(const void* x, const void* w, const void* b, const void* r, void* y,
                             const convsel_linear_desc_t* desc, void* workspace, size_t workspace_bytes,
                             void* stream) {
  conv_status_t st = linear_sizes(desc);
  if (st != CONV_OK || desc->m == 0) return st;
  if (!x || !w || !y || (desc->has_bias != 0) != (b != nullptr) || (desc->has_residual != 0) != (r != nullptr))
    return CONV_ERR_INVALID_ARG;
  const int64_t es = esize(desc->dtype), m = desc->m, in = desc->in_features, out = desc->out_features;
  if (!aligned(x, es) || !aligned(w, es) || !aligned(b, es) || !aligned(r, es) || !aligned(y, es))
    return CONV_ERR_INVALID_ARG;
  const convsel::LinearArgs a = linear_args(desc, x, w, b, r, y);
  const size_t need = convsel::linear_workspace(a);
  if (workspace_bytes < need || (need > 0 && !workspace)) return CONV_ERR_WORKSPACE;
  if (need > 0 && !aligned(workspace, 256)) return CONV_ERR_INVALID_ARG;
  const int64_t ybytes = span(m, a.ldy, 1, 0, out, es);
  if (overlaps(y, ybytes, x, span(m, a.ldx, 1, 0, in, es)) || overlaps(y, ybytes, w, out * in * es) ||
      overlaps(y, ybytes, b, b ? out * es : 0) || overlaps(y, ybytes, workspace, (int64_t)need))
    return CONV_ERR_INVALID_ARG;
  if (r && !(r == y && a.ldr == a.ldy) && overlaps(y, ybytes, r, span(m, a.ldr, 1, 0, out, es)))
    return CONV_ERR_INVALID_ARG;
  st = convsel::device_ready();
  if (st != CONV_OK) return st;
  return from_hip(convsel::launch_linear(a, workspace, (hipStream_t)stream));
}

conv_status_t convsel_linear_describe(const convsel_linear_desc_t* desc, char* buf, size_t len) {
  const conv_status_t st = linear_sizes(desc);
  if (st != CONV_OK) return st;
  if (!buf || len == 0) return CONV_ERR_INVALID_ARG;
  convsel::linear_describe(linear_args(desc, nullptr, nullptr, nullptr, nullptr, nullptr), buf, len);
  return CONV_OK;
}

conv_status_t convsel_qk_norm_rope(const void* q, const void* k, const void* q_weight, const void* k_weight,
                                   const int32_t* positions, const float* cos, const float* sin, void* q_out,
                                   void* k_out, const convsel_qk_desc_t* desc, void* stream) {
  const convsel_qk_desc_t* d = desc;
  if (!d || d->tokens < 0 || d->tokens > kInt31 || d->q_heads < 0 || d->k_heads < 0 || d->q_heads > 65535 ||
      d->k_heads > 65535)
    return CONV_ERR_INVALID_ARG;
  if (d->head_dim < 1 || d->head_dim > 1024 || d->rotary_dim < 0 || d->rotary_dim > d->head_dim || d->rotary_dim % 2)
    return CONV_ERR_INVALID_ARG;
  if (!dtype_ok(d->dtype) || !flag_ok(d->norm) || !flag_ok(d->interleaved) || !(d->eps >= 0.f) || !isfinite(d->eps))
    return CONV_ERR_INVALID_ARG;
  if (d->rotary_dim > 0 && (d->max_position < 1 || d->max_position > kInt31)) return CONV_ERR_INVALID_ARG;
  convsel::QkArgs a;
  a.in[0] = q; a.in[1] = k;
  a.weight[0] = q_weight; a.weight[1] = k_weight;
  a.out[0] = q_out; a.out[1] = k_out;
  a.heads[0] = d->q_heads; a.heads[1] = d->k_heads;
  a.in_token[0] = d->q_token_stride; a.in_head[0] = d->q_head_stride;
  a.in_token[1] = d->k_token_stride; a.in_head[1] = d->k_head_stride;
  a.out_token[0] = d->q_out_token_stride; a.out_head[0] = d->q_out_head_stride;
  a.out_token[1] = d->k_out_token_stride; a.out_head[1] = d->k_out_head_stride;
  a.positions = positions; a.cos = cos; a.sin = sin;
  a.tokens = d->tokens; a.max_position = d->max_position;
  a.dim = d->head_dim; a.rotary = d->rotary_dim; a.dtype = d->dtype; a.norm = d->norm;
  a.interleaved = d->interleaved; a.eps = d->eps;
  const int64_t es = esize(d->dtype), t = d->tokens;
  for (int i = 0; i < 2; ++i) {
    if (!stride_ok(a.in_token[i], t) || !stride_ok(a.in_head[i], a.heads[i]) || !stride_ok(a.out_token[i], t) ||
        !stride_ok(a.out_head[i], a.heads[i]))
      return CONV_ERR_INVALID_ARG;
  }
  if (t == 0 || a.heads[0] + a.heads[1] == 0) return CONV_OK;
  if (a.rotary > 0 && (!positions || !cos || !sin || !aligned(positions, 4) || !aligned(cos, 4) || !aligned(sin, 4)))
    return CONV_ERR_INVALID_ARG;
  for (int i = 0; i < 2; ++i) {
    if (a.heads[i] == 0) continue;
    if (!a.in[i] || !a.out[i] || !aligned(a.in[i], es) || !aligned(a.out[i], es) || !aligned(a.weight[i], es))
      return CONV_ERR_INVALID_ARG;
    if (!rows_apart(t, a.out_token[i], a.heads[i], a.out_head[i], a.dim)) return CONV_ERR_INVALID_ARG;
  }
  // What is written may be a head's own input, and nothing else that the call reads or writes.
  Rows in[2], out[2];
  for (int i = 0; i < 2; ++i) {
    const bool there = a.heads[i] > 0;
    in[i] = {there ? a.in[i] : nullptr, t, a.in_token[i] * es, a.heads[i], a.in_head[i] * es, a.dim * es};
    out[i] = {there ? a.out[i] : nullptr, t, a.out_token[i] * es, a.heads[i], a.out_head[i] * es, a.dim * es};
  }
  const int64_t table = a.rotary > 0 ? a.max_position * (a.rotary / 2) * 4 : 0;
  for (int i = 0; i < 2; ++i) {
    if (!same_rows(out[i], in[i]) && share_bytes(out[i], in[i])) return CONV_ERR_INVALID_ARG;
    if (share_bytes(out[i], in[1 - i])) return CONV_ERR_INVALID_ARG;
    for (int j = 0; j < 2; ++j)
      if (a.heads[j] > 0 && share_bytes(out[i], run_of(a.weight[j], a.dim * es))) return CONV_ERR_INVALID_ARG;
    if (table > 0 && (share_bytes(out[i], run_of(cos, table)) || share_bytes(out[i], run_of(sin, table)) ||
                      share_bytes(out[i], run_of(positions, t * 4))))
      return CONV_ERR_INVALID_ARG;
  }
  if (share_bytes(out[0], out[1])) return CONV_ERR_INVALID_ARG;
  const conv_status_t st = convsel::device_ready();
  if (st != CONV_OK) return st;
  return from_hip(convsel::launch_qk_norm_rope(a, (hipStream_t)stream));
}

conv_status_t convsel_kv_cache_bytes(const convsel_kv_cache_t* cache, size_t* bytes) {
  const conv_status_t st = cache_sizes(cache);
  if (st != CONV_OK) return st;
  if (!bytes) return CONV_ERR_INVALID_ARG;
  *bytes = (size_t)code_bytes(cache);
  return CONV_OK;
}

conv_status_t convsel_kv_write(const convsel_kv_cache_t* cache, const convsel_kv_batch_t* batch, const void* k,
                               const void* v, int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                               int64_t v_head_stride, int32_t dtype, void* stream) {
  conv_status_t st = cache_sizes(cache);
  if (st == CONV_OK) st = batch_sizes(cache, batch);
  if (st != CONV_OK) return st;
  if (!dtype_ok(dtype) || !stride_ok(k_token_stride, batch->tokens) || !stride_ok(k_head_stride, cache->kv_heads) ||
      !stride_ok(v_token_stride, batch->tokens) || !stride_ok(v_head_stride, cache->kv_heads))
    return CONV_ERR_INVALID_ARG;
  if (batch->seqs == 0 || batch->tokens == 0 || batch->table_width == 0) return CONV_OK;
  st = cache_pointers(cache);
  if (st == CONV_OK) st = batch_pointers(batch);
  if (st != CONV_OK) return st;
  const int64_t es = esize(dtype);
  if (!k || !v || !aligned(k, es) || !aligned(v, es)) return CONV_ERR_INVALID_ARG;
  if (hits_cache(k, span(batch->tokens, k_token_stride, cache->kv_heads, k_head_stride, cache->head_dim, es), cache) ||
      hits_cache(v, span(batch->tokens, v_token_stride, cache->kv_heads, v_head_stride, cache->head_dim, es), cache))
    return CONV_ERR_INVALID_ARG;
  st = convsel::device_ready();
  if (st != CONV_OK) return st;
  const convsel::KvTokens t = {k, v, k_token_stride, k_head_stride, v_token_stride, v_head_stride, dtype};
  return from_hip(convsel::launch_kv_write(*cache, *batch, t, (hipStream_t)stream));
}

conv_status_t convsel_kv_read(const convsel_kv_cache_t* cache, const convsel_kv_batch_t* batch, void* k, void* v,
                              int32_t dtype, void* stream) {
  conv_status_t st = cache_sizes(cache);
  if (st == CONV_OK) st = batch_sizes(cache, batch);
  if (st != CONV_OK) return st;
  if (!dtype_ok(dtype)) return CONV_ERR_INVALID_ARG;
  if (batch->seqs == 0 || batch->tokens == 0) return CONV_OK;
  st = cache_pointers(cache);
  if (st == CONV_OK) st = batch_pointers(batch);
  if (st != CONV_OK) return st;
  const int64_t es = esize(dtype), bytes = batch->tokens * cache->kv_heads * cache->head_dim * es;
  if (!k || !v || !aligned(k, es) || !aligned(v, es) || overlaps(k, bytes, v, bytes)) return CONV_ERR_INVALID_ARG;
  if (hits_cache(k, bytes, cache) || hits_cache(v, bytes, cache) || hits_batch(k, bytes, batch) ||
      hits_batch(v, bytes, batch))
    return CONV_ERR_INVALID_ARG;
  st = convsel::device_ready();
  if (st != CONV_OK) return st;
  const convsel::KvTokens t = {k, v, 0, 0, 0, 0, dtype};
  return from_hip(convsel::launch_kv_read(*cache, *batch, t, (hipStream_t)stream));
}

conv_status_t convsel_attention_workspace_bytes(const convsel_kv_cache_t* cache, const convsel_kv_batch_t* batch,
                                                const convsel_attention_desc_t* desc, size_t* bytes) {
  const conv_status_t st = attention_sizes(cache, batch, desc);
  if (st != CONV_OK) return st;
  if (!bytes) return CONV_ERR_INVALID_ARG;
  *bytes = batch->seqs == 0 || batch->tokens == 0 ? 0 : convsel::attention_workspace(*cache, *batch, *desc);
  return CONV_OK;
}

conv_status_t convsel_attention(const void* q, const convsel_kv_cache_t* cache, const convsel_kv_batch_t* batch,
                                void* y, const convsel_attention_desc_t* desc, void* workspace,
                                size_t workspace_bytes, void* stream) {
  conv_status_t st = attention_sizes(cache, batch, desc);
  if (st != CONV_OK) return st;
  if (batch->seqs == 0 || batch->tokens == 0) return CONV_OK;
  st = cache_pointers(cache);
  if (st == CONV_OK) st = batch_pointers(batch);
  if (st != CONV_OK) return st;
  const int64_t es = esize(desc->dtype), t = batch->tokens, h = desc->q_heads, d = cache->head_dim;
  if (!q || !y || !aligned(q, es) || !aligned(y, es)) return CONV_ERR_INVALID_ARG;
  if (!rows_apart(t, desc->y_token_stride, h, desc->y_head_stride, d)) return CONV_ERR_INVALID_ARG;
  const size_t need = convsel::attention_workspace(*cache, *batch, *desc);
  if (workspace_bytes < need || (need > 0 && !workspace)) return CONV_ERR_WORKSPACE;
  if (need > 0 && !aligned(workspace, 256)) return CONV_ERR_INVALID_ARG;
  const int64_t ybytes = span(t, desc->y_token_stride, h, desc->y_head_stride, d, es);
  const int64_t qbytes = span(t, desc->q_token_stride, h, desc->q_head_stride, d, es);
  if (overlaps(y, ybytes, q, qbytes) || hits_cache(y, ybytes, cache) || hits_batch(y, ybytes, batch) ||
      overlaps(y, ybytes, workspace, (int64_t)need))
    return CONV_ERR_INVALID_ARG;
  st = convsel::device_ready();
  if (st != CONV_OK) return st;
  return from_hip(convsel::launch_attention(q, *cache, *batch, y, *desc, workspace, (hipStream_t)stream));
}

conv_status_t convsel_attention_describe(const convsel_kv_cache_t* cache, const convsel_kv_batch_t* batch,
                                         const convsel_attention_desc_t* desc, char* buf, size_t len) {
  const conv_status_t st = attention_sizes(cache, batch, desc);
  if (st != CONV_OK) return st;
  if (!buf || len == 0) return CONV_ERR_INVALID_ARG;
  convsel::attention_describe(*cache, *batch, *desc, buf, len);
  return CONV_OK;
}

}  // extern "C"
