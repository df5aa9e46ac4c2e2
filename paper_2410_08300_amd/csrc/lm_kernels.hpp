// Host-side interface between the entry points of the decoder operators
// (lm_api.hip, declared in include/convsel_lm.h) and their kernel launchers.
// Arguments are validated by the caller; every launcher enqueues on `stream`
// and returns the HIP status of its last launch.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/convsel_lm.h"

namespace convsel {

struct LinearArgs {
  const void* x;
  const void* w;
  const void* b;  // or nullptr
  const void* r;  // or nullptr
  void* y;
  int64_t m, in, out;
  int64_t ldx, ldr, ldy;
  int dtype, act;
};

size_t linear_workspace(const LinearArgs& a);
hipError_t launch_linear(const LinearArgs& a, void* workspace, hipStream_t stream);
void linear_describe(const LinearArgs& a, char* buf, size_t len);

struct QkArgs {
  const void* in[2];  // q, k
  const void* weight[2];
  void* out[2];
  int heads[2];
  int64_t in_token[2], in_head[2], out_token[2], out_head[2];
  const int32_t* positions;
  const float* cos;
  const float* sin;
  int64_t tokens, max_position;
  int dim, rotary, dtype, norm, interleaved;
  float eps;
};

hipError_t launch_qk_norm_rope(const QkArgs& a, hipStream_t stream);

// Bytes of one page's codes of one head, and of a row of it.
__host__ __device__ inline int kv_row_bytes(int head_dim) { return (head_dim + 31) / 32 * 32; }

struct KvTokens {
  const void* k;  // write: sources; read: destinations (cast)
  const void* v;
  int64_t k_token, k_head, v_token, v_head;
  int dtype;
};

hipError_t launch_kv_write(const convsel_kv_cache_t& c, const convsel_kv_batch_t& b, const KvTokens& t,
                           hipStream_t stream);
hipError_t launch_kv_read(const convsel_kv_cache_t& c, const convsel_kv_batch_t& b, const KvTokens& t,
                          hipStream_t stream);

size_t attention_workspace(const convsel_kv_cache_t& c, const convsel_kv_batch_t& b,
                           const convsel_attention_desc_t& d);
hipError_t launch_attention(const void* q, const convsel_kv_cache_t& c, const convsel_kv_batch_t& b, void* y,
                            const convsel_attention_desc_t& d, void* workspace, hipStream_t stream);
void attention_describe(const convsel_kv_cache_t& c, const convsel_kv_batch_t& b, const convsel_attention_desc_t& d,
                        char* buf, size_t len);

}  // namespace convsel
