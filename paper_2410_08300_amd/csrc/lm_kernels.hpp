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

// With `codes`, x and w are 8-bit whole numbers, their rows ldx and ldw bytes apart, with fp32 scales; dtype is then that
// of b, r and y alone, and w's rows are dense without.
struct LinearArgs {
  const void* x;
  const void* w;
  const void* b;  // or nullptr
  const void* r;  // or nullptr
  void* y;
  int64_t m, in, out;
  int64_t ldx, ldr, ldy;
  int dtype, act;
  int codes = 0;
  int64_t ldw = 0;
  const float* x_scale = nullptr;
  const float* w_scale = nullptr;
  int64_t numbers = 0;  // of a row of x that the product's kernel codes itself; `in` is then that in whole 16-byte units
};

size_t linear_workspace(const LinearArgs& a);
hipError_t launch_linear(const LinearArgs& a, void* workspace, hipStream_t stream);
void linear_describe(const LinearArgs& a, char* buf, size_t len);

// Rows of fp32 or bf16 numbers coded in 8 bits, a scale each; codes behind the row are zero up to ldc.
struct CodeArgs {
  const void* x;
  int8_t* codes;
  float* scales;
  int64_t m, in, ldx, ldc;
  int dtype;
};
hipError_t launch_quantize_rows(const CodeArgs& a, hipStream_t stream);

// The same product on codes; x's rows are fp32 or bf16 (x_dtype) and coded on the way, or codes already (-1).
size_t linear_int8_workspace(const LinearArgs& a, int x_dtype);
hipError_t launch_linear_int8(const LinearArgs& a, int x_dtype, void* workspace, hipStream_t stream);
void linear_int8_describe(const LinearArgs& a, int x_dtype, char* buf, size_t len);

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

// Attention of packed prompts over their own keys and values.
struct PromptArgs {
  const void* q;
  const void* k;
  const void* v;
  const int32_t* offsets;
  void* y;
  int64_t seqs, tokens;
  int64_t q_token, q_head, k_token, k_head, v_token, v_head, y_token, y_head;
  int q_heads, kv_heads, dim, dtype, causal, window;
  float scale;
};

size_t prompt_attention_workspace(const PromptArgs& a);
hipError_t launch_prompt_attention(const PromptArgs& a, void* workspace, hipStream_t stream);
void prompt_attention_describe(const PromptArgs& a, char* buf, size_t len);

struct LogitsArgs {
  const void* x;
  const int32_t* history;  // or nullptr, as what follows
  const int32_t* offsets;
  const int32_t* prompt_lengths;
  const float* repetition;
  const float* presence;
  const float* frequency;
  const float* bias;
  const uint32_t* mask;
  void* y;
  int64_t rows, vocab, tokens;
  int64_t ldx, ldy, ldbias, ldmask;
  int dtype;
};
hipError_t launch_adjust_logits(const LogitsArgs& a, hipStream_t stream);

}  // namespace convsel
