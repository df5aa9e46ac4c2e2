/*
 * convsel decoder operators -- the pieces of a decoder (language-model) layer
 * that run beside the convolutions of convsel.h: the linear layer with a fused
 * epilogue, the norm and position rotation of query and key heads, a paged
 * key/value cache held in 8 bits, and attention over that cache; linear layers
 * whose weights are held in 8 bits, attention of prompts over their own keys and
 * values, and the adjustments of logits before a token is chosen.
 *
 * Conventions are those of convsel.h: device pointers, status codes, every
 * check of arguments on the host before the first HIP call, work enqueued on
 * `stream` (hipStream_t as void*, NULL = the default stream) without
 * synchronising, no device memory allocated inside a call, no state kept
 * between calls, nothing recorded that a HIP graph may not replay.  Element
 * types are conv_dtype_t (CONV_F32, CONV_BF16); every sum, norm and softmax
 * statistic is held in fp32 and results are rounded once, on their way out.
 * Strides are in elements; the innermost dimension is dense.  A call over no
 * tokens is a valid no-op.
 *
 * Numbers that live on the device (positions, lengths, block tables) cannot be
 * checked by the host without waiting for the GPU.  The kernels bound every
 * one of them before it becomes an address, as each entry point states.
 */
#ifndef CONVSEL_LM_H
#define CONVSEL_LM_H

#include <stddef.h>
#include <stdint.h>

#include "convsel.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- linear layer --------------------------------------------------------
 *   y[m][o] = act(sum_i x[m][i] * w[o][i] + b[o]) + r[m][o]
 * w is O x I dense; x, r and y are rows of stride ldx >= I, ldr >= O,
 * ldy >= O.  The sum, the activation and the residual add are fp32; y is
 * rounded once.  gelu is z * Phi(z) (erf), gelu_tanh its tanh form, silu
 * z / (1 + exp(-z)). */
typedef enum convsel_act {
  CONVSEL_ACT_NONE = 0,
  CONVSEL_ACT_RELU = 1,
  CONVSEL_ACT_GELU = 2,
  CONVSEL_ACT_GELU_TANH = 3,
  CONVSEL_ACT_SILU = 4
} convsel_act_t;

typedef struct convsel_linear_desc {
  int64_t m, in_features, out_features;  /* out_features < 2^26, m * out_features <= 2^35 */
  int64_t ldx, ldr, ldy;  /* ldr is read only with a residual */
  int32_t dtype;          /* conv_dtype_t of x, w, b, r and y */
  int32_t act;            /* convsel_act_t */
  int32_t has_bias;       /* 0: b must be NULL; 1: b holds O values */
  int32_t has_residual;   /* 0: r must be NULL */
} convsel_linear_desc_t;

/* Device bytes the call needs as workspace (0: none; else 256-byte aligned). */
conv_status_t convsel_linear_workspace_bytes(const convsel_linear_desc_t* desc, size_t* bytes);

/* Any alignment of elements is served; more than 16 rows run fastest where x
 * and w start on 16 bytes.  y may be r itself (same address and stride: the
 * residual is updated in place); otherwise the span of y, first to last
 * element, must not overlap that of x, w, b or r.  INVALID_ARG for a malformed
 * descriptor, a NULL or overlapping pointer, a pointer not aligned to its
 * element; WORKSPACE for too little of it. */
conv_status_t convsel_linear(const void* x, const void* w, const void* b, const void* r, void* y,
                             const convsel_linear_desc_t* desc, void* workspace, size_t workspace_bytes,
                             void* stream);

/* One line: kernel, tile, grid, split and workspace of the call. */
conv_status_t convsel_linear_describe(const convsel_linear_desc_t* desc, char* buf, size_t len);

/* ---- norm and rotation of query and key heads ------------------------------
 * For every token t and every head of q and of k, x = its head_dim values:
 *   norm 1 (RMS):  z_d = x_d / sqrt(mean_d x_d^2 + eps) * weight_d
 *   norm 0:        z_d = x_d * weight_d
 * (weight NULL: ones), then the first rotary_dim = R values are rotated by
 * the angle whose cosine and sine are cos[p][i], sin[p][i], p = positions[t],
 * i < R/2, fp32 tables of max_position rows of R/2:
 *   a' = a cos - b sin,   b' = b cos + a sin
 * for the pairs (a, b) = (z_i, z_{i+R/2}), or (z_{2i}, z_{2i+1}) with
 * `interleaved`.  R = 0 rotates nothing (positions, cos and sin are ignored).
 * One pass over q and k.
 *
 * A token whose position lies outside [0, max_position) is written as NaN.
 * q_out may be q (same address and strides), k_out may be k.  Beyond that no
 * value of an output may lie where one of q, k, the weights, the tables, the
 * positions or the other output does; slices of one projection, whose rows only
 * interleave, are apart. */
typedef struct convsel_qk_desc {
  int64_t tokens;
  int32_t q_heads, k_heads;  /* either may be 0 (its pointers are then ignored) */
  int32_t head_dim;          /* 1 .. 1024 */
  int32_t rotary_dim;        /* even, <= head_dim */
  int64_t q_token_stride, q_head_stride, k_token_stride, k_head_stride;
  int64_t q_out_token_stride, q_out_head_stride, k_out_token_stride, k_out_head_stride;
  int64_t max_position;      /* rows of cos and sin */
  int32_t dtype;             /* of q, k, the weights and the outputs */
  int32_t norm;              /* 0 none, 1 RMS */
  int32_t interleaved;
  float eps;
} convsel_qk_desc_t;

conv_status_t convsel_qk_norm_rope(const void* q, const void* k, const void* q_weight, const void* k_weight,
                                   const int32_t* positions, const float* cos, const float* sin, void* q_out,
                                   void* k_out, const convsel_qk_desc_t* desc, void* stream);

/* ---- paged key/value cache in 8 bits ---------------------------------------
 * A cache is `pages` pages of page_size tokens of kv_heads heads.  A page
 * holds, for each head, the tokens' keys and values as 8-bit codes and one
 * fp32 scale for the block's keys and one for its values: value = code * scale.
 * Codes are whole numbers -127..127 (int8) or e4m3 numbers up to 448 (fp8).
 *
 * Sequence b's position p lives in page table[b][p / page_size] at row
 * p % page_size.  A table entry outside [0, pages) stands for no page: its
 * tokens are not written, read as zeros, and masked by attention (a sliding
 * window may have handed its old pages back).
 *
 * Layout of the code buffers (also what a copy or a swap to host moves; each
 * page is one contiguous piece).  With Dp = head_dim rounded up to a multiple
 * of 32, the code at page g, head h, row t, column d is byte
 *   keys:    ((g*H + h)*page_size + t)*Dp + d
 *   values:  ((g*H + h)*page_size + t/16*16)*Dp
 *            + ((t%16)/4*16 + d%16)*(Dp/4) + (d/16)*4 + t%4
 * (values lie in the order in which a wave's lanes feed them to the matrix
 * cores: no transposition while they are read).  Columns d >= head_dim hold
 * zeros.  Scales are [pages][kv_heads]. */
typedef enum convsel_kv_format {
  CONVSEL_KV_INT8 = 0,
  CONVSEL_KV_FP8 = 1 /* e4m3: 1 sign, 4 exponent (bias 7), 3 mantissa bits, no infinities */
} convsel_kv_format_t;

typedef struct convsel_kv_cache {
  int64_t pages;
  int32_t kv_heads;
  int32_t head_dim;   /* 1 .. 256 */
  int32_t page_size;  /* 16, 32, 64 or 128 */
  int32_t format;     /* convsel_kv_format_t */
  void* k_codes;      /* 16-byte aligned, convsel_kv_cache_bytes() each */
  void* v_codes;
  float* k_scales;    /* pages * kv_heads each */
  float* v_scales;
} convsel_kv_cache_t;

/* The sequences of a call.  Sequence b owns the packed tokens
 * offsets[b] .. offsets[b+1]-1 of the call's q, k, v or output (rising from 0;
 * the kernels clamp them to [0, tokens]).  No output may lie over these three. */
typedef struct convsel_kv_batch {
  int64_t seqs;
  int64_t tokens;          /* packed tokens of the call */
  int64_t table_width;     /* pages a sequence may have; * page_size <= 2^30 */
  const int32_t* table;    /* seqs x table_width */
  const int32_t* lengths;  /* seqs: what it means is said at each call */
  const int32_t* offsets;  /* seqs + 1 */
} convsel_kv_batch_t;

/* Bytes of each of the two code buffers (pointers in `cache` are not read). */
conv_status_t convsel_kv_cache_bytes(const convsel_kv_cache_t* cache, size_t* code_bytes);

/* Writes the tokens of k and v ([tokens][kv_heads][head_dim], strides given)
 * behind the lengths[b] tokens that sequence b already holds: token i of it
 * goes to position lengths[b] + i.  For each page and head, with A the largest
 * finite magnitude among the tokens written there by this call:
 *   scale = max(A / qmax, 2^-100)            (qmax 127 or 448, fp32 quotient)
 *   if the page held earlier tokens of the sequence (the first position
 *   written there is not its row 0): scale = max(scale, old scale), and where
 *   it grew, the earlier tokens are coded again from code * old scale;
 *   code  = round(x / scale)                 (fp32 quotient, ties to even)
 * Infinities become the largest code of their sign and NaN becomes 0.  Rows
 * that the call does not write keep their codes.  Positions outside the table
 * and pages outside the cache are skipped.  Two sequences of one call must not
 * write to one page. */
conv_status_t convsel_kv_write(const convsel_kv_cache_t* cache, const convsel_kv_batch_t* batch, const void* k,
                               const void* v, int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                               int64_t v_head_stride, int32_t dtype, void* stream);

/* Reads positions lengths[b] .. lengths[b] + (offsets[b+1] - offsets[b]) - 1
 * of every sequence as values: k and v are dense [tokens][kv_heads][head_dim]
 * of `dtype`.  Positions outside the table and tokens of no page are zeros. */
conv_status_t convsel_kv_read(const convsel_kv_cache_t* cache, const convsel_kv_batch_t* batch, void* k, void* v,
                              int32_t dtype, void* stream);

/* ---- attention over the cache ------------------------------------------------
 * lengths[b] is the number of tokens of sequence b in the cache, its new
 * tokens included (they have been written before).  Its n = offsets[b+1] -
 * offsets[b] queries stand at the last n positions: query i at
 * p = lengths[b] - n + i.  Head h of q reads key/value head h / (q_heads /
 * kv_heads), and
 *   y[i][h] = sum_j softmax_j(scale * q[i][h] . K[j]) V[j]
 * over the positions 0 <= j < lengths[b] with a page, with causal only
 * j <= p, and with window > 0 only j > p - window.  A row whose mask leaves
 * nothing is zero.  What lies in masked places (rows never written, pages
 * handed back) has no influence, whatever bits it holds. */
typedef struct convsel_attention_desc {
  int32_t q_heads; /* tokens * q_heads <= 2^31 - 2^20 */
  int32_t dtype;   /* of q and y */
  int32_t causal;
  int32_t window;  /* 0: none */
  float scale;     /* finite */
  int64_t q_token_stride, q_head_stride, y_token_stride, y_head_stride;
} convsel_attention_desc_t;

/* Pointers in `cache` and `batch` are not read: sizes only. */
conv_status_t convsel_attention_workspace_bytes(const convsel_kv_cache_t* cache, const convsel_kv_batch_t* batch,
                                                const convsel_attention_desc_t* desc, size_t* bytes);
conv_status_t convsel_attention(const void* q, const convsel_kv_cache_t* cache, const convsel_kv_batch_t* batch,
                                void* y, const convsel_attention_desc_t* desc, void* workspace,
                                size_t workspace_bytes, void* stream);
/* One line: kernel, rows and keys of a tile, grid, split and workspace. */
conv_status_t convsel_attention_describe(const convsel_kv_cache_t* cache, const convsel_kv_batch_t* batch,
                                         const convsel_attention_desc_t* desc, char* buf, size_t len);

/* ---- attention of prompts ----------------------------------------------------
 * The packed tokens of a call are whole sequences: sequence b owns the tokens
 * offsets[b] .. offsets[b+1]-1 of q, k, v and y (rising from 0; the kernels clamp
 * them to [0, tokens]), and no cache is read.  Head h of q reads key/value head
 * h / (q_heads / kv_heads), and for token i of a sequence of n
 *   y[i][h] = sum_j softmax_j(scale * q[i][h] . k[j]) v[j]
 * over its tokens 0 <= j < n, with causal only j <= i, and with window > 0 only
 * j > i - window.  What lies in masked places has no influence, infinities and
 * NaN included.  Rows of y behind the last sequence are left as they were. */
typedef struct convsel_prompt_desc {
  int64_t seqs, tokens;
  int32_t q_heads, kv_heads; /* tokens * q_heads <= 2^31 - 2^20 */
  int32_t head_dim;          /* 1 .. 256 */
  int32_t dtype;             /* of q, k, v and y */
  int32_t causal;
  int32_t window; /* 0: none */
  float scale;    /* of magnitude 2^127 at most */
  int64_t q_token_stride, q_head_stride, k_token_stride, k_head_stride;
  int64_t v_token_stride, v_head_stride, y_token_stride, y_head_stride;
} convsel_prompt_desc_t;

/* Device bytes the call needs as workspace (0: none; else 256-byte aligned).
 * Of q, k and v the addresses' alignment is looked at, nothing else: rows that do
 * not lie in whole 16-byte units are copied there first. */
conv_status_t convsel_prompt_attention_workspace_bytes(const void* q, const void* k, const void* v,
                                                       const convsel_prompt_desc_t* desc, size_t* bytes);
/* No value of y may lie where the call reads: q, k, v (slices whose rows only
 * interleave are apart), offsets or the workspace. */
conv_status_t convsel_prompt_attention(const void* q, const void* k, const void* v, const int32_t* offsets, void* y,
                                       const convsel_prompt_desc_t* desc, void* workspace, size_t workspace_bytes,
                                       void* stream);
/* One line: kernels, rows and keys of a tile, and workspace of the call. */
conv_status_t convsel_prompt_attention_describe(const void* q, const void* k, const void* v,
                                                const convsel_prompt_desc_t* desc, char* buf, size_t len);

/* ---- linear layer on 8-bit codes ----------------------------------------------
 * Rows of numbers are coded with a scale each: with A a row's largest finite
 * magnitude
 *   scale = max(A / 127, 2^-100)             (fp32 quotient)
 *   code  = round(x / scale)                 (fp32 quotient, ties to even)
 * Infinities become the largest code of their sign and NaN becomes 0.
 *
 * x: m rows of in_features numbers of `dtype`, ldx apart; codes: rows of ldc >=
 * in_features bytes, of which those behind the row are written as zeros; scales:
 * m values.  No output may lie over x or the other output. */
typedef struct convsel_quantize_desc {
  int64_t m, in_features;
  int64_t ldx, ldc;
  int32_t dtype;
} convsel_quantize_desc_t;

conv_status_t convsel_quantize_rows(const void* x, int8_t* codes, float* scales, const convsel_quantize_desc_t* desc,
                                    void* stream);

/*   y[m][o] = act((sum_i X[m][i] * W[o][i]) * sx[m] * sw[o] + b[o]) + r[m][o]
 * W: codes, O rows of in_features bytes, ldw apart (up to 15 bytes behind a row,
 * less where ldw is, can be read; what they hold does not matter), sw their O scales.  x is
 * codes with m scales sx (x_dtype CONVSEL_CODES) or numbers (CONV_F32, CONV_BF16;
 * sx NULL), which are coded by rows as above within the call.  The sum is exact;
 * scales (any: their product may leave fp32 where the result does not), bias,
 * activation and residual are fp32, and y is rounded once. */
#define CONVSEL_CODES (-1)
typedef struct convsel_linear_int8_desc {
  int64_t m, in_features, out_features; /* in < 2^17, out < 2^26, m * out <= 2^35 */
  int64_t ldx, ldw, ldr, ldy;           /* ldr is read only with a residual */
  int32_t x_dtype;                      /* CONVSEL_CODES, or conv_dtype_t of x */
  int32_t dtype;                        /* of b, r and y */
  int32_t act;                          /* convsel_act_t */
  int32_t has_bias, has_residual;
} convsel_linear_int8_desc_t;

/* Device bytes the call needs as workspace (0: none; else 256-byte aligned).
 * Codes run fastest where their rows start on 16 bytes, every one of them:
 * others are copied first.  Of x and w the addresses' alignment is looked at. */
conv_status_t convsel_linear_int8_workspace_bytes(const void* x, const void* w, const convsel_linear_int8_desc_t* desc,
                                                  size_t* bytes);
/* y may be r itself (same address and stride); otherwise its span must not
 * overlap what the call reads, nor the workspace. */
conv_status_t convsel_linear_int8(const void* x, const float* x_scale, const int8_t* w, const float* w_scale,
                                  const void* b, const void* r, void* y, const convsel_linear_int8_desc_t* desc,
                                  void* workspace, size_t workspace_bytes, void* stream);
/* One line: kernels, tile, split and workspace of the call. */
conv_status_t convsel_linear_int8_describe(const void* x, const void* w, const convsel_linear_int8_desc_t* desc,
                                           char* buf, size_t len);

/* ---- logits before a token is chosen --------------------------------------------
 * Row b is a sequence's logits over `vocab` tokens.  Its history are the tokens
 * history[offsets[b]] .. history[offsets[b+1]-1] (rising from 0; clamped to
 * [0, tokens]), the first prompt_lengths[b] of them its prompt (NULL: none) and
 * the others generated; tokens outside [0, vocab) are ignored.  With c(t) the
 * number of times t was generated, for z = x[b][t] in this order:
 *   t in the history:  z = z > 0 ? z / repetition[b] : z * repetition[b]
 *   c(t) > 0:          z = z - (frequency[b] * c(t) + presence[b])
 *   bias:              z = z + bias[b][t]          (ldbias 0: one row for all)
 *   mask:              z = -inf where bit t % 32 of mask[b][t / 32] is clear
 * in fp32; y is rounded once.  Each of them is left out where its pointer is NULL
 * (history NULL leaves out the first two).  A row whose mask allows nothing is
 * -inf throughout.  y may be x itself (same address and stride). */
typedef struct convsel_logits_desc {
  int64_t rows, vocab; /* each < 2^31 */
  int64_t tokens;      /* of the history */
  int64_t ldx, ldy;
  int64_t ldbias; /* 0, or at least vocab */
  int64_t ldmask; /* words: 0 (one row for all), or at least vocab / 32, rounded up */
  int32_t dtype;  /* of x and y */
} convsel_logits_desc_t;

conv_status_t convsel_adjust_logits(const void* x, const int32_t* history, const int32_t* offsets,
                                    const int32_t* prompt_lengths, const float* repetition, const float* presence,
                                    const float* frequency, const float* bias, const uint32_t* mask, void* y,
                                    const convsel_logits_desc_t* desc, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CONVSEL_LM_H */
