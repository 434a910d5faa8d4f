/*
 * nvfp4_attention.h -- C ABI of the attention between two W4A4 projections:
 * the norm and rotation of query and key heads, the append of keys and values
 * to a paged 8-bit cache, and the attention over that cache.
 *
 * The paper serves its attention layers with an FP8 KV cache (section 7
 * "KV-cache recipe": E4M3 keys and values with calibrated scales).  Here the
 * cache holds E4M3 (OCP E4M3FN) codes with one FP32 scale for each page (a
 * block of page_size tokens) and head, taken from the values themselves
 * (NVFP4_DYNAMIC) or given (NVFP4_STATIC): value = code * scale.
 *
 * Conventions are those of nvfp4.h (whose status codes and scale modes these
 * functions use): device pointers owned by the caller, synchronous checks
 * before anything is enqueued, work enqueued on ``stream``, no host
 * synchronization, no allocation, safe from several host threads.  Inputs are
 * finite; buffers do not overlap except where stated.
 *
 * Values in device memory (lengths, positions, page numbers) are not checked
 * on the host.  The kernels bound every access by the sizes given here: rows
 * outside [0, rows), slots before 0 and pages outside [0, num_pages) are not
 * read or written; such a page's tokens are dropped by the append and masked
 * in the attention.  Lengths are cut to max_pages * page_size.
 *
 * A launch holds fewer than 2^32 work-items.  A step that would take more in one is
 * refused with NVFP4_EINVAL: with one row for each sequence, an attention from n_seqs
 * * kv_heads = 2^24 on (q_heads / kv_heads <= 16), an append from n_seqs *
 * ceil(kv_heads * head_dim / 512) = 2^23 on.
 */
#ifndef NVFP4_ATTENTION_H
#define NVFP4_ATTENTION_H

#include "nvfp4.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * A paged cache of keys and values of one layer.
 *
 * Page p and head h hold page_size * head_dim bytes of keys at
 * k + p * k_page_stride + h * page_size * head_dim, and as many of values at
 * v (with v_page_stride); their scales are k_scale[p * scale_page_stride + h]
 * and v_scale[same].  Inside, tokens come in groups of 16, in the order in
 * which the attention's matrix instructions take them:
 *   keys    [page_size / 16][head_dim / 16][16: t][16: e % 16]
 *   values  [page_size / 16][head_dim / 64][4: t / 4][16: e % 16]
 *           [4: e / 16 % 4][4: t % 4]
 * for token t of the group and element e of the head.
 * Requirements: num_pages >= 1; kv_heads >= 1; head_dim 64, 128 or 256;
 * page_size 16, 32, 64 or 128 with page_size * head_dim <= 16384; page strides
 * in bytes, at least kv_heads * page_size * head_dim and multiples of 16;
 * scale_page_stride >= kv_heads; k and v 16-byte aligned, scales 4-byte.
 */
typedef struct nvfp4_kv_cache {
  void* k;
  void* v;
  float* k_scale;
  float* v_scale;
  int64_t num_pages;
  int64_t page_size;
  int64_t kv_heads;
  int64_t head_dim;
  int64_t k_page_stride;
  int64_t v_page_stride;
  int64_t scale_page_stride;
} nvfp4_kv_cache;

/*
 * The sequences of one step.  Sequence b's new rows are rows
 * [cu_rows[b], cu_rows[b + 1]) of q, k, v and y, n_b of them; kv_len[b] counts
 * its tokens with the new ones, so new row i is token kv_len[b] - n_b + i
 * (rows whose token would be before 0 are dropped by the append, and see
 * nothing under a causal mask, without one what the others see).  Token t is in page page_table[b * page_table_stride +
 * t / page_size], slot t % page_size; entries of the table behind its last token,
 * or wholly in front of the attention's windows, may hold anything, and so may
 * their pages and scales (scales of the others are finite).  Sequences may have no
 * rows, no tokens, or share pages that are only read.
 *
 *   page_table   device int32 [n_seqs x max_pages], row stride
 *                page_table_stride >= max_pages entries.
 *   kv_len       device int32 [n_seqs].
 *   cu_rows      device int32 [n_seqs + 1], not decreasing, from 0; NULL: one
 *                row for each sequence (rows == n_seqs).  Rows from
 *                cu_rows[n_seqs] on are left as they are.
 *   rows         rows of the tensors.
 *   max_kv_len   the largest kv_len as far as the host knows it: the work is
 *                divided by it.  A longer sequence is computed all the same,
 *                with less of it side by side.
 * Requirements: 0 <= n_seqs, rows < 2^24; 0 <= max_pages; max_pages *
 * page_size <= 2^30; max_kv_len >= 0; pointers 4-byte aligned.
 */
typedef struct nvfp4_kv_batch {
  const int32_t* page_table;
  const int32_t* kv_len;
  const int32_t* cu_rows;
  int64_t page_table_stride;
  int64_t max_pages;
  int64_t n_seqs;
  int64_t rows;
  int64_t max_kv_len;
} nvfp4_kv_batch;

/*
 * RMSNorm of each head of the queries and of the keys, with the rotation of
 * its first elements in the same pass:
 *   y = x * gamma / sqrt(sum_e x^2 / head_dim + eps)     (y = x: gamma NULL)
 *   angle_i = position * inv_freq[i],  0 <= i < rot_dim / 2
 *   (y_a, y_b) <- (y_a cos_i - y_b sin_i, y_b cos_i + y_a sin_i)
 *   with (a, b) = (i, i + rot_dim / 2), or (2 i, 2 i + 1) if interleaved;
 * evaluated in binary32 (the angle's whole turns are taken off in binary64;
 * sum_e x^2 has to stay below 2^128) and rounded to bf16 once.
 *
 *   q, q_out     bf16 [rows x q_heads x head_dim], row strides ldq, ldq_out
 *                (elements).  q_out may be q itself with the same stride.
 *   k, k_out     the same for the keys.  q_heads or k_heads may be 0.
 *   q_gamma, k_gamma   bf16 [head_dim] or NULL.
 *   positions    device int32 [rows] (NULL if rot_dim is 0).
 *   inv_freq     device float [rot_dim / 2] (NULL if rot_dim is 0).
 * Requirements: head_dim 64, 128 or 256; rot_dim a multiple of 16, 0 <=
 * rot_dim <= head_dim; rows < 2^24; heads <= 1024; strides multiples of 8, at
 * least heads * head_dim and below 2^31; eps >= 0, finite; bf16 pointers
 * 16-byte aligned, the others 4-byte.
 * Errors: NVFP4_EINVAL, NVFP4_EUNSUPPORTED, NVFP4_EHIP.
 */
int nvfp4_qk_norm_rope(const void* q, int64_t ldq, int64_t q_heads, const void* q_gamma, void* q_out, int64_t ldq_out,
                       const void* k, int64_t ldk, int64_t k_heads, const void* k_gamma, void* k_out, int64_t ldk_out,
                       int64_t rows, int64_t head_dim, float eps, const int32_t* positions, const float* inv_freq,
                       int64_t rot_dim, int interleaved, void* stream);

/*
 * Appends a step's keys and values to the cache; keys are normed (k_gamma not
 * NULL) and rotated (rot_dim > 0) on the way, as by nvfp4_qk_norm_rope but
 * without the rounding to bf16: each code is one rounding (to nearest, ties to
 * even) of the value over the scale, computed in binary64 (with a scale that is
 * no power of two, of the value cut to binary32, over the scale in binary64).
 *   NVFP4_DYNAMIC: a page and head's scale is the smallest power of two s >=
 *     2^-100 with |value| <= 448 s for all its tokens.  A call that writes slot
 *     0 starts the page anew; one that writes behind tokens that the page
 *     holds keeps the larger of its scale and theirs, and where the scale
 *     grows the held codes are brought to it (one more rounding, which changes
 *     only values below 2^-6 of the new scale).  Held scales are powers of two,
 *     as this mode leaves them: a page is written in one mode.
 *   NVFP4_STATIC: the scales (> 0, finite) are read and kept; values over
 *     448 s are cut to it.
 * Slots that the step does not write to keep their codes (those held ones
 * apart).  A page that a call writes to belongs to one sequence, once.
 *
 *   k, v         bf16 [rows x kv_heads x head_dim], row strides ldk, ldv.
 *   k_gamma      bf16 [head_dim] or NULL.
 *   positions    device int32 [rows]: the positions to rotate by; NULL: each
 *                token's own number in its sequence.
 *   inv_freq, rot_dim, interleaved   as for nvfp4_qk_norm_rope.
 * Requirements: those of the structures and of nvfp4_qk_norm_rope.
 * Errors: NVFP4_EINVAL, NVFP4_EUNSUPPORTED, NVFP4_EHIP.
 */
int nvfp4_kv_append(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch, const void* k, int64_t ldk,
                    const void* v, int64_t ldv, const void* k_gamma, float eps, const int32_t* positions,
                    const float* inv_freq, int64_t rot_dim, int interleaved, int mode, void* stream);

/* Workspace bytes of nvfp4_kv_attention (partial results of long sequences
 * that are computed in pieces side by side); 0: none is used, or the arguments
 * are invalid. */
size_t nvfp4_kv_attention_workspace(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch, int64_t q_heads);

/*
 * Attention of a step's queries over the cache (which holds the step's own
 * tokens already): for row i of sequence b, at token t = kv_len[b] - n_b + i,
 * and query head a (key head h = a * kv_heads / q_heads)
 *   s_j = softmax_scale * q . k_j,   y = sum_j exp(s_j) v_j / sum_j exp(s_j)
 *   lse = log sum_j exp(s_j)
 * over the tokens j < kv_len[b] with j <= t if causal and j > t - window if
 * window > 0.  A row that sees no token gets y = 0 and lse = -infinity.
 * Scores (which have to stay below 2^23 in magnitude), exponentials and sums are
 * binary32, and k is taken exactly.  The product with v is one of binary16
 * factors, summed in binary32: a token's probability is rounded by at most 2^-11
 * of itself or 2^-34 of the largest one that the row has met (2^-33 with value
 * scales that are no powers of two), whichever is more: exp(-15) of the largest
 * keeps its 11 bits, exp(-20) is off by 2% (4%) at most;
 * v is exact, but in pages whose scale is under 2^-22 of the largest value scale
 * among the pages that the row's workgroup looks at, where it is off by 2^-31 of
 * that scale at most.
 *
 *   q            bf16 [rows x q_heads x head_dim], row stride ldq.
 *   q_heads      a multiple of kv_heads, at most 1024.
 *   y            out, bf16 [rows x q_heads x head_dim], row stride ldy.
 *   lse          optional out (may be NULL): float [rows x q_heads].
 *   causal       0 or 1.   window   0 (none) or the number of tokens.
 *   workspace, workspace_bytes   at least nvfp4_kv_attention_workspace bytes,
 *                16-byte aligned (NULL if that is 0).  Its contents on entry
 *                do not matter; calls sharing one must be ordered.
 * Requirements: those of the structures; strides multiples of 8, at least
 * q_heads * head_dim and below 2^31; q, y 16-byte aligned, lse 4-byte;
 * softmax_scale finite; 0 <= window < 2^31; rows * q_heads < 2^31.
 * Errors: NVFP4_EINVAL, NVFP4_EWORKSPACE, NVFP4_EUNSUPPORTED, NVFP4_EHIP.
 */
int nvfp4_kv_attention(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch, const void* q, int64_t ldq,
                       int64_t q_heads, void* y, int64_t ldy, float* lse, float softmax_scale, int causal,
                       int64_t window, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Which kernels nvfp4_kv_attention launches for a step (diagnostics: tests and
 * profiles name the kernel that they mean), from the sizes alone: no device value
 * is read.  part 0: the attention; part 1: the launch that joins its pieces.
 * Returns a static string, or NULL where there is no such launch (no rows, a single
 * piece) or the arguments are invalid (part not 0 or 1) or refused.
 */
const char* nvfp4_kv_attention_kernel(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch, int64_t q_heads,
                                      int64_t window, int part);

#ifdef __cplusplus
}
#endif

#endif /* NVFP4_ATTENTION_H */
