// Checks of the attention entry points' arguments, and the kernels' parameters
// made of them (attention_api.cpp, paging_api.cpp).  Host code.
#pragma once

#include <math.h>
#include <stdint.h>

#include "attention_launch.h"
#include "nvfp4_attention.h"

namespace nvfp4 {

constexpr int64_t kI32Lim = (int64_t)1 << 31;
constexpr int64_t kMaxRows = (int64_t)1 << 24;
constexpr int64_t kMaxHeads = 1024;
constexpr int64_t kMaxTokens = (int64_t)1 << 30;

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

inline bool valid_dim(int64_t d) { return d == 64 || d == 128 || d == 256; }

// A tensor of `heads` heads per row; one without rows or heads may be NULL.
inline bool valid_rows(const void* p, int64_t ld, int64_t heads, int64_t dim, int64_t rows) {
  if (heads < 0 || heads > kMaxHeads) return false;
  if (heads == 0 || rows == 0) return true;
  return p != nullptr && aligned(p, 16) && ld >= heads * dim && ld % 8 == 0 && ld < kI32Lim;
}

inline bool valid_rope(int64_t dim, const float* inv_freq, int64_t rot_dim, int interleaved) {
  if (rot_dim < 0 || rot_dim > dim || rot_dim % 16 != 0 || (interleaved != 0 && interleaved != 1)) return false;
  return rot_dim == 0 || (inv_freq != nullptr && aligned(inv_freq, 4));
}

inline bool valid_eps(float eps) { return eps >= 0.0f && isfinite(eps); }

inline bool valid_cache(const nvfp4_kv_cache* c) {
  if (c == nullptr || !valid_dim(c->head_dim)) return false;
  const int64_t p = c->page_size, bytes = p * c->head_dim;
  if ((p != 16 && p != 32 && p != 64 && p != 128) || bytes > 16384) return false;
  if (c->num_pages < 1 || c->num_pages >= kI32Lim || c->kv_heads < 1 || c->kv_heads > kMaxHeads) return false;
  if (c->k_page_stride < c->kv_heads * bytes || c->v_page_stride < c->kv_heads * bytes) return false;
  if (c->k_page_stride % 16 != 0 || c->v_page_stride % 16 != 0 || c->scale_page_stride < c->kv_heads) return false;
  if (c->k == nullptr || c->v == nullptr || c->k_scale == nullptr || c->v_scale == nullptr) return false;
  return aligned(c->k, 16) && aligned(c->v, 16) && aligned(c->k_scale, 4) && aligned(c->v_scale, 4);
}

inline bool valid_batch(const nvfp4_kv_batch* b, int64_t page_size) {
  if (b == nullptr || b->n_seqs < 0 || b->n_seqs >= kMaxRows || b->rows < 0 || b->rows >= kMaxRows) return false;
  if (b->max_pages < 0 || b->max_pages >= kI32Lim || b->max_pages * page_size > kMaxTokens) return false;
  if (b->max_kv_len < 0 || b->page_table_stride < b->max_pages) return false;
  if (b->n_seqs == 0) return true;
  if (b->cu_rows == nullptr && b->rows != b->n_seqs) return false;
  if (b->kv_len == nullptr || (b->max_pages > 0 && b->page_table == nullptr)) return false;
  return aligned(b->page_table, 4) && aligned(b->kv_len, 4) && aligned(b->cu_rows, 4);
}

inline KvCacheArgs cache_args(const nvfp4_kv_cache* c) {
  KvCacheArgs a;
  a.kv[0] = static_cast<uint8_t*>(c->k);
  a.kv[1] = static_cast<uint8_t*>(c->v);
  a.scale[0] = c->k_scale;
  a.scale[1] = c->v_scale;
  a.page_stride[0] = c->k_page_stride;
  a.page_stride[1] = c->v_page_stride;
  a.scale_stride = c->scale_page_stride;
  a.num_pages = (int)c->num_pages;
  a.page_size = (int)c->page_size;
  a.page_shift = __builtin_ctzll((unsigned long long)c->page_size);
  a.heads = (int)c->kv_heads;
  a.dim = (int)c->head_dim;
  return a;
}

inline KvBatchArgs batch_args(const nvfp4_kv_batch* b, int64_t page_size) {
  KvBatchArgs a;
  a.table = b->page_table;
  a.kv_len = b->kv_len;
  a.cu_rows = b->cu_rows;
  a.table_stride = b->page_table_stride;
  a.max_tokens = (int)(b->max_pages * page_size);
  a.seqs = (int)b->n_seqs;
  a.rows = (int)b->rows;
  a.max_kv_len = (int)(b->max_kv_len < a.max_tokens ? b->max_kv_len : a.max_tokens);
  return a;
}

inline bool valid_q_heads(int64_t q_heads, int64_t kv_heads) {
  return q_heads >= kv_heads && q_heads <= kMaxHeads && q_heads % kv_heads == 0;
}

}  // namespace nvfp4
