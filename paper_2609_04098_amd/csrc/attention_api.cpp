// C ABI of the attention operators (include/nvfp4_attention.h): synchronous
// argument validation, the gfx950 device check and dispatch to the launchers.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "attention_launch.h"
#include "attention_plan.h"
#include "nvfp4_attention.h"

namespace {

constexpr int64_t kI32Lim = (int64_t)1 << 31;
constexpr int64_t kMaxRows = (int64_t)1 << 24;
constexpr int64_t kMaxHeads = 1024;
constexpr int64_t kMaxTokens = (int64_t)1 << 30;

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

bool valid_dim(int64_t d) { return d == 64 || d == 128 || d == 256; }

// A tensor of `heads` heads per row; one without rows or heads may be NULL.
bool valid_rows(const void* p, int64_t ld, int64_t heads, int64_t dim, int64_t rows) {
  if (heads < 0 || heads > kMaxHeads) return false;
  if (heads == 0 || rows == 0) return true;
  return p != nullptr && aligned(p, 16) && ld >= heads * dim && ld % 8 == 0 && ld < kI32Lim;
}

bool valid_rope(int64_t dim, const float* inv_freq, int64_t rot_dim, int interleaved) {
  if (rot_dim < 0 || rot_dim > dim || rot_dim % 16 != 0 || (interleaved != 0 && interleaved != 1)) return false;
  return rot_dim == 0 || (inv_freq != nullptr && aligned(inv_freq, 4));
}

bool valid_eps(float eps) { return eps >= 0.0f && isfinite(eps); }

bool valid_cache(const nvfp4_kv_cache* c) {
  if (c == nullptr || !valid_dim(c->head_dim)) return false;
  const int64_t p = c->page_size, bytes = p * c->head_dim;
  if ((p != 16 && p != 32 && p != 64 && p != 128) || bytes > 16384) return false;
  if (c->num_pages < 1 || c->num_pages >= kI32Lim || c->kv_heads < 1 || c->kv_heads > kMaxHeads) return false;
  if (c->k_page_stride < c->kv_heads * bytes || c->v_page_stride < c->kv_heads * bytes) return false;
  if (c->k_page_stride % 16 != 0 || c->v_page_stride % 16 != 0 || c->scale_page_stride < c->kv_heads) return false;
  if (c->k == nullptr || c->v == nullptr || c->k_scale == nullptr || c->v_scale == nullptr) return false;
  return aligned(c->k, 16) && aligned(c->v, 16) && aligned(c->k_scale, 4) && aligned(c->v_scale, 4);
}

bool valid_batch(const nvfp4_kv_batch* b, int64_t page_size) {
  if (b == nullptr || b->n_seqs < 0 || b->n_seqs >= kMaxRows || b->rows < 0 || b->rows >= kMaxRows) return false;
  if (b->max_pages < 0 || b->max_pages >= kI32Lim || b->max_pages * page_size > kMaxTokens) return false;
  if (b->max_kv_len < 0 || b->page_table_stride < b->max_pages) return false;
  if (b->n_seqs == 0) return true;
  if (b->cu_rows == nullptr && b->rows != b->n_seqs) return false;
  if (b->kv_len == nullptr || (b->max_pages > 0 && b->page_table == nullptr)) return false;
  return aligned(b->page_table, 4) && aligned(b->kv_len, 4) && aligned(b->cu_rows, 4);
}

nvfp4::KvCacheArgs cache_args(const nvfp4_kv_cache* c) {
  nvfp4::KvCacheArgs a;
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

nvfp4::KvBatchArgs batch_args(const nvfp4_kv_batch* b, int64_t page_size) {
  nvfp4::KvBatchArgs a;
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

bool valid_q_heads(int64_t q_heads, int64_t kv_heads) {
  return q_heads >= kv_heads && q_heads <= kMaxHeads && q_heads % kv_heads == 0;
}

// The kernels of a head size, in the order of kernel_name().
#define NVFP4_KERNELS(D)                                                                            \
  {"kv_attention_rows_kernel<" #D ",1,4,false>", "kv_attention_rows_kernel<" #D ",1,4,true>",       \
   "kv_attention_rows_kernel<" #D ",1,8,false>", "kv_attention_rows_kernel<" #D ",2,4,false>",      \
   "kv_attention_rows_kernel<" #D ",2,4,true>",  "kv_attention_tile_kernel<" #D ",false>",          \
   "kv_attention_tile_kernel<" #D ",true>",      "kv_attention_join_kernel<" #D ",1,1>",            \
   "kv_attention_join_kernel<" #D ",1,4>",       "kv_attention_join_kernel<" #D ",2,1>",            \
   "kv_attention_join_kernel<" #D ",2,4>",       "kv_attention_join_kernel<" #D ",8,1>",            \
   "kv_attention_join_kernel<" #D ",8,4>"}
constexpr const char* kKernels[3][13] = {NVFP4_KERNELS(64), NVFP4_KERNELS(128), NVFP4_KERNELS(256)};
#undef NVFP4_KERNELS

const char* kernel_name(int dim, const nvfp4::AttentionPlan& p, int part) {
  const auto& names = kKernels[dim == 64 ? 0 : dim == 128 ? 1 : 2];
  const int split = p.splits > 1 ? 1 : 0;
  if (part == 1) return split == 0 ? nullptr : names[7 + (p.tiles == 1 ? 0 : p.tiles == 2 ? 2 : 4) + (p.splits > 8 ? 1 : 0)];
  return names[p.waves == 8 ? 2 : (p.tiles == 1 ? 0 : p.tiles == 2 ? 3 : 5) + split];
}

}  // namespace

extern "C" {

int nvfp4_qk_norm_rope(const void* q, int64_t ldq, int64_t q_heads, const void* q_gamma, void* q_out, int64_t ldq_out,
                       const void* k, int64_t ldk, int64_t k_heads, const void* k_gamma, void* k_out, int64_t ldk_out,
                       int64_t rows, int64_t head_dim, float eps, const int32_t* positions, const float* inv_freq,
                       int64_t rot_dim, int interleaved, void* stream) {
  if (!valid_dim(head_dim) || rows < 0 || rows >= kMaxRows || !valid_eps(eps)) return NVFP4_EINVAL;
  if (!valid_rope(head_dim, inv_freq, rot_dim, interleaved)) return NVFP4_EINVAL;
  if (rot_dim > 0 && rows > 0 && (positions == nullptr || !aligned(positions, 4))) return NVFP4_EINVAL;
  if (!valid_rows(q, ldq, q_heads, head_dim, rows) || !valid_rows(q_out, ldq_out, q_heads, head_dim, rows) ||
      !valid_rows(k, ldk, k_heads, head_dim, rows) || !valid_rows(k_out, ldk_out, k_heads, head_dim, rows))
    return NVFP4_EINVAL;
  if (!aligned(q_gamma, 16) || !aligned(k_gamma, 16)) return NVFP4_EINVAL;
  if (q == q_out && q != nullptr && ldq != ldq_out) return NVFP4_EINVAL;
  if (k == k_out && k != nullptr && ldk != ldk_out) return NVFP4_EINVAL;
  const int st = nvfp4::check_device();
  if (st != NVFP4_OK) return st;
  if (rows == 0 || q_heads + k_heads == 0) return NVFP4_OK;
  nvfp4::NormRopeArgs a;
  a.x[0] = static_cast<const uint16_t*>(q);
  a.x[1] = static_cast<const uint16_t*>(k);
  a.y[0] = static_cast<uint16_t*>(q_out);
  a.y[1] = static_cast<uint16_t*>(k_out);
  a.gamma[0] = static_cast<const uint16_t*>(q_gamma);
  a.gamma[1] = static_cast<const uint16_t*>(k_gamma);
  a.ldx[0] = ldq;
  a.ldx[1] = ldk;
  a.ldy[0] = ldq_out;
  a.ldy[1] = ldk_out;
  a.heads[0] = (int)q_heads;
  a.heads[1] = (int)k_heads;
  a.rows = (int)rows;
  a.eps = eps;
  a.rope = {positions, inv_freq, (int)rot_dim, interleaved};
  const hipError_t e = nvfp4::launch_qk_norm_rope(a, (int)head_dim, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? NVFP4_OK : nvfp4::fail_hip(e);
}

int nvfp4_kv_append(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch, const void* k, int64_t ldk,
                    const void* v, int64_t ldv, const void* k_gamma, float eps, const int32_t* positions,
                    const float* inv_freq, int64_t rot_dim, int interleaved, int mode, void* stream) {
  if (mode != NVFP4_DYNAMIC && mode != NVFP4_STATIC) return NVFP4_EINVAL;
  if (!valid_cache(cache) || !valid_batch(batch, cache->page_size) || !valid_eps(eps)) return NVFP4_EINVAL;
  if (!valid_rope(cache->head_dim, inv_freq, rot_dim, interleaved) || !aligned(positions, 4)) return NVFP4_EINVAL;
  if (!valid_rows(k, ldk, cache->kv_heads, cache->head_dim, batch->rows) ||
      !valid_rows(v, ldv, cache->kv_heads, cache->head_dim, batch->rows) || !aligned(k_gamma, 16))
    return NVFP4_EINVAL;
  nvfp4::AppendArgs a;
  a.cache = cache_args(cache);
  a.batch = batch_args(batch, cache->page_size);
  const nvfp4::AppendPlan p = nvfp4::append_plan(a.cache, a.batch);
  if (!nvfp4::one_grid(p.workgroups, p.threads)) return NVFP4_EINVAL;
  const int st = nvfp4::check_device();
  if (st != NVFP4_OK) return st;
  if (a.batch.seqs == 0 || a.batch.rows == 0 || a.batch.max_tokens == 0) return NVFP4_OK;
  a.x[0] = static_cast<const uint16_t*>(k);
  a.x[1] = static_cast<const uint16_t*>(v);
  a.ld[0] = ldk;
  a.ld[1] = ldv;
  a.gamma = static_cast<const uint16_t*>(k_gamma);
  a.eps = eps;
  a.rope = {positions, inv_freq, (int)rot_dim, interleaved};
  a.dynamic = mode == NVFP4_DYNAMIC;
  const hipError_t e = nvfp4::launch_kv_append(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? NVFP4_OK : nvfp4::fail_hip(e);
}

size_t nvfp4_kv_attention_workspace(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch, int64_t q_heads) {
  if (!valid_cache(cache) || !valid_batch(batch, cache->page_size) || !valid_q_heads(q_heads, cache->kv_heads))
    return 0;
  const nvfp4::KvCacheArgs c = cache_args(cache);
  const nvfp4::KvBatchArgs b = batch_args(batch, cache->page_size);
  if (b.seqs == 0 || b.rows == 0) return 0;
  const int group = (int)(q_heads / cache->kv_heads);
  const nvfp4::AttentionPlan p = nvfp4::attention_plan(c, b, group, 0, nvfp4::kAnyRoom);
  return nvfp4::attention_fits(c, b, group, p) ? nvfp4::part_bytes(c, b, group, p) : 0;
}

int nvfp4_kv_attention(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch, const void* q, int64_t ldq,
                       int64_t q_heads, void* y, int64_t ldy, float* lse, float softmax_scale, int causal,
                       int64_t window, void* workspace, size_t workspace_bytes, void* stream) {
  if (!valid_cache(cache) || !valid_batch(batch, cache->page_size) || !valid_q_heads(q_heads, cache->kv_heads))
    return NVFP4_EINVAL;
  if (!valid_rows(q, ldq, q_heads, cache->head_dim, batch->rows) ||
      !valid_rows(y, ldy, q_heads, cache->head_dim, batch->rows) || !aligned(lse, 4))
    return NVFP4_EINVAL;
  const double scale = (double)softmax_scale * 1.4426950408889634;      // (powers of two)
  if (batch->rows * q_heads >= kI32Lim) return NVFP4_EINVAL;
  if (!isfinite((float)scale) || (causal != 0 && causal != 1) || window < 0 || window >= kI32Lim) return NVFP4_EINVAL;
  nvfp4::AttentionArgs a;
  a.cache = cache_args(cache);
  a.batch = batch_args(batch, cache->page_size);
  a.q_heads = (int)q_heads;
  a.group = (int)(q_heads / cache->kv_heads);
  const bool none = a.batch.seqs == 0 || a.batch.rows == 0;
  nvfp4::AttentionPlan p = {};
  if (!none) {
    p = nvfp4::attention_plan(a.cache, a.batch, a.group, 0, nvfp4::kAnyRoom);
    if (!nvfp4::attention_fits(a.cache, a.batch, a.group, p)) return NVFP4_EINVAL;
    const size_t need = nvfp4::part_bytes(a.cache, a.batch, a.group, p);
    if (need > 0) {
      if (workspace == nullptr || !aligned(workspace, 16)) return NVFP4_EINVAL;
      if (workspace_bytes < need) return NVFP4_EWORKSPACE;
    }
    if (window > 0) p = nvfp4::attention_plan(a.cache, a.batch, a.group, (int)window, p.splits);
  }
  const int st = nvfp4::check_device();
  if (st != NVFP4_OK) return st;
  if (none) return NVFP4_OK;
  a.row_tiles = p.tiles;
  a.waves = p.waves;
  a.chunk = p.chunk;
  a.splits = p.splits;
  a.q = static_cast<const uint16_t*>(q);
  a.y = static_cast<uint16_t*>(y);
  a.lse = lse;
  a.ldq = ldq;
  a.ldy = ldy;
  a.scale = (float)scale;
  a.causal = causal;
  a.window = (int)window;
  const hipError_t e = nvfp4::launch_kv_attention(a, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? NVFP4_OK : nvfp4::fail_hip(e);
}

const char* nvfp4_kv_attention_kernel(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch, int64_t q_heads,
                                      int64_t window, int part) {
  if (!valid_cache(cache) || !valid_batch(batch, cache->page_size) || !valid_q_heads(q_heads, cache->kv_heads))
    return nullptr;
  if (window < 0 || window >= kI32Lim || (part != 0 && part != 1) || batch->rows * q_heads >= kI32Lim) return nullptr;
  const nvfp4::KvCacheArgs c = cache_args(cache);
  const nvfp4::KvBatchArgs b = batch_args(batch, cache->page_size);
  if (b.seqs == 0 || b.rows == 0) return nullptr;
  const int group = (int)(q_heads / cache->kv_heads);
  nvfp4::AttentionPlan p = nvfp4::attention_plan(c, b, group, 0, nvfp4::kAnyRoom);
  if (!nvfp4::attention_fits(c, b, group, p)) return nullptr;
  if (window > 0) p = nvfp4::attention_plan(c, b, group, (int)window, p.splits);
  return kernel_name(c.dim, p, part);
}

}  // extern "C"
