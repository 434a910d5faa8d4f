// C ABI of serving over the paged cache (include/nvfp4_paging.h): synchronous
// argument validation, the gfx950 device check and dispatch to the launchers.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attention_checks.h"
#include "nvfp4_paging.h"
#include "paging_launch.h"

using namespace nvfp4;

namespace {

bool valid_requests(const nvfp4_requests* r) {
  if (r == nullptr || r->n_seqs < 0 || r->n_seqs >= kMaxRows) return false;
  const int64_t p = r->page_size;
  if ((p != 16 && p != 32 && p != 64 && p != 128) || r->num_pages < 1 || r->num_pages >= kI32Lim) return false;
  if (r->max_pages < 0 || r->max_pages >= kI32Lim || r->max_pages * p > kMaxTokens) return false;
  if (r->page_table_stride < r->max_pages) return false;
  if (r->free_pages == nullptr || r->free_count == nullptr || !aligned(r->free_pages, 4) || !aligned(r->free_count, 4))
    return false;
  if (r->n_seqs == 0) return true;
  if (r->kv_len == nullptr || (r->max_pages > 0 && r->page_table == nullptr)) return false;
  return aligned(r->page_table, 4) && aligned(r->kv_len, 4);
}

bool valid_shared(const nvfp4_shared_prefix* s, const nvfp4_kv_batch* b) {
  if (s == nullptr || s->n_groups < 0 || s->n_groups > b->n_seqs || s->max_prefix < 0 || s->max_own < 0) return false;
  if (s->n_groups == 0) return true;
  return s->cu_seqs != nullptr && s->prefix != nullptr && aligned(s->cu_seqs, 4) && aligned(s->prefix, 4);
}

SharedArgs shared_args(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch, const nvfp4_shared_prefix* shared,
                       int64_t q_heads) {
  SharedArgs a = {};
  a.cache = cache_args(cache);
  a.batch = batch_args(batch, cache->page_size);
  a.q_heads = (int)q_heads;
  a.group = (int)(q_heads / cache->kv_heads);
  a.cu_seqs = shared->cu_seqs;
  a.prefix = shared->prefix;
  a.groups = (int)shared->n_groups;
  a.max_prefix = (int)(shared->max_prefix < a.batch.max_tokens ? shared->max_prefix : a.batch.max_tokens);
  a.max_own = (int)(shared->max_own < a.batch.max_kv_len ? shared->max_own : a.batch.max_kv_len);
  return a;
}

bool valid_bounds(const nvfp4_kv_bounds* b, const nvfp4_kv_cache* c) {
  if (b == nullptr || b->codes == nullptr || b->step == nullptr || !aligned(b->codes, 16) || !aligned(b->step, 4)) return false;
  return b->page_stride >= 2 * c->kv_heads * c->head_dim && b->page_stride % 16 == 0 && b->page_stride < kI32Lim &&
         b->step_stride >= c->kv_heads && b->step_stride < kI32Lim;
}

PageBoundsArgs bounds_args(const nvfp4_kv_bounds* b) {
  return {static_cast<int8_t*>(b->codes), b->step, b->page_stride, b->step_stride};
}

// Pages that a row may take: 1 to 2^30 tokens' in all.
bool valid_choice(const nvfp4_kv_cache* c, int64_t rows, int64_t count) {
  return rows >= 0 && rows < kMaxRows && count >= 1 && count <= kMaxTokens / c->page_size;
}

SelectedArgs selected_args(const nvfp4_kv_cache* cache, int64_t rows, int64_t q_heads, int64_t count) {
  SelectedArgs a = {};
  a.cache = cache_args(cache);
  a.q_heads = (int)q_heads;
  a.group = (int)(q_heads / cache->kv_heads);
  a.count = (int)count;
  a.batch.seqs = a.batch.rows = (int)rows;
  a.batch.max_tokens = a.batch.max_kv_len = (int)(count * cache->page_size);
  return a;
}

// (By the rows of a prefix's and of a sequence's own workgroups: 16 both, more of the
// prefix's, more of both.)
constexpr const char* kSharedKernels[3][3] = {
    {"kv_attention_shared_kernel<64,1,1>", "kv_attention_shared_kernel<64,2,1>", "kv_attention_shared_kernel<64,2,2>"},
    {"kv_attention_shared_kernel<128,1,1>", "kv_attention_shared_kernel<128,3,1>", "kv_attention_shared_kernel<128,3,2>"},
    {"kv_attention_shared_kernel<256,1,1>", nullptr, "kv_attention_shared_kernel<256,8,8>"}};
constexpr const char* kSharedJoins[3][2] = {
    {"kv_attention_shared_join_kernel<64,1>", "kv_attention_shared_join_kernel<64,4>"},
    {"kv_attention_shared_join_kernel<128,1>", "kv_attention_shared_join_kernel<128,4>"},
    {"kv_attention_shared_join_kernel<256,1>", "kv_attention_shared_join_kernel<256,4>"}};

}  // namespace

extern "C" {

size_t nvfp4_step_tables_workspace(int64_t n_seqs) {
  return n_seqs < 0 || n_seqs >= kMaxRows ? 0 : step_tables_workspace_bytes(n_seqs);
}

int nvfp4_step_tables(const nvfp4_requests* requests, const int32_t* new_rows, const int32_t* drop, const int32_t* kept,
                      int32_t* cu_rows, int32_t* positions, int64_t* slots, int64_t rows, void* workspace,
                      size_t workspace_bytes, void* stream) {
  if (!valid_requests(requests) || rows < 0 || rows >= kMaxRows) return NVFP4_EINVAL;
  if ((requests->n_seqs > 0 && new_rows == nullptr) || cu_rows == nullptr || workspace == nullptr) return NVFP4_EINVAL;
  if (!aligned(new_rows, 4) || !aligned(drop, 4) || !aligned(kept, 4) || !aligned(cu_rows, 4) || !aligned(positions, 4) ||
      !aligned(slots, 8) || !aligned(workspace, 8))
    return NVFP4_EINVAL;
  if (workspace_bytes < step_tables_workspace_bytes(requests->n_seqs)) return NVFP4_EWORKSPACE;
  const int st = check_device();
  if (st != NVFP4_OK) return st;
  TablesArgs a;
  a.table = requests->page_table;
  a.kv_len = requests->kv_len;
  a.free_pages = requests->free_pages;
  a.free_count = requests->free_count;
  a.new_rows = new_rows;
  a.drop = drop;
  a.kept = kept;
  a.cu_rows = cu_rows;
  a.positions = positions;
  a.slots = slots;
  a.table_stride = requests->page_table_stride;
  a.max_pages = (int)requests->max_pages;
  a.seqs = (int)requests->n_seqs;
  a.num_pages = (int)requests->num_pages;
  a.page_shift = __builtin_ctzll((unsigned long long)requests->page_size);
  a.rows = (int)rows;
  a.plan = static_cast<int32_t*>(workspace);
  const hipError_t e = launch_step_tables(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? NVFP4_OK : fail_hip(e);
}

size_t nvfp4_kv_attention_shared_workspace(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch,
                                           const nvfp4_shared_prefix* shared, int64_t q_heads) {
  if (!valid_cache(cache) || !valid_batch(batch, cache->page_size) || !valid_shared(shared, batch) ||
      !valid_q_heads(q_heads, cache->kv_heads))
    return 0;
  const SharedArgs a = shared_args(cache, batch, shared, q_heads);
  if (a.batch.seqs == 0 || a.batch.rows == 0) return 0;
  const SharedPlan p = shared_plan(a);
  return shared_fits(a, p) ? p.bytes : 0;
}

int nvfp4_kv_attention_shared(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch, const nvfp4_shared_prefix* shared,
                              const void* q, int64_t ldq, int64_t q_heads, void* y, int64_t ldy, float* lse,
                              float softmax_scale, int causal, void* workspace, size_t workspace_bytes, void* stream) {
  if (!valid_cache(cache) || !valid_batch(batch, cache->page_size) || !valid_shared(shared, batch) ||
      !valid_q_heads(q_heads, cache->kv_heads))
    return NVFP4_EINVAL;
  if (!valid_rows(q, ldq, q_heads, cache->head_dim, batch->rows) ||
      !valid_rows(y, ldy, q_heads, cache->head_dim, batch->rows) || !aligned(lse, 4))
    return NVFP4_EINVAL;
  const double scale = (double)softmax_scale * 1.4426950408889634;      // (powers of two)
  if (batch->rows * q_heads >= kI32Lim || !isfinite((float)scale) || (causal != 0 && causal != 1)) return NVFP4_EINVAL;
  SharedArgs a = shared_args(cache, batch, shared, q_heads);
  const bool none = a.batch.seqs == 0 || a.batch.rows == 0;
  SharedPlan p = {};
  if (!none) {
    p = shared_plan(a);
    if (!shared_fits(a, p)) return NVFP4_EINVAL;
    if (p.bytes > 0) {
      if (workspace == nullptr || !aligned(workspace, 16)) return NVFP4_EINVAL;
      if (workspace_bytes < p.bytes) return NVFP4_EWORKSPACE;
    }
  }
  const int st = check_device();
  if (st != NVFP4_OK) return st;
  if (none) return NVFP4_OK;
  a.q = static_cast<const uint16_t*>(q);
  a.y = static_cast<uint16_t*>(y);
  a.lse = lse;
  a.ldq = ldq;
  a.ldy = ldy;
  a.scale = (float)scale;
  a.causal = causal;
  a.window = 0;
  a.part = static_cast<float*>(workspace);
  const hipError_t e = launch_kv_attention_shared(a, p, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? NVFP4_OK : fail_hip(e);
}

const char* nvfp4_kv_attention_shared_kernel(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch,
                                             const nvfp4_shared_prefix* shared, int64_t q_heads, int part) {
  if (!valid_cache(cache) || !valid_batch(batch, cache->page_size) || !valid_shared(shared, batch) ||
      !valid_q_heads(q_heads, cache->kv_heads) || (part != 0 && part != 1) || batch->rows * q_heads >= kI32Lim)
    return nullptr;
  const SharedArgs a = shared_args(cache, batch, shared, q_heads);
  if (a.batch.seqs == 0 || a.batch.rows == 0) return nullptr;
  const SharedPlan p = shared_plan(a);
  if (!shared_fits(a, p)) return nullptr;
  if (p.apart) return nvfp4_kv_attention_kernel(cache, batch, q_heads, 0, part);
  const int dim = a.cache.dim == 64 ? 0 : a.cache.dim == 128 ? 1 : 2;
  if (part == 1) return kSharedJoins[dim][p.join_share == 4 ? 1 : 0];
  return kSharedKernels[dim][p.prefix.tiles == 1 ? 0 : p.own.tiles == 1 ? 1 : 2];
}

int nvfp4_kv_page_bounds(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch, const nvfp4_kv_bounds* bounds,
                         void* stream) {
  if (!valid_cache(cache) || !valid_batch(batch, cache->page_size) || !valid_bounds(bounds, cache)) return NVFP4_EINVAL;
  const BoundsArgs a = {cache_args(cache), batch_args(batch, cache->page_size), bounds_args(bounds)};
  if (!bounds_fit(a)) return NVFP4_EINVAL;
  const int st = check_device();
  if (st != NVFP4_OK) return st;
  if (a.batch.seqs == 0 || a.batch.rows == 0 || a.batch.max_tokens == 0) return NVFP4_OK;
  const hipError_t e = launch_kv_page_bounds(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? NVFP4_OK : fail_hip(e);
}

size_t nvfp4_kv_select_pages_workspace(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch) {
  if (!valid_cache(cache) || !valid_batch(batch, cache->page_size)) return 0;
  SelectArgs a = {};
  a.cache = cache_args(cache);
  a.batch = batch_args(batch, cache->page_size);
  a.max_pages = (int)batch->max_pages;
  return kv_select_workspace_bytes(a);
}

int nvfp4_kv_select_pages(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch, const nvfp4_kv_bounds* bounds,
                          const void* q, int64_t ldq, int64_t q_heads, int64_t count, int64_t first, int64_t recent, int causal,
                          int32_t* index, int32_t* pages, int32_t* tokens, void* workspace, size_t workspace_bytes,
                          void* stream) {
  if (!valid_cache(cache) || !valid_batch(batch, cache->page_size) || !valid_bounds(bounds, cache) ||
      !valid_q_heads(q_heads, cache->kv_heads) || !valid_choice(cache, batch->rows, count))
    return NVFP4_EINVAL;
  if (first < 0 || recent < 1 || first > count || recent > count - first || (causal != 0 && causal != 1)) return NVFP4_EINVAL;
  if (!valid_rows(q, ldq, q_heads, cache->head_dim, batch->rows)) return NVFP4_EINVAL;
  const bool none = batch->rows == 0 || batch->n_seqs == 0;
  if (batch->rows > 0 && (index == nullptr || pages == nullptr || tokens == nullptr)) return NVFP4_EINVAL;
  if (!aligned(index, 4) || !aligned(pages, 4) || !aligned(tokens, 4)) return NVFP4_EINVAL;
  if (batch->rows > 0 && batch->n_seqs == 0) return NVFP4_EINVAL;      // (rows of no sequence)
  SelectArgs a;
  a.cache = cache_args(cache);
  a.batch = batch_args(batch, cache->page_size);
  a.bounds = bounds_args(bounds);
  a.q = static_cast<const uint16_t*>(q);
  a.ldq = ldq;
  a.group = (int)(q_heads / cache->kv_heads);
  a.count = (int)count;
  a.first = (int)first;
  a.recent = (int)recent;
  a.causal = causal;
  a.max_pages = (int)batch->max_pages;
  a.index = index;
  a.pages = pages;
  a.tokens = tokens;
  if (!none) {
    if (!select_fits(a)) return NVFP4_EINVAL;
    const size_t need = kv_select_workspace_bytes(a);
    if (need > 0 && (workspace == nullptr || !aligned(workspace, 16))) return NVFP4_EINVAL;
    if (workspace_bytes < need) return NVFP4_EWORKSPACE;
  }
  a.scores = static_cast<uint32_t*>(workspace);
  const int st = check_device();
  if (st != NVFP4_OK) return st;
  if (none) return NVFP4_OK;
  const hipError_t e = launch_kv_select(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? NVFP4_OK : fail_hip(e);
}

size_t nvfp4_kv_attention_selected_workspace(const nvfp4_kv_cache* cache, int64_t rows, int64_t q_heads, int64_t count) {
  if (!valid_cache(cache) || !valid_q_heads(q_heads, cache->kv_heads) || !valid_choice(cache, rows, count) || rows == 0)
    return 0;
  const SelectedArgs a = selected_args(cache, rows, q_heads, count);
  const AttentionPlan p = attention_plan(a.cache, a.batch, a.group, 0, kAnyRoom);
  return attention_fits(a.cache, a.batch, a.group, p) ? part_bytes(a.cache, a.batch, a.group, p) : 0;
}

int nvfp4_kv_attention_selected(const nvfp4_kv_cache* cache, const void* q, int64_t ldq, int64_t q_heads, int64_t rows,
                                int64_t count, const int32_t* pages, const int32_t* tokens, void* y, int64_t ldy, float* lse,
                                float softmax_scale, void* workspace, size_t workspace_bytes, void* stream) {
  if (!valid_cache(cache) || !valid_q_heads(q_heads, cache->kv_heads) || !valid_choice(cache, rows, count))
    return NVFP4_EINVAL;
  if (!valid_rows(q, ldq, q_heads, cache->head_dim, rows) || !valid_rows(y, ldy, q_heads, cache->head_dim, rows) ||
      !aligned(lse, 4))
    return NVFP4_EINVAL;
  if (rows > 0 && (pages == nullptr || tokens == nullptr || !aligned(pages, 4) || !aligned(tokens, 4))) return NVFP4_EINVAL;
  const double scale = (double)softmax_scale * 1.4426950408889634;      // (powers of two)
  if (rows * q_heads >= kI32Lim || !isfinite((float)scale)) return NVFP4_EINVAL;
  SelectedArgs a = selected_args(cache, rows, q_heads, count);
  if (rows > 0) {
    const AttentionPlan p = attention_plan(a.cache, a.batch, a.group, 0, kAnyRoom);
    if (!attention_fits(a.cache, a.batch, a.group, p)) return NVFP4_EINVAL;
    const size_t need = part_bytes(a.cache, a.batch, a.group, p);
    if (need > 0) {
      if (workspace == nullptr || !aligned(workspace, 16)) return NVFP4_EINVAL;
      if (workspace_bytes < need) return NVFP4_EWORKSPACE;
    }
    a.row_tiles = p.tiles;
    a.waves = p.waves;
    a.chunk = p.chunk;
    a.splits = p.splits;
  }
  const int st = check_device();
  if (st != NVFP4_OK) return st;
  if (rows == 0) return NVFP4_OK;
  a.batch.kv_len = tokens;
  a.pages = pages;
  a.q = static_cast<const uint16_t*>(q);
  a.y = static_cast<uint16_t*>(y);
  a.lse = lse;
  a.ldq = ldq;
  a.ldy = ldy;
  a.scale = (float)scale;
  a.part = static_cast<float*>(workspace);
  const hipError_t e = launch_kv_attention_selected(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? NVFP4_OK : fail_hip(e);
}

}  // extern "C"
