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

}  // extern "C"
