// Host-only stand-ins for the launchers behind nvfp4_paging.h (csrc/paging_launch.h), so
// that the validation layer (csrc/paging_api.cpp) can be built for the CPU with
// sanitizers.  Without a device, every call that passes validation stops at the device
// check, so none is reached.
#include "paging_launch.h"

namespace nvfp4 {

size_t step_tables_workspace_bytes(int64_t seqs) { return (size_t)(8 + 3 * (seqs + 1)) * 4; }
hipError_t launch_step_tables(const TablesArgs&, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_kv_attention_shared(const SharedArgs&, const SharedPlan&, hipStream_t) { return hipErrorNoDevice; }
bool bounds_fit(const BoundsArgs& a) { return (int64_t)a.batch.seqs * a.cache.heads < (int64_t)1 << 26; }
hipError_t launch_kv_page_bounds(const BoundsArgs&, hipStream_t) { return hipErrorNoDevice; }
size_t kv_select_workspace_bytes(const SelectArgs& a) {
  return a.max_pages > 256 ? (size_t)a.batch.rows * a.cache.heads * a.max_pages * 4 : 0;
}
bool select_fits(const SelectArgs& a) { return (int64_t)a.batch.rows * a.cache.heads < (int64_t)1 << 22; }
hipError_t launch_kv_select(const SelectArgs&, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_kv_attention_selected(const SelectedArgs&, hipStream_t) { return hipErrorNoDevice; }

}  // namespace nvfp4
