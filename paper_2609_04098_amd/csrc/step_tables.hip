// A step's page tables, row offsets, positions and slots from the requests'
// lengths (definition: nvfp4_paging.h), for gfx950.
//
// Three sums over the sequences in order: of pages given back, pages taken and
// rows.  One workgroup computes them (plan); what hangs on them, an entry of the
// pool, of a table or a row each, is then independent: a thread finds its sequence
// by bisection of the sums.  Small steps do all of it in that one workgroup, one
// launch; where there are many rows (prompts) two more launches share it out: pages
// go back to the pool before any is taken from it.
#include "paging_launch.h"

namespace nvfp4 {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kHeld = 2048;              // sequences whose sums are held in LDS
constexpr int kOneLaunchRows = 8192;

// The workspace: a head, then three vectors of seqs + 1.
struct PlanHead {
  int32_t given, taken, before, left;    // pages given back and taken; the pool before, and behind the step
  int32_t rows;
};
constexpr int kHead = 8;

struct Plan {
  int32_t *given, *taken, *base;         // sums of pages given back, taken; tokens after the drop
};

__device__ __forceinline__ Plan plan_of(int32_t* at, int seqs) {
  return {at + kHead, at + kHead + seqs + 1, at + kHead + 2 * ((int64_t)seqs + 1)};
}

__device__ __forceinline__ int ceil_shift(int x, int shift) { return (x + (1 << shift) - 1) >> shift; }

// A sequence's own numbers.
struct Request {
  int held, base, back0, back, need, rows;      // back0: the first entry given back
};

__device__ __forceinline__ Request request(const TablesArgs& a, int b, int held, int drop, int kept, int rows) {
  const int most = a.max_pages << a.page_shift;
  Request r;
  r.held = min(max(held, 0), most);
  r.base = max(r.held - max(drop, 0), 0);
  r.back0 = ceil_shift(max(r.base, min(max(kept, 0), r.held)), a.page_shift);
  r.back = max(ceil_shift(r.held, a.page_shift) - r.back0, 0);
  r.rows = max(rows, 0);
  if (r.rows > most - r.base) r.rows = 0;
  r.need = ceil_shift(r.base + r.rows, a.page_shift) - ceil_shift(r.base, a.page_shift);
  return r;
}

// Sums over the lanes up to this one.
__device__ __forceinline__ int64_t wave_scan(int64_t x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t other = __shfl_up((long long)x, d);
    if (lane >= d) x += other;
  }
  return x;
}

// The last entry of sums[0 .. n] (not decreasing, from 0) that is at most `item`,
// which is below sums[n].
__device__ __forceinline__ int owner(const int32_t* sums, int n, int item) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] <= item) lo = mid; else hi = mid;
  }
  return lo;
}

// Pages back onto the pool: item of `given`, the pages' sums of all sequences.
__device__ __forceinline__ void give_back(const TablesArgs& a, const int32_t* sums, const int32_t* base, int item,
                                          int before) {
  const int b = owner(sums, a.seqs, item);
  const int64_t to = (int64_t)before + item;
  // (The first entry given back is a kept one's end, or the base's.)
  const int kept = a.kept == nullptr ? 0 : max(a.kept[b], 0);
  const int first = ceil_shift(max(base[b], min(kept, a.max_pages << a.page_shift)), a.page_shift);
  if (to < a.num_pages) a.free_pages[to] = a.table[(int64_t)b * a.table_stride + first + (item - sums[b])];
}

__device__ __forceinline__ int page_from_pool(const TablesArgs& a, int64_t at) {
  return at >= 0 && at < a.num_pages ? a.free_pages[at] : -1;
}

__device__ __forceinline__ void take(const TablesArgs& a, const int32_t* sums, const int32_t* base, int item, int left) {
  const int b = owner(sums, a.seqs, item);
  a.table[(int64_t)b * a.table_stride + ceil_shift(base[b], a.page_shift) + (item - sums[b])] =
      page_from_pool(a, (int64_t)left + item);
}

// Position and slot of a row, whose page may be among those that this step takes.
__device__ __forceinline__ void place(const TablesArgs& a, const int32_t* cu, const int32_t* taken, const int32_t* base,
                                      int row, int left) {
  const int b = owner(cu, a.seqs, row);
  const int start = base[b], at = start + (row - cu[b]);
  if (a.positions != nullptr) a.positions[row] = at;
  if (a.slots == nullptr) return;
  const int entry = at >> a.page_shift, have = ceil_shift(start, a.page_shift);
  const int page = entry >= have ? page_from_pool(a, (int64_t)left + taken[b] + (entry - have))
                                 : a.table[(int64_t)b * a.table_stride + entry];
  const bool there = page >= 0 && page < a.num_pages;
  a.slots[row] = there ? ((int64_t)page << a.page_shift) + (at & ((1 << a.page_shift) - 1)) : -1;
}

// The sums, and with kAll the rest of the step; kLds: they stay in LDS.
template <bool kAll, bool kLds>
__global__ __launch_bounds__(kThreads) void step_plan_kernel(TablesArgs a) {
  __shared__ int64_t totals[3][kWaves];
  __shared__ int ends[2];
  __shared__ int32_t held_sums[4][kLds ? kHeld + 1 : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Plan ws = plan_of(a.plan, a.seqs);
  int32_t* const given = kLds ? held_sums[0] : ws.given;
  int32_t* const taken = kLds ? held_sums[1] : ws.taken;
  int32_t* const base = kLds ? held_sums[2] : ws.base;
  int32_t* const cu = kLds ? held_sums[3] : a.cu_rows;
  const int before = min(max(a.free_count[0], 0), a.num_pages);
  // Pages given back first: what is served hangs on all of them.
  int64_t carry = 0;
  for (int b0 = 0; b0 < a.seqs; b0 += kThreads) {
    const int b = b0 + threadIdx.x;
    int64_t mine = 0;
    if (b < a.seqs) {
      const Request r = request(a, b, a.kv_len[b], a.drop == nullptr ? 0 : a.drop[b], a.kept == nullptr ? 0 : a.kept[b], 0);
      mine = r.back;
    }
    const int64_t up = wave_scan(mine);
    if (lane == 63) totals[0][wave] = up;
    __syncthreads();
    int64_t sum = carry + up - mine;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) sum += totals[0][w];
      carry += totals[0][w];
    }
    // (Behind the pool's room nothing is put back, so a sum beyond 32 bits may stop there.)
    if (b < a.seqs) given[b] = (int32_t)min(sum, (int64_t)0x7FFFFFFF);
    __syncthreads();
  }
  const int backs = (int)min(carry, (int64_t)a.num_pages - before);
  const int room = before + backs;
  int64_t pages = 0, rows = 0;
  int last_pages = 0, last_rows = 0;      // of those that are served
  for (int b0 = 0; b0 < a.seqs; b0 += kThreads) {
    const int b = b0 + threadIdx.x;
    Request r = {};
    if (b < a.seqs)
      r = request(a, b, a.kv_len[b], a.drop == nullptr ? 0 : a.drop[b], a.kept == nullptr ? 0 : a.kept[b], a.new_rows[b]);
    const int64_t up_pages = wave_scan(r.need), up_rows = wave_scan(r.rows);
    if (lane == 63) totals[1][wave] = up_pages, totals[2][wave] = up_rows;
    __syncthreads();
    int64_t to_pages = pages + up_pages, to_rows = rows + up_rows;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) to_pages += totals[1][w], to_rows += totals[2][w];
      pages += totals[1][w];
      rows += totals[2][w];
    }
    // Both sums grow, so those that are served are the first ones.
    const bool served = b < a.seqs && to_pages <= room && to_rows <= a.rows;
    const int64_t from_pages = to_pages - r.need, from_rows = to_rows - r.rows;
    // Sums of the served: those of the last one stay behind it.
    if (threadIdx.x == 0) ends[0] = last_pages, ends[1] = last_rows;
    __syncthreads();
    if (served) atomicMax(&ends[0], (int)to_pages), atomicMax(&ends[1], (int)to_rows);
    __syncthreads();
    last_pages = ends[0], last_rows = ends[1];
    if (b < a.seqs) {
      taken[b] = served ? (int)from_pages : last_pages;
      const int first = served ? (int)from_rows : last_rows;
      a.cu_rows[b] = first;
      if (kLds) cu[b] = first;
      base[b] = r.base;
      a.kv_len[b] = r.base + (served ? r.rows : 0);
    }
    __syncthreads();
  }
  const int left = room - last_pages;
  if (threadIdx.x == 0) {
    given[a.seqs] = (int32_t)min(carry, (int64_t)0x7FFFFFFF);
    taken[a.seqs] = last_pages;
    a.cu_rows[a.seqs] = last_rows;
    if (kLds) cu[a.seqs] = last_rows;
    a.free_count[0] = left;
    if (!kAll) {
      PlanHead* head = reinterpret_cast<PlanHead*>(a.plan);
      *head = {backs, last_pages, before, left, last_rows};
    }
  }
  if constexpr (kAll) {
    __syncthreads();
    for (int i = threadIdx.x; i < backs; i += kThreads) give_back(a, given, base, i, before);
    __syncthreads();
    for (int i = threadIdx.x; i < last_rows; i += kThreads) place(a, cu, taken, base, i, left);
    __syncthreads();
    for (int i = threadIdx.x; i < last_pages; i += kThreads) take(a, taken, base, i, left);
  }
}

__global__ __launch_bounds__(256) void step_give_back_kernel(TablesArgs a) {
  const PlanHead head = *reinterpret_cast<const PlanHead*>(a.plan);
  const Plan ws = plan_of(a.plan, a.seqs);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < head.given; i += (int64_t)gridDim.x * 256)
    give_back(a, ws.given, ws.base, (int)i, head.before);
}

__global__ __launch_bounds__(256) void step_fill_kernel(TablesArgs a) {
  const PlanHead head = *reinterpret_cast<const PlanHead*>(a.plan);
  const Plan ws = plan_of(a.plan, a.seqs);
  const int64_t all = (int64_t)gridDim.x * 256, first = (int64_t)blockIdx.x * 256 + threadIdx.x;
  for (int64_t i = first; i < head.rows; i += all) place(a, a.cu_rows, ws.taken, ws.base, (int)i, head.left);
  // (New entries are those that no row of place() reads: behind the base's pages.)
  for (int64_t i = first; i < head.taken; i += all) take(a, ws.taken, ws.base, (int)i, head.left);
}

}  // namespace

size_t step_tables_workspace_bytes(int64_t seqs) { return (size_t)(kHead + 3 * (seqs + 1)) * sizeof(int32_t); }

hipError_t launch_step_tables(const TablesArgs& a, hipStream_t stream) {
  if (a.rows <= kOneLaunchRows) {
    if (a.seqs <= kHeld)
      step_plan_kernel<true, true><<<1, kThreads, 0, stream>>>(a);
    else
      step_plan_kernel<true, false><<<1, kThreads, 0, stream>>>(a);
    return hipGetLastError();
  }
  step_plan_kernel<false, false><<<1, kThreads, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  step_give_back_kernel<<<256, 256, 0, stream>>>(a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  step_fill_kernel<<<512, 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace nvfp4
