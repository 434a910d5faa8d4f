// A step's page tables, row offsets, positions and slots from the requests'
// lengths (definition: nvfp4_paging.h), for gfx950.
//
// Three sums over the sequences in order: of pages given back, pages taken and rows.
// What hangs on them, an entry of the pool, of a table or a row each, is then independent.
// Steps of up to 1024 sequences with up to 8192 rows are one workgroup's: a thread has a
// sequence; where none has more than a few rows and pages to move (decoding), it moves its
// own, and a page that comes back and is taken again stays in LDS; else a thread takes an
// entry and finds its sequence by bisection of the sums.  Where there are more rows
// (prompts) many workgroups compute the same sums and put pages back, and a second launch
// takes pages and places rows: pages go back to the pool before any is taken from it.
//
// Bound by latency: a launch, then the lengths, the tables' entries and the pool's, each a
// load's.  500 sequences with up to 5 rows take 3.8 us, one of 1000 tokens 2.7; with bisections and 64-bit sums for all 11.9 and 5.3.
// Over 1024 sequences one workgroup computes the sums of 1024 at a time: 1500 take 19.2 us and 20000 201, and the
// launches behind it 4.6 + 6.7 and 6.8 + 10.1.  Where many pages come back with few rows, one workgroup moves them:
// 223632 of 150 ended requests 190 us.
#include "paging_launch.h"

namespace nvfp4 {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
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

// Sums that stay at 2^32 - 1: in any grouping the same, and exact below.
__device__ __forceinline__ uint32_t add_sat(uint32_t x, uint32_t y) { return __builtin_elementwise_add_sat(x, y); }

template <int kHow, int kRows>
__device__ __forceinline__ uint32_t from_below(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kHow, kRows, 0xF, false);
}

// Over the lanes up to this one (all lanes active).
__device__ __forceinline__ uint32_t scan_up(uint32_t x) {
  x = add_sat(x, from_below<0x111, 0xF>(x));      // one lane below, in a row of 16; two, four, eight
  x = add_sat(x, from_below<0x112, 0xF>(x));
  x = add_sat(x, from_below<0x114, 0xF>(x));
  x = add_sat(x, from_below<0x118, 0xF>(x));
  x = add_sat(x, from_below<0x142, 0xA>(x));      // the last lane of the row below, into rows 1 and 3
  return add_sat(x, from_below<0x143, 0xC>(x));   // lane 31, into rows 2 and 3
}

template <int kHow>
__device__ __forceinline__ uint32_t row_other(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kHow, 0xF, 0xF, true);
}

// Over a row of 16 lanes.
__device__ __forceinline__ uint32_t row_sum(uint32_t v) {
  v = add_sat(v, row_other<0xB1>(v));
  v = add_sat(v, row_other<0x4E>(v));
  v = add_sat(v, row_other<0x141>(v));
  return add_sat(v, row_other<0x140>(v));
}

__device__ __forceinline__ uint32_t row_high(uint32_t v) {
  v = max(v, row_other<0xB1>(v));
  v = max(v, row_other<0x4E>(v));
  v = max(v, row_other<0x141>(v));
  return max(v, row_other<0x140>(v));
}

// The step's sums for up to 1024 sequences, one of them a thread's: what is before it.
struct Sums {
  Request r;
  bool served;
  uint32_t given, taken, rows;           // of the sequences before this one
  int before, backs, pages, all_rows, left;      // the pool, pages given back and taken, rows given, the pool behind
};

struct SumsLds {
  uint32_t totals[3][kWaves], ends[2][kWaves], most[kWaves];
};

// An entry's share of items of a sequence that a thread moves by itself.
constexpr int kOwnBack = 2, kOwnRows = 8;

__device__ __forceinline__ Sums step_sums(const TablesArgs& a, SumsLds& lds) {
  static_assert(kWaves == 16, "a wave for each lane of a row");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, b = threadIdx.x;
  Sums s;
  const int count = a.free_count[0];
  int held = 0, drop = 0, kept = 0, rows = 0;
  if (b < a.seqs) {
    held = a.kv_len[b];
    rows = a.new_rows[b];
    if (a.drop != nullptr) drop = a.drop[b];
    if (a.kept != nullptr) kept = a.kept[b];
  }
  s.before = min(max(count, 0), a.num_pages);
  s.r = request(a, b, held, drop, kept, rows);
  const uint32_t mine[3] = {(uint32_t)s.r.back, (uint32_t)s.r.need, (uint32_t)s.r.rows};
  uint32_t up[3], own[3], all[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    up[i] = scan_up(mine[i]);
    if (lane == 63) lds.totals[i][wave] = up[i];
  }
  const bool many = s.r.back > kOwnBack || s.r.rows > kOwnRows;
  if (lane == 0) lds.most[wave] = 0;
  if (__any(many) && lane == 0) lds.most[wave] = 1;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const uint32_t of_wave = lds.totals[i][col], ahead = row_sum(col < wave ? of_wave : 0u);
    all[i] = row_sum(of_wave);
    own[i] = add_sat(ahead, up[i]);      // with this sequence
  }
  s.backs = (int)min(all[0], (uint32_t)(a.num_pages - s.before));
  const uint32_t room = (uint32_t)(s.before + s.backs);
  // Both sums grow, so those that are served are the first ones.
  s.served = b < a.seqs && own[1] <= room && own[2] <= (uint32_t)a.rows;
  const int served = __popcll(__ballot(s.served));
  const int last = max(served - 1, 0);
  const uint32_t end_pages = (uint32_t)__builtin_amdgcn_readlane((int)own[1], last), end_rows = (uint32_t)__builtin_amdgcn_readlane((int)own[2], last);
  if (lane == 0) lds.ends[0][wave] = served ? end_pages : 0u, lds.ends[1][wave] = served ? end_rows : 0u;
  __syncthreads();
  s.pages = (int)row_high(lds.ends[0][col]);
  s.all_rows = (int)row_high(lds.ends[1][col]);
  s.left = (int)room - s.pages;
  s.given = own[0] == ~0u ? ~0u : own[0] - mine[0];      // (behind 2^32 - 1 pages nothing is put back)
  s.taken = s.served ? own[1] - mine[1] : (uint32_t)s.pages;
  s.rows = s.served ? own[2] - mine[2] : (uint32_t)s.all_rows;
  return s;
}

// Offsets and lengths.
__device__ __forceinline__ void put_lengths(const TablesArgs& a, const Sums& s) {
  const int b = threadIdx.x;
  if (b < a.seqs) {
    a.cu_rows[b] = (int)s.rows;
    a.kv_len[b] = s.r.base + (s.served ? s.r.rows : 0);
  }
  if (b == 0) {
    a.cu_rows[a.seqs] = s.all_rows;
    a.free_count[0] = s.left;
  }
}

// A whole step of up to 1024 sequences in one workgroup.
__global__ __launch_bounds__(kThreads) void step_small_kernel(TablesArgs a) {
  __shared__ SumsLds lds;
  __shared__ int32_t sums[4][kThreads + 1];      // or, in the first of them, the pages that come back
  const int b = threadIdx.x, shift = a.page_shift;
  const Sums s = step_sums(a, lds);
  const bool many = row_high(lds.most[threadIdx.x & 15]) != 0 || s.backs > kThreads;
  int32_t* const table = a.table + (int64_t)b * a.table_stride;
  if (!many) {
    // Each thread its own sequence's few: at most kOwnBack pages back, one new page, kOwnRows rows.
    const int have = ceil_shift(s.r.base, shift);
    int back[kOwnBack], open = -1;
#pragma unroll
    for (int i = 0; i < kOwnBack; ++i)
      if (i < s.r.back) back[i] = table[s.r.back0 + i];
    if (s.served && s.r.rows > 0 && (s.r.base & ((1 << shift) - 1))) open = table[have - 1];      // the page that is filled on
    // (a page of the pool that was there before: known now)
    const int64_t at = (int64_t)s.left + s.taken;
    const bool takes = s.served && s.r.need > 0;
    int fresh = takes && at < s.before ? a.free_pages[at] : -1;
#pragma unroll
    for (int i = 0; i < kOwnBack; ++i) {
      const uint32_t to = s.given + i;
      if (i < s.r.back && to < (uint32_t)s.backs) {
        sums[0][to] = back[i];
        a.free_pages[s.before + to] = back[i];
      }
    }
    put_lengths(a, s);
    __syncthreads();
    if (takes) {
      if (at >= s.before) fresh = sums[0][at - s.before];
      table[have] = fresh;
    }
    if (s.served) {
#pragma unroll
      for (int i = 0; i < kOwnRows; ++i) {
        if (i >= s.r.rows) break;
        const int row = (int)s.rows + i, position = s.r.base + i, page = (position >> shift) >= have ? fresh : open;
        if (a.positions != nullptr) a.positions[row] = position;
        if (a.slots != nullptr)
          a.slots[row] = page >= 0 && page < a.num_pages ? ((int64_t)page << shift) + (position & ((1 << shift) - 1)) : -1;
      }
    }
    return;
  }
  if (b < a.seqs) sums[0][b] = (int)min(s.given, 0x7FFFFFFFu), sums[1][b] = (int)s.taken, sums[2][b] = s.r.base, sums[3][b] = (int)s.rows;
  if (b == 0) sums[0][a.seqs] = 0x7FFFFFFF, sums[1][a.seqs] = s.pages, sums[3][a.seqs] = s.all_rows;
  put_lengths(a, s);
  __syncthreads();
  for (int i = b; i < s.backs; i += kThreads) give_back(a, sums[0], sums[2], i, s.before);
  __syncthreads();
  for (int i = b; i < s.all_rows; i += kThreads) place(a, sums[3], sums[1], sums[2], i, s.left);
  for (int i = b; i < s.pages; i += kThreads) take(a, sums[1], sums[2], i, s.left);
}

// The first of two launches for up to 1024 sequences with many rows: every workgroup
// computes the sums for itself and puts its share of the pages back; the first one leaves
// them, and the lengths, for the second launch (here they are still read).
__global__ __launch_bounds__(kThreads) void step_begin_kernel(TablesArgs a) {
  __shared__ SumsLds lds;
  __shared__ int32_t sums[2][kThreads + 1];
  const int b = threadIdx.x;
  const Sums s = step_sums(a, lds);
  if (b < a.seqs) sums[0][b] = (int)min(s.given, 0x7FFFFFFFu), sums[1][b] = s.r.base;
  if (b == 0) sums[0][a.seqs] = 0x7FFFFFFF;
  if (blockIdx.x == 0) {
    const Plan ws = plan_of(a.plan, a.seqs);
    if (b < a.seqs) {
      ws.given[b] = s.r.base + (s.served ? s.r.rows : 0);      // (the lengths to be)
      ws.taken[b] = (int)s.taken;
      ws.base[b] = s.r.base;
      a.cu_rows[b] = (int)s.rows;
    }
    if (b == 0) {
      ws.taken[a.seqs] = s.pages;
      a.cu_rows[a.seqs] = s.all_rows;
      *reinterpret_cast<PlanHead*>(a.plan) = {s.backs, s.pages, s.before, s.left, s.all_rows};
    }
  }
  __syncthreads();
  for (int64_t i = (int64_t)blockIdx.x * kThreads + b; i < s.backs; i += (int64_t)gridDim.x * kThreads)
    give_back(a, sums[0], sums[1], (int)i, s.before);
}

// The sums for more sequences.
__global__ __launch_bounds__(kThreads) void step_plan_kernel(TablesArgs a) {
  __shared__ int64_t totals[3][kWaves];
  __shared__ int ends[2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Plan ws = plan_of(a.plan, a.seqs);
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
    if (b < a.seqs) ws.given[b] = (int32_t)min(sum, (int64_t)0x7FFFFFFF);
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
      ws.taken[b] = served ? (int)from_pages : last_pages;
      a.cu_rows[b] = served ? (int)from_rows : last_rows;
      ws.base[b] = r.base;
      a.kv_len[b] = r.base + (served ? r.rows : 0);
    }
    __syncthreads();
  }
  const int left = room - last_pages;
  if (threadIdx.x == 0) {
    ws.given[a.seqs] = (int32_t)min(carry, (int64_t)0x7FFFFFFF);
    ws.taken[a.seqs] = last_pages;
    a.cu_rows[a.seqs] = last_rows;
    a.free_count[0] = left;
    *reinterpret_cast<PlanHead*>(a.plan) = {backs, last_pages, before, left, last_rows};
  }
}

__global__ __launch_bounds__(256) void step_give_back_kernel(TablesArgs a) {
  const PlanHead head = *reinterpret_cast<const PlanHead*>(a.plan);
  const Plan ws = plan_of(a.plan, a.seqs);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < head.given; i += (int64_t)gridDim.x * 256)
    give_back(a, ws.given, ws.base, (int)i, head.before);
}

// Rows and new pages.  Behind step_begin_kernel (up to 1024 sequences) the sums are searched in LDS,
// and its lengths are still to be put down.
template <bool kFew>
__global__ __launch_bounds__(256) void step_fill_kernel(TablesArgs a) {
  __shared__ int32_t sums[3][kFew ? kThreads + 1 : 1];
  const PlanHead head = *reinterpret_cast<const PlanHead*>(a.plan);
  const Plan ws = plan_of(a.plan, a.seqs);
  const int64_t all = (int64_t)gridDim.x * 256, first = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const auto fill = [&](const int32_t* cu, const int32_t* taken, const int32_t* base) {
    for (int64_t i = first; i < head.rows; i += all) place(a, cu, taken, base, (int)i, head.left);
    // (New entries are those that no row of place() reads: behind the base's pages.)
    for (int64_t i = first; i < head.taken; i += all) take(a, taken, base, (int)i, head.left);
  };
  if constexpr (kFew) {
    for (int b = threadIdx.x; b <= a.seqs; b += 256) {
      sums[0][b] = a.cu_rows[b];
      sums[1][b] = ws.taken[b];
      if (b < a.seqs) sums[2][b] = ws.base[b];
    }
    if (blockIdx.x == 0) {
      for (int b = threadIdx.x; b < a.seqs; b += 256) a.kv_len[b] = ws.given[b];
      if (threadIdx.x == 0) a.free_count[0] = head.left;
    }
    __syncthreads();
    fill(sums[0], sums[1], sums[2]);
  } else {
    fill(a.cu_rows, ws.taken, ws.base);
  }
}

}  // namespace

size_t step_tables_workspace_bytes(int64_t seqs) { return (size_t)(kHead + 3 * (seqs + 1)) * sizeof(int32_t); }

hipError_t launch_step_tables(const TablesArgs& a, hipStream_t stream) {
  hipError_t e;
  if (a.seqs <= kThreads && a.rows <= kOneLaunchRows) {
    step_small_kernel<<<1, kThreads, 0, stream>>>(a);
    return hipGetLastError();
  }
  const bool two = a.seqs <= kThreads;
  if (two) {
    step_begin_kernel<<<32, kThreads, 0, stream>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  } else {
    step_plan_kernel<<<1, kThreads, 0, stream>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    step_give_back_kernel<<<256, 256, 0, stream>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (two) step_fill_kernel<true><<<512, 256, 0, stream>>>(a);
  else step_fill_kernel<false><<<512, 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace nvfp4
