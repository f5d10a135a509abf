// Block tables and slot maps of a paged cache from the requests' lengths, and the pool's free pages.
//
// Every row asks for some pages (or gives its pages back).  Where a row's pages lie in the ring of free pages follows from
// the sum of the needs of the rows before it: one scan over the rows, after which every entry of the table, the ring and
// the slot map is computed on its own.  Pages are taken at the ring's head and given back at its tail: the entries read lie
// in [head, head + free), those written in [head + free, head + free + given), and as no page is held twice the two never
// meet in a ring of n_pages entries.  So nothing that one thread reads is written by another, except the lengths and the
// ring's state themselves, which are written after everybody has read them.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/meda.h"
#include "paged.hpp"

namespace meda {

struct PageUpdate {
  const int32_t* lens;
  const int32_t* n_new;
  int32_t* table;
  int32_t* ring;
  const int64_t* state;
  int32_t* lens_out;
  int64_t* state_out;
  int64_t* slots;
  int32_t* granted;
  int4* plan;      // [R]: ring position of the first page taken, of the first page given back, old length, new positions
                   // granted (-1: ended)
  int n_pages, R, max_blocks, page_log2, max_new;
  int group;       // consecutive rows that are granted together (1: every row on its own)
};

constexpr int kPlanThreads = 1024;
constexpr int kMaxRows = 65536;
constexpr int kAloneSlots = 8192;   // slots that one workgroup writes on its own

struct RowNeed {
  int len, held, want;   // length, pages held, new positions asked for (negative: ended)
  int need, give;        // pages asked for, pages given back
  bool fits;
};
__device__ __forceinline__ RowNeed row_need(const PageUpdate& a, int r) {
  const int page = 1 << a.page_log2, most = a.max_blocks << a.page_log2;
  RowNeed n;
  n.len = min(max(a.lens[r], 0), most);
  n.want = a.n_new[r];
  n.held = (n.len + page - 1) >> a.page_log2;
  n.fits = n.want >= 0 && n.want <= most - n.len;
  n.need = n.fits ? (int)(((long long)n.len + n.want + page - 1) >> a.page_log2) - n.held : 0;
  n.give = n.want < 0 ? n.held : 0;
  return n;
}

// head in [0, n_pages), free in [0, n_pages]: whatever the caller's array holds
__device__ __forceinline__ void ring_state(const PageUpdate& a, int& head, int& free) {
  const long long h = a.state[0] % a.n_pages, f = a.state[1];
  head = (int)(h < 0 ? h + a.n_pages : h);
  free = (int)(f < 0 ? 0 : (f > a.n_pages ? a.n_pages : f));
}

// position `at` + `by` of the ring; at in [0, n_pages), by >= 0
__device__ __forceinline__ int ring_at(const PageUpdate& a, int at, long long by) {
  const long long x = at + by;
  return (int)(x < a.n_pages ? x : x % a.n_pages);
}

// One entry each: the table's block `held + j` of a row that takes pages, the ring's entry for block b of a row that has
// ended, the i-th slot of a row.
__device__ __forceinline__ void take_page(const PageUpdate& a, int r, int pop, int held, int j) {
  a.table[(size_t)r * a.max_blocks + held + j] = a.ring[ring_at(a, pop, j)];
}
__device__ __forceinline__ void give_page(const PageUpdate& a, int r, int push, int b) {
  a.ring[ring_at(a, push, b)] = a.table[(size_t)r * a.max_blocks + b];
}
__device__ __forceinline__ void write_slot(const PageUpdate& a, int r, int pop, int held, int len, int count, int i) {
  long long slot = -1;
  if (i < count) {
    const int p = len + i, b = p >> a.page_log2;
    // (a block that this call enters is read from the ring, not from the table: another thread enters it)
    const int page = b >= held ? a.ring[ring_at(a, pop, b - held)] : a.table[(size_t)r * a.max_blocks + b];
    if (page >= 0 && page < a.n_pages)
      slot = ((long long)page << a.page_log2) + (p & ((1 << a.page_log2) - 1));
  }
  a.slots[(size_t)r * a.max_new + i] = slot;
}

// What a row's place in the scan says: pages needed by the rows before it, pages given back before it, its length, the new
// positions it is granted (-1: ended).
struct RowPlan {
  int base, behind, len, count;
};
struct PlanTotals {
  int head, free;    // of the ring before the call
  int taken, given;  // pages
};

// The scan over the rows by one workgroup of kPlanThreads threads: keep(r, plan) for every row, in the thread that has it.
// (Sums stay below R * max_blocks <= 2^30.)  Everything of lens and the ring's state has been read when it returns.
//
// Rows in groups: a row that does not fit into its table marks its group, whose needs then do not count; what is granted
// follows from the sum at the group's end, once every row's place in the scan is known: put(r, plan) keeps it as it is then
// (count: what was asked for), get(r) gives it back.  (512 rows, a token each, in place or not: 3.8 us, in groups of 32 4.9;
// with ended rows among them, whose pages go back, 4.6.)
template <bool GROUPS, typename Keep, typename Put, typename Get>
__device__ __forceinline__ PlanTotals plan_rows(const PageUpdate& a, Keep keep, Put put, Get get) {
  __shared__ int wave_need[kPlanThreads / 64], wave_give[kPlanThreads / 64];
  __shared__ unsigned refused[kMaxRows / 2 / 32];   // a bit per group
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, groups = a.R / a.group;
  auto refuse = [&](int g) { atomicOr(&refused[g >> 5], 1u << (g & 31)); };
  auto is_refused = [&](int g) { return ((refused[g >> 5] >> (g & 31)) & 1u) != 0u; };
  if constexpr (GROUPS) {
    for (int i = tid; i < (groups + 31) / 32; i += kPlanThreads) refused[i] = 0u;
    __syncthreads();
    for (int r = tid; r < a.R; r += kPlanThreads) {
      const RowNeed n = row_need(a, r);
      if (n.want >= 0 && !n.fits) refuse(r / a.group);
    }
    __syncthreads();
  }
  PlanTotals t{0, 0, 0, 0};
  ring_state(a, t.head, t.free);
  int need_before = 0, give_before = 0, taken = 0;
  for (int base = 0; base < a.R; base += kPlanThreads) {
    const int r = base + tid;
    RowNeed n{0, 0, 0, 0, 0, false};
    if (r < a.R) n = row_need(a, r);
    if (GROUPS && r < a.R && is_refused(r / a.group)) {
      n.fits = false;
      n.need = 0;
    }
    const int need_in = wave_inclusive_sum(n.need), give_in = wave_inclusive_sum(n.give);
    if (base > 0) __syncthreads();
    if (lane == 63) {
      wave_need[wave] = need_in;
      wave_give[wave] = give_in;
    }
    __syncthreads();
    int need_to = need_before + need_in, give_to = give_before + give_in;
#pragma unroll
    for (int w = 0; w < kPlanThreads / 64; ++w) {
      need_to += w < wave ? wave_need[w] : 0;
      give_to += w < wave ? wave_give[w] : 0;
      need_before += wave_need[w];
      give_before += wave_give[w];
    }
    if constexpr (GROUPS) {
      if (r < a.R) put(r, RowPlan{need_to - n.need, give_to - n.give, n.len, n.want < 0 ? -1 : (n.fits ? n.want : 0)});
    } else if (r < a.R) {
      const bool grant = n.fits && (n.need == 0 || need_to <= t.free);
      if (grant && n.need > 0) taken = need_to;   // (granted needs are a prefix of the sum)
      keep(r, RowPlan{need_to - n.need, give_to - n.give, n.len, n.want < 0 ? -1 : (grant ? n.want : 0)});
    }
  }
  if constexpr (GROUPS) {
    __syncthreads();
    for (int g = tid; g < groups; g += kPlanThreads) {
      const int from = get(g * a.group).base, to = g + 1 < groups ? get((g + 1) * a.group).base : need_before;
      if (to > from && to > t.free) refuse(g);
      else if (to > from) taken = to;
    }
    __syncthreads();
    for (int r = tid; r < a.R; r += kPlanThreads) {
      RowPlan p = get(r);
      if (p.count > 0 && is_refused(r / a.group)) p.count = 0;
      keep(r, p);
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) taken = max(taken, __shfl_xor(taken, o, kWave));
  __syncthreads();
  if (lane == 0) wave_need[wave] = taken;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) t.taken = max(t.taken, wave_need[w]);
  t.given = give_before;
  return t;
}

__device__ __forceinline__ void write_row(const PageUpdate& a, int r, const RowPlan& p) {
  a.lens_out[r] = p.count < 0 ? 0 : p.len + p.count;
  if (a.granted) a.granted[r] = p.count;
}
__device__ __forceinline__ void write_state(const PageUpdate& a, const PlanTotals& t) {
  const long long left = (long long)t.free - t.taken + t.given;
  a.state_out[0] = ring_at(a, t.head, t.taken);
  a.state_out[1] = left > a.n_pages ? a.n_pages : left;
}

// Everything in one launch, up to kFusedRows rows: the scan, and then every entry on its own, whatever row it belongs to
// (the row of the n-th page taken or given back is searched in the scan's sums).  grid: one workgroup, or, where lens_out and
// state_out are arrays of their own, any number: every workgroup scans all rows and takes a part of the entries.
constexpr int kFusedRows = 2048;
template <bool GROUPS>
__global__ void __launch_bounds__(kPlanThreads) page_update_kernel(PageUpdate a) {
  __shared__ RowPlan rows[kFusedRows];
  const PlanTotals t = plan_rows<GROUPS>(
      a,
      [&](int r, const RowPlan& p) {
        rows[r] = p;
        if (blockIdx.x == 0) write_row(a, r, p);
      },
      [&](int r, const RowPlan& p) { rows[r] = p; }, [&](int r) { return rows[r]; });
  if (blockIdx.x == 0 && threadIdx.x == 0) write_state(a, t);
  const int at = blockIdx.x * kPlanThreads + threadIdx.x, step = gridDim.x * kPlanThreads, page = 1 << a.page_log2;
  // the last row whose sum is not above n
  auto row_of = [&](int n, int RowPlan::*sum) {
    int lo = 0, hi = a.R;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (rows[mid].*sum <= n) lo = mid; else hi = mid;
    }
    return lo;
  };
  for (int n = at; n < t.taken; n += step) {
    const int r = row_of(n, &RowPlan::base), held = (rows[r].len + page - 1) >> a.page_log2;
    a.table[(size_t)r * a.max_blocks + held + (n - rows[r].base)] = a.ring[ring_at(a, t.head, n)];
  }
  for (int n = at; n < t.given; n += step) {
    const int r = row_of(n, &RowPlan::behind);
    a.ring[ring_at(a, t.head, (long long)t.free + n)] = a.table[(size_t)r * a.max_blocks + (n - rows[r].behind)];
  }
  const unsigned entries = (unsigned)a.R * (unsigned)a.max_new;
  for (unsigned n = at; n < entries; n += step) {
    const int r = (int)(n / (unsigned)a.max_new), i = (int)(n - (unsigned)r * (unsigned)a.max_new);
    const RowPlan p = rows[r];
    write_slot(a, r, ring_at(a, t.head, p.count > 0 ? p.base : 0), (p.len + page - 1) >> a.page_log2, p.len, p.count, i);
  }
}

// More rows, or many slots beside lengths that are updated in place: the scan by itself, plan[r] for every row ...
template <bool GROUPS>
__global__ void __launch_bounds__(kPlanThreads) page_plan_kernel(PageUpdate a) {
  int head, free;
  ring_state(a, head, free);
  const PlanTotals t = plan_rows<GROUPS>(
      a,
      [&](int r, const RowPlan& p) {
        a.plan[r] = make_int4(ring_at(a, head, p.count > 0 ? p.base : 0), ring_at(a, head, (long long)free + p.behind), p.len, p.count);
        write_row(a, r, p);
      },
      [&](int r, const RowPlan& p) { a.plan[r] = make_int4(p.base, p.behind, p.len, p.count); },
      [&](int r) {
        const int4 p = a.plan[r];
        return RowPlan{p.x, p.y, p.z, p.w};
      });
  if (threadIdx.x == 0) write_state(a, t);
}

// ... and the entries of one row.  grid (R, parts).
__global__ void __launch_bounds__(256) page_fill_kernel(PageUpdate a) {
  const int r = blockIdx.x, at = blockIdx.y * 256 + threadIdx.x, step = gridDim.y * 256;
  const int4 plan = a.plan[r];
  const int page = 1 << a.page_log2, len = plan.z, count = plan.w;
  const int held = (len + page - 1) >> a.page_log2;
  if (count < 0) {
    for (int b = at; b < held; b += step) give_page(a, r, plan.y, b);
  } else {
    const int need = (int)(((long long)len + count + page - 1) >> a.page_log2) - held;
    for (int j = at; j < need; j += step) take_page(a, r, plan.x, held, j);
  }
  // (unsigned: a step behind the last of nearly 2^31 slots is past the range of int)
  for (unsigned i = at; i < (unsigned)a.max_new; i += step) write_slot(a, r, plan.x, held, len, count, (int)i);
}

static hipError_t launch_page_update(const PageUpdate& a, hipStream_t s) {
  const long long entries = (long long)a.R * a.max_new;
  const bool in_place = a.lens_out == a.lens || a.state_out == a.state;
  if (a.R <= kFusedRows && (entries <= kAloneSlots || (!in_place && entries < (1ll << 31)))) {
    long long groups = entries <= kAloneSlots ? 1 : (entries + 4 * kPlanThreads - 1) / (4 * kPlanThreads);
    if (groups > 256) groups = 256;
    if (a.group > 1) hipLaunchKernelGGL(page_update_kernel<true>, dim3((unsigned)groups), dim3(kPlanThreads), 0, s, a);
    else hipLaunchKernelGGL(page_update_kernel<false>, dim3((unsigned)groups), dim3(kPlanThreads), 0, s, a);
    return hipGetLastError();
  }
  if (a.group > 1) hipLaunchKernelGGL(page_plan_kernel<true>, dim3(1), dim3(kPlanThreads), 0, s, a);
  else hipLaunchKernelGGL(page_plan_kernel<false>, dim3(1), dim3(kPlanThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int longest = a.max_new > a.max_blocks ? a.max_new : a.max_blocks;
  int parts = (longest - 1) / 1024 + 1;
  if (parts > 16) parts = 16;
  hipLaunchKernelGGL(page_fill_kernel, dim3(a.R, parts), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace meda

extern "C" {

size_t meda_page_update_workspace_bytes(int32_t n_rows) {
  if (n_rows < 1) return 0;
  return ((size_t)n_rows * sizeof(int4) + 255) / 256 * 256;
}

meda_status meda_page_update(const meda_page_params* params, const int32_t* lens, const int32_t* n_new, int32_t* table,
                             int32_t* free_ring, const int64_t* free_state, int32_t* lens_out, int64_t* free_state_out,
                             int64_t* slots, int32_t* granted, void* workspace, size_t workspace_bytes, void* hip_stream) {
  using namespace meda;
  if (!params) return MEDA_ERR_INVALID_ARG;
  const meda_page_params& p = *params;
  if (p.n_pages < 1 || p.n_rows < 1 || p.max_blocks < 1 || p.max_new < 0) return MEDA_ERR_INVALID_ARG;
  if (p.rows_per_seq < 0 || (p.rows_per_seq > 1 && p.n_rows % p.rows_per_seq != 0)) return MEDA_ERR_INVALID_ARG;
  if (p.n_pages > INT32_MAX || p.n_rows > kMaxRows || !valid_page_size(p.page_size)) return MEDA_ERR_UNSUPPORTED;
  if ((int64_t)p.n_rows * p.max_blocks > (1 << 30) || (int64_t)p.max_blocks * p.page_size > INT32_MAX) return MEDA_ERR_UNSUPPORTED;
  if (!lens || !n_new || !table || !free_ring || !free_state || !lens_out || !free_state_out) return MEDA_ERR_INVALID_ARG;
  if (p.max_new > 0 && !slots) return MEDA_ERR_INVALID_ARG;
  const uintptr_t words = (uintptr_t)lens | (uintptr_t)n_new | (uintptr_t)table | (uintptr_t)free_ring | (uintptr_t)lens_out | (uintptr_t)granted;
  const uintptr_t longs = (uintptr_t)free_state | (uintptr_t)free_state_out | (uintptr_t)slots;
  if ((words & 3u) || (longs & 7u)) return MEDA_ERR_INVALID_ARG;
  // What is written overlaps nothing else that the call reads or writes; lens_out and free_state_out may be lens and free_state.
  struct Range { const void* at; uint64_t bytes; };
  const uint64_t R = (uint64_t)p.n_rows;
  const Range all[] = {{table, R * p.max_blocks * 4}, {free_ring, (uint64_t)p.n_pages * 4}, {lens_out, R * 4}, {free_state_out, 16},
                       {p.max_new > 0 ? slots : nullptr, R * p.max_new * 8}, {granted, R * 4},
                       {lens, R * 4}, {n_new, R * 4}, {free_state, 16}};
  for (int x = 0; x < 6; ++x)
    for (int y = x + 1; y < 9; ++y) {
      if (!all[x].at || !all[y].at || (x == 2 && y == 6 && lens_out == lens) || (x == 3 && y == 8 && free_state_out == free_state)) continue;
      const uintptr_t u = (uintptr_t)all[x].at, v = (uintptr_t)all[y].at;
      if (u < v + all[y].bytes && v < u + all[x].bytes) return MEDA_ERR_INVALID_ARG;
    }
  if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < meda_page_update_workspace_bytes(p.n_rows)) return MEDA_ERR_WORKSPACE;

  PageUpdate a;
  a.lens = lens; a.n_new = n_new; a.table = table; a.ring = free_ring; a.state = free_state;
  a.lens_out = lens_out; a.state_out = free_state_out; a.slots = p.max_new > 0 ? slots : nullptr; a.granted = granted;
  a.plan = static_cast<int4*>(workspace);
  a.n_pages = (int)p.n_pages; a.R = p.n_rows; a.max_blocks = p.max_blocks;
  a.page_log2 = __builtin_ctz((unsigned)p.page_size); a.max_new = p.max_new;
  a.group = p.rows_per_seq > 1 ? p.rows_per_seq : 1;
  return launch_page_update(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? MEDA_OK : MEDA_ERR_HIP;
}

}  // extern "C"
