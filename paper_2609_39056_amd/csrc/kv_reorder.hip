// Page tables after a choice of beams (sq_kv_reorder): row r becomes a copy of
// row parent[r], pages that no row holds any more are free again, and the rows
// behind the first that go on from the same parent get a page of their own for
// the copy of its partly filled last one.
//
// Nothing is counted from step to step: a page is held by the rows of the table.
// Which pages come free is found with one word per page of scratch, in phases:
//   A  new rows; the words of the pages of rows that nobody goes on from
//      (dropped rows) become "largest"
//   B  every entry of a kept row puts -1 into its page's word, every entry of a
//      dropped row its own index, by minimum: the word names the entry that
//      frees the page, in an order that does not depend on the run
//   C  freed pages per dropped row
//   D  their places in the list of freed pages (a sum over the rows before), of
//      which the first go to the copies and the rest back to the free list
// Many entries take a launch per phase, a wave per row; few one workgroup, with
// barriers between the phases.
#include <algorithm>

#include "token_internal.h"

namespace sq {
namespace {

constexpr int kMaxRows = kPlanMaxRequests;
constexpr int32_t kLargest = 0x7FFFFFFF;

// The scratch: words of the pages, rows that freed pages are counted in, the
// rows that want a copy in order, and how many of them there are.
struct Scratch {
  int32_t *mark, *first, *count, *copy_of, *copies;
};
__device__ __forceinline__ Scratch scratch(const ReorderArgs& a) {
  Scratch s;
  s.mark = a.ws;
  s.first = s.mark + a.num_pages;
  s.count = s.first + a.R;
  s.copy_of = s.count + a.R;
  s.copies = s.copy_of + a.R;
  return s;
}

__device__ __forceinline__ int32_t load(const int32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void store(int32_t* p, int32_t v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Tokens of an old row and its pages.
__device__ __forceinline__ int32_t length(const ReorderArgs& a, int s) {
  const int64_t most = static_cast<int64_t>(a.max_pages) << a.page_shift;
  return static_cast<int32_t>(min(static_cast<int64_t>(max(a.kv_len[s], 0)), most));
}
__device__ __forceinline__ int32_t pages_of(const ReorderArgs& a, int32_t n) {
  return static_cast<int32_t>((static_cast<uint32_t>(n) + ((1u << a.page_shift) - 1)) >> a.page_shift);
}
__device__ __forceinline__ bool is_page(const ReorderArgs& a, int32_t p) { return p >= 0 && p < a.num_pages; }
__device__ __forceinline__ const int32_t* row_of(const ReorderArgs& a, int s) {
  return a.table + static_cast<size_t>(s) * a.max_pages;
}

// The lowest row that goes on from each, in LDS.
__device__ void find_first(const ReorderArgs& a, int32_t* first) {
  for (int s = threadIdx.x; s < a.R; s += blockDim.x) first[s] = kLargest;
  __syncthreads();
  for (int r = threadIdx.x; r < a.R; r += blockDim.x) {
    const int32_t p = a.parent[r];
    if (p >= 0 && p < a.R) atomicMin(&first[p], r);
  }
  __syncthreads();
}

// Whether row r, which goes on from p, wants a copy of p's last page, and which.
__device__ __forceinline__ bool wants_copy(const ReorderArgs& a, int r, int p, int32_t first, int32_t n, int32_t& page) {
  if (first == r || (n & ((1 << a.page_shift) - 1)) == 0) return false;
  page = row_of(a, p)[n >> a.page_shift];
  return is_page(a, page);
}

// A, one row by one wave.
__device__ void new_row(const ReorderArgs& a, const Scratch& w, const int32_t* first, int r) {
  const int lane = threadIdx.x & 63;
  if (first[r] == kLargest) {
    const int32_t* row = row_of(a, r);
    const int32_t pages = pages_of(a, length(a, r));
    for (int j = lane; j < pages; j += 64)
      if (is_page(a, row[j])) store(&w.mark[row[j]], kLargest);
  }
  const int32_t p = a.parent[r];
  int32_t n = 0, src = -1, rows = 0;
  if (p >= 0 && p < a.R) {
    n = length(a, p);
    int32_t page = -1;
    const bool copy = wants_copy(a, r, p, first[p], n, page);
    if (copy) {
      src = page;
      rows = n & ((1 << a.page_shift) - 1);
    }
    const int32_t* row = row_of(a, p);
    int32_t* out = a.table_out + static_cast<size_t>(r) * a.max_pages;
    const int32_t entries = pages_of(a, n) - (copy ? 1 : 0);
    for (int j = lane; j < entries; j += 64) out[j] = row[j];
  }
  if (lane == 0) {
    a.kv_len_out[r] = n;
    a.copy_src[r] = src;
    a.copy_dst[r] = -1;
    a.copy_rows[r] = rows;
  }
}

// A, by one workgroup: the rows that want a copy, in order.
__device__ void list_copies(const ReorderArgs& a, const Scratch& w, const int32_t* first, int32_t* sums) {
  const int threads = blockDim.x, tid = threadIdx.x, per = (a.R + threads - 1) / threads;
  const int r0 = min(tid * per, a.R), r1 = min(r0 + per, a.R);
  int32_t mine = 0;
  for (int pass = 0; pass < 2; ++pass) {
    int32_t at = 0;
    if (pass == 1) {
      int32_t incl = mine;
      for (int o = 1; o < 64; o <<= 1) {
        const int32_t v = __shfl_up(incl, o, 64);
        if ((tid & 63) >= o) incl += v;
      }
      if ((tid & 63) == 63) sums[tid >> 6] = incl;
      __syncthreads();
      at = incl - mine;
      for (int v = 0; v < tid >> 6; ++v) at += sums[v];
      if (tid == threads - 1) store(w.copies, at + mine);
    }
    for (int r = r0; r < r1; ++r) {
      const int32_t p = a.parent[r];
      int32_t page;
      if (p < 0 || p >= a.R || !wants_copy(a, r, p, first[p], length(a, p), page)) continue;
      if (pass == 0)
        ++mine;
      else
        store(&w.copy_of[at++], r);
    }
  }
}

// B, one old row by one wave.
__device__ void mark_row(const ReorderArgs& a, const Scratch& w, bool dropped, int s) {
  const int32_t* row = row_of(a, s);
  const int32_t pages = pages_of(a, length(a, s));
  for (int j = threadIdx.x & 63; j < pages; j += 64)
    if (is_page(a, row[j])) atomicMin(&w.mark[row[j]], dropped ? s * a.max_pages + j : -1);
}

// C and D, one dropped row by one wave: `each` gets the row's freed pages in
// order; returns how many there are.
template <typename Each>
__device__ int32_t freed_of(const ReorderArgs& a, const Scratch& w, int s, Each each) {
  const int lane = threadIdx.x & 63;
  const int32_t* row = row_of(a, s);
  const int32_t pages = pages_of(a, length(a, s));
  int32_t found = 0;
  for (int j0 = 0; j0 < pages; j0 += 64) {
    const int j = j0 + lane;
    const int32_t page = j < pages ? row[j] : -1;
    const bool mine = is_page(a, page) && load(&w.mark[page]) == s * a.max_pages + j;
    const uint64_t all = __ballot(mine);
    if (mine) each(found + static_cast<int32_t>(__popcll(all & ((1ull << lane) - 1))), page);
    found += static_cast<int32_t>(__popcll(all));
  }
  return found;
}

// The freed pages of the rows before each thread's share of rows, and of all.
__device__ void sum_counts(const ReorderArgs& a, const Scratch& w, int32_t* base, int32_t* sums, int32_t& all) {
  const int threads = blockDim.x, tid = threadIdx.x, per = (a.R + threads - 1) / threads;
  const int r0 = min(tid * per, a.R), r1 = min(r0 + per, a.R);
  int32_t mine = 0;
  for (int r = r0; r < r1; ++r) {
    base[r] = load(&w.count[r]);
    mine += base[r];
  }
  int32_t incl = mine;
  for (int o = 1; o < 64; o <<= 1) {
    const int32_t v = __shfl_up(incl, o, 64);
    if ((tid & 63) >= o) incl += v;
  }
  if ((tid & 63) == 63) sums[tid >> 6] = incl;
  __syncthreads();
  int32_t at = incl - mine;
  all = 0;
  for (int v = 0; v < threads >> 6; ++v) {
    if (v < tid >> 6) at += sums[v];
    all += sums[v];
  }
  for (int r = r0; r < r1; ++r) {
    const int32_t c = base[r];
    base[r] = at;
    at += c;
  }
  __syncthreads();
}

// Where freed pages and the free list's go.
struct Places {
  int32_t head, freed, copies, taken, new_head, back;
};
__device__ __forceinline__ Places places(const ReorderArgs& a, int32_t copies, int32_t freed) {
  Places p;
  p.head = a.free_head == nullptr ? 0 : min(max(*a.free_head, 0), a.num_free);
  p.freed = freed;
  p.copies = copies;
  p.taken = min(copies, freed + (a.num_free - p.head));
  p.new_head = max(p.head + p.taken - freed, 0);
  p.back = min(max(freed - p.taken, 0), p.head);  // pages that return to the list
  return p;
}

// The last entry of the c-th copying row, and its page.
__device__ __forceinline__ void place_copy(const ReorderArgs& a, const Scratch& w, const Places& p, int32_t c, int32_t page) {
  const int r = load(&w.copy_of[c]);
  const int32_t n = length(a, a.parent[r]);
  const bool ok = c < p.taken;
  a.table_out[static_cast<size_t>(r) * a.max_pages + (n >> a.page_shift)] = ok ? page : -1;
  if (ok) {
    a.copy_dst[r] = page;
  } else {
    a.kv_len_out[r] = 0;
    a.copy_src[r] = -1;
    a.copy_rows[r] = 0;
  }
}

// D: the freed pages of a dropped row, the first of which start at `base`.
__device__ void give_row(const ReorderArgs& a, const Scratch& w, const Places& p, int s, int32_t base) {
  freed_of(a, w, s, [&](int32_t k, int32_t page) {
    const int32_t f = base + k;
    if (f < p.taken)
      place_copy(a, w, p, f, page);
    else if (f - p.taken < p.back)
      a.free_pages[p.new_head + f - p.taken] = page;
  });
}

// D: copies past the freed pages take the free list's, as far as there are any.
// (Then no freed page goes back to the list that is read here.)
__device__ void give_listed(const ReorderArgs& a, const Scratch& w, const Places& p) {
  for (int32_t c = p.freed + static_cast<int32_t>(threadIdx.x); c < p.copies; c += blockDim.x)
    place_copy(a, w, p, c, c < p.taken ? a.free_pages[p.head + c - p.freed] : -1);
  if (threadIdx.x == 0) *a.free_head_out = p.new_head;
}

constexpr int kThreads = 256, kWaves = kThreads / 64;

__global__ __launch_bounds__(kThreads) void reorder_rows_kernel(ReorderArgs a) {
  __shared__ int32_t first[kMaxRows], sums[kWaves];
  const Scratch w = scratch(a);
  find_first(a, first);
  for (int r = blockIdx.x * kWaves + (threadIdx.x >> 6); r < a.R; r += gridDim.x * kWaves) {
    new_row(a, w, first, r);
    if ((threadIdx.x & 63) == 0) store(&w.first[r], first[r]);
  }
  if (blockIdx.x == 0) list_copies(a, w, first, sums);
}

__global__ __launch_bounds__(kThreads) void reorder_mark_kernel(ReorderArgs a) {
  const Scratch w = scratch(a);
  const int s = blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (s < a.R) mark_row(a, w, w.first[s] == kLargest, s);
}

__global__ __launch_bounds__(kThreads) void reorder_count_kernel(ReorderArgs a) {
  const Scratch w = scratch(a);
  const int s = blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (s >= a.R) return;
  int32_t found = 0;
  if (w.first[s] == kLargest) found = freed_of(a, w, s, [](int32_t, int32_t) {});
  if ((threadIdx.x & 63) == 0) w.count[s] = found;
}

__global__ __launch_bounds__(kThreads) void reorder_give_kernel(ReorderArgs a) {
  __shared__ int32_t base[kMaxRows], sums[kWaves];
  const Scratch w = scratch(a);
  int32_t freed;
  sum_counts(a, w, base, sums, freed);
  const Places p = places(a, load(w.copies), freed);
  for (int s = blockIdx.x * kWaves + (threadIdx.x >> 6); s < a.R; s += gridDim.x * kWaves)
    if (w.first[s] == kLargest) give_row(a, w, p, s, base[s]);
  if (blockIdx.x == 0) give_listed(a, w, p);
}

}  // namespace

size_t reorder_ws_ints(int32_t R, int32_t num_pages) { return static_cast<size_t>(num_pages) + 3 * static_cast<size_t>(R) + 1; }

hipError_t launch_kv_reorder(const ReorderArgs& a, hipStream_t s) {
  const unsigned rows = static_cast<unsigned>((a.R + kWaves - 1) / kWaves);
  reorder_rows_kernel<<<rows, kThreads, 0, s>>>(a);
  reorder_mark_kernel<<<rows, kThreads, 0, s>>>(a);
  reorder_count_kernel<<<rows, kThreads, 0, s>>>(a);
  reorder_give_kernel<<<rows, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace sq
