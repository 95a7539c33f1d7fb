// Page tables after a choice of beams (sq_kv_reorder): row r becomes a copy of
// row parent[r], pages that no row holds any more are free again, and the rows
// behind the first that go on from the same parent get a page of their own for
// the copy of its partly filled last one.
//
// Nothing is counted from step to step: a page is held by the rows of the table.
// Which pages come free is found with two words per page of scratch, in phases:
//   A  new rows; the words of the pages of rows that nobody goes on from
//      (dropped rows) become "largest" and "not held"
//   B  every entry of a kept row makes its page held, every entry of a dropped
//      row puts its own index into its page's word, by minimum: the word names the
//      entry that frees the page, in an order that does not depend on the run
//   C  freed pages per dropped row
//   D  their places in the list of freed pages (a sum over the rows before), of
//      which the first go to the copies and the rest back to the free list
// What bounds it is dependent loads and launches, not data.  Large tables take a launch
// per phase, a wave per row (1024 rows of up to 290 pages: 25 us, of which the phases take
// 7.0, 6.4, 6.3 and 6.4).  Small ones take one workgroup with barriers between the phases,
// which has the entries and the scratch in LDS, so that only the lengths, the entries and
// the last pages are dependent loads (64 rows of up to 142 pages: 11.3 us, in four
// launches 15.7).
#include <algorithm>

#include "token_internal.h"

namespace sq {
namespace {

constexpr int kMaxRows = kPlanMaxRequests;
constexpr int32_t kLargest = 0x7FFFFFFF;

// The scratch: words of the pages, the lowest row that goes on from each, freed pages of
// each row, the entries that want a page of their own in order, and how many there are.
struct Scratch {
  int32_t *mark, *held, *first, *count, *copy_of, *copies;
};
__device__ inline Scratch scratch(int32_t* p, int32_t R, int32_t num_pages) {
  Scratch s;
  s.mark = p;
  s.held = s.mark + num_pages;
  s.first = s.held + num_pages;
  s.count = s.first + R;
  s.copy_of = s.count + R;
  s.copies = s.copy_of + R;
  return s;
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

// The sum of the threads' values before this one's, and of all.
__device__ int32_t before(int32_t mine, int32_t* sums, int32_t& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int32_t incl = mine;
  for (int o = 1; o < 64; o <<= 1) {
    const int32_t v = __shfl_up(incl, o, 64);
    if (lane >= o) incl += v;
  }
  __syncthreads();  // `sums` may still be read
  if (lane == 63) sums[wave] = incl;
  __syncthreads();
  int32_t at = incl - mine;
  all = 0;
  for (int v = 0; v < static_cast<int>(blockDim.x >> 6); ++v) {
    if (v < wave) at += sums[v];
    all += sums[v];
  }
  return at;
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

// A, the entries of one row by one wave, without the last where that is to be a
// copy: then it is returned, else -1.
__device__ int32_t new_row(const ReorderArgs& a, const int32_t* first, int r) {
  const int lane = threadIdx.x & 63;
  const int32_t p = a.parent[r];
  if (p < 0 || p >= a.R) return -1;
  const int32_t n = length(a, p);
  int32_t page = -1;
  const bool copy = wants_copy(a, r, p, first[p], n, page);
  const int32_t* row = row_of(a, p);
  int32_t* out = a.table_out + static_cast<size_t>(r) * a.max_pages;
  const int32_t entries = pages_of(a, n) - (copy ? 1 : 0);
  for (int j = lane; j < entries; j += 64) out[j] = row[j];
  return copy ? page : -1;
}

// A, by one workgroup: where the rows that want a copy have it, in order (a thread
// has 32 rows at most).  wants(r) says which do, tokens_of(r) gives their tokens.
template <typename Wants, typename Tokens>
__device__ void list_copies(const ReorderArgs& a, const Scratch& w, Wants wants, Tokens tokens_of, int32_t* sums) {
  const int threads = blockDim.x, tid = threadIdx.x, per = (a.R + threads - 1) / threads;
  const int r0 = min(tid * per, a.R), r1 = min(r0 + per, a.R);
  uint32_t wanted = 0;
#pragma unroll 4
  for (int r = r0; r < r1; ++r)
    if (wants(r)) wanted |= 1u << (r - r0);
  const int32_t mine = __popc(wanted);
  int32_t all;
  int32_t at = before(mine, sums, all);
  for (; wanted != 0; wanted &= wanted - 1) {
    const int r = r0 + __ffs(wanted) - 1;
    w.copy_of[at++] = r * a.max_pages + (tokens_of(r) >> a.page_shift);
  }
  if (tid == 0) *w.copies = all;
}

// B, one old row by one wave.
__device__ void mark_row(const ReorderArgs& a, const Scratch& w, bool dropped, int s) {
  const int32_t* row = row_of(a, s);
  const int32_t pages = pages_of(a, length(a, s));
  for (int j = threadIdx.x & 63; j < pages; j += 64)
    if (is_page(a, row[j])) {
      if (dropped)
        atomicMin(&w.mark[row[j]], s * a.max_pages + j);
      else
        w.held[row[j]] = 1;  // (by many: the words are not counted)
    }
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
    const bool mine = is_page(a, page) && w.mark[page] == s * a.max_pages + j && w.held[page] == 0;
    const uint64_t all = __ballot(mine);
    if (mine) each(found + static_cast<int32_t>(__popcll(all & ((1ull << lane) - 1))), page);
    found += static_cast<int32_t>(__popcll(all));
  }
  return found;
}

// The freed pages of the rows before each, into `base`, and of all.
__device__ void sum_counts(const ReorderArgs& a, const int32_t* count, int32_t* base, int32_t* sums, int32_t& all) {
  const int threads = blockDim.x, tid = threadIdx.x, per = (a.R + threads - 1) / threads;
  const int r0 = min(tid * per, a.R), r1 = min(r0 + per, a.R);
  int32_t mine = 0;
  for (int r = r0; r < r1; ++r) mine += count[r];
  int32_t at = before(mine, sums, all);
  for (int r = r0; r < r1; ++r) {
    const int32_t c = count[r];
    base[r] = at;
    at += c;
  }
  __syncthreads();
}

// Where freed pages and the free list's go.
struct Places {
  int32_t head, freed, copies, taken, new_head, back;
};
__device__ __forceinline__ int32_t free_head(const ReorderArgs& a) {
  return a.free_head == nullptr ? 0 : min(max(*a.free_head, 0), a.num_free);
}
__device__ __forceinline__ Places places(const ReorderArgs& a, int32_t head, int32_t copies, int32_t freed) {
  Places p;
  p.head = head;
  p.freed = freed;
  p.copies = copies;
  p.taken = min(copies, freed + min(a.num_free - p.head, copies));
  p.new_head = max(p.head + (p.taken - freed), 0);
  p.back = min(max(freed - p.taken, 0), p.head);  // pages that return to the list
  return p;
}

// The last entry of the c-th row that wants a copy.
__device__ __forceinline__ void place_copy(const ReorderArgs& a, const Scratch& w, const Places& p, int32_t c, int32_t page) {
  const int32_t at = w.copy_of[c], r = at / a.max_pages;
  const bool ok = c < p.taken;
  a.table_out[at] = ok ? page : -1;
  if (ok) {
    a.copy_dst[r] = page;
  } else {
    a.kv_len_out[r] = 0;
    a.copy_src[r] = -1;
    a.copy_rows[r] = 0;
  }
}

// D: the f-th freed page.
__device__ __forceinline__ void give(const ReorderArgs& a, const Scratch& w, const Places& p, int32_t f, int32_t page) {
  if (f < p.taken)
    place_copy(a, w, p, f, page);
  else if (f - p.taken < p.back)
    a.free_pages[p.new_head + (f - p.taken)] = page;
}

// D: copies past the freed pages take the free list's, as far as there are any.
// (Then no freed page goes back to the list that is read here.)
__device__ void give_listed(const ReorderArgs& a, const Scratch& w, const Places& p) {
  for (int32_t c = p.freed + static_cast<int32_t>(threadIdx.x); c < p.copies; c += blockDim.x)
    place_copy(a, w, p, c, c < p.taken ? a.free_pages[p.head + (c - p.freed)] : -1);
  if (threadIdx.x == 0) *a.free_head_out = p.new_head;
}

constexpr int kThreads = 256, kWaves = kThreads / 64;

// The last workgroup lists the copies.
__global__ __launch_bounds__(kThreads) void reorder_rows_kernel(ReorderArgs a) {
  __shared__ int32_t first[kMaxRows], sums[kWaves];
  const Scratch w = scratch(a.ws, a.R, a.num_pages);
  find_first(a, first);
  if (blockIdx.x == gridDim.x - 1) {
    auto wants = [&](int r) {
      const int32_t p = a.parent[r];
      int32_t page;
      return p >= 0 && p < a.R && wants_copy(a, r, p, first[p], length(a, p), page);
    };
    return list_copies(a, w, wants, [&](int r) { return length(a, a.parent[r]); }, sums);
  }
  const int r = blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (r >= a.R) return;
  const int lane = threadIdx.x & 63;
  if (first[r] == kLargest) {
    const int32_t* row = row_of(a, r);
    const int32_t pages = pages_of(a, length(a, r));
    for (int j = lane; j < pages; j += 64)
      if (is_page(a, row[j])) {
        w.mark[row[j]] = kLargest;
        w.held[row[j]] = 0;
      }
  }
  const int32_t copy = new_row(a, first, r);
  if (lane == 0) {
    const int32_t p = a.parent[r];
    const int32_t n = p >= 0 && p < a.R ? length(a, p) : 0;
    w.first[r] = first[r];
    a.kv_len_out[r] = n;
    a.copy_src[r] = copy;
    a.copy_dst[r] = -1;
    a.copy_rows[r] = copy >= 0 ? n & ((1 << a.page_shift) - 1) : 0;
  }
}

__global__ __launch_bounds__(kThreads) void reorder_mark_kernel(ReorderArgs a) {
  const Scratch w = scratch(a.ws, a.R, a.num_pages);
  const int s = blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (s < a.R) mark_row(a, w, w.first[s] == kLargest, s);
}

__global__ __launch_bounds__(kThreads) void reorder_count_kernel(ReorderArgs a) {
  const Scratch w = scratch(a.ws, a.R, a.num_pages);
  const int s = blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (s >= a.R) return;
  int32_t found = 0;
  if (w.first[s] == kLargest) found = freed_of(a, w, s, [](int32_t, int32_t) {});
  if ((threadIdx.x & 63) == 0) w.count[s] = found;
}

__global__ __launch_bounds__(kThreads) void reorder_give_kernel(ReorderArgs a) {
  __shared__ int32_t base[kMaxRows], sums[kWaves];
  const Scratch w = scratch(a.ws, a.R, a.num_pages);
  int32_t freed;
  sum_counts(a, w.count, base, sums, freed);
  const Places p = places(a, free_head(a), *w.copies, freed);
  for (int s = blockIdx.x * kWaves + (threadIdx.x >> 6); s < a.R; s += gridDim.x * kWaves)
    if (w.first[s] == kLargest) freed_of(a, w, s, [&](int32_t k, int32_t page) { give(a, w, p, base[s] + k, page); });
  if (blockIdx.x == 0) give_listed(a, w, p);
}

// Small tables, one launch: workgroup 0 takes all phases with the scratch and the
// dropped rows' entries in its LDS, a row per thread and runs of 64 entries per
// wave; the others copy the rows' entries.  What takes its time is one load or LDS
// access after the other, so runs go through each step several at a time.
constexpr int kOneThreads = 1024, kOneWaves = kOneThreads / 64;
constexpr int64_t kOneWords = 36 << 10;  // LDS words
constexpr int kTogether = 6;             // runs of a wave at a time

// Runs of up to 64 entries that a row has.
__host__ __device__ inline int runs_of(int32_t max_pages) { return (max_pages + 63) / 64; }
// LDS words: two per page, two per row, its first follower, the entries by runs.
__host__ __device__ inline int64_t one_words(int32_t R, int32_t max_pages, int32_t num_pages) {
  return 2 * static_cast<int64_t>(num_pages) + R * (3 + 64 * static_cast<int64_t>(runs_of(max_pages)));
}

__global__ __launch_bounds__(kOneThreads) void reorder_one_kernel(ReorderArgs a) {
  extern __shared__ int32_t lds[];
  __shared__ int32_t copies[kOneWaves], freed[kOneWaves];
  int32_t *mark = lds, *held = mark + a.num_pages, *first = held + a.num_pages, *tokens = first + a.R,
          *copy_of = tokens + a.R, *entry = copy_of + a.R;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (blockIdx.x > 0) {
    find_first(a, first);
    const int r = (blockIdx.x - 1) * kOneWaves + wave;
    if (r < a.R) new_row(a, first, r);
    return;
  }
  const int32_t head = free_head(a), mask = (1 << a.page_shift) - 1;
  int32_t parent = -1;
  if (tid < a.R) {
    parent = a.parent[tid];
    tokens[tid] = length(a, tid);
    first[tid] = kLargest;
  }
  for (int i = tid; i < a.num_pages; i += kOneThreads) {
    mark[i] = kLargest;
    held[i] = 0;
  }
  const bool some = parent >= 0 && parent < a.R;
  __syncthreads();
  if (some) atomicMin(&first[parent], tid);
  __syncthreads();

  // the rows that want a copy
  int32_t n = 0, last_page = -1;
  bool copy = false;
  if (some) {
    n = tokens[parent];
    copy = wants_copy(a, tid, parent, first[parent], n, last_page);
  }
  // The wave has consecutive runs, in the order of rows and entries.
  const int runs = runs_of(a.max_pages), each = (a.R * runs + kOneWaves - 1) / kOneWaves;
  const int run0 = min(wave * each, a.R * runs), run1 = min(run0 + each, a.R * runs);
  auto row_at = [&](int run, int& j) {
    const int s = run / runs;
    j = (run - s * runs) * 64 + lane;
    return s;
  };
  for (int run = run0; run < run1; run += kTogether) {
    int32_t page[kTogether];
#pragma unroll
    for (int u = 0; u < kTogether; ++u) {
      page[u] = -1;
      int j;
      const int s = row_at(run + u, j);
      if (run + u < run1 && j < pages_of(a, tokens[s])) page[u] = row_of(a, s)[j];
    }
#pragma unroll
    for (int u = 0; u < kTogether; ++u) {
      if (run + u >= run1) break;
      int j;
      const int s = row_at(run + u, j);
      const bool ok = is_page(a, page[u]), dropped = first[s] == kLargest;
      if (ok && dropped) atomicMin(&mark[page[u]], s * a.max_pages + j);
      if (ok && !dropped) held[page[u]] = 1;
      entry[(run + u) * 64 + lane] = ok && dropped ? page[u] : -1;
    }
  }
  const uint64_t copying = __ballot(copy);
  if (lane == 0) copies[wave] = static_cast<int32_t>(__popcll(copying));
  __syncthreads();

  // The sum of what the waves before this one have, and of all.
  auto sum = [&](const int32_t* of, int32_t& all) {
    int32_t at = 0;
    all = 0;
#pragma unroll
    for (int v = 0; v < kOneWaves; ++v) {
      const int32_t c = of[v];
      at += v < wave ? c : 0;
      all += c;
    }
    return at;
  };
  int32_t all_copies, all_freed;
  const int32_t copy_at = sum(copies, all_copies) + static_cast<int32_t>(__popcll(copying & ((1ull << lane) - 1)));
  if (copy) copy_of[copy_at] = tid * a.max_pages + (n >> a.page_shift);
  if (tid < a.R) {
    a.kv_len_out[tid] = n;
    a.copy_src[tid] = copy ? last_page : -1;
    a.copy_dst[tid] = -1;
    a.copy_rows[tid] = copy ? n & mask : 0;
  }
  // `each` for every run with the page that its entry frees, or -1
  auto freed_pages = [&](auto then) {
    for (int run = run0; run < run1; run += kTogether) {
      int32_t page[kTogether];
      bool free[kTogether];
#pragma unroll
      for (int u = 0; u < kTogether; ++u) page[u] = run + u < run1 ? entry[(run + u) * 64 + lane] : -1;
#pragma unroll
      for (int u = 0; u < kTogether; ++u) {
        int j;
        const int s = row_at(run + u, j);
        free[u] = page[u] >= 0 && mark[max(page[u], 0)] == s * a.max_pages + j && held[max(page[u], 0)] == 0;
      }
#pragma unroll
      for (int u = 0; u < kTogether; ++u) then(free[u] ? page[u] : -1);
    }
  };
  int32_t found = 0;
  freed_pages([&](int32_t page) { found += static_cast<int32_t>(__popcll(__ballot(page >= 0))); });
  if (lane == 0) freed[wave] = found;
  __syncthreads();
  int32_t at = sum(freed, all_freed);
  Scratch w{};
  w.copy_of = copy_of;
  const Places p = places(a, head, all_copies, all_freed);
  if (found > 0)
    freed_pages([&](int32_t page) {
      const uint64_t which = __ballot(page >= 0);
      if (page >= 0) give(a, w, p, at + static_cast<int32_t>(__popcll(which & ((1ull << lane) - 1))), page);
      at += static_cast<int32_t>(__popcll(which));
    });
  give_listed(a, w, p);
}

}  // namespace

size_t reorder_ws_ints(int32_t R, int32_t num_pages) {
  return 2 * static_cast<size_t>(num_pages) + 3 * static_cast<size_t>(R) + 1;
}

hipError_t launch_kv_reorder(const ReorderArgs& a, hipStream_t s) {
  const int64_t words = one_words(a.R, a.max_pages, a.num_pages);
  if (a.R <= kOneThreads && words <= kOneWords) {
    reorder_one_kernel<<<1 + (a.R + kOneWaves - 1) / kOneWaves, kOneThreads, 4 * words, s>>>(a);
    return hipGetLastError();
  }
  const unsigned rows = static_cast<unsigned>((a.R + kWaves - 1) / kWaves);
  reorder_rows_kernel<<<rows + 1, kThreads, 0, s>>>(a);
  reorder_mark_kernel<<<rows, kThreads, 0, s>>>(a);
  reorder_count_kernel<<<rows, kThreads, 0, s>>>(a);
  reorder_give_kernel<<<rows, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace sq
