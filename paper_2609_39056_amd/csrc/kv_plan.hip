// Block tables and slot maps of a paged key-value cache from request lengths
// (sq_kv_plan): two exclusive sums over the requests (new tokens, new pages),
// then one table entry per taken page and one slot and position per token.
//
// One launch: every workgroup forms both sums of all requests in its LDS (at
// most 8192 lengths, from L2) and takes its share of the pages and tokens,
// found by bisection in the sums, so that one long prompt is spread like many
// short ones and no workgroup waits for another.  Workgroup 0 writes the
// per-request outputs.
#include <algorithm>

#include "token_internal.h"

namespace sq {
namespace {

__device__ __forceinline__ int32_t saturate(uint64_t v) { return static_cast<int32_t>(v < 0x7FFFFFFFu ? v : 0x7FFFFFFFu); }

// What one request holds and asks for.
struct Ask {
  int32_t cached, fresh;  // tokens
  uint32_t have, take;    // pages held, pages wanted
  bool room;              // the table's row holds them
};

__device__ __forceinline__ Ask ask(const PlanArgs& a, int r) {
  Ask q;
  q.cached = max(a.cached[r], 0);
  q.fresh = max(a.fresh[r], 0);
  const uint32_t mask = (1u << a.page_shift) - 1;
  q.have = (static_cast<uint32_t>(q.cached) + mask) >> a.page_shift;
  const uint32_t need =
      static_cast<uint32_t>((static_cast<uint64_t>(q.cached) + static_cast<uint32_t>(q.fresh) + mask) >> a.page_shift);
  q.room = need <= static_cast<uint32_t>(a.max_pages);
  q.take = q.room ? need - q.have : 0;
  return q;
}

// Placed: the row, the free list and the token arrays hold it.
__device__ __forceinline__ bool placed(const PlanArgs& a, const Ask& q, int32_t head, int32_t first, int32_t start) {
  return q.room && (q.take == 0 || static_cast<int64_t>(head) + first + q.take <= a.num_free) &&
         static_cast<int64_t>(start) + q.fresh <= a.max_tokens;
}

// The last r with sum[r] <= i (sum[0] = 0).
__device__ __forceinline__ int owner(const int32_t* sum, int R, int32_t i) {
  int lo = 0, hi = R;  // sum[lo] <= i; hi is past the end or sum[hi] > i
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sum[mid] <= i) {
      lo = mid;
    } else {
      hi = mid;
    }
  }
  return lo;
}

// THREADS threads for at most MOST requests.
template <int THREADS, int MOST>
__global__ __launch_bounds__(THREADS) void kv_plan_kernel(PlanArgs a) {
  __shared__ int32_t start[MOST], first[MOST];
  __shared__ uint64_t wave_sum[2][THREADS / 64];
  __shared__ int32_t used;
  const int tid = threadIdx.x, R = a.R;
  const int lane = tid & 63, wave = tid >> 6;
  const int32_t head = a.free_head == nullptr ? 0 : min(max(*a.free_head, 0), a.num_free);
  if (tid == 0) used = 0;

  // a thread sums consecutive requests, the threads' sums are scanned
  const int per = (R + THREADS - 1) / THREADS;
  const int r0 = min(tid * per, R), r1 = min(r0 + per, R);
  uint64_t tokens = 0, pages = 0;
  for (int r = r0; r < r1; ++r) {
    const Ask q = ask(a, r);
    tokens += static_cast<uint32_t>(q.fresh);
    pages += q.take;
  }
  uint64_t t_incl = tokens, p_incl = pages;
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t tv = __shfl_up(t_incl, o, 64), pv = __shfl_up(p_incl, o, 64);
    if (lane >= o) {
      t_incl += tv;
      p_incl += pv;
    }
  }
  if (lane == 63) {
    wave_sum[0][wave] = t_incl;
    wave_sum[1][wave] = p_incl;
  }
  __syncthreads();
  uint64_t t_at = t_incl - tokens, p_at = p_incl - pages, t_all = 0, p_all = 0;
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w < wave) {
      t_at += wave_sum[0][w];
      p_at += wave_sum[1][w];
    }
    t_all += wave_sum[0][w];
    p_all += wave_sum[1][w];
  }
  const bool writer = blockIdx.x == 0;
  int32_t most = 0;
  for (int r = r0; r < r1; ++r) {
    const Ask q = ask(a, r);
    start[r] = saturate(t_at);
    first[r] = saturate(p_at);
    if (writer) {
      const bool ok = placed(a, q, head, first[r], start[r]);
      if (ok && q.take > 0) most = max(most, first[r] + static_cast<int32_t>(q.take));
      a.token_start[r] = start[r];
      a.kv_len[r] = ok ? q.cached + q.fresh : q.cached;
    }
    t_at += static_cast<uint32_t>(q.fresh);
    p_at += q.take;
  }
  if (most > 0) atomicMax(&used, most);
  __syncthreads();
  if (writer && tid == 0) {
    a.token_start[R] = saturate(t_all);
    *a.free_head_out = head + used;
  }

  // one table entry per page that a placed request takes
  const int32_t pages_end = min(saturate(p_all), a.num_free - head);
  const int64_t at = static_cast<int64_t>(blockIdx.x) * THREADS + tid, step = static_cast<int64_t>(gridDim.x) * THREADS;
  for (int64_t i = at; i < pages_end; i += step) {
    const int r = owner(first, R, static_cast<int32_t>(i));
    const Ask q = ask(a, r);
    if (placed(a, q, head, first[r], start[r]))
      a.table[static_cast<size_t>(r) * a.max_pages + q.have + (i - first[r])] = a.free_pages[head + i];
  }
  // one slot and position per token; fresh pages are read from the free list,
  // not from the table entries written above
  const int32_t tokens_end = saturate(t_all);
  for (int64_t t = at; t < a.max_tokens; t += step) {
    int32_t slot = -1, pos = -1;
    if (t < tokens_end) {
      const int r = owner(start, R, static_cast<int32_t>(t));
      const Ask q = ask(a, r);
      if (placed(a, q, head, first[r], start[r])) {
        pos = q.cached + static_cast<int32_t>(t) - start[r];
        const uint32_t j = static_cast<uint32_t>(pos) >> a.page_shift;
        const int32_t page = j < q.have ? a.table[static_cast<size_t>(r) * a.max_pages + j]
                                        : a.free_pages[head + first[r] + (j - q.have)];
        slot = static_cast<int32_t>((static_cast<uint32_t>(page) << a.page_shift) +
                                    (static_cast<uint32_t>(pos) & ((1u << a.page_shift) - 1)));
      }
    }
    a.slot[t] = slot;
    a.pos[t] = pos;
  }
}

}  // namespace

hipError_t launch_kv_plan(const PlanArgs& a, hipStream_t s) {
  // One token per thread and pass.  Up to 1024 requests their sums take a
  // workgroup little, so up to eight of them per CU share the tokens (512 prompts,
  // 327000 tokens: 9.4 us, with one per CU 13.4, in workgroups of 1024 threads
  // 11.6); more take 1024 threads and 64 KB of LDS, one per CU.
  constexpr int32_t kFew = 1024;
  const int64_t items = static_cast<int64_t>(a.max_tokens) + a.R;
  if (a.R <= kFew) {
    const int64_t grid = std::min<int64_t>((items + 255) / 256, 8 * device_cus());
    kv_plan_kernel<256, kFew><<<static_cast<unsigned>(grid), 256, 0, s>>>(a);
  } else {
    const int64_t grid = std::min<int64_t>((items + 1023) / 1024, device_cus());
    kv_plan_kernel<1024, kPlanMaxRequests><<<static_cast<unsigned>(grid), 1024, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace sq
