// Copies of partly filled or whole pages inside the caches of several layers
// (sq_kv_copy_pages).  A page is [heads][page_size][head_dim], so the first rows
// of its heads are runs of rows * head_dim values; a workgroup takes a share of
// one page of one tensor, in 16-byte pieces.
//
// Memory bounds it (128 copies in 28 layers, 846 MB read and written: 175 to 191 us, 4.4 to
// 4.8 TB/s, as fast as a plain copy of 4 GiB), and at little data the launch (48 copies in
// one layer: 3.0 us).  Four pieces of a thread in flight: with 1, 2, 4 and 8 the former
// takes 219, 188, 187 and 182 us, the latter 3.4, 3.7, 3.2 and 3.7, 64 copies of small pages
// in 28 layers 30.5, 24.5, 23.2 and 22.9.  Loads and stores past the caches gained nothing.
#include <algorithm>

#include "token_internal.h"

namespace sq {
namespace {

typedef unsigned int Piece __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kAhead = 4;  // pieces of a thread in flight

__global__ __launch_bounds__(kThreads) void kv_copy_kernel(CopyArgs a, unsigned parts) {
  const int i = blockIdx.y;
  const int32_t src = a.src[i], dst = a.dst[i];
  if (src < 0 || src >= a.num_pages || dst < 0 || dst >= a.num_pages || src == dst) return;
  const uint32_t P = 1u << a.page_shift;
  const uint32_t rows = a.rows == nullptr ? P : static_cast<uint32_t>(min(max(a.rows[i], 0), static_cast<int32_t>(P)));
  const uint32_t run = rows * (static_cast<uint32_t>(a.row_bytes) / 16);  // pieces of a head
  const uint32_t total = run * static_cast<uint32_t>(a.heads);
  const unsigned tensor = blockIdx.x / parts, part = blockIdx.x % parts;
  const uint32_t head = P * (static_cast<uint32_t>(a.row_bytes) / 16);  // pieces from one head to the next
  Piece* pages = static_cast<Piece*>(a.pages[tensor]);
  const size_t page = static_cast<size_t>(head) * a.heads;
  const Piece* from = pages + src * page;
  Piece* to = pages + dst * page;
  const uint32_t step = parts * kThreads;
  for (uint32_t p = part * kThreads + threadIdx.x; p < total; p += kAhead * step) {
    Piece v[kAhead];
    uint32_t at[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const uint32_t q = min(p + u * step, total - 1);  // (a piece past the end repeats the last)
      at[u] = q / run * head + q % run;
      v[u] = from[at[u]];
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) to[at[u]] = v[u];
  }
}

}  // namespace

hipError_t launch_kv_copy(const CopyArgs& a, hipStream_t s) {
  const size_t page = (static_cast<size_t>(a.row_bytes) << a.page_shift) * a.heads;
  const unsigned parts = static_cast<unsigned>(std::max<size_t>(1, page / (kThreads * 16 * kAhead)));
  const dim3 grid(2 * static_cast<unsigned>(a.caches) * parts, static_cast<unsigned>(a.n));
  kv_copy_kernel<<<grid, kThreads, 0, s>>>(a, parts);
  return hipGetLastError();
}

}  // namespace sq
