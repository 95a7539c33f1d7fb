// Attention of one new token per request over a paged key-value cache
// (sq_attn_paged).
#include "half_types.h"
#include "token_internal.h"

namespace sq {
namespace {

constexpr int kWaves = 4;

// One workgroup per query head; its waves take tokens in turn, each with its
// own running maximum, sum and weighted values, joined in wave order.
template <bool F16>
__global__ __launch_bounds__(64 * kWaves) void attn_simple_kernel(AttnArgs a) {
  const size_t wg = flat_wg();
  if (wg >= static_cast<size_t>(a.R) * a.Hq) return;
  const int r = static_cast<int>(wg / a.Hq), h = static_cast<int>(wg % a.Hq);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int D = a.D, kvh = h / (a.Hq / a.Hk);
  const int n = min(max(a.kv_len[r], 0), a.max_kv_len);
  const int begin = a.window > 0 ? max(0, n - a.window) : 0;
  float q[4], o[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int d = 4 * lane + i;
    q[i] = d < D ? half_lo<F16>(a.q[r * a.q_stride + static_cast<size_t>(h) * D + d]) : 0.0f;
  }
  float m = -INFINITY, l = 0.0f;
  for (int j = begin + wave; j < n; j += kWaves) {
    const int32_t page = a.table[static_cast<size_t>(r) * a.max_pages + (j >> a.page_shift)];
    if (page < 0 || page >= a.num_pages) continue;
    const size_t row = ((static_cast<size_t>(page) * a.Hk + kvh) << a.page_shift) + (j & ((1 << a.page_shift) - 1));
    float s = 0.0f, v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = 4 * lane + i;
      s += d < D ? q[i] * half_lo<F16>(a.k[row * D + d]) : 0.0f;
      v[i] = d < D ? half_lo<F16>(a.v[row * D + d]) : 0.0f;
    }
#pragma unroll
    for (int k = 32; k >= 1; k >>= 1) s += __shfl_xor(s, k, 64);
    s *= a.scale;
    const float mn = fmaxf(m, s), f = __expf(m - mn), p = __expf(s - mn);
    m = mn;
    l = l * f + p;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = o[i] * f + p * v[i];
  }
  __shared__ float sm[kWaves], sl[kWaves], so[kWaves][256];
  if (lane == 0) {
    sm[wave] = m;
    sl[wave] = l;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) so[wave][4 * lane + i] = o[i];
  __syncthreads();
  float M = -INFINITY, L = 0.0f;
  for (int w = 0; w < kWaves; ++w) M = fmaxf(M, sm[w]);
  float f[kWaves];
  for (int w = 0; w < kWaves; ++w) {
    f[w] = sl[w] > 0.0f ? __expf(sm[w] - M) : 0.0f;
    L += sl[w] * f[w];
  }
  for (int d = threadIdx.x; d < D; d += 64 * kWaves) {
    float y = 0.0f;
    for (int w = 0; w < kWaves; ++w) y += so[w][d] * f[w];
    store_out(a.out, wg * D + d, L > 0.0f ? y / L : 0.0f, a.out_dtype);
  }
  if (threadIdx.x == 0 && a.lse != nullptr) a.lse[wg] = L > 0.0f ? M + logf(L) : -INFINITY;
}

}  // namespace

size_t attn_partial_bytes(int32_t, int32_t, int32_t, int32_t, int32_t) { return 0; }

hipError_t launch_attn_paged(const AttnArgs& a, bool f16, hipStream_t s) {
  const dim3 grid = wg_grid(static_cast<size_t>(a.R) * a.Hq);
  if (f16) {
    attn_simple_kernel<true><<<grid, 64 * kWaves, 0, s>>>(a);
  } else {
    attn_simple_kernel<false><<<grid, 64 * kWaves, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace sq
