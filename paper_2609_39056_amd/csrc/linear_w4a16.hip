// The few-token linear on packed int4 weights with bf16 activations
// (sq_linear_w4a16).
#include "half_types.h"
#include "token_internal.h"

namespace sq {
namespace {

// One wave per output channel and row: fp32 products over the lanes' chunks of
// 8 codes, each with its group's step.
__global__ __launch_bounds__(256) void linear_w4a16_kernel(LinearArgs a) {
  const int lane = threadIdx.x & 63;
  const int n = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int m = blockIdx.y;
  float acc = 0.0f;
  for (int c = lane; c < a.K / 8; c += 64) {
    const uint32_t p = *reinterpret_cast<const uint32_t*>(a.qw + static_cast<size_t>(n) * (a.K / 2) + 4 * c);
    float x[8];
    widen8<false>(*reinterpret_cast<const uint4*>(a.x + static_cast<size_t>(m) * a.K + 8 * c), x);
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int code = static_cast<int>(p << (28 - (8 * (i & 3) + 4 * (i >> 2)))) >> 28;
      s = __builtin_fmaf(a.dinv != nullptr ? x[i] * a.dinv[8 * c + i] : x[i], static_cast<float>(code), s);
    }
    acc = __builtin_fmaf(s, f16_to_f32(a.w_scale[static_cast<size_t>((8 * c) / a.w_group) * a.N + n]), acc);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) acc += __shfl_xor(acc, o, 64);
  if (lane == 0)
    store_out(a.y, static_cast<size_t>(m) * a.N + n, a.bias != nullptr ? acc + bf16_to_f32(a.bias[n]) : acc, a.out_dtype);
}

}  // namespace

hipError_t launch_linear_w4a16(const LinearArgs& a, hipStream_t s) {
  linear_w4a16_kernel<<<dim3(a.N / 4, a.M), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace sq
