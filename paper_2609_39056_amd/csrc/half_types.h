// The 16-bit types of the token step's tensors, bf16 and f16: widening is
// exact, narrowing rounds to nearest even with the hardware conversion (NaN
// stays NaN).
#pragma once

#include "sq_internal.h"

namespace sq {
namespace {

template <bool F16>
__device__ __forceinline__ float half_lo(uint32_t w) {
  if constexpr (F16) return f16_to_f32(w & 0xFFFFu);
  return __uint_as_float(w << 16);
}
template <bool F16>
__device__ __forceinline__ float half_hi(uint32_t w) {
  if constexpr (F16) return f16_to_f32(w >> 16);
  return __uint_as_float(w & 0xFFFF0000u);
}
template <bool F16>
__device__ __forceinline__ uint32_t to_half(float v) {
  if constexpr (F16) return f32_to_f16(v);
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
}
// Both halves with one conversion.
template <bool F16>
__device__ __forceinline__ uint32_t to_half2(float lo, float hi) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
  const f32x2_t v = {lo, hi};
  if constexpr (F16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2_t));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}

// 8 values of 16 bits <-> 8 floats
template <bool F16>
__device__ __forceinline__ void widen8(const uint4& r, float (&v)[8]) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = half_lo<F16>(w[i]);
    v[2 * i + 1] = half_hi<F16>(w[i]);
  }
}
template <bool F16>
__device__ __forceinline__ uint4 narrow8(const float (&v)[8]) {
  return make_uint4(to_half2<F16>(v[0], v[1]), to_half2<F16>(v[2], v[3]), to_half2<F16>(v[4], v[5]),
                    to_half2<F16>(v[6], v[7]));
}

// One output value of SQ_OUT_F32 / BF16 / F16.
__device__ __forceinline__ void store_out(void* y, size_t i, float v, int32_t out_dtype) {
  if (out_dtype == SQ_OUT_F32) {
    static_cast<float*>(y)[i] = v;
  } else {
    static_cast<uint16_t*>(y)[i] = static_cast<uint16_t>(out_dtype == SQ_OUT_BF16 ? to_half<false>(v) : to_half<true>(v));
  }
}

// Four of them from index 4 i on.
__device__ __forceinline__ void store_out4(void* y, size_t i, const float4& v, int32_t out_dtype) {
  if (out_dtype == SQ_OUT_F32) {
    static_cast<float4*>(y)[i] = v;
  } else if (out_dtype == SQ_OUT_BF16) {
    static_cast<uint2*>(y)[i] = make_uint2(to_half2<false>(v.x, v.y), to_half2<false>(v.z, v.w));
  } else {
    static_cast<uint2*>(y)[i] = make_uint2(to_half2<true>(v.x, v.y), to_half2<true>(v.z, v.w));
  }
}

}  // namespace
}  // namespace sq
