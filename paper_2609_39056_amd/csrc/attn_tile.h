// What the attention kernels share: 16 x 16 x 32 matrix-core tiles, loads of keys
// and values, softmax pieces.  Scores are in units of log 2.
#pragma once

#include "half_types.h"

namespace sq {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kLowest = -3.402823466e38f;  // no score yet

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef unsigned int v2u __attribute__((ext_vector_type(2)));

template <bool F16>
__device__ __forceinline__ v4f mfma(const uint4& x, const uint4& y, v4f c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
}

__device__ __forceinline__ bool is_nan(float v) { return v != v; }

// Maximum / sum over the four lanes that share lane & 15.
__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float quad_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// Loads of a row's pieces: past the caches where a row is read once (STREAM).
template <bool STREAM = true>
__device__ __forceinline__ uint4 load16(const uint16_t* p) {
  typedef unsigned int vec __attribute__((ext_vector_type(4)));
  const vec* q = reinterpret_cast<const vec*>(p);
  return __builtin_bit_cast(uint4, STREAM ? __builtin_nontemporal_load(q) : *q);
}
// N dwords from a 4-byte boundary.
template <int N, bool STREAM = true>
__device__ __forceinline__ void load_words(const uint16_t* p, uint32_t* w) {
  typedef unsigned int vec __attribute__((ext_vector_type(N), aligned(4)));
  const vec* q = reinterpret_cast<const vec*>(p);
  const vec r = STREAM ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = r[i];
}

__device__ __forceinline__ void add_scaled(float4& y, const float4& v, float al) {
  y.x = __builtin_fmaf(v.x, al, y.x);
  y.y = __builtin_fmaf(v.y, al, y.y);
  y.z = __builtin_fmaf(v.z, al, y.z);
  y.w = __builtin_fmaf(v.w, al, y.w);
}

}  // namespace
}  // namespace sq
