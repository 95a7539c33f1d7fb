// Codes of the quantizers from scaled fp32 values.
#pragma once

#include "sq_internal.h"

namespace sq {
namespace {

// t rounded to the nearest integer, ties to even, for abs(t) <= 2^22: adding
// 1.5 * 2^23 leaves exactly the rounded value in the low mantissa bits, so the
// two's-complement code is the low byte (8-bit) or nibble (4-bit) of the sum.
__device__ __forceinline__ uint32_t rne_code_bits(float t) { return __float_as_uint(t + 12582912.0f); }

// Bytes b0 of four words, in order, as one word.
__device__ __forceinline__ uint32_t pack_low_bytes(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3) {
  const uint32_t lo = __builtin_amdgcn_perm(w1, w0, 0x0c0c0400u);  // [w0.b0, w1.b0, 0, 0]
  const uint32_t hi = __builtin_amdgcn_perm(w3, w2, 0x0c0c0400u);  // [w2.b0, w3.b0, 0, 0]
  return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
}

}  // namespace
}  // namespace sq
