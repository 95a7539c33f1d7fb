// Internal declarations of a decoder's token step: page plan, head norm and
// rotation, paged attention, the bf16 linear on int4 weights.
#pragma once

#include "sq_internal.h"

namespace sq {

struct PlanArgs {
  const int32_t *cached, *fresh, *free_pages, *free_head;
  int32_t *table, *slot, *pos, *token_start, *kv_len, *free_head_out;
  int32_t R, max_pages, max_tokens, num_free, page_shift;
};
constexpr int32_t kPlanMaxRequests = 8192;
hipError_t launch_kv_plan(const PlanArgs& a, hipStream_t s);

struct RopeArgs {
  const uint16_t *q, *k, *v;  // v NULL: no cache
  int64_t q_stride, k_stride, v_stride;
  const float *q_weight, *k_weight, *cos, *sin;
  const int32_t *pos, *slot;  // pos NULL: no rotation
  uint16_t *q_out, *k_out, *k_cache, *v_cache;
  int32_t T, Hq, Hk, D, rot, num_pos, num_pages, page_shift;
  float eps;
};
hipError_t launch_qk_norm_rope(const RopeArgs& a, bool f16, bool interleaved, hipStream_t s);

struct AttnArgs {
  const uint16_t *q, *k, *v;
  int64_t q_stride;
  const int32_t *table, *kv_len;
  void* out;
  float* lse;   // or NULL
  float* part;  // partial results of split histories, part_bytes of them
  size_t part_bytes;
  int32_t R, Hq, Hk, D, max_pages, num_pages, page_shift, max_kv_len, window, out_dtype;
  float scale;
};
// for every batch of at most R requests of at most max_kv_len tokens
size_t attn_partial_bytes(int32_t R, int32_t Hq, int32_t Hk, int32_t D, int32_t max_kv_len);
hipError_t launch_attn_paged(const AttnArgs& a, bool f16, hipStream_t s);

struct LinearArgs {
  const uint16_t* x;
  const float* dinv;  // or NULL
  const uint8_t* qw;
  const uint16_t* w_scale;
  const uint16_t* bias;  // or NULL
  void* y;
  int32_t M, N, K, w_group, out_dtype;
};
constexpr int32_t kLinear16MaxM = 64;
hipError_t launch_linear_w4a16(const LinearArgs& a, hipStream_t s);

}  // namespace sq
