// Internal declarations of a decoder's token step: page plan, head norm and
// rotation, paged attention, the bf16 linear on int4 weights, the residual norm;
// and of its beams: their choice, the tables and pages that follow it, attention
// over a shared prefix.
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

struct NormArgs {
  const void *x, *residual;  // residual NULL: none
  int64_t x_stride, residual_stride, sum_stride;
  const float* weight;  // or NULL
  void *sum, *y;        // each or NULL
  int8_t* qx;           // or NULL
  float* scale;
  const int32_t* tok2stream;
  const float *gamma, *clip, *dinv;
  int32_t M, K, x_dtype, residual_dtype, y_dtype, S, step, range_mode;
  float eps;
};
hipError_t launch_add_rmsnorm(const NormArgs& a, hipStream_t s);

struct ReorderArgs {
  const int32_t *parent, *kv_len, *table, *free_head;
  int32_t *free_pages, *table_out, *kv_len_out, *copy_src, *copy_dst, *copy_rows, *free_head_out;
  int32_t* ws;  // reorder_ws_ints()
  int32_t R, max_pages, num_pages, num_free, page_shift;
};
size_t reorder_ws_ints(int32_t R, int32_t num_pages);
hipError_t launch_kv_reorder(const ReorderArgs& a, hipStream_t s);

constexpr int32_t kCopyMaxCaches = 64;  // of one launch: their pointers are its arguments
struct CopyArgs {
  void* pages[2 * kCopyMaxCaches];  // keys and values of every cache
  const int32_t *src, *dst, *rows;  // rows NULL: whole pages
  int32_t n, caches, num_pages, heads, page_shift, row_bytes;
};
hipError_t launch_kv_copy(const CopyArgs& a, hipStream_t s);

struct SharedArgs {
  const uint16_t *q, *k, *v;
  int64_t q_stride;
  const int32_t *table, *kv_len, *group_start, *shared_len;
  void* out;
  float* lse;  // or NULL
  void* ws;    // attn_shared_bytes()
  size_t ws_bytes;
  int32_t R, groups, Hq, Hk, D, max_pages, num_pages, page_shift, max_shared, max_own, out_dtype;
  float scale;
};
size_t attn_shared_bytes(int32_t R, int32_t Hq, int32_t Hk, int32_t D, int32_t max_shared, int32_t max_own);
hipError_t launch_attn_shared(const SharedArgs& a, bool f16, hipStream_t s);

struct BeamArgs {
  const void* logits;
  int64_t stride;
  const float* scores;
  const int32_t* done;  // or NULL
  int32_t *parent, *token, *done_out;
  float* score_out;
  void* ws;  // beam_ws_bytes()
  int32_t rows, beams, vocab, width, end_token, dtype;
};
size_t beam_ws_bytes(int32_t rows, int32_t vocab, int32_t width);
hipError_t launch_beam_select(const BeamArgs& a, hipStream_t s);

}  // namespace sq
