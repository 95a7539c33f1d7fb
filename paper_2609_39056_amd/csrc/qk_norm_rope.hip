// Per-head norm of queries and keys, position rotation and cache write in one
// pass (sq_qk_norm_rope).
#include "half_types.h"
#include "token_internal.h"

namespace sq {
namespace {

constexpr int kRopeThreads = 256;

// A group of GL lanes takes one head; a lane holds two chunks of 8 values that
// the rotation pairs with each other (halves: chunk c and c + rot / 16), or
// two adjacent chunks (adjacent pairs, and the values past rot).  So the
// rotation needs no exchange between lanes, and the norm a sum over GL lanes.
// A workgroup takes `per` heads of one token, whose cos and sin stay in
// registers over the heads; the next head is loaded ahead.
template <bool F16, bool INTER, int GL>
__global__ __launch_bounds__(kRopeThreads) void qk_norm_rope_kernel(RopeArgs a, uint32_t parts, int per) {
  constexpr int kGroups = kRopeThreads / GL;
  const uint32_t wg = static_cast<uint32_t>(flat_wg());  // at most 2^24 tokens of 96 parts
  const int heads = a.Hq + a.Hk + (a.v != nullptr ? a.Hk : 0);
  if (wg >= static_cast<uint32_t>(a.T) * parts) return;
  const uint32_t t32 = parts == 1 ? wg : wg / parts;
  const size_t t = t32;
  const int h0 = static_cast<int>(wg - t32 * parts) * per, end = min(h0 + per, heads);
  const int u = threadIdx.x % GL;  // pair of chunks
  const int D = a.D, rot = a.rot;
  const int pairs = D / 16, rpairs = rot / 16;
  const int uc = min(u, pairs - 1);
  const bool rotated = uc < rpairs;
  const int ca = INTER || !rotated ? 2 * uc : uc;
  const int cb = INTER || !rotated ? 2 * uc + 1 : uc + rpairs;

  uint4 na = make_uint4(0, 0, 0, 0), nb = na;  // the next head's chunks
  auto load = [&](int h) {
    if (h >= end || u >= pairs) return;
    const uint16_t* src = h < a.Hq          ? a.q + t * a.q_stride + static_cast<size_t>(h) * D
                          : h < a.Hq + a.Hk ? a.k + t * a.k_stride + static_cast<size_t>(h - a.Hq) * D
                                            : a.v + t * a.v_stride + static_cast<size_t>(h - a.Hq - a.Hk) * D;
    na = *reinterpret_cast<const uint4*>(src + 8 * ca);
    nb = *reinterpret_cast<const uint4*>(src + 8 * cb);
  };
  load(h0 + threadIdx.x / GL);

  float c[8], n[8];
  if (rot > 0) {
    const int32_t p = a.pos[t];
    if (p < 0 || p >= a.num_pos) return;
    const size_t at = static_cast<size_t>(p) * (rot / 2) + 8 * (rotated ? uc : 0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      c[i] = a.cos[at + i];
      n[i] = a.sin[at + i];
    }
  }
  const int32_t slot = a.slot != nullptr ? a.slot[t] : -1;
  const bool cached = slot >= 0 && (slot >> a.page_shift) < a.num_pages;
  const size_t page = cached ? slot >> a.page_shift : 0;
  const int in_page = slot & ((1 << a.page_shift) - 1);

  for (int hb = h0; hb < end; hb += kGroups) {
    const int h = hb + threadIdx.x / GL;
    const bool live = h < end && u < pairs;
    const int kind = h < a.Hq ? 0 : (h < a.Hq + a.Hk ? 1 : 2);
    const int hh = kind == 0 ? h : (kind == 1 ? h - a.Hq : h - a.Hq - a.Hk);
    const uint4 ra = na, rb = nb;
    if (hb + kGroups < end) load(h + kGroups);
    const size_t row = ((page * a.Hk + hh) << a.page_shift) + in_page;
    if (kind == 2) {
      if (live && cached) {
        *reinterpret_cast<uint4*>(a.v_cache + row * D + 8 * ca) = ra;
        *reinterpret_cast<uint4*>(a.v_cache + row * D + 8 * cb) = rb;
      }
      continue;
    }
    float va[8], vb[8];
    widen8<F16>(ra, va);
    widen8<F16>(rb, vb);
    const float* w = kind == 0 ? a.q_weight : a.k_weight;
    if (w != nullptr) {
      float ss = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(va[i], va[i], __builtin_fmaf(vb[i], vb[i], ss));
#pragma unroll
      for (int o = GL / 2; o >= 1; o >>= 1) ss += __shfl_xor(ss, o, 64);
      const float r = 1.0f / sqrtf(ss / static_cast<float>(D) + a.eps);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        va[i] = va[i] * r * w[8 * ca + i];
        vb[i] = vb[i] * r * w[8 * cb + i];
      }
    }
    if (rotated) {
      if constexpr (INTER) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = va[2 * i], y = va[2 * i + 1];
          va[2 * i] = x * c[i] - y * n[i];
          va[2 * i + 1] = y * c[i] + x * n[i];
          const float z = vb[2 * i], m = vb[2 * i + 1];
          vb[2 * i] = z * c[4 + i] - m * n[4 + i];
          vb[2 * i + 1] = m * c[4 + i] + z * n[4 + i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = va[i], y = vb[i];
          va[i] = x * c[i] - y * n[i];
          vb[i] = y * c[i] + x * n[i];
        }
      }
    }
    if (!live) continue;
    const uint4 oa = narrow8<F16>(va), ob = narrow8<F16>(vb);
    if (kind == 0) {
      uint16_t* o = a.q_out + (t * a.Hq + hh) * D;
      *reinterpret_cast<uint4*>(o + 8 * ca) = oa;
      *reinterpret_cast<uint4*>(o + 8 * cb) = ob;
    } else {
      if (a.k_out != nullptr) {
        uint16_t* o = a.k_out + (t * a.Hk + hh) * D;
        *reinterpret_cast<uint4*>(o + 8 * ca) = oa;
        *reinterpret_cast<uint4*>(o + 8 * cb) = ob;
      }
      if (cached) {
        *reinterpret_cast<uint4*>(a.k_cache + row * D + 8 * ca) = oa;
        *reinterpret_cast<uint4*>(a.k_cache + row * D + 8 * cb) = ob;
      }
    }
  }
}

template <bool F16, bool INTER, int GL>
void launch_groups(const RopeArgs& a, hipStream_t s) {
  constexpr int kGroups = kRopeThreads / GL;
  const int heads = a.Hq + a.Hk + (a.v != nullptr ? a.Hk : 0);
  const int rounds = (heads + kGroups - 1) / kGroups;
  // few tokens: their heads over more workgroups, a round each (8 tokens of 120
  // heads: 6.8 us in four rounds, 5.9; from 512 on the parts only repeat cos and sin)
  const uint32_t parts = a.T < 512 ? rounds : 1;
  const int per = (rounds + static_cast<int>(parts) - 1) / static_cast<int>(parts) * kGroups;
  qk_norm_rope_kernel<F16, INTER, GL><<<wg_grid(static_cast<size_t>(a.T) * parts), kRopeThreads, 0, s>>>(a, parts, per);
}

template <bool F16, bool INTER>
void launch_head_width(const RopeArgs& a, hipStream_t s) {
  if (a.D <= 64) {
    launch_groups<F16, INTER, 4>(a, s);
  } else if (a.D <= 128) {
    launch_groups<F16, INTER, 8>(a, s);
  } else {
    launch_groups<F16, INTER, 16>(a, s);
  }
}

}  // namespace

hipError_t launch_qk_norm_rope(const RopeArgs& a, bool f16, bool interleaved, hipStream_t s) {
  if (f16) {
    interleaved ? launch_head_width<true, true>(a, s) : launch_head_width<true, false>(a, s);
  } else {
    interleaved ? launch_head_width<false, true>(a, s) : launch_head_width<false, false>(a, s);
  }
  return hipGetLastError();
}

}  // namespace sq
