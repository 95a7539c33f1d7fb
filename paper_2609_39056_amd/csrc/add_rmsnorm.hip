// Residual addition and root-mean-square norm of token rows, to 16 or 32 bits
// and / or to the quantizer's 8-bit codes (sq_add_rmsnorm):
//     h = x + residual,  u = h / sqrt(mean(h^2) + eps) * weight
// One pass: a row's sum stays in registers between the mean and the output, the
// codes take u itself, without a rounding to 16 bits in between.
//
// WPR waves share a row; lane l of the row owns its 8-value chunks l, l + 64 WPR, ..
//
// Memory bounds it without codes (8384 rows of 5120 with a 32-bit residual: 515 MB in 92 us,
// 5.6 TB/s); with codes the vector units are busy 72 % of the time (4192 rows of 2048: 15 us,
// 60 MB), and weights and D^-1 come from the cache.
#include "code_bits.h"
#include "half_types.h"
#include "token_internal.h"

namespace sq {
namespace {

struct Raw8 {
  uint4 a, b;  // b: 32-bit values 4 .. 7
};

__device__ __forceinline__ Raw8 load_raw8(const void* p, size_t at, int32_t dtype) {
  Raw8 r;
  if (dtype == SQ_OUT_F32) {
    const uint4* q = reinterpret_cast<const uint4*>(static_cast<const float*>(p) + at);
    r.a = q[0];
    r.b = q[1];
  } else {
    r.a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at);
    r.b = r.a;
  }
  return r;
}

__device__ __forceinline__ void widen_raw8(const Raw8& r, int32_t dtype, float (&v)[8]) {
  if (dtype == SQ_OUT_BF16) {
    widen8<false>(r.a, v);
  } else if (dtype == SQ_OUT_F16) {
    widen8<true>(r.a, v);
  } else {
    const uint32_t w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
  }
}

__device__ __forceinline__ void store8(void* p, size_t at, const float (&v)[8], int32_t dtype) {
  if (dtype == SQ_OUT_F32) {
    float4* q = reinterpret_cast<float4*>(static_cast<float*>(p) + at);
    q[0] = make_float4(v[0], v[1], v[2], v[3]);
    q[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    uint4* q = reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + at);
    *q = dtype == SQ_OUT_BF16 ? narrow8<false>(v) : narrow8<true>(v);
  }
}

__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}

// Sum or maximum over a row's lanes.
template <int WPR, bool SUM>
__device__ __forceinline__ float over_row(float v, float* red) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    const float w = __shfl_xor(v, o, 64);
    v = SUM ? v + w : fmaxf(v, w);
  }
  if constexpr (WPR > 1) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int w = 1; w < WPR; ++w) v = SUM ? v + red[w] : fmaxf(v, red[w]);
  }
  return v;
}

template <int WPR, int NCH>
__global__ __launch_bounds__(WPR == 1 ? 256 : 64 * WPR) void add_rmsnorm_kernel(NormArgs a) {
  constexpr int kRows = WPR == 1 ? 4 : 1;  // of a workgroup
  constexpr int kLanes = 64 * WPR;
  __shared__ float red[2][WPR];
  const int lr = threadIdx.x % kLanes;
  const size_t row = flat_wg() * kRows + threadIdx.x / kLanes;
  if (row >= static_cast<size_t>(a.M)) return;  // a row's lanes leave together
  const int nch = a.K >> 3;

  Raw8 xr[NCH], rr[NCH];
#pragma unroll
  for (int j = 0; j < NCH; ++j) {
    const int c = lr + j * kLanes;
    if (c < nch) {
      xr[j] = load_raw8(a.x, row * a.x_stride + 8 * c, a.x_dtype);
      if (a.residual != nullptr) rr[j] = load_raw8(a.residual, row * a.residual_stride + 8 * c, a.residual_dtype);
    }
  }
  float v[NCH][8];
  float ss = 0.0f;
#pragma unroll
  for (int j = 0; j < NCH; ++j) {
    const int c = lr + j * kLanes;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[j][i] = 0.0f;
    if (c < nch) {
      widen_raw8(xr[j], a.x_dtype, v[j]);
      if (a.residual != nullptr) {
        float w[8];
        widen_raw8(rr[j], a.residual_dtype, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[j][i] += w[i];
        if (a.sum != nullptr) store8(a.sum, row * a.sum_stride + 8 * c, v[j], a.residual_dtype);
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(v[j][i], v[j][i], ss);
  }
  ss = over_row<WPR, true>(ss, red[0]);
  const float r = 1.0f / sqrtf(ss / static_cast<float>(a.K) + a.eps);
#pragma unroll
  for (int j = 0; j < NCH; ++j) {
    const int c = lr + j * kLanes;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[j][i] *= r;
    if (a.weight != nullptr && c < nch) {
      float w[8];
      load8(a.weight + 8 * c, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j][i] *= w[i];
    }
    if (a.y != nullptr && c < nch) store8(a.y, row * a.K + 8 * c, v[j], a.y_dtype);
  }
  if (a.qx == nullptr) return;

  // the quantizer's chain (sq.h) on u in the place of x
  const bool dynamic = a.range_mode == SQ_RANGE_DYNAMIC;
  float m = 0.0f;
#pragma unroll
  for (int j = 0; j < NCH; ++j) {
    const int c = lr + j * kLanes;
    if (a.dinv != nullptr && c < nch) {
      float d[8];
      load8(a.dinv + 8 * c, d);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j][i] *= d[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(v[j][i]));
  }
  m = dynamic ? over_row<WPR, false>(m, red[1]) : a.clip[a.step];
  const float g = a.gamma[static_cast<size_t>(a.step) * a.S + a.tok2stream[row]];
  const float delta = m / 127.0f;
  float inv = 1.0f / delta;
  if (__builtin_isinf(inv)) inv = 0.0f;
#pragma unroll
  for (int j = 0; j < NCH; ++j) {
    const int c = lr + j * kLanes;
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = rne_code_bits(fminf(fmaxf((v[j][i] * g) * inv, -127.0f), 127.0f));
    if (c < nch)
      *reinterpret_cast<uint2*>(a.qx + row * a.K + 8 * c) =
          make_uint2(pack_low_bytes(b[0], b[1], b[2], b[3]), pack_low_bytes(b[4], b[5], b[6], b[7]));
  }
  if (lr == 0) a.scale[row] = delta / g;
}

template <int WPR, int NCH>
hipError_t launch_rows(const NormArgs& a, hipStream_t s) {
  constexpr int kRows = WPR == 1 ? 4 : 1;
  add_rmsnorm_kernel<WPR, NCH>
      <<<wg_grid((static_cast<size_t>(a.M) + kRows - 1) / kRows), WPR == 1 ? 256 : 64 * WPR, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

// One 8-value chunk per lane, so that a row's loads are all in flight at once and no
// lane does its divisions for more than it holds: a row of 1024 takes 2 waves (4096 rows
// 8.5 us, with 4 waves 9.2), of 2048 4 waves (64 rows 3.2, with one wave 5.4), of 4096 8
// waves (4096 rows 27.3, with 4 waves 29.1), of 8192 16 waves (4096 rows 50.2, with 4 waves
// 55.9).  Between 4096 and 6144 values half to a quarter of 16 waves' lanes has none.  Few rows
// (1 of 5120: 3.1, with 4 waves 4.5; 512 with codes 7.2 and 9.0) and rows without codes (4096
// with a 32-bit residual 48.7 and 53.6) gain all the same; many with codes, whose two
// divisions and two sums every wave repeats, are left at 4 waves (4096 rows 38.8, with 16
// waves 47.1, with 8 43.4).
hipError_t launch_add_rmsnorm(const NormArgs& a, hipStream_t s) {
  const int nch = a.K / 8;
  if (nch <= 64) return launch_rows<1, 1>(a, s);
  if (nch <= 128) return launch_rows<2, 1>(a, s);
  if (nch <= 256) return launch_rows<4, 1>(a, s);
  if (nch <= 512) return launch_rows<8, 1>(a, s);
  if (nch <= 768 && a.qx != nullptr && a.M > 1024) return launch_rows<4, 3>(a, s);
  if (nch <= 1024) return launch_rows<16, 1>(a, s);
  return nch <= 2048 ? launch_rows<16, 2>(a, s) : launch_rows<16, 4>(a, s);
}

}  // namespace sq
