// Attention of one new token per request over a paged key-value cache
// (sq_attn_paged).
#include <algorithm>

#include "half_types.h"
#include "token_internal.h"

namespace sq {
namespace {

constexpr int kWaves = 4;    // of a workgroup
constexpr int kTile = 32;    // tokens a wave takes at a time
constexpr int kQTile = 16;   // query heads of a workgroup: the columns of a 16 x 16 matrix-core tile
constexpr int kMaxChunk = 2048, kMinChunk = 512;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

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

// Maximum / sum over the four lanes that share lane & 15.
__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float quad_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// How a history is split over workgroups.
struct Split {
  int32_t chunk;  // tokens of a workgroup, a multiple of kTile
  int32_t count;  // workgroups of a history of `span` tokens
};
Split split_of(int64_t heads, int32_t span) {
  const int64_t want = std::max<int64_t>(1, 2048 / std::max<int64_t>(1, heads));
  const int64_t even = (span + want - 1) / want;
  int64_t chunk = std::min<int64_t>(kMaxChunk, std::max<int64_t>(kMinChunk, (even + 127) / 128 * 128));
  Split s;
  s.chunk = static_cast<int32_t>(chunk);
  s.count = static_cast<int32_t>(std::max<int64_t>(1, (static_cast<int64_t>(span) + chunk - 1) / chunk));
  return s;
}
int64_t max_splits(int64_t heads, int32_t longest) {
  const int64_t want = std::max<int64_t>(1, 2048 / std::max<int64_t>(1, heads));
  return std::max(std::min<int64_t>(want, (static_cast<int64_t>(longest) + kMinChunk - 1) / kMinChunk),
                  (static_cast<int64_t>(longest) + kMaxChunk - 1) / kMaxChunk);
}
int q_tiles(int32_t Hq, int32_t Hk) { return (Hq / Hk + kQTile - 1) / kQTile; }

// The tokens [first, n) of a request.
__device__ __forceinline__ void range_of(const AttnArgs& a, int r, int& first, int& n) {
  n = min(max(a.kv_len[r], 0), a.max_kv_len);
  first = a.window > 0 ? max(0, n - a.window) : 0;
}

template <bool F16, int D, int NP>
__global__ __launch_bounds__(64 * kWaves, D <= 128 ? 2 : 1) void attn_kernel(AttnArgs a, Split sp, int qtiles) {
  constexpr int KF = D / 32;  // fragments of a key row
  constexpr int E = D / 16;   // dimensions of a lane's part of a value row
  constexpr int EW = E / 2;   // the same in dwords
  constexpr float kShift = F16 ? 11.0f : 0.0f;
  constexpr float kSlack = F16 ? 4.0f : 8.0f;
  __shared__ int32_t pages[kMaxChunk / 8 + 1];
  __shared__ float s_m[kWaves][kQTile], s_l[kWaves][kQTile], s_o[kWaves][kQTile][D + 4];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;

  size_t wg = flat_wg();
  if (wg >= static_cast<size_t>(a.R) * a.Hk * qtiles * sp.count) return;
  const int kvh = static_cast<int>(wg % a.Hk);
  wg /= a.Hk;
  const int qt = static_cast<int>(wg % qtiles);
  wg /= qtiles;
  const int split = static_cast<int>(wg % sp.count);
  const int r = static_cast<int>(wg / sp.count);
  const int G = a.Hq / a.Hk;
  const int gq = min(G - qt * kQTile, kQTile);  // query heads here
  const int h0 = kvh * G + qt * kQTile;

  int first, n;
  range_of(a, r, first, n);
  const int span = n - (first & ~(kTile - 1));
  const bool whole = span <= sp.chunk;  // one workgroup has all of it
  if (split > 0 && static_cast<int64_t>(split) * sp.chunk >= span) return;
  const int begin = (first & ~(kTile - 1)) + split * sp.chunk;
  const int end = begin + min(n - begin, sp.chunk);

  const int shift = a.page_shift, mask = (1 << shift) - 1;
  const int page0 = begin >> shift;
  const int npages = begin < end ? ((end - 1) >> shift) - page0 + 1 : 0;
  for (int i = threadIdx.x; i < npages; i += 64 * kWaves) {
    const int32_t p = a.table[static_cast<size_t>(r) * a.max_pages + page0 + i];
    pages[i] = p >= 0 && p < a.num_pages ? p : -1;
  }

  // queries: column c is head h0 + c, the lane's values 32 j + 8 g ..
  uint4 q[KF];
  const uint16_t* qrow = a.q + r * a.q_stride + static_cast<size_t>(h0 + min(c, gq - 1)) * D + 8 * g;
#pragma unroll
  for (int j = 0; j < KF; ++j) {
    q[j] = *reinterpret_cast<const uint4*>(qrow + 32 * j);
    if (c >= gq) q[j] = make_uint4(0, 0, 0, 0);
  }
  __syncthreads();

  v4f o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = v4f{0, 0, 0, 0};
  float m = -3.402823466e38f, l = 0.0f;
  const float scale = a.scale * kLog2e;

  auto page_of = [&](int tok) { return pages[max(0, min((tok >> shift) - page0, npages - 1))]; };
  auto row_of = [&](int page, int tok) {
    return ((static_cast<size_t>(max(page, 0)) * a.Hk + kvh) << shift) + (tok & mask);
  };
  const int tiles = (end - begin + kTile - 1) / kTile;
  for (int t = wave; t < tiles; t += kWaves) {
    const int b = begin + t * kTile;
    uint4 k[2][KF];
    int kp[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int tok = b + 16 * i + c;
      kp[i] = page_of(tok);
      const uint16_t* p = a.k + row_of(kp[i], tok) * D + 8 * g;
#pragma unroll
      for (int j = 0; j < KF; ++j) k[i][j] = *reinterpret_cast<const uint4*>(p + 32 * j);
    }
    uint32_t v[8][EW];
    int vp[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int tok = b + 16 * i + 4 * g;
      vp[i] = page_of(tok);
      const uint16_t* p = a.v + row_of(vp[i], tok) * D + E * c;
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int w = 0; w < EW; ++w) v[4 * i + x][w] = reinterpret_cast<const uint32_t*>(p + x * D)[w];
    }
    v4f s[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s[i] = v4f{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < KF; ++j) s[i] = mfma<F16>(k[i][j], q[j], s[i]);
    }
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = s[i / 4][i % 4] * scale;
    const bool full = b >= first && b + kTile <= end && __all(kp[0] >= 0 && kp[1] >= 0);
    if (!full) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int tok = b + 16 * (i / 4) + 4 * g + i % 4;
        const bool live = (tok >= first) & (tok < end) & (vp[i / 4] >= 0);
        f[i] = live ? f[i] : -INFINITY;
#pragma unroll
        for (int w = 0; w < EW; ++w) v[i][w] = live ? v[i][w] : 0;
      }
    }
    float top = f[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, f[i]);
    if (__any(top > m + kSlack)) {
      const float mn = fmaxf(m, quad_max(top));
      const float al = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= al;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] *= al;
    }
    uint32_t p[NP][4];
    const float base = m - kShift;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      float x = __builtin_amdgcn_exp2f(f[i] - base), y = __builtin_amdgcn_exp2f(f[i + 1] - base);
      l += x + y;
#pragma unroll
      for (int u = 0; u < NP; ++u) {
        p[u][i / 2] = to_half2<F16>(x, y);
        x -= half_lo<F16>(p[u][i / 2]);
        y -= half_hi<F16>(p[u][i / 2]);
      }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      uint4 vt;
      const uint32_t sel = e & 1 ? 0x07060302u : 0x05040100u;
      vt.x = __builtin_amdgcn_perm(v[1][e / 2], v[0][e / 2], sel);
      vt.y = __builtin_amdgcn_perm(v[3][e / 2], v[2][e / 2], sel);
      vt.z = __builtin_amdgcn_perm(v[5][e / 2], v[4][e / 2], sel);
      vt.w = __builtin_amdgcn_perm(v[7][e / 2], v[6][e / 2], sel);
#pragma unroll
      for (int u = 0; u < NP; ++u) o[e] = mfma<F16>(vt, make_uint4(p[u][0], p[u][1], p[u][2], p[u][3]), o[e]);
    }
  }

  // the waves' parts: column c, dimensions 4 E g + E x + e
  l = quad_sum(l);
  if (g == 0) {
    s_m[wave][c] = m - kShift;
    s_l[wave][c] = l;
  }
#pragma unroll
  for (int e = 0; e < E; ++e)
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (c < gq) s_o[wave][c][E * (4 * g + x) + e] = o[e][x];
  __syncthreads();
  for (int i = threadIdx.x; i < gq * D; i += 64 * kWaves) {
    const int qh = i / D, d = i % D;
    float M = s_m[0][qh];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, s_m[w][qh]);
    float y = 0.0f, L = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float al = __builtin_amdgcn_exp2f(s_m[w][qh] - M);
      L = __builtin_fmaf(s_l[w][qh], al, L);
      y = __builtin_fmaf(s_o[w][qh][d], al, y);
    }
    const size_t row = static_cast<size_t>(r) * a.Hq + h0 + qh;
    if (whole) {
      store_out(a.out, row * D + d, L > 0.0f ? y / L : 0.0f, a.out_dtype);
      if (d == 0 && a.lse != nullptr) a.lse[row] = L > 0.0f ? (M + __builtin_amdgcn_logf(L)) * kLn2 : -INFINITY;
    } else {
      float* part = a.part + (row * sp.count + split) * (D + 2);
      part[2 + d] = y;
      if (d == 0) {
        part[0] = M;
        part[1] = L;
      }
    }
  }
}

// Joins the parts of one query head of a split history, in their order.
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a, Split sp) {
  const size_t row = flat_wg();
  if (row >= static_cast<size_t>(a.R) * a.Hq) return;
  int first, n;
  range_of(a, static_cast<int>(row / a.Hq), first, n);
  const int span = n - (first & ~(kTile - 1));
  if (span <= sp.chunk) return;
  const int count = (span + sp.chunk - 1) / sp.chunk;
  const int D = a.D, d = threadIdx.x;
  const float* part = a.part + row * sp.count * (D + 2);
  float M = -3.402823466e38f;
  for (int s = 0; s < count; ++s) M = fmaxf(M, part[static_cast<size_t>(s) * (D + 2)]);
  float L = 0.0f, y = 0.0f;
  for (int s = 0; s < count; ++s) {
    const float* p = part + static_cast<size_t>(s) * (D + 2);
    const float al = __builtin_amdgcn_exp2f(p[0] - M);
    L = __builtin_fmaf(p[1], al, L);
    if (d < D) y = __builtin_fmaf(p[2 + d], al, y);
  }
  if (d < D) store_out(a.out, row * D + d, L > 0.0f ? y / L : 0.0f, a.out_dtype);
  if (d == 0 && a.lse != nullptr) a.lse[row] = L > 0.0f ? (M + __builtin_amdgcn_logf(L)) * kLn2 : -INFINITY;
}

template <bool F16, int NP>
void launch_dim(const AttnArgs& a, const Split& sp, hipStream_t s) {
  const int qt = q_tiles(a.Hq, a.Hk);
  const dim3 grid = wg_grid(static_cast<size_t>(a.R) * a.Hk * qt * sp.count);
  switch (a.D) {
    case 64: attn_kernel<F16, 64, NP><<<grid, 64 * kWaves, 0, s>>>(a, sp, qt); break;
    case 96: attn_kernel<F16, 96, NP><<<grid, 64 * kWaves, 0, s>>>(a, sp, qt); break;
    case 128: attn_kernel<F16, 128, NP><<<grid, 64 * kWaves, 0, s>>>(a, sp, qt); break;
    case 192: attn_kernel<F16, 192, NP><<<grid, 64 * kWaves, 0, s>>>(a, sp, qt); break;
    default: attn_kernel<F16, 256, NP><<<grid, 64 * kWaves, 0, s>>>(a, sp, qt); break;
  }
}

}  // namespace

size_t attn_partial_bytes(int32_t R, int32_t Hq, int32_t Hk, int32_t D, int32_t max_kv_len) {
  const int64_t splits = max_splits(static_cast<int64_t>(R) * Hk * q_tiles(Hq, Hk), max_kv_len);
  return splits <= 1 ? 0 : static_cast<size_t>(R) * Hq * splits * (D + 2) * 4;
}

hipError_t launch_attn_paged(const AttnArgs& a, bool f16, hipStream_t s) {
  const int32_t span = a.window > 0 ? static_cast<int32_t>(std::min<int64_t>(a.max_kv_len, a.window + int64_t{kTile - 1}))
                                    : a.max_kv_len;
  const Split sp = split_of(static_cast<int64_t>(a.R) * a.Hk * q_tiles(a.Hq, a.Hk), span);
  if (f16)
    launch_dim<true, 2>(a, sp, s);
  else if (a.out_dtype == SQ_OUT_F32)
    launch_dim<false, 3>(a, sp, s);
  else
    launch_dim<false, 2>(a, sp, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || sp.count == 1) return e;
  attn_join_kernel<<<wg_grid(static_cast<size_t>(a.R) * a.Hq), 256, 0, s>>>(a, sp);
  return hipGetLastError();
}

}  // namespace sq
