// The few-token linear on packed int4 weights with bf16 activations
// (sq_linear_w4a16).
//
// y[m][n] = sum over 128-channel blocks b of Delta[b][n] * sum_k x~[m][k] code[n][k]
// on the bf16 matrix cores (16 x 16 x 32): the codes are exact in bf16, x~ is
// a sum of NP bf16 parts (x itself without a channel scaling, 16 bits of
// x * dinv for 16-bit outputs, all 24 for fp32 ones), products are exact and
// sums fp32.  A code is met as code + 8 (widen_codes); the matrix cores also
// take the block's -8 * sum_k x~, as one more operand of constants.
//
// The work is reading the weights once.  A workgroup owns 16 NT output
// channels; its waves take the 128-channel blocks of K in turn (a lane 16
// bytes of one channel's row per block) and their sums are added in wave
// order through LDS.
#include <algorithm>

#include "half_types.h"
#include "token_internal.h"

namespace sq {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kBlock = 128;              // channels of a block
constexpr int kStageBytes = 64 << 10;    // LDS for staged activations

__device__ __forceinline__ v4f mfma(const uint4& x, const uint4& w, v4f c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, w), c, 0, 0, 0);
}

// Eight codes of a packed dword as bf16 (code + 8) * 2^-9: a nibble with its
// sign bit flipped is code + 8 in 0 .. 15, which as an fp8 e4m3 byte is that
// number times 2^-9, exactly (subnormal up to 7, then the first binade).
// Byte b holds codes b and b + 4: the low nibbles are codes 0 .. 3.
constexpr float kCodeUnit = 512.0f;
constexpr uint32_t kMinus8 = 0xBC80BC80u;  // two bf16 -8 * 2^-9
__device__ __forceinline__ uint4 widen_codes(uint32_t p) {
  const uint32_t lo = (p & 0x0F0F0F0Fu) ^ 0x08080808u, hi = ((p >> 4) & 0x0F0F0F0Fu) ^ 0x08080808u;
  uint4 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false));
  r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true));
  r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false));
  r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true));
  return r;
}

// The NP bf16 parts of eight x~: each takes what the earlier ones left.
template <int NP>
__device__ __forceinline__ void parts_of(const uint4& raw, const float* dinv, uint4 (&p)[NP]) {
  if constexpr (NP == 1) {
    p[0] = raw;
  } else {
    float v[8];
    widen8<false>(raw, v);
    const float4 d0 = *reinterpret_cast<const float4*>(dinv), d1 = *reinterpret_cast<const float4*>(dinv + 4);
    const float d[8] = {d0.x, d0.y, d0.z, d0.w, d1.x, d1.y, d1.z, d1.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= d[i];
#pragma unroll
    for (int u = 0; u < NP; ++u) {
      p[u] = narrow8<false>(v);
      if (u + 1 < NP) {
        float h[8];
        widen8<false>(p[u], h);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] -= h[i];
      }
    }
  }
}

// The weights and steps of one block for a wave: lane (c, g) holds channels
// 32 g .. of the rows n0 + 16 t + c.
template <int NT>
struct Block {
  uint4 w[NT];
  uint16_t step[NT];
};
template <int NT>
__device__ __forceinline__ void load_block(const LinearArgs& a, int n0, int b, Block<NT>& o) {
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const uint16_t* step = a.w_scale + static_cast<size_t>((b * kBlock) / a.w_group) * a.N + n0 + c;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    o.w[t] = *reinterpret_cast<const uint4*>(a.qw + static_cast<size_t>(n0 + 16 * t + c) * (a.K / 2) + b * (kBlock / 2) + 16 * g);
    o.step[t] = step[16 * t];
  }
}

// total += Delta * (block sums) of the rows whose fragments f[0 .. 4) hold.
template <int NT, int NP>
__device__ __forceinline__ void add_block(const uint4 (&f)[4][NP], const Block<NT>& blk, v4f (&total)[NT]) {
  const uint4 m8 = make_uint4(kMinus8, kMinus8, kMinus8, kMinus8);
  v4f base = v4f{0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int u = 0; u < NP; ++u) base = mfma(f[j][u], m8, base);
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    v4f acc = base;
    const uint32_t w[4] = {blk.w[t].x, blk.w[t].y, blk.w[t].z, blk.w[t].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint4 codes = widen_codes(w[j]);
#pragma unroll
      for (int u = 0; u < NP; ++u) acc = mfma(f[j][u], codes, acc);
    }
    const float step = f16_to_f32(blk.step[t]) * kCodeUnit;
#pragma unroll
    for (int i = 0; i < 4; ++i) total[t][i] = __builtin_fmaf(acc[i], step, total[t][i]);
  }
}

// Adds the waves' sums (rows m * np .. + np make output row m), bias, store.
template <int NT>
__device__ __forceinline__ void finish(const LinearArgs& a, const float* sums, int waves, int rows, int np, int n0) {
  for (int i = threadIdx.x; i < a.M * 16 * NT; i += blockDim.x) {
    const int m = i / (16 * NT), t = (i / 16) % NT, c = i % 16;
    float y = 0.0f;
    for (int w = 0; w < waves; ++w)
      for (int u = 0; u < np; ++u) y += sums[((w * NT + t) * rows + m * np + u) * 16 + c];
    const int n = n0 + 16 * t + c;
    if (a.bias != nullptr) y += bf16_to_f32(a.bias[n]);
    store_out(a.y, static_cast<size_t>(m) * a.N + n, y, a.out_dtype);
  }
}

// Few rows (M * NP <= 16): the parts of x~ are rows of one matrix-core tile.
// The workgroup stages them for `iters` blocks per wave at a time in LDS, in
// 16-byte pieces ((block * 4 + j) * 4 + g) * R + row, so every x~ is split
// once per workgroup and a wave reads its fragments as whole lines.
template <int NP, int NT>
__global__ __launch_bounds__(1024) void linear_staged_kernel(LinearArgs a, int iters) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  uint4* stage = reinterpret_cast<uint4*>(lds);
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int R = a.M * NP, nblk = a.K / kBlock;
  const int n0 = blockIdx.x * 16 * NT;
  v4f total[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) total[t] = v4f{0, 0, 0, 0};
  Block<NT> next;
  if (wave < nblk) load_block<NT>(a, n0, wave, next);
  for (int b0 = 0; b0 < nblk; b0 += iters * waves) {
    const int blocks = min(iters * waves, nblk - b0);
    if (b0 > 0) __syncthreads();
    for (int i = threadIdx.x; i < blocks * 16 * a.M; i += blockDim.x) {
      const int piece = i % (blocks * 16), m = i / (blocks * 16);
      const int k = b0 * kBlock + piece * 8;
      uint4 p[NP];
      parts_of<NP>(*reinterpret_cast<const uint4*>(a.x + static_cast<size_t>(m) * a.K + k), a.dinv + k, p);
      const int at = ((piece / 16) * 16 + (piece & 3) * 4 + ((piece >> 2) & 3)) * R + m * NP;
#pragma unroll
      for (int u = 0; u < NP; ++u) stage[at + u] = p[u];
    }
    __syncthreads();
    for (int b = wave; b < blocks; b += waves) {
      const Block<NT> blk = next;
      if (b0 + b + waves < nblk) load_block<NT>(a, n0, b0 + b + waves, next);
      uint4 f[4][1];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f[j][0] = make_uint4(0, 0, 0, 0);
        if (c < R) f[j][0] = stage[(b * 16 + j * 4 + g) * R + c];
      }
      add_block<NT, 1>(f, blk, total);
    }
  }
  __syncthreads();
  float* sums = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[((wave * NT + t) * 16 + 4 * g + i) * 16 + c] = total[t][i];
  __syncthreads();
  finish<NT>(a, sums, waves, 16, NP, n0);
}

// More rows: RT tiles of 16 rows, whose parts each wave splits in registers
// as it needs them (rows past M repeat the last one and are not stored).
template <int NP, int NT, int RT>
__global__ __launch_bounds__(512) void linear_rows_kernel(LinearArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int nblk = a.K / kBlock;
  const int n0 = blockIdx.x * 16 * NT;
  v4f total[RT][NT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int t = 0; t < NT; ++t) total[r][t] = v4f{0, 0, 0, 0};
  Block<NT> next;
  if (wave < nblk) load_block<NT>(a, n0, wave, next);
  for (int b = wave; b < nblk; b += waves) {
    const Block<NT> blk = next;
    if (b + waves < nblk) load_block<NT>(a, n0, b + waves, next);
    const int k = b * kBlock + 32 * g;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const uint16_t* x = a.x + static_cast<size_t>(min(16 * r + c, a.M - 1)) * a.K + k;
      uint4 f[4][NP];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        parts_of<NP>(*reinterpret_cast<const uint4*>(x + 8 * j), a.dinv + k + 8 * j, f[j]);
      add_block<NT, NP>(f, blk, total[r]);
    }
  }
  float* sums = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) sums[((wave * NT + t) * 16 * RT + 16 * r + 4 * g + i) * 16 + c] = total[r][t][i];
  __syncthreads();
  finish<NT>(a, sums, waves, 16 * RT, 1, n0);
}

template <int NP, int NT>
void launch_tiles(const LinearArgs& a, hipStream_t s) {
  const int nblk = a.K / kBlock;
  const int R = a.M * NP;
  const unsigned grid = static_cast<unsigned>(a.N / (16 * NT));
  if (R <= 16) {
    const int waves = nblk >= 16 ? 16 : (nblk >= 8 ? 8 : 4);
    const int iters = std::max(1, std::min((nblk + waves - 1) / waves, kStageBytes / (waves * R * 2 * kBlock)));
    const size_t bytes = std::max(static_cast<size_t>(iters) * waves * R * 2 * kBlock, static_cast<size_t>(waves) * NT * 1024);
    linear_staged_kernel<NP, NT><<<grid, 64 * waves, bytes, s>>>(a, iters);
    return;
  }
  const int waves = nblk >= 8 ? 8 : 4;
  const int rt = a.M <= 16 ? 1 : (a.M <= 32 ? 2 : 4);
  const size_t bytes = static_cast<size_t>(waves) * NT * rt * 1024;
  if (rt == 1) {
    linear_rows_kernel<NP, NT, 1><<<grid, 64 * waves, bytes, s>>>(a);
  } else if (rt == 2) {
    linear_rows_kernel<NP, NT, 2><<<grid, 64 * waves, bytes, s>>>(a);
  } else if constexpr (NT <= 2) {
    linear_rows_kernel<NP, NT, 4><<<grid, 64 * waves, bytes, s>>>(a);
  }
}

template <int NP>
void launch_parts(const LinearArgs& a, hipStream_t s) {
  const int strips = a.N / 16;
  if (strips <= 256) {
    launch_tiles<NP, 1>(a, s);
  } else if (strips <= 512 || a.M > 32) {
    launch_tiles<NP, 2>(a, s);
  } else {
    launch_tiles<NP, 4>(a, s);
  }
}

}  // namespace

hipError_t launch_linear_w4a16(const LinearArgs& a, hipStream_t s) {
  if (a.dinv == nullptr)
    launch_parts<1>(a, s);
  else if (a.out_dtype == SQ_OUT_F32)
    launch_parts<3>(a, s);
  else
    launch_parts<2>(a, s);
  return hipGetLastError();
}

}  // namespace sq
