// The few-token linear on packed int4 weights with bf16 activations
// (sq_linear_w4a16).
//
// y[m][n] = sum over 128-channel blocks b of Delta[b][n] * sum_k x~[m][k] code[n][k]
// on the bf16 matrix cores (16 x 16 x 32): the codes are exact in bf16, x~ is
// a sum of NP bf16 parts (x itself without a channel scaling, 16 bits of
// x * dinv for 16-bit outputs, all 24 for fp32 ones), products are exact and
// sums fp32.  A code is met as code + 8 (widen_codes); the matrix cores also
// take the block's -8 * sum_k x~, as one more operand of constants, so that the
// fp32 sums of a block are several times its products (16 rows of 13824 -> 5120
// against 64 bits: 5.6e-7 relative, the plain fp32 product 9.7e-7).
//
// The two parts leave up to 2^-17 of a term: before the output's rounding (2^-9 or
// 2^-12 of the result) several times what fp32 does, after it 1.1 to 1.2 % of the f16
// and 0.2 % of the bf16 outputs are not the nearest value (plain fp32 0.2 to 0.5 and
// 0.04 to 0.07 %; 16 rows of 2048 -> 2048 and 13824 -> 5120).  Three parts are 15 to
// 30 % slower from three rows on (8 rows of 5120 -> 5120 12.8 us, two 10.9; 64 of
// 5120 -> 13824 47.7 and 36.4).
//
// The work is reading the weights once.  A workgroup owns 16 NT output
// channels; its waves take the 128-channel blocks of K in turn (a lane 16
// bytes of one channel's row per block) and their sums are added in wave
// order through LDS.
#include <algorithm>

#include "gemm_frag.h"
#include "half_types.h"
#include "token_internal.h"

namespace sq {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kBlock = 128;              // channels of a block

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
    const uint8_t* row = a.qw + static_cast<size_t>(n0 + 16 * t + c) * (a.K / 2);
    o.w[t] = *reinterpret_cast<const uint4*>(row + b * (kBlock / 2) + 16 * g);
    o.step[t] = step[16 * t];
  }
}

// total += Delta * (block sums); fragment(j) gives the NP parts of the rows at
// the lane's channels 8 j ..
template <int NT, int NP, typename Fragment>
__device__ __forceinline__ void add_block(Fragment fragment, const Block<NT>& blk, v4f (&total)[NT]) {
  const uint4 m8 = make_uint4(kMinus8, kMinus8, kMinus8, kMinus8);
  v4f base = v4f{0, 0, 0, 0}, acc[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) acc[t] = v4f{0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint4 f[NP];
    fragment(j, f);
#pragma unroll
    for (int u = 0; u < NP; ++u) base = mfma(f[u], m8, base);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const uint32_t w[4] = {blk.w[t].x, blk.w[t].y, blk.w[t].z, blk.w[t].w};
      const uint4 codes = widen_codes(w[j]);
#pragma unroll
      for (int u = 0; u < NP; ++u) acc[t] = mfma(f[u], codes, acc[t]);
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const float step = f16_to_f32(blk.step[t]) * kCodeUnit;
#pragma unroll
    for (int i = 0; i < 4; ++i) total[t][i] = __builtin_fmaf(acc[t][i] + base[i], step, total[t][i]);
  }
}

// y[m][n] without the bias as the formula reads, one product after the other.
__device__ float plain_sum(const LinearArgs& a, int m, int n) {
  const uint32_t* codes = reinterpret_cast<const uint32_t*>(a.qw + static_cast<size_t>(n) * (a.K / 2));
  const uint16_t* x = a.x + static_cast<size_t>(m) * a.K;
  float y = 0.0f;
  for (int k0 = 0; k0 < a.K && y == y; k0 += 8) {  // NaN stays
    const float step = f16_to_f32(a.w_scale[static_cast<size_t>(k0 / a.w_group) * a.N + n]);
    const uint32_t p = codes[k0 / 8];
    for (int i = 0; i < 8; ++i) {
      const int code = static_cast<int>(p << (28 - 8 * (i & 3) - 4 * (i >> 2))) >> 28;
      const float v = bf16_to_f32(x[k0 + i]);
      y = __builtin_fmaf(a.dinv != nullptr ? v * a.dinv[k0 + i] : v, static_cast<float>(code) * step, y);
    }
  }
  return y;
}

// Adds the waves' sums (tile rows m * np .. + np make output row m0 + m), bias,
// store.  The parts of an infinite x~ (or of one past bf16's range) and code + 8
// beside -8 leave NaN or infinities that its products do not have: such a sum is
// formed again.
template <int NT>
__device__ __forceinline__ void finish(const LinearArgs& a, const float* sums, int waves, int tile_rows, int np, int m0,
                                       int rows, int n0) {
  auto sum_of = [&](int i) {
    const int m = i / (16 * NT), t = (i / 16) % NT, c = i % 16;
    float y = 0.0f;
    for (int u = 0; u < np; ++u) {
      const float* p = sums + (t * tile_rows + m * np + u) * 16 + c;
#pragma unroll 4
      for (int w = 0; w < waves; ++w) y += p[w * NT * tile_rows * 16];
    }
    return y;
  };
  auto put = [&](int i, float y) {
    const int m = m0 + i / (16 * NT), n = n0 + 16 * ((i / 16) % NT) + i % 16;
    if (a.bias != nullptr) y += bf16_to_f32(a.bias[n]);
    store_out(a.y, static_cast<size_t>(m) * a.N + n, y, a.out_dtype);
  };
  bool odd = false;
  for (int i = threadIdx.x; i < rows * 16 * NT; i += blockDim.x) {
    const float y = sum_of(i);
    odd |= y - y != 0.0f;
    put(i, y);
  }
  if (!odd) return;
  for (int i = threadIdx.x; i < rows * 16 * NT; i += blockDim.x) {
    const float y = sum_of(i);
    if (y - y != 0.0f) put(i, plain_sum(a, m0 + i / (16 * NT), n0 + 16 * ((i / 16) % NT) + i % 16));
  }
}

// A row or a few with a channel scaling: the parts of x~ are rows of one
// matrix-core tile.  The workgroup stages all of them in LDS, in 16-byte pieces
// ((block * 4 + j) * 4 + g) * R + row, so that only the rows there are get split,
// by all its lanes (one row of 13824 -> 5120: 13.4 us, with the kernel below
// 21.0); the wave's next block is loaded ahead.
template <int NP, int NT>
__global__ __launch_bounds__(1024) void linear_staged_kernel(LinearArgs a) {
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
  const int pieces = nblk * 16;
  for (int i = threadIdx.x; i < pieces * a.M; i += blockDim.x) {
    const int piece = i % pieces, m = i / pieces;
    uint4 p[NP];
    parts_of<NP>(*reinterpret_cast<const uint4*>(a.x + static_cast<size_t>(m) * a.K + piece * 8), a.dinv + piece * 8, p);
    const int at = ((piece / 16) * 16 + (piece & 3) * 4 + ((piece >> 2) & 3)) * R + m * NP;
#pragma unroll
    for (int u = 0; u < NP; ++u) stage[at + u] = p[u];
  }
  __syncthreads();
  for (int b = wave; b < nblk; b += waves) {
    const Block<NT> blk = next;
    if (b + waves < nblk) load_block<NT>(a, n0, b + waves, next);
    add_block<NT, 1>(
        [&](int j, uint4(&f)[1]) {
          f[0] = make_uint4(0, 0, 0, 0);
          if (c < R) f[0] = stage[(b * 16 + j * 4 + g) * R + c];
        },
        blk, total);
  }
  __syncthreads();
  float* sums = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[((wave * NT + t) * 16 + 4 * g + i) * 16 + c] = total[t][i];
  __syncthreads();
  finish<NT>(a, sums, waves, 16, NP, 0, a.M, n0);
}

// The rest: RT tiles of 16 rows.  Each wave copies its blocks (activation rows,
// weights, weight steps and the channel scaling) by direct global -> LDS loads
// into a ring of its own, SLOTS - 1 blocks ahead, and splits x~ in registers as
// it takes the fragments.  The copies go along the rows, four rows of 256
// bytes (16 of 64) per instruction; loads in the fragments' own layout touch a
// line with every lane, and those kept the address unit busy for the whole
// kernel (16 rows of 13824 -> 5120 without a channel scaling: 22.8 us, now 13.8).
// A wave reads only what it copied: the loop has no barriers.  W waves: eight,
// twelve for strips of 16 channels (16 rows of 8192 -> 2048 11.7 us, eight 12.7).
// With two row tiles there is no block ahead (64 rows of 5120 -> 13824, scaled: 38.4
// us, 42.6 in four waves with one), and where workgroups outnumber the CUs they are
// of four waves, two to a CU (36.0; unscaled 22.5, eight waves 25.6; but 64 rows of
// 5120 -> 5120, unscaled, with CUs to spare 17.0 and 13.5).  With a
// scaling and 16 rows what is left is the splitting of x~ in every workgroup, 7.5
// vector operations a value (13824 -> 5120, fp32 out: 23.4 us, 25.0 on weights that
// come from memory, vector units 74 % busy; 13.8 without).
template <int NP, int NT, int RT, int NW>
struct Ring {
  static constexpr int X = RT * 16 * 2 * kBlock;    // row r, 16-byte chunk k at r * 256 + 16 * (k ^ (r & 15))
  static constexpr int W = NT * 16 * (kBlock / 2);  // channel n, chunk k at n * 64 + 16 * (k ^ ((n >> 2) & 3))
  static constexpr int W_OFF = X, S_OFF = X + W, D_OFF = S_OFF + 256;
  static constexpr int SLOT = D_OFF + (NP > 1 ? 4 * kBlock : 0);
  static constexpr int COPIES = RT * 4 + NT + 1 + (NP > 1 ? 2 : 0);
  static constexpr int SLOTS = RT == 1 ? 2 : 1;
  static constexpr int WAVES = NW;
  static_assert(WAVES * SLOTS * SLOT <= 160 * 1024, "the rings fit in the LDS");
  static_assert(NT * RT * 1024 <= SLOTS * SLOT, "the waves' sums fit in the rings");
};

template <int NP, int NT, int RT, int W>
__global__ __launch_bounds__(64 * W, W == 4 ? 2 : 1) void linear_rows_kernel(LinearArgs a) {
  using L = Ring<NP, NT, RT, W>;
  __shared__ __attribute__((aligned(16))) uint8_t ring[L::WAVES][L::SLOTS][L::SLOT];
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nblk = a.K / kBlock;
  const int n0 = blockIdx.x * 16 * NT, m0 = blockIdx.y * 16 * RT;
  const int rows = min(a.M - m0, 16 * RT);
  const uint16_t* xs = a.x + static_cast<size_t>(m0) * a.K;
  uint32_t xoff[RT * 4], woff[NT];
#pragma unroll
  for (int i = 0; i < RT * 4; ++i) {
    const int r = 4 * i + g;
    xoff[i] = static_cast<uint32_t>(min(r, rows - 1) * a.K * 2 + 16 * (c ^ (r & 15)));
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int n = 16 * t + (lane >> 2);
    woff[t] = static_cast<uint32_t>(n * (a.K / 2) + 16 * ((lane & 3) ^ ((n >> 2) & 3)));
  }
  const uint32_t soff = 4 * (lane & (8 * NT - 1));  // lanes past the steps repeat them
  const uint32_t ring0 = lds_offset(&ring[wave][0][0]);
  const uint8_t* qw = a.qw + static_cast<size_t>(n0) * (a.K / 2);
  auto copy = [&](int b, int slot) {
    const uint32_t at = ring0 + slot * L::SLOT;
#pragma unroll
    for (int t = 0; t < NT; ++t) dma<16>(qw + b * (kBlock / 2), woff[t], at + L::W_OFF + t * 1024);
    dma<4>(a.w_scale + static_cast<size_t>((b * kBlock) / a.w_group) * a.N + n0, soff, at + L::S_OFF);
#pragma unroll
    for (int i = 0; i < RT * 4; ++i) dma<16>(xs + b * kBlock, xoff[i], at + i * 1024);
    if constexpr (NP > 1) {
      dma<4>(a.dinv + b * kBlock, 4 * lane, at + L::D_OFF);
      dma<4>(a.dinv + b * kBlock + 64, 4 * lane, at + L::D_OFF + 256);
    }
  };
  v4f total[RT][NT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int t = 0; t < NT; ++t) total[r][t] = v4f{0, 0, 0, 0};

  constexpr int DIST = L::SLOTS - 1;  // blocks ahead
#pragma unroll
  for (int u = 0; u < DIST; ++u)
    if (wave + u * L::WAVES < nblk) copy(wave + u * L::WAVES, u);
  int slot = 0;
  for (int b = wave; b < nblk; b += L::WAVES) {
    // the slot that is filled next was read in the last pass: its reads are done
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (b + DIST * L::WAVES < nblk) {
      copy(b + DIST * L::WAVES, slot == 0 ? DIST : slot - 1);
      wait_vm<DIST * L::COPIES>();
    } else {
      wait_vm<0>();
    }
    const uint8_t* st = &ring[wave][slot][0];
    Block<NT> blk;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int n = 16 * t + c;
      blk.w[t] = *reinterpret_cast<const uint4*>(st + L::W_OFF + n * 64 + 16 * (g ^ ((n >> 2) & 3)));
      blk.step[t] = *reinterpret_cast<const uint16_t*>(st + L::S_OFF + 2 * n);
    }
    const float* d = reinterpret_cast<const float*>(st + L::D_OFF) + 32 * g;
#pragma unroll
    for (int r = 0; r < RT; ++r)
      add_block<NT, NP>(
          [&](int j, uint4(&f)[NP]) {
            const uint4 x = *reinterpret_cast<const uint4*>(st + (16 * r + c) * 256 + 16 * ((4 * g + j) ^ c));
            parts_of<NP>(x, d + 8 * j, f);
          },
          blk, total[r]);
    slot = slot == DIST ? 0 : slot + 1;
  }
  __syncthreads();
  float* sums = reinterpret_cast<float*>(&ring[0][0][0]);
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) sums[((wave * NT + t) * 16 * RT + 16 * r + 4 * g + i) * 16 + c] = total[r][t][i];
  __syncthreads();
  finish<NT>(a, sums, L::WAVES, 16 * RT, 1, m0, rows, n0);
}

template <int NP, int NT>
void launch_staged(const LinearArgs& a, hipStream_t s) {
  const int nblk = a.K / kBlock;
  const unsigned grid = static_cast<unsigned>(a.N / (16 * NT));
  // sixteen waves where a CU has one workgroup (13824 -> 5120, one row: 13.4 us,
  // eight 14.2), eight where it has two (5120 -> 15360: 12.2, sixteen 13.8)
  const int waves = nblk >= 16 && grid <= 256 ? 16 : (nblk >= 8 ? 8 : 4);
  const size_t bytes = std::max(static_cast<size_t>(a.M) * NP * a.K * 2, static_cast<size_t>(waves) * NT * 1024);
  linear_staged_kernel<NP, NT><<<grid, 64 * waves, bytes, s>>>(a);
}

template <int NP, int NT, int RT, int W>
void launch_rows(const LinearArgs& a, hipStream_t s) {
  const dim3 grid(a.N / (16 * NT), (a.M + 16 * RT - 1) / (16 * RT));
  linear_rows_kernel<NP, NT, RT, W><<<grid, 64 * W, 0, s>>>(a);
}

// Whether the staged kernel takes the layer: up to six rows of parts (two rows
// of 5120 -> 5120: 9.1 us, 11.0 by the other; eight rows of 2048 -> 8192 8.6, 7.2),
// as far as the LDS holds them beside a second workgroup where there is one (three
// rows of 11264 -> 9792, 135 KB: 27.3, 23.3 by the other).
template <int NP>
bool staged(const LinearArgs& a) {
  const size_t bytes = static_cast<size_t>(a.M) * NP * a.K * 2;
  return NP > 1 && a.M * NP <= 6 && bytes <= (a.N / 16 <= 512 ? 144 << 10 : 80 << 10);
}

// The rows kernel's tiles: strips of 16 NT channels by 16 RT rows.  Narrow ones
// make more workgroups, of which a CU has one at a time; wide ones share the
// splitting of x~ (by channels) and the widening of codes (by rows).  A workgroup
// takes about 4 + RT (3 NP - 1 + NT) + NT (measured with CUs to spare, 8192 channels
// in, scaled: NT, RT = 1, 1 9.1 us, 2, 1 11.5, 4, 1 15, 4, 2 24.8 beside 3 of launch;
// unscaled 5.6, 7, 9.7, 13.8), the call that many rounds over the CUs: 64 rows of
// 5120 -> 5120, scaled, 4, 2 20.5 us, 4, 1 23.7, 2, 1 25.7, 1, 1 32.8; 64 of
// 8192 -> 2048 27.9, 18.1, 14.9, 21.0; 24 of 5120 -> 5120 fp32 out 26.8, 16.4, 21.8,
// 26.1.  Strips of 16 or 32 by 32 rows are never the best of these.
template <int NP>
void launch_parts(const LinearArgs& a, hipStream_t s) {
  const int strips = a.N / 16;
  if (staged<NP>(a)) {
    if constexpr (NP > 1) {
      if (strips <= 256)
        launch_staged<NP, 1>(a, s);
      else
        launch_staged<NP, 2>(a, s);
    }
    return;
  }
  const int cus = device_cus();
  auto cost = [&](int nt, int rt) {
    const int wgs = strips / nt * ((a.M + 16 * rt - 1) / (16 * rt));
    return (wgs + cus - 1) / cus * (4 + rt * (3 * NP - 1 + nt) + nt);
  };
  const int c11 = cost(1, 1), c21 = cost(2, 1), c41 = cost(4, 1), c42 = cost(4, 2);
  const int least = std::min(std::min(c11, c21), std::min(c41, c42));
  if (c11 == least)
    launch_rows<NP, 1, 1, 12>(a, s);
  else if (c21 == least)
    launch_rows<NP, 2, 1, 8>(a, s);
  else if (c41 == least)
    launch_rows<NP, 4, 1, 8>(a, s);
  else if (strips / 4 * ((a.M + 31) / 32) <= cus)
    launch_rows<NP, 4, 2, 8>(a, s);
  else
    launch_rows<NP, 4, 2, 4>(a, s);
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
