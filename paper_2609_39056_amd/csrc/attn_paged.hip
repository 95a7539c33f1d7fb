// Attention of one new token per request over a paged key-value cache
// (sq_attn_paged): one pass over the keys and values with a running maximum m
// and sum l per query head, p_j = 2^(s_j - m) with s_j in units of log 2, and
// out = sum p_j v_j / l.  The work is reading the cache once; 2 D flops per 2 D
// bytes and query head of a group leave the matrix cores mostly idle.
//
// A wave takes 32 tokens at a time for up to 16 query heads of one key-value
// head (or two such tiles), with 16 x 16 x 32 matrix-core tiles and nothing passed between lanes:
//   scores   A = 16 keys (lane: key lane & 15, values 32 j + 8 (lane >> 4) ..),
//            B = the queries; lane (c, g) gets head c, tokens 4 g .. 4 g + 3 of
//            each half of the tile
//   values   the product's 32 tokens are ordered so that lane group g holds the
//            tokens whose probabilities it has: 4 g .. and 16 + 4 g ..; a lane
//            loads its dimensions of those eight rows (whole lines across the
//            lanes) and transposes them in registers (v_perm), so that the
//            sums come as lane (c, g): head c, dimensions of lanes 4 g ..
// The maximum is only moved when some score exceeds it by 8 (bf16: p up to
// 2^8) or 4 (f16, whose p are scaled by 2^11 to keep small ones off its
// subnormals), which leaves out most rescaling.  p enters its product as three
// 16-bit parts, each holding what the ones before left: all 24 bits of it, whatever
// the output's type.  The products are hidden behind the loads (64 requests up to
// 8192 tokens, 8 heads of 128: 171 us, two parts 170; 100 of 64 tokens, 40 heads
// 18.2 and 18.0).  The sum l is fp32 over the unrounded p.  Parts of p may be 0 or
// negative, so an infinite value leaves NaN in its dimension's sum; where one is
// NaN (and l is not) the infinities are summed by themselves at the end.
//
// Reading the keys and values goes at 5.2 to 5.9 TB/s where there is enough of
// it (64 requests of 1024 to 8192 tokens, 8 heads of 128: 162 to 172 us; two histories
// of up to 131072: 113 to 151 us; a copy of 4 GiB runs at 4.8 TB/s).  Nontemporal loads
// are 2 to 13 % faster than cached ones, the most on long histories.  A call with
// little to read is bound by its chain of loads (length, table entry, keys) and
// one launch: 5 to 7 us.
#include <type_traits>

#include "attn_split.h"
#include "attn_tile.h"
#include "token_internal.h"

namespace sq {
namespace {

constexpr int kTile = kAttnTile, kQTile = kAttnQTile;  // kQTile: the columns of a 16 x 16 matrix-core tile
constexpr int kMinPage = 8;
constexpr int kParts = 3;  // 16-bit parts of a probability

// The tokens [first, n) of a request.
__device__ __forceinline__ void range_of(const AttnArgs& a, int r, int& first, int& n) {
  n = min(max(a.kv_len[r], 0), a.max_kv_len);
  first = a.window > 0 ? max(0, n - a.window) : 0;
}

// The parts of split histories: values [row][split][D], then maximum and sum
// [row][split].
__device__ __forceinline__ float2* part_stats(const AttnArgs& a, const AttnSplit& sp) {
  return reinterpret_cast<float2*>(a.part + static_cast<size_t>(a.R) * a.Hq * sp.count * a.D);
}

// Four outputs of a query head, and its lse once, from the maximum (in units
// of log 2), the sum and the weighted values.  An empty sum gives 0; one that is
// NaN (of a NaN score, or one of +infinity) goes into both.
__device__ __forceinline__ void finish_row(const AttnArgs& a, size_t row, int d4, float M, float L, const float4& y) {
  const bool empty = L == 0.0f;
  const float inv = empty ? 0.0f : 1.0f / L;
  store_out4(a.out, row * (a.D / 4) + d4, make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv), a.out_dtype);
  if (d4 == 0 && a.lse != nullptr) a.lse[row] = empty ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * kLn2;
}

// W waves take a chunk, for Q tiles of 16 query heads.
template <bool F16, int D, int W, int Q>
__global__ __launch_bounds__(64 * W, D <= 128 ? 2 : 1) void attn_kernel(AttnArgs a, AttnSplit sp, int qtiles) {
  constexpr int KF = D / 32;  // fragments of a key row
  // a lane's part of a value row: E dimensions, E0 c .. of the first 16 E0 and
  // E1 c .. of the rest, so that a load covers whole lines across the lanes
  constexpr int E = D / 16, E0 = E < 8 ? E : 8, E1 = E - E0;
  constexpr int EW = E / 2;   // the same in dwords
  // The next tile's keys are loaded once this tile's scores are formed, its
  // values after the products (3 to 4 % at head dimension 128); at 256 the
  // registers that takes leave one workgroup per CU (64 histories up to 8192, 8 heads
  // on one: 91 us, without 66).
  constexpr bool kAhead = D < 256 && W > 1;
  constexpr int kPages = (W == 1 ? kAttnLone : kAttnWhole) / kMinPage + 1;  // of a chunk: one for each of as many threads
  static_assert(kPages <= 64 * W, "one table entry per thread");
  constexpr float kShift = F16 ? 11.0f : 0.0f;
  constexpr float kSlack = F16 ? 4.0f : 8.0f;
  __shared__ int32_t pages[kPages];
  constexpr int kHeads = Q * kQTile;
  __shared__ float s_m[W][kHeads], s_l[W][kHeads], s_o[W][kHeads][D + 4];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;

  // blockIdx.x: key-value head, tile of query heads, split (past the last one in a
  // workgroup that only fills the row); blockIdx.y: request
  const int r = blockIdx.y;
  uint32_t wg = blockIdx.x;
  const int kvh = static_cast<int>(wg % static_cast<uint32_t>(a.Hk));
  wg /= static_cast<uint32_t>(a.Hk);
  const int qt = static_cast<int>(wg % static_cast<uint32_t>(qtiles));
  const int split = static_cast<int>(wg / static_cast<uint32_t>(qtiles));
  const int G = a.Hq / a.Hk;
  const int gq = min(G - qt * kHeads, kHeads);  // query heads here
  const int h0 = kvh * G + qt * kHeads;

  // Without a window the chunk's table entries do not wait for the length
  // (those past it are in the row all the same, and not used).
  int first, n;
  range_of(a, r, first, n);
  const int base = a.window > 0 ? first & ~(kTile - 1) : 0;
  const int64_t begin64 = base + static_cast<int64_t>(split) * sp.chunk;
  const int shift = a.page_shift, mask = (1 << shift) - 1;
  const int64_t at = (begin64 >> shift) + threadIdx.x;
  if (threadIdx.x < kPages && at < a.max_pages) {
    const int32_t p = a.table[static_cast<size_t>(r) * a.max_pages + at];
    pages[threadIdx.x] = p >= 0 && p < a.num_pages ? p : -1;
  }
  const bool whole = n - base <= sp.chunk;  // one workgroup has all of it
  if (split > 0 && begin64 >= n) return;
  const int begin = static_cast<int>(begin64);
  const int end = begin + min(n - begin, sp.chunk);
  const int page0 = begin >> shift;
  const int npages = begin < end ? ((end - 1) >> shift) - page0 + 1 : 0;

  // queries: column c of tile y is head h0 + 16 y + c, the lane's values 32 j + 8 g ..
  uint4 q[Q][KF];
#pragma unroll
  for (int y = 0; y < Q; ++y) {
    const int h = kQTile * y + c;
    const uint16_t* qrow = a.q + r * a.q_stride + static_cast<size_t>(h0 + min(h, gq - 1)) * D + 8 * g;
#pragma unroll
    for (int j = 0; j < KF; ++j) {
      q[y][j] = *reinterpret_cast<const uint4*>(qrow + 32 * j);
      if (h >= gq) q[y][j] = make_uint4(0, 0, 0, 0);
    }
  }
  __syncthreads();

  v4f o[Q][E];
  float m[Q], l[Q];
#pragma unroll
  for (int y = 0; y < Q; ++y) {
#pragma unroll
    for (int e = 0; e < E; ++e) o[y][e] = v4f{0, 0, 0, 0};
    m[y] = kLowest;
    l[y] = 0.0f;
  }
  const float scale = a.scale * kLog2e;

  auto page_of = [&](int tok) { return pages[max(0, min((tok >> shift) - page0, npages - 1))]; };
  auto row_of = [&](int page, int tok) {
    return ((static_cast<size_t>(max(page, 0)) * a.Hk + kvh) << shift) + (tok & mask);
  };
  // a tile's keys: tokens b + 16 i + c, the lane's values 32 j + 8 g ..;
  // its values: tokens b + 16 i + 4 g + x, the lane's dimensions
  const int tiles = (end - begin + kTile - 1) / kTile;
  uint4 k[2][KF];
  uint32_t v[8][EW];
  int kp[2], vp[2];
  // Tokens outside [first, end) are not loaded: their lanes repeat the nearest
  // row inside (a short history would otherwise cost a whole tile of 16 KB).
  auto inside = [&](int b) { return b >= first && b + kTile <= end; };
  auto load_v_row = [&](const uint16_t* p, uint32_t* w) {
    load_words<E0 / 2>(p + E0 * c, w);
    if constexpr (E1 > 0) load_words<E1 / 2>(p + 16 * E0 + E1 * c, w + E0 / 2);
  };
  auto load_k = [&](int b) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int tok = max(first, min(b + 16 * i + c, end - 1));
      kp[i] = page_of(tok);
      const uint16_t* p = a.k + row_of(kp[i], tok) * D + 8 * g;
#pragma unroll
      for (int j = 0; j < KF; ++j) k[i][j] = load16(p + 32 * j);
    }
  };
  auto load_v = [&](int b) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int tok = b + 16 * i + 4 * g, tc = max(first, min(tok, end - 1));
      vp[i] = page_of(tc);
      const uint16_t* p = a.v + row_of(vp[i], tc) * D;
      if (inside(b)) {
#pragma unroll
        for (int x = 0; x < 4; ++x) load_v_row(p + x * D, v[4 * i + x]);
      } else {
#pragma unroll
        for (int x = 0; x < 4; ++x) load_v_row(p + max(0, min(tok + x, end - 1) - tc) * D, v[4 * i + x]);
      }
    }
  };
  if (kAhead && wave < tiles) {
    load_k(begin + wave * kTile);
    load_v(begin + wave * kTile);
  }
  for (int t = wave; t < tiles; t += W) {
    const int b = begin + t * kTile;
    if (!kAhead) {
      load_k(b);
      load_v(b);
    }
    float f[Q][8];
#pragma unroll
    for (int y = 0; y < Q; ++y) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        v4f s = v4f{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < KF; ++j) s = mfma<F16>(k[i][j], q[y][j], s);
#pragma unroll
        for (int x = 0; x < 4; ++x) f[y][4 * i + x] = s[x] * scale;
      }
    }
    const bool whole_tile = inside(b) && __all(kp[0] >= 0 && kp[1] >= 0);
    if (kAhead && t + W < tiles) load_k(b + W * kTile);
    if (!whole_tile) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int tok = b + 16 * (i / 4) + 4 * g + i % 4;
        const bool live = (tok >= first) & (tok < end) & (vp[i / 4] >= 0);
#pragma unroll
        for (int y = 0; y < Q; ++y) f[y][i] = live ? f[y][i] : -INFINITY;
#pragma unroll
        for (int w = 0; w < EW; ++w) v[i][w] = live ? v[i][w] : 0;
      }
    }
    uint32_t p[Q][kParts][4];
#pragma unroll
    for (int y = 0; y < Q; ++y) {
      float top = f[y][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, f[y][i]);
      if (__any(top > m[y] + kSlack)) {
        const float mn = fmaxf(m[y], quad_max(top));
        const float al = __builtin_amdgcn_exp2f(m[y] - mn);
        m[y] = mn;
        l[y] *= al;
#pragma unroll
        for (int e = 0; e < E; ++e) o[y][e] *= al;
      }
      const float base = m[y] - kShift;
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        float x0 = __builtin_amdgcn_exp2f(f[y][i] - base), x1 = __builtin_amdgcn_exp2f(f[y][i + 1] - base);
        l[y] += x0 + x1;
#pragma unroll
        for (int u = 0; u < kParts; ++u) {
          p[y][u][i / 2] = to_half2<F16>(x0, x1);
          x0 -= half_lo<F16>(p[y][u][i / 2]);
          x1 -= half_hi<F16>(p[y][u][i / 2]);
        }
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
      for (int y = 0; y < Q; ++y)
#pragma unroll
        for (int u = 0; u < kParts; ++u)
          o[y][e] = mfma<F16>(vt, make_uint4(p[y][u][0], p[y][u][1], p[y][u][2], p[y][u][3]), o[y][e]);
    }
    if (kAhead && t + W < tiles) load_v(b + W * kTile);
  }

  // the waves' parts: column c, and the dimensions that lane 4 g + x loaded
#pragma unroll
  for (int y = 0; y < Q; ++y) {
    const int h = kQTile * y + c;
    const float ls = quad_sum(l[y]);
    if (g == 0) {
      s_m[wave][h] = m[y] - kShift;
      s_l[wave][h] = ls;
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (h < gq) s_o[wave][h][e < E0 ? E0 * (4 * g + x) + e : 16 * E0 + E1 * (4 * g + x) + e - E0] = o[y][e][x];
  }
  __syncthreads();
  // four dimensions of a query head: maximum and sum, and the weighted values
  auto joined = [&](int qh, int d4, float& M, float& L) {
    M = s_m[0][qh];
#pragma unroll
    for (int w = 1; w < W; ++w) M = fmaxf(M, s_m[w][qh]);
    float4 y = make_float4(0, 0, 0, 0);
    L = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float al = __builtin_amdgcn_exp2f(s_m[w][qh] - M);
      L = __builtin_fmaf(s_l[w][qh], al, L);
      add_scaled(y, *reinterpret_cast<const float4*>(&s_o[w][qh][4 * d4]), al);
    }
    return y;
  };
  auto put = [&](int qh, int d4, float M, float L, const float4& y) {
    const size_t row = static_cast<size_t>(r) * a.Hq + h0 + qh;
    if (whole) {
      finish_row(a, row, d4, M, L, y);
    } else {
      const size_t part = row * sp.count + split;
      reinterpret_cast<float4*>(a.part)[part * (D / 4) + d4] = y;
      if (d4 == 0) part_stats(a, sp)[part] = make_float2(M, L);
    }
  };
  float M, L;
  bool odd = false;
  for (int i = threadIdx.x; i < gq * (D / 4); i += 64 * W) {
    const int qh = i / (D / 4), d4 = i % (D / 4);
    const float4 y = joined(qh, d4, M, L);
    odd |= is_nan(y.x + y.y + y.z + y.w);
    put(qh, d4, M, L, y);
  }
  if (!odd) return;
  // NaN where l is none: the sum of the attended values that are not finite
  for (int i = threadIdx.x; i < gq * (D / 4); i += 64 * W) {
    const int qh = i / (D / 4), d4 = i % (D / 4);
    float4 y = joined(qh, d4, M, L);
    if (!is_nan(y.x + y.y + y.z + y.w) || is_nan(L)) continue;
    const float was[4] = {y.x, y.y, y.z, y.w};
    float sum[4] = {0, 0, 0, 0};
    bool open = true;  // some dimension's sum may still change
    for (int tok = max(first, begin); tok < end && open; ++tok) {
      const int page = page_of(tok);
      if (page < 0) continue;
      const size_t at = row_of(page, tok) * D;
      const uint2 raw = *reinterpret_cast<const uint2*>(a.v + at + 4 * d4);
      const float w[4] = {half_lo<F16>(raw.x), half_hi<F16>(raw.x), half_lo<F16>(raw.y), half_hi<F16>(raw.y)};
      bool odd_here = false, infinite = false;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        odd_here |= w[x] - w[x] != 0.0f;
        infinite |= fabsf(w[x]) == INFINITY;
      }
      if (!odd_here) continue;
      float factor = 1.0f;  // or 0, which makes an infinity NaN: where the probability is 0
      if (infinite) {
        const uint4* qr = reinterpret_cast<const uint4*>(a.q + r * a.q_stride + static_cast<size_t>(h0 + qh) * D);
        const uint4* kr = reinterpret_cast<const uint4*>(a.k + at);
        float dot = 0.0f;
#pragma unroll 1  // its registers are the kernel's
        for (int j = 0; j < D / 8; ++j) {
          float u[8], v8[8];
          widen8<F16>(qr[j], u);
          widen8<F16>(kr[j], v8);
#pragma unroll
          for (int x = 0; x < 8; ++x) dot = __builtin_fmaf(u[x], v8[x], dot);
        }
        if (dot * scale == -INFINITY) factor = 0.0f;
      }
      open = false;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if (w[x] - w[x] != 0.0f) sum[x] += w[x] * factor;
        open |= is_nan(was[x]) && !is_nan(sum[x]);
      }
    }
    auto pick = [](float v, float w) { return is_nan(v) && w != 0.0f ? w : v; };
    put(qh, d4, M, L, make_float4(pick(y.x, sum[0]), pick(y.y, sum[1]), pick(y.z, sum[2]), pick(y.w, sum[3])));
  }
}

// Joins the parts of split histories, few of them: a thread takes four
// dimensions of one query head and its parts in order.
__global__ __launch_bounds__(256) void attn_join_few_kernel(AttnArgs a, AttnSplit sp) {
  const int D4 = a.D / 4;
  const size_t i = flat_wg() * 256 + threadIdx.x, row = i / D4;
  if (row >= static_cast<size_t>(a.R) * a.Hq) return;
  int first, n;
  range_of(a, static_cast<int>(row / a.Hq), first, n);
  const int span = n - (first & ~(kTile - 1));
  if (span <= sp.chunk) return;
  const int count = (span + sp.chunk - 1) / sp.chunk;
  const int d4 = static_cast<int>(i % D4);
  const float4* po = reinterpret_cast<const float4*>(a.part) + row * sp.count * D4 + d4;
  const float2* pm = part_stats(a, sp) + row * sp.count;
  float M = kLowest, L = 0.0f;
  float4 v = make_float4(0, 0, 0, 0);
  constexpr int kAhead = 8;  // parts whose loads are in flight together
  for (int s0 = 0; s0 < count; s0 += kAhead) {
    float2 ml[kAhead];
    float4 o[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int s = min(s0 + u, count - 1);
      ml[u] = pm[s];
      o[u] = po[static_cast<size_t>(s) * D4];
      if (s0 + u >= count) ml[u] = make_float2(kLowest, 0.0f);
    }
    float mn = M;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) mn = fmaxf(mn, ml[u].x);
    const float was = __builtin_amdgcn_exp2f(M - mn);
    M = mn;
    L *= was;
    v = make_float4(v.x * was, v.y * was, v.z * was, v.w * was);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const float al = s0 + u < count ? __builtin_amdgcn_exp2f(ml[u].x - mn) : 0.0f;
      L = __builtin_fmaf(ml[u].y, al, L);
      add_scaled(v, o[u], al);
    }
  }
  finish_row(a, row, d4, M, L, v);
}

// Joins the parts of a split history, many of them: a workgroup takes 32 dimensions of one
// query head, eight threads with four dimensions each for every THREADS / 8-th
// part; their sums are added in a fixed order.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void attn_join_kernel(AttnArgs a, AttnSplit sp) {
  constexpr int kParts = THREADS / 8, kWavesHere = THREADS / 64;
  __shared__ float s_max[kWavesHere], s_l[kWavesHere];
  __shared__ float4 s_sum[kWavesHere][8];
  const int strips = a.D / 32;
  const size_t wg = flat_wg(), row = wg / strips;
  if (row >= static_cast<size_t>(a.R) * a.Hq) return;
  int first, n;
  range_of(a, static_cast<int>(row / a.Hq), first, n);
  const int span = n - (first & ~(kTile - 1));
  if (span <= sp.chunk) return;
  const int count = (span + sp.chunk - 1) / sp.chunk;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int d4 = static_cast<int>(wg % strips) * 8 + (tid & 7), D4 = a.D / 4;
  const float4* po = reinterpret_cast<const float4*>(a.part) + row * sp.count * D4 + d4;
  const float2* pm = part_stats(a, sp) + row * sp.count;
  float M = kLowest;
  for (int s = tid; s < count; s += THREADS) M = fmaxf(M, pm[s].x);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
  if (lane == 0) s_max[wave] = M;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWavesHere; ++w) M = fmaxf(M, s_max[w]);
  float4 v = make_float4(0, 0, 0, 0);
  float L = 0.0f;
  for (int s = tid / 8; s < count; s += kParts) {
    const float2 ml = pm[s];
    const float al = __builtin_amdgcn_exp2f(ml.x - M);
    add_scaled(v, po[static_cast<size_t>(s) * D4], al);
    L = __builtin_fmaf(ml.y, al, L);
  }
#pragma unroll
  for (int o = 8; o < 64; o <<= 1) {
    v.x += __shfl_xor(v.x, o, 64);
    v.y += __shfl_xor(v.y, o, 64);
    v.z += __shfl_xor(v.z, o, 64);
    v.w += __shfl_xor(v.w, o, 64);
    L += __shfl_xor(L, o, 64);
  }
  if (lane < 8) {
    s_sum[wave][lane] = v;
    if (lane == 0) s_l[wave] = L;
  }
  __syncthreads();
  if (tid >= 8) return;
  for (int w = 1; w < kWavesHere; ++w) {
    add_scaled(v, s_sum[w][tid], 1.0f);
    L += s_l[w];
  }
  finish_row(a, row, d4, M, L, v);
}

// Workgroups of a request.  They go to the XCDs in turn, and in an XCD to its
// shader engines, so a request's row of a multiple of 8 (or of 32) of them
// would put split s of every request in the same place, and the last splits are
// empty for all but the longest histories.  Split rows are therefore made odd,
// with workgroups that find nothing and end: the splits where the heads go
// evenly over the XCDs (128 histories up to 2048, 8 heads: 90 us, 130 in four
// splits without), the row itself elsewhere (64 up to 8192, one head: 36 us, 47).
unsigned grid_row(int heads, int splits) {
  const unsigned h = static_cast<unsigned>(heads), s = static_cast<unsigned>(splits);
  if (s == 1) return h;
  return h % 8 == 0 ? h * (s | 1u) : (h * s) | 1u;
}

// More than 16 query heads on a key-value head (head dimensions up to 128, whose
// registers leave room): where one tile each would make as many workgroups as
// CUs, for spans past 384, a workgroup takes two and reads the keys and values
// once for them (32 heads on one, 64 histories up to 8192: 45 us, 62 in workgroups
// of a tile; 200 up to 600: 18.1, 22.6; 10 up to 2000: 12.8, 13.1; but 4 up to 2000
// 12.1 and 10.9, 130 up to 300 9.7 and 9.3).
template <bool F16, int W, int D>
void launch_tiles(const AttnArgs& a, const AttnSplit& sp, hipStream_t s) {
  const int G = a.Hq / a.Hk;
  auto launch = [&](auto tiles) {
    constexpr int Q = decltype(tiles)::value;
    const int qt = (G + Q * kQTile - 1) / (Q * kQTile);
    const dim3 grid(grid_row(a.Hk * qt, sp.count), static_cast<unsigned>(a.R));
    attn_kernel<F16, D, W, Q><<<grid, 64 * W, 0, s>>>(a, sp, qt);
  };
  if constexpr (D <= 128 && W == 4) {
    if (G > kQTile && attn_span(a.max_kv_len, a.window) > 384 &&
        attn_heads(a.R, a.Hq, a.Hk) * sp.count >= device_cus())
      return launch(std::integral_constant<int, 2>{});
  }
  launch(std::integral_constant<int, 1>{});
}

template <bool F16, int W>
void launch_dim(const AttnArgs& a, const AttnSplit& sp, hipStream_t s) {
  switch (a.D) {
    case 64: return launch_tiles<F16, W, 64>(a, sp, s);
    case 96: return launch_tiles<F16, W, 96>(a, sp, s);
    case 128: return launch_tiles<F16, W, 128>(a, sp, s);
    case 192: return launch_tiles<F16, W, 192>(a, sp, s);
    default: return launch_tiles<F16, W, 256>(a, sp, s);
  }
}

}  // namespace

size_t attn_partial_bytes(int32_t R, int32_t Hq, int32_t Hk, int32_t D, int32_t max_kv_len) {
  return attn_part_bytes(1, Hq, D, attn_most_parts(R, attn_heads(1, Hq, Hk), max_kv_len));
}

hipError_t launch_attn_paged(const AttnArgs& a, bool f16, hipStream_t s) {
  const int64_t heads = attn_heads(a.R, a.Hq, a.Hk);
  const int64_t span = attn_span(a.max_kv_len, a.window);
  const AttnSplit sp = attn_split(heads, span);
  if (attn_part_bytes(a.R, a.Hq, a.D, sp.count) > a.part_bytes) return hipErrorInvalidValue;
  if (heads / a.R * (sp.count + 1) >= (1 << 24)) return hipErrorInvalidConfiguration;  // 2^32 threads in a grid's row
  // A whole span is a chain of tiles: eight waves shorten it where a workgroup has
  // a CU to itself (30 requests of up to 350 tokens, 8 heads of 64: 8.0 us, four
  // waves 8.9; 28 of 600 with heads of 128 14.1, 15.7; with 512 heads of 500 20.3, 19.5).
  if (attn_lone(heads, span))
    f16 ? launch_dim<true, 1>(a, sp, s) : launch_dim<false, 1>(a, sp, s);
  else if (sp.count == 1 && span > 128 && heads <= device_cus())
    f16 ? launch_dim<true, 8>(a, sp, s) : launch_dim<false, 8>(a, sp, s);
  else
    f16 ? launch_dim<true, 4>(a, sp, s) : launch_dim<false, 4>(a, sp, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || sp.count == 1) return e;
  const dim3 rows = wg_grid(static_cast<size_t>(a.R) * a.Hq * (a.D / 32));
  if (sp.count <= 32) {
    const size_t n = static_cast<size_t>(a.R) * a.Hq * (a.D / 4);
    attn_join_few_kernel<<<wg_grid((n + 255) / 256), 256, 0, s>>>(a, sp);
  } else if (sp.count <= 64) {
    attn_join_kernel<256><<<rows, 256, 0, s>>>(a, sp);
  } else {
    attn_join_kernel<1024><<<rows, 1024, 0, s>>>(a, sp);
  }
  return hipGetLastError();
}

}  // namespace sq
