// Attention of one new token per request where groups of requests share their
// first tokens (sq_attn_shared).  Those are read once for a group instead of once
// for each of its requests: the group's query rows (requests x query heads of a
// key-value head) meet each tile of keys together.
//
// Two kernels: the prefix in chunks for tiles of a group's query rows beside each
// request's own tokens, and the join of both kinds of parts.  A part holds a running
// maximum m (in units of log 2), a sum l and the weighted values.
//
// A wave takes 32 tokens at a time for Q tiles of 16 query rows, as in the paged
// attention: scores as keys x queries, so that a lane has the probabilities that it
// needs for the values, which it transposes in registers; nothing is passed
// between lanes.
//
// Probabilities enter their product as three 16-bit parts, all 24 bits of fp32, for every
// output type: with two of bf16 a sum that cancels was off by twice the bound of fp32
// probabilities.  The third costs nothing where memory bounds, and up to 8 % where the
// arithmetic does (64 rows of 5 heads on 8 by 8192 tokens: 45.7 us with two, 49 to 50).
#include <type_traits>

#include "attn_shared_split.h"
#include "attn_tile.h"
#include "gemm_frag.h"
#include "token_internal.h"

namespace sq {
namespace {

constexpr int kTile = kAttnTile, kQTile = kAttnQTile;
constexpr int kMinPage = 8;
constexpr int kParts = 3;  // 16-bit parts of a probability
constexpr int kWaves = 4;

// The parts of the prefix and of the requests' own tokens, [row][chunk] of each
// kind: D values, then maximum and sum; then the token ranges of the requests.
struct Parts {
  float *prefix, *mine;
  float2 *prefix_stat, *mine_stat;
  int2* range;  // own tokens [x, y)
};
__host__ __device__ inline Parts parts_of(const SharedArgs& a, const SharedSplit& sp) {
  const size_t rows = static_cast<size_t>(a.R) * a.Hq;
  Parts p;
  p.prefix = static_cast<float*>(a.ws);
  p.mine = p.prefix + rows * sp.count * a.D;
  p.prefix_stat = reinterpret_cast<float2*>(p.mine + rows * sp.mine.count * a.D);
  p.mine_stat = p.prefix_stat + rows * sp.count;
  p.range = reinterpret_cast<int2*>(p.mine_stat + rows * sp.mine.count);
  return p;
}

__device__ __forceinline__ int group_start(const SharedArgs& a, int g) { return min(max(a.group_start[g], 0), a.R); }
__device__ __forceinline__ int64_t capacity(const SharedArgs& a) { return static_cast<int64_t>(a.max_pages) << a.page_shift; }
__device__ __forceinline__ int shared_len(const SharedArgs& a, int g) {
  return static_cast<int>(min(static_cast<int64_t>(min(max(a.shared_len[g], 0), a.max_shared)), capacity(a)));
}
__device__ __forceinline__ int kv_len(const SharedArgs& a, int r) {
  return static_cast<int>(min(static_cast<int64_t>(max(a.kv_len[r], 0)), capacity(a)));
}

// The last group g with place(g) <= x, by all lanes of a wave (place does not fall).
template <typename Place>
__device__ int last_group(const SharedArgs& a, int64_t x, Place place) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  for (int step = a.groups > 4096 ? 4096 : a.groups > 64 ? 64 : 1;; step /= 64) {
    const int64_t g = lo + static_cast<int64_t>(lane) * step;
    const uint64_t before = __ballot(g < a.groups && place(static_cast<int>(g)) <= x);
    lo += max(static_cast<int>(__popcll(before)) - 1, 0) * step;
    if (step == 1) return lo;
  }
}

// Four dimensions of a query head over the tokens [first, last), one after the other,
// as the formula reads: sum of 2^(score - M) v.
template <bool F16, int D, typename PageOf>
__device__ float4 follow_tokens(const SharedArgs& a, int req, int head, int kvh, int first, int last, int d4, float M,
                                PageOf page_of) {
  const int mask = (1 << a.page_shift) - 1;
  const float scale = a.scale * kLog2e;
  const uint4* qr = reinterpret_cast<const uint4*>(a.q + req * a.q_stride + static_cast<size_t>(head) * D);
  float4 sum = make_float4(0, 0, 0, 0);
#pragma unroll 1
  for (int tok = first; tok < last; ++tok) {
    const int page = page_of(tok);
    if (page < 0) continue;
    const size_t row = (((static_cast<size_t>(page) * a.Hk + kvh) << a.page_shift) + (tok & mask)) * D;
    const uint4* kr = reinterpret_cast<const uint4*>(a.k + row);
    float dot = 0.0f;
#pragma unroll 1  // its registers are the kernel's
    for (int j = 0; j < D / 8; ++j) {
      float u[8], w8[8];
      widen8<F16>(qr[j], u);
      widen8<F16>(kr[j], w8);
#pragma unroll
      for (int x = 0; x < 8; ++x) dot = __builtin_fmaf(u[x], w8[x], dot);
    }
    const uint2 raw = *reinterpret_cast<const uint2*>(a.v + row + 4 * d4);
    add_scaled(sum, make_float4(half_lo<F16>(raw.x), half_hi<F16>(raw.x), half_lo<F16>(raw.y), half_hi<F16>(raw.y)),
               __builtin_amdgcn_exp2f(dot * scale - M));
  }
  return sum;
}

// A workgroup's part of a group's prefix: query rows row0 .. row0 + rows - 1 of one
// key-value head (row i is head kvh * each + i % each of request req0 + i / each)
// against the tokens [begin, end), which are read through the row of request `reader`.
struct Chunk {
  int kvh, split, req0, row0, rows, reader, begin, end;
};

template <int ROWS>
__device__ bool find_chunk(const SharedArgs& a, const SharedSplit& sp, uint32_t id, int each, Chunk& ch) {
  const int lane = threadIdx.x & 63;
  // tiles of one (key-value head, chunk) stand 8 apart: on one XCD, whose cache
  // then has the keys and values
  const uint32_t slots = static_cast<uint32_t>(sp.slots);
  const uint32_t pair = id / 8 / slots * 8 + id % 8, slot = id / 8 % slots;
  if (pair >= static_cast<uint32_t>(a.Hk * sp.count)) return false;
  ch.kvh = static_cast<int>(pair % static_cast<uint32_t>(a.Hk));
  ch.split = static_cast<int>(pair / static_cast<uint32_t>(a.Hk));
  // group i has the slots from start * each / ROWS + i on, at least as many as it needs
  auto place = [&](int i) { return static_cast<int64_t>(group_start(a, i)) * each / ROWS + i; };
  const int group = last_group(a, slot, place);
  const int s0 = group_start(a, group), s1 = group_start(a, group + 1);
  ch.row0 = static_cast<int>(slot - place(group)) * ROWS;
  if (ch.row0 < 0 || s1 <= s0 || ch.row0 >= (s1 - s0) * each) return false;
  ch.rows = min((s1 - s0) * each - ch.row0, ROWS);
  ch.req0 = s0;
  const int p = shared_len(a, group);
  const int64_t begin = static_cast<int64_t>(ch.split) * sp.chunk;
  if (begin >= p) return false;
  // through the first request that has the most of them
  int stop = 0;
  ch.reader = s0;
  for (int m = s0; m < s1 && stop < p; m += 64) {
    const int n = m + lane < s1 ? min(kv_len(a, m + lane), p) : 0;
    int top = n;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) top = max(top, __shfl_xor(top, o, 64));
    if (top > stop) {
      stop = top;
      ch.reader = m + __ffsll(static_cast<unsigned long long>(__ballot(n == top))) - 1;
    }
  }
  if (begin >= stop) return false;
  ch.begin = static_cast<int>(begin);
  ch.end = ch.begin + min(stop - ch.begin, sp.chunk);
  // the same in all lanes: kept in scalar registers
  for (int* v : {&ch.kvh, &ch.split, &ch.req0, &ch.row0, &ch.rows, &ch.reader, &ch.begin, &ch.end})
    *v = __builtin_amdgcn_readfirstlane(*v);
  return true;
}

// Q tiles of query rows against one chunk: the prefix of a group (OWN false) or a
// request's own tokens.  The waves take the chunk's tiles of tokens in turn, each for
// itself (no barrier), and are joined through LDS.
// Keys and values pass through LDS, a tile per wave, with direct loads whose lanes read
// along the lines.  Straight into registers (as past a workgroup's share of LDS, at head
// dimension 192) consecutive lanes read different rows of keys, four times the accesses
// to the cache: 64 rows of 5 heads on 8 by 8192 tokens took 51.3 us (50.4), two groups of 16
// rows on 8 by 32000 68.5 (61.0), 8 groups of 32 rows of 64 on 8 with 2000 tokens of their own
// 60.7 (47.1), 32 rows of 4 on 4 of 256 with 400 own 41.5 (38.3).  At 192 the LDS would leave
// one workgroup on a CU for two (32 rows on 8 heads, 800 own tokens: 53.6 us, 40.5 in registers).
template <int D>
constexpr bool kThroughLds = D != 192;

template <int D>
struct Lds {
  union {
    uint8_t tile[kWaves][2][kThroughLds<D> ? kTile * 2 * D : 16];  // keys and values
    struct {
      float values[kWaves][kQTile][D + 4], top[kWaves][kQTile], sum[kWaves][kQTile];
    };
  };
  int32_t pages[static_cast<int>(kSharedMost) / kMinPage + 2];
};
static_assert(kAttnWhole <= kSharedMost, "one array holds the pages of either chunk");

// N dwords of LDS from a 4-byte boundary.
template <int N>
__device__ __forceinline__ void read_words(const uint8_t* p, uint32_t* w) {
  typedef unsigned int vec __attribute__((ext_vector_type(N), aligned(N == 3 ? 4 : 4 * N)));
  const vec r = *reinterpret_cast<const vec*>(p);
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = r[i];
}

template <bool F16, int D, int Q, bool OWN>
__device__ __forceinline__ void take_tokens(const SharedArgs& a, const SharedSplit& sp, uint32_t id, Lds<D>& lds) {
  constexpr int W = kWaves;
  constexpr int KF = D / 32;  // fragments of a key row
  constexpr int E = D / 16, E0 = E < 8 ? E : 8, E1 = E - E0;  // a lane's dimensions of a value row
  constexpr int EW = E / 2;
  constexpr bool kStaged = kThroughLds<D>;
  constexpr int kRows = Q * kQTile;
  constexpr float kShift = F16 ? 11.0f : 0.0f;
  constexpr float kSlack = F16 ? 4.0f : 8.0f;
  int32_t* pages = lds.pages;
  auto& s_o = lds.values;
  auto& s_m = lds.top;
  auto& s_l = lds.sum;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  const int each = a.Hq / a.Hk;
  const Parts parts = parts_of(a, sp);

  Chunk ch;
  int first = 0;
  if constexpr (OWN) {
    const uint32_t qtiles = static_cast<uint32_t>((each + kRows - 1) / kRows);
    uint32_t wg = id;
    ch.kvh = static_cast<int>(wg % static_cast<uint32_t>(a.Hk));
    wg /= static_cast<uint32_t>(a.Hk);
    ch.row0 = static_cast<int>(wg % qtiles) * kRows;
    wg /= qtiles;
    ch.split = static_cast<int>(wg % static_cast<uint32_t>(sp.mine.count));
    const int r = static_cast<int>(wg / static_cast<uint32_t>(sp.mine.count));
    const int group = last_group(a, r, [&](int i) { return static_cast<int64_t>(group_start(a, i)); });
    const bool member = a.groups > 0 && group_start(a, group) <= r && r < group_start(a, group + 1);
    const int p = member ? shared_len(a, group) : 0;
    const int n = kv_len(a, r);
    first = min(p, n);
    const int stop = static_cast<int>(min(static_cast<int64_t>(n), static_cast<int64_t>(p) + a.max_own));
    if (ch.kvh == 0 && ch.row0 == 0 && ch.split == 0 && threadIdx.x == 0) parts.range[r] = make_int2(first, stop);
    ch.reader = ch.req0 = r;
    ch.rows = min(each - ch.row0, kRows);
    const int64_t begin = (first & ~(kTile - 1)) + static_cast<int64_t>(ch.split) * sp.mine.chunk;
    if (begin >= stop) return;
    ch.begin = static_cast<int>(begin);
    ch.end = ch.begin + min(stop - ch.begin, sp.mine.chunk);
  } else if (!find_chunk<kRows>(a, sp, id, each, ch)) {
    return;
  }
  const int kvh = ch.kvh, split = ch.split, req0 = ch.req0, row0 = ch.row0, rows = ch.rows, begin = ch.begin, end = ch.end;
  const int shift = a.page_shift, mask = (1 << shift) - 1;
  const int page0 = begin >> shift, npages = ((end - 1) >> shift) - page0 + 1;

  // queries (with a negative scale their negatives): column c of tile y is row
  // 16 y + c, the lane's values 32 j + 8 g ..
  const float scale = fabsf(a.scale) * kLog2e;
  const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u;
  uint4 q[Q][KF];
  int limit[Q];  // tokens of the rows' requests
  int least = end;
#pragma unroll
  for (int y = 0; y < Q; ++y) {
    const int i = kQTile * y + c, at = row0 + min(i, rows - 1);
    const int req = req0 + at / each, head = kvh * each + at % each;
    limit[y] = OWN ? end : kv_len(a, req);
    least = min(least, limit[y]);
    const uint16_t* qrow = a.q + req * a.q_stride + static_cast<size_t>(head) * D + 8 * g;
#pragma unroll
    for (int j = 0; j < KF; ++j) {
      q[y][j] = *reinterpret_cast<const uint4*>(qrow + 32 * j);
      q[y][j].x ^= flip, q[y][j].y ^= flip, q[y][j].z ^= flip, q[y][j].w ^= flip;
      if (i >= rows) q[y][j] = make_uint4(0, 0, 0, 0);
    }
  }
  if constexpr (!OWN) {
#pragma unroll
    for (int o = 8; o >= 1; o >>= 1) least = min(least, __shfl_xor(least, o, 64));
  }
  bool pages_ok = true;
  for (int i = threadIdx.x; i < npages; i += 64 * W) {
    const int32_t p = a.table[static_cast<size_t>(ch.reader) * a.max_pages + page0 + i];
    const bool ok = p >= 0 && p < a.num_pages;
    pages[i] = ok ? p : -1;
    pages_ok &= ok;
  }
  pages_ok = __syncthreads_and(pages_ok);

  v4f o[Q][E];
  float m[Q], l[Q];
#pragma unroll
  for (int y = 0; y < Q; ++y) {
#pragma unroll
    for (int e = 0; e < E; ++e) o[y][e] = v4f{0, 0, 0, 0};
    m[y] = kLowest;
    l[y] = 0.0f;
  }

  auto page_of = [&](int tok) { return pages[max(0, min((tok >> shift) - page0, npages - 1))]; };
  auto row_of = [&](int page, int tok) {
    return ((static_cast<size_t>(max(page, 0)) * a.Hk + kvh) << shift) + (tok & mask);
  };
  // a tile's keys: tokens b + 16 i + c, the lane's values 32 j + 8 g ..; its
  // values: tokens b + 16 i + 4 g + x, the lane's dimensions.  Where the tile lies
  // within one page of the range its address is the same for all lanes; tokens
  // outside [first, end) are not loaded: their lanes repeat the nearest row inside.
  uint4 k[2][KF];
  uint32_t v[8][EW];
  auto inside = [&](int b) { return b >= first && b + kTile <= end; };
  const bool half_page = shift >= 4;
  size_t half[2];  // rows of the cache where the halves of a tile begin
  auto find_halves = [&](int b) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int page = __builtin_amdgcn_readfirstlane(page_of(b + 16 * i));
      half[i] = ((static_cast<size_t>(max(page, 0)) * a.Hk + kvh) << shift) + ((b + 16 * i) & mask);
    }
  };
  auto load_k_row = [&](int i, const uint16_t* p) {
#pragma unroll
    for (int j = 0; j < KF; ++j) k[i][j] = load16<OWN>(p + 32 * j);
  };
  auto load_v_row = [&](const uint16_t* p, uint32_t* w) {
    load_words<E0 / 2, OWN>(p + E0 * c, w);
    if constexpr (E1 > 0) load_words<E1 / 2, OWN>(p + 16 * E0 + E1 * c, w + E0 / 2);
  };
  auto load_k = [&](int b) {
    if (half_page && inside(b)) {
#pragma unroll
      for (int i = 0; i < 2; ++i) load_k_row(i, a.k + half[i] * D + static_cast<uint32_t>(c * D + 8 * g));
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int tok = max(first, min(b + 16 * i + c, end - 1));
        load_k_row(i, a.k + row_of(page_of(tok), tok) * D + 8 * g);
      }
    }
  };
  auto load_v = [&](int b) {
    if (half_page && inside(b)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) load_v_row(a.v + half[i / 4] * D + static_cast<uint32_t>((4 * g + i % 4) * D), v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int tok = b + 16 * i + 4 * g, tc = max(first, min(tok, end - 1));
        const uint16_t* p = a.v + row_of(page_of(tc), tc) * D;
#pragma unroll
        for (int x = 0; x < 4; ++x) load_v_row(p + max(0, min(tok + x, end - 1) - tc) * D, v[4 * i + x]);
      }
    }
  };
  // Staged: 16-byte pieces go from memory into the wave's part of LDS, 64 to a load: piece
  // 64 j + lane of 16 rows.  Those of a key row are turned by the row, so that the 16 rows that
  // lanes read together lie in different banks.
  constexpr int S = D / 8, kSame = D % 128 == 0 ? 1 : D == 96 ? 4 : 2;
  constexpr int kLoads = 2 * KF;  // of 32 rows
  auto turn = [&](int row) { return row / kSame; };
  uint32_t k_from[KF], k_at[KF], v_from[KF];
#pragma unroll
  for (int j = 0; j < KF; ++j) {
    const int row = (64 * j + lane) / S, piece = (64 * j + lane) % S - turn(row), at = 4 * j + g + turn(c);
    k_from[j] = static_cast<uint32_t>(2 * D * row + 16 * (piece < 0 ? piece + S : piece));
    v_from[j] = static_cast<uint32_t>(1024 * j + 16 * lane);
    k_at[j] = static_cast<uint32_t>(2 * D * c + 16 * (at >= S ? at - S : at));
  }
  const uint8_t *keys = lds.tile[wave][0], *values = lds.tile[wave][1];
  // kLoads loads, after find_halves.  Where a half of the tile may lie in two pages or
  // tokens of it outside [first, end), each lane has an address of its own, and those
  // tokens repeat the nearest inside.
  auto load_tile = [&](const uint16_t* cache, const uint32_t (&from)[KF], const uint8_t* to, int b) {
    const uint32_t at = lds_offset(to);
    if (half_page && inside(b)) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the tile before has been read
#pragma unroll
      for (int i = 0; i < 2; ++i)
        dma_run(cache + half[i] * D, from, at + 32 * D * i);
    } else {
      auto token = [&](int i, int j) {
        return max(first, min(b + 16 * i + static_cast<int>(from[j] / (2 * D)), end - 1));
      };
      int page[2][KF];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < KF; ++j) page[i][j] = page_of(token(i, j));
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < KF; ++j)
          dma16_lanes(cache + row_of(page[i][j], token(i, j)) * D + from[j] % (2 * D) / 2, at + 32 * D * i + 1024 * j);
    }
  };
  auto start_k = [&](int b) {
    find_halves(b);
    if constexpr (kStaged)
      load_tile(a.k, k_from, keys, b);
    else
      load_k(b);
  };
  auto start_v = [&](int b) {
    if constexpr (kStaged)
      load_tile(a.v, v_from, values, b);
    else
      load_v(b);
  };
  if (begin + wave * kTile < end) {
    start_k(begin + wave * kTile);
    start_v(begin + wave * kTile);
  }
  for (int b = begin + wave * kTile; b < end; b += W * kTile) {
    const int next = b + W * kTile;
    const bool more = next < end;
    if constexpr (kStaged) wait_vm<kLoads>();  // the keys; the values are behind them
    float f[Q][8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      v4f s[Q];
#pragma unroll
      for (int y = 0; y < Q; ++y) s[y] = v4f{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < KF; ++j) {
        if constexpr (kStaged) k[i][j] = *reinterpret_cast<const uint4*>(keys + 32 * D * i + k_at[j]);
#pragma unroll
        for (int y = 0; y < Q; ++y) s[y] = mfma<F16>(k[i][j], q[y][j], s[y]);
      }
#pragma unroll
      for (int y = 0; y < Q; ++y)
#pragma unroll
        for (int x = 0; x < 4; ++x) f[y][4 * i + x] = s[y][x];
    }
    if (more) start_k(next);
    float unit = scale;  // of f, in units of log 2
    const bool masked = !(pages_ok && inside(b) && b + kTile <= least);
    uint32_t dead = 0;
    if (masked) {
      unit = 1.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int tok = b + 16 * (i / 4) + 4 * g + i % 4;
        const bool live = (tok >= first) & (tok < end) & (page_of(tok) >= 0);
#pragma unroll
        for (int y = 0; y < Q; ++y) f[y][i] = (live & (tok < limit[y])) ? f[y][i] * scale : -INFINITY;
        dead |= static_cast<uint32_t>(!live) << i;
      }
    }
    uint32_t p[Q][kParts][4];
#pragma unroll
    for (int y = 0; y < Q; ++y) {
      float top = f[y][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, f[y][i]);
      top *= unit;
      if (__any(top > m[y] + kSlack)) {
        const float mn = fmaxf(m[y], quad_max(top));
        const float al = __builtin_amdgcn_exp2f(m[y] - mn);
        m[y] = mn;
        l[y] *= al;
#pragma unroll
        for (int e = 0; e < E; ++e) o[y][e] *= al;
      }
      const float from = kShift - m[y];
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        float x0 = __builtin_amdgcn_exp2f(__builtin_fmaf(f[y][i], unit, from));
        float x1 = __builtin_amdgcn_exp2f(__builtin_fmaf(f[y][i + 1], unit, from));
        l[y] += x0 + x1;
#pragma unroll
        for (int u = 0; u < kParts; ++u) {
          p[y][u][i / 2] = to_half2<F16>(x0, x1);
          if (u + 1 < kParts) {
            x0 -= half_lo<F16>(p[y][u][i / 2]);
            x1 -= half_hi<F16>(p[y][u][i / 2]);
          }
        }
      }
    }
    if constexpr (kStaged) {
      if (more)
        wait_vm<kLoads>();  // the values; the next keys are behind them
      else
        wait_vm<0>();
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint8_t* row = values + 2 * D * (16 * (i / 4) + 4 * g + i % 4);
        read_words<E0 / 2>(row + 2 * E0 * c, v[i]);
        if constexpr (E1 > 0) read_words<E1 / 2>(row + 32 * E0 + 2 * E1 * c, v[i] + E0 / 2);
      }
    }
    if (masked) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int w = 0; w < EW; ++w) v[i][w] = dead >> i & 1 ? 0 : v[i][w];
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
    if (more) start_v(next);
  }

  // the waves' parts, a tile of rows at a time: column c, and the dimensions that lane 4 g + x loaded
  float* out = OWN ? parts.mine : parts.prefix;
  float2* stat = OWN ? parts.mine_stat : parts.prefix_stat;
  const int count = OWN ? sp.mine.count : sp.count;
#pragma unroll
  for (int y = 0; y < Q; ++y) {
    if (kQTile * y >= rows) break;
    const float ls = quad_sum(l[y]);
    __syncthreads();
    if (g == 0) {
      s_m[wave][c] = m[y] - kShift;
      s_l[wave][c] = ls;
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        s_o[wave][c][e < E0 ? E0 * (4 * g + x) + e : 16 * E0 + E1 * (4 * g + x) + e - E0] = o[y][e][x];
    __syncthreads();
    const int here = min(rows - kQTile * y, kQTile);
    for (int i = threadIdx.x; i < here * (D / 4); i += 64 * W) {
      const int qh = i / (D / 4), d4 = i % (D / 4);
      float M = s_m[0][qh], L = 0.0f;
#pragma unroll
      for (int w = 1; w < W; ++w) M = fmaxf(M, s_m[w][qh]);
      float4 sum = make_float4(0, 0, 0, 0);
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float al = __builtin_amdgcn_exp2f(s_m[w][qh] - M);
        L = __builtin_fmaf(s_l[w][qh], al, L);
        add_scaled(sum, *reinterpret_cast<const float4*>(&s_o[w][qh][4 * d4]), al);
      }
      const int at = row0 + kQTile * y + qh, req = req0 + at / each, head = kvh * each + at % each;
      // Parts of a probability may be 0 or negative, and 0 meets values of tokens that a
      // shorter request does not attend: where that leaves NaN the formula is followed token by token.
      if (is_nan(sum.x + sum.y + sum.z + sum.w) && !is_nan(L)) {
        sum = follow_tokens<F16, D>(a, req, head, kvh, max(first, begin), OWN ? end : min(end, kv_len(a, req)), d4, M,
                                    page_of);
      }
      const size_t part = (static_cast<size_t>(req) * a.Hq + head) * count + split;
      reinterpret_cast<float4*>(out)[part * (D / 4) + d4] = sum;
      if (d4 == 0) stat[part] = make_float2(M, L);
    }
  }
}

// The prefixes' workgroups, ROWS query rows each, then those of the requests' own
// tokens: the former compute, the latter wait for memory, and run beside them.
template <bool F16, int D, int ROWS>
__global__ __launch_bounds__(64 * kWaves, D <= 128 ? 2 : 1) void shared_kernel(SharedArgs a, SharedSplit sp) {
  __shared__ Lds<D> lds;
  const uint32_t id = static_cast<uint32_t>(flat_wg());
  if (id < sp.prefix_wgs)
    take_tokens<F16, D, ROWS / kQTile, false>(a, sp, id, lds);
  else if (id - sp.prefix_wgs < sp.own_wgs)
    take_tokens<F16, D, 1, true>(a, sp, id - sp.prefix_wgs, lds);
}

// Joins the parts of a query head: a thread takes four dimensions.
__global__ __launch_bounds__(256) void shared_join_kernel(SharedArgs a, SharedSplit sp) {
  const int D4 = a.D / 4;
  const size_t i = flat_wg() * 256 + threadIdx.x, row = i / D4;
  if (row >= static_cast<size_t>(a.R) * a.Hq) return;
  const int d4 = static_cast<int>(i % D4);
  const Parts parts = parts_of(a, sp);
  const int2 range = parts.range[row / a.Hq];
  const int np = (range.x + sp.chunk - 1) / sp.chunk;
  const int from = range.x & ~(kTile - 1);
  const int nm = range.y > range.x ? (range.y - from + sp.mine.chunk - 1) / sp.mine.chunk : 0;
  float M = kLowest, L = 0.0f;
  float4 v = make_float4(0, 0, 0, 0);
  auto join = [&](const float* part, const float2* stat, int count, int n) {
    const float4* po = reinterpret_cast<const float4*>(part) + row * count * D4 + d4;
    const float2* ps = stat + row * count;
    constexpr int kTogether = 8;  // parts whose loads are in flight together
    for (int s0 = 0; s0 < n; s0 += kTogether) {
      float2 ml[kTogether];
      float4 o[kTogether];
#pragma unroll
      for (int u = 0; u < kTogether; ++u) {
        const int s = min(s0 + u, n - 1);
        ml[u] = ps[s];
        o[u] = po[static_cast<size_t>(s) * D4];
        if (s0 + u >= n) ml[u] = make_float2(kLowest, 0.0f);
      }
      float mn = M;
#pragma unroll
      for (int u = 0; u < kTogether; ++u) mn = fmaxf(mn, ml[u].x);
      const float was = __builtin_amdgcn_exp2f(M - mn);
      M = mn;
      L *= was;
      v = make_float4(v.x * was, v.y * was, v.z * was, v.w * was);
#pragma unroll
      for (int u = 0; u < kTogether; ++u) {
        if (s0 + u >= n) break;
        const float al = __builtin_amdgcn_exp2f(ml[u].x - mn);
        L = __builtin_fmaf(ml[u].y, al, L);
        add_scaled(v, o[u], al);
      }
    }
  };
  join(parts.prefix, parts.prefix_stat, sp.count, np);
  join(parts.mine, parts.mine_stat, sp.mine.count, nm);
  // an empty sum gives 0; a NaN one (of a NaN score, or one of +infinity) goes into both
  const bool empty = L == 0.0f;
  const float inv = empty ? 0.0f : 1.0f / L;
  store_out4(a.out, row * D4 + d4, make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv), a.out_dtype);
  if (d4 == 0 && a.lse != nullptr) a.lse[row] = empty ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * kLn2;
}

template <bool F16, int D>
void launch_dim(const SharedArgs& a, const SharedSplit& sp, hipStream_t s) {
  const dim3 grid = wg_grid(static_cast<size_t>(sp.prefix_wgs) + sp.own_wgs);
  if (sp.rows == 16) {
    shared_kernel<F16, D, 16><<<grid, 64 * kWaves, 0, s>>>(a, sp);
  } else if constexpr (D <= 192) {
    shared_kernel<F16, D, 32><<<grid, 64 * kWaves, 0, s>>>(a, sp);
  }
}

template <bool F16>
void launch_type(const SharedArgs& a, const SharedSplit& sp, hipStream_t s) {
  switch (a.D) {
    case 64: return launch_dim<F16, 64>(a, sp, s);
    case 96: return launch_dim<F16, 96>(a, sp, s);
    case 128: return launch_dim<F16, 128>(a, sp, s);
    case 192: return launch_dim<F16, 192>(a, sp, s);
    default: return launch_dim<F16, 256>(a, sp, s);
  }
}

}  // namespace

size_t attn_shared_bytes(int32_t R, int32_t Hq, int32_t Hk, int32_t D, int32_t max_shared, int32_t max_own) {
  return shared_ws_bytes(R, Hq, Hk, D, max_shared, max_own);
}

hipError_t launch_attn_shared(const SharedArgs& a, bool f16, hipStream_t s) {
  const SharedSplit sp = shared_split(a.R, a.groups, a.Hq, a.Hk, a.D, a.max_shared, a.max_own);
  const Parts p = parts_of(a, sp);
  const size_t used = reinterpret_cast<const char*>(p.range + a.R) - static_cast<const char*>(a.ws);
  if (used > a.ws_bytes) return hipErrorInvalidValue;
  if (shared_wgs(a.R, a.groups, a.Hq, a.Hk, sp) >= (int64_t{1} << 31)) return hipErrorInvalidConfiguration;
  f16 ? launch_type<true>(a, sp, s) : launch_type<false>(a, sp, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const size_t n = static_cast<size_t>(a.R) * a.Hq * (a.D / 4);
  shared_join_kernel<<<wg_grid((n + 255) / 256), 256, 0, s>>>(a, sp);
  return hipGetLastError();
}

}  // namespace sq
