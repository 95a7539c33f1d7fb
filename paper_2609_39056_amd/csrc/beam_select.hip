// The best continuations of groups of beams (sq_beam_select): for the rows b of
// a group
//     total(b, t) = score[b] + x[b][t] - log sum_u exp(x[b][u])
// and the `width` pairs (b, t) with the largest totals, in order.
//
// One pass over the logits.  A workgroup takes a chunk of a row in registers and
// leaves its maximum, its sum of exponentials and its `width` best tokens: the
// width-th largest of 64 groups' maxima bounds them from below, the few values
// that reach it are listed and ordered by their keys, the logit's bits in the
// order of its value above the inverted token number: unique whole numbers whose
// order is that of the definition within a row.  A second kernel joins the chunks
// of each row of a group, in the same way, and the rows.  Totals are fp64: beams
// of one prompt lie next to each other.
//
// Reading bounds the chunks where there is much to read, with the vector units at 55 %
// (128 rows of 131071 bf16, 34 MB: 13 us, and 7 for the join of 16 workgroups); else the
// two launches do (4 rows of 8192: 3.9 and 4.5 us).
#include "beam_split.h"
#include "half_types.h"
#include "token_internal.h"

namespace sq {
namespace {

typedef unsigned long long Key;  // 0: none

constexpr int kThreads = kBeamThreads, kWaves = kThreads / 64;
constexpr int kMaxWidth = 64;
constexpr int kList = 1024;  // values that a workgroup orders; more only where very many are equal
constexpr float kLog2e = 1.44269504088896340736f;

// Of one chunk of a row.
struct Stat {
  double sum;  // of 2^((x - top) log2 e)
  float top;
  int32_t unused;
};
static_assert(sizeof(Stat) + sizeof(Key) == beam_chunk_bytes(1), "what the workspace holds of a chunk");

// Bits whose order is that of the values (-0 counts as 0).
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t u = __float_as_uint(v + 0.0f);
  return u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ Key key_of(float v, uint32_t token) {
  return (static_cast<Key>(order_of(v)) << 32) | (0xFFFFFFFFu - token);
}
__device__ __forceinline__ uint32_t token_of(Key k) { return 0xFFFFFFFFu - static_cast<uint32_t>(k); }
__device__ __forceinline__ float value_of_order(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ float value_of(Key k) { return value_of_order(static_cast<uint32_t>(k >> 32)); }

__device__ __forceinline__ Key max_key(Key a, Key b) { return a > b ? a : b; }
// A lower bound of the n-th largest of the lanes' values, 0 where there are fewer:
// its upper 16 bits (what may reach it beside the n largest is ordered with them).
__device__ __forceinline__ uint32_t nth_largest(uint32_t o, int n) {
  uint32_t t = 0;
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t u = t | (1u << bit);
    if (__popcll(__ballot(o >= u)) >= n) t = u;
  }
  return t;
}

template <typename T>
__device__ __forceinline__ T wave_max(T v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    const T w = __shfl_xor(v, o, 64);
    v = v > w ? v : w;
  }
  return v;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// Eight values from token t of a row on (past the vocabulary: not read).
__device__ __forceinline__ void load_values(const BeamArgs& a, size_t row, int t, float (&v)[8]) {
  if (t + 8 <= a.vocab) {
    if (a.dtype == SQ_OUT_F32) {
      const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(a.logits) + row * a.stride + t);
      const float4 x = p[0], y = p[1];
      v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w, v[4] = y.x, v[5] = y.y, v[6] = y.z, v[7] = y.w;
    } else {
      const uint4 r = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.logits) + row * a.stride + t);
      if (a.dtype == SQ_OUT_BF16)
        widen8<false>(r, v);
      else
        widen8<true>(r, v);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = -INFINITY;
    if (t + i < a.vocab) {
      const size_t at = row * a.stride + t + i;
      if (a.dtype == SQ_OUT_F32) {
        v[i] = static_cast<const float*>(a.logits)[at];
      } else {
        const uint32_t h = static_cast<const uint16_t*>(a.logits)[at];
        v[i] = a.dtype == SQ_OUT_BF16 ? half_lo<false>(h) : half_lo<true>(h);
      }
    }
  }
}

// EACH values of a thread.
template <int EACH>
__global__ __launch_bounds__(kThreads) void beam_chunk_kernel(BeamArgs a, Key* keys, Stat* stats) {
  __shared__ float tops[kWaves][64];
  __shared__ float sums[kThreads];
  __shared__ Key list[kList];
  __shared__ int count;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int chunk = blockIdx.x, chunks = gridDim.x;
  const size_t row = blockIdx.y;
  if (a.done != nullptr && a.done[row] != 0) return;  // its logits do not count
  const int t0 = chunk * (kThreads * EACH);
  auto token = [&](int i) { return t0 + (i / 8 * kThreads + tid) * 8 + i % 8; };
  float v[EACH / 8][8];
#pragma unroll
  for (int i = 0; i < EACH / 8; ++i) load_values(a, row, token(8 * i), v[i]);
  float best = -INFINITY;
#pragma unroll
  for (int i = 0; i < EACH; ++i) best = fmaxf(best, v[i / 8][i % 8]);
  tops[wave][lane] = best;
  if (tid == 0) count = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) best = fmaxf(best, tops[w][lane]);
  const float top = wave_max(best);
  // (-infinity is never taken)
  const float least = value_of_order(max(nth_largest(order_of(best), a.width), order_of(-INFINITY) + 1));

  // exponentials; a NaN or an infinity leaves NaN
  const float from = top == -INFINITY ? 0.0f : top;
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const float x = v[i / 8][i % 8];
    sum += __builtin_amdgcn_exp2f((x - from) * kLog2e);
    if (x >= least) {
      const int at = atomicAdd(&count, 1);
      if (at < kList) list[at] = key_of(x, token(i));
    }
  }
  sums[tid] = sum;
  __syncthreads();
  if (wave == kWaves - 1) {
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) s += sums[w * 64 + lane];
    s = wave_sum(s);
    if (lane == 0) stats[row * chunks + chunk] = Stat{s, top, 0};
  }
  const int n = count;
  Key* out = keys + (row * chunks + chunk) * a.width;
  if (n <= kList) {
    for (int i = tid; i < max(n, a.width); i += kThreads) {
      if (i >= n) {
        out[i] = 0;
        continue;
      }
      const Key k = list[i];
      int rank = 0;
#pragma unroll 8
      for (int j = 0; j < n; ++j) rank += list[j] > k ? 1 : 0;
      if (rank < a.width) out[rank] = k;
    }
    return;
  }
  // very many equal values: the largest key below the last one, again and again
  Key last = ~static_cast<Key>(0);
  for (int r = 0; r < a.width; ++r) {
    Key mine = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const Key k = token(i) < a.vocab ? key_of(v[i / 8][i % 8], token(i)) : 0;
      if (k < last) mine = max_key(mine, k);
    }
    mine = wave_max(mine);
    __syncthreads();
    if (lane == 0) list[wave] = mine;
    __syncthreads();
    last = list[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) last = max_key(last, list[w]);
    if (tid == 0) out[r] = last;
  }
}

// One workgroup per group of beams: a wave per row joins its chunks, then the
// rows' best are ordered.
constexpr int kJoinThreads = 512, kJoinWaves = kJoinThreads / 64;
constexpr int kJoinList = 512;                                   // keys of a wave that are ordered together
constexpr int kLists = (1 << 20) / (kThreads * kBeamMostEach) / 64;  // chunks of a lane, of the largest vocabulary

__global__ __launch_bounds__(kJoinThreads) void beam_join_kernel(BeamArgs a, const Key* keys, const Stat* stats, int chunks) {
  extern __shared__ double totals[];  // [beams][width], then their tokens
  int32_t* tokens = reinterpret_cast<int32_t*>(totals + a.beams * a.width);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int group = blockIdx.x, width = a.width;
  __shared__ Key found[kJoinWaves][kJoinList];
  __shared__ bool ended[kMaxWidth];  // done_out may be done
  for (int b = wave; b < a.beams; b += kJoinWaves) {
    const size_t row = static_cast<size_t>(group) * a.beams + b;
    const double score = a.scores[row];
    const bool live = score - score == 0.0;
    const bool end = a.done != nullptr && a.done[row] != 0;
    if (lane == 0) ended[b] = end;
    if (end) {
      for (int i = lane; i < width; i += 64) {
        totals[b * width + i] = i == 0 && live ? score : -INFINITY;
        tokens[b * width + i] = a.end_token;
      }
      continue;
    }
    const Stat* st = stats + row * chunks;
    Stat part[kLists];
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < kLists; ++u) {
      const int c = lane + 64 * u;
      part[u] = c < chunks ? st[c] : Stat{0.0, -INFINITY, 0};
      top = fmaxf(top, part[u].top);
    }
    top = wave_max(top);
    double sum = 0.0;
#pragma unroll
    for (int u = 0; u < kLists; ++u)
      if (part[u].sum != 0.0) sum += part[u].sum * exp(static_cast<double>(part[u].top) - top);
    sum = wave_sum(sum);
    const double lse = top + log(sum);
    auto put = [&](int i, Key k) {
      const double total = score + (static_cast<double>(value_of(k)) - lse);
      totals[b * width + i] = k != 0 && live && total - total == 0.0 ? total : -INFINITY;
      tokens[b * width + i] = static_cast<int32_t>(token_of(k));
    };
    const Key* lists = keys + row * chunks * width;
    const int all = chunks * width;
    // up to 512 keys stay in registers between the threshold and the list
    constexpr int kHold = 8;
    Key held[kHold];
    uint32_t best = 0;
#pragma unroll
    for (int u = 0; u < kHold; ++u) held[u] = lane + 64 * u < all ? lists[lane + 64 * u] : 0;
#pragma unroll
    for (int u = 0; u < kHold; ++u) best = max(best, static_cast<uint32_t>(held[u] >> 32));
    for (int i = lane + 64 * kHold; i < all; i += 64) best = max(best, static_cast<uint32_t>(lists[i] >> 32));
    const uint32_t least = max(nth_largest(best, width), 1u);
    int n = 0;
    auto keep = [&](Key k) {
      const bool mine = static_cast<uint32_t>(k >> 32) >= least;
      const uint64_t which = __ballot(mine);
      const int at = n + static_cast<int>(__popcll(which & ((1ull << lane) - 1)));
      if (mine && at < kJoinList) found[wave][at] = k;
      n += static_cast<int>(__popcll(which));
    };
#pragma unroll
    for (int u = 0; u < kHold; ++u) keep(held[u]);
    for (int i0 = 64 * kHold; i0 < all; i0 += 64) keep(i0 + lane < all ? lists[i0 + lane] : 0);
    if (n <= kJoinList) {
      for (int i = lane; i < max(n, width); i += 64) {
        int rank = i;
        Key k = 0;
        if (i < n) {
          k = found[wave][i];
          rank = 0;
#pragma unroll 8
          for (int j = 0; j < n; ++j) rank += found[wave][j] > k ? 1 : 0;
        }
        if (rank < width) put(rank, k);
      }
      continue;
    }
    // many equal ones: the chunks' lists are in order, the largest of their heads is next
    int at[kLists];
    Key head[kLists];
#pragma unroll
    for (int u = 0; u < kLists; ++u) {
      const int c = lane + 64 * u;
      at[u] = 0;
      head[u] = c < chunks ? lists[static_cast<size_t>(c) * width] : 0;
    }
    for (int i = 0; i < width; ++i) {
      Key mine = 0;
#pragma unroll
      for (int u = 0; u < kLists; ++u) mine = max_key(mine, head[u]);
      const Key next = wave_max(mine);
#pragma unroll
      for (int u = 0; u < kLists; ++u)
        if (next != 0 && head[u] == next) {
          ++at[u];
          head[u] = at[u] < width ? lists[static_cast<size_t>(lane + 64 * u) * width + at[u]] : 0;
        }
      if (lane == 0) put(i, next);
    }
  }
  __syncthreads();
  // Rows stand in order, and a row's tokens in the order of its totals: where there
  // are many, how many of each row stand before a total is found by bisection.
  const int n = a.beams * width;
  const size_t out = static_cast<size_t>(group) * width;
  for (int i = tid; i < n; i += kJoinThreads) {
    const double total = totals[i];
    const int own = i / width;
    int rank = 0;
    if (n <= 256) {
#pragma unroll 8
      for (int j = 0; j < n; ++j) rank += totals[j] > total || (totals[j] == total && j < i) ? 1 : 0;
    }
    for (int b = n <= 256 ? a.beams : 0; b < a.beams && rank < width; ++b) {
      if (b == own) {
        rank += i % width;
        continue;
      }
      int lo = 0, hi = width;  // those below lo stand before it, those from hi on do not
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        const double t = totals[b * width + mid];
        if (t > total || (t == total && b < own)) {
          lo = mid + 1;
        } else {
          hi = mid;
        }
      }
      rank += lo;
    }
    if (rank >= width) continue;
    const bool some = total != -INFINITY;
    const size_t row = static_cast<size_t>(group) * a.beams + i / width;
    a.parent[out + rank] = some ? static_cast<int32_t>(row) : -1;
    a.token[out + rank] = some ? tokens[i] : -1;
    a.score_out[out + rank] = static_cast<float>(total);
    if (a.done_out != nullptr)
      a.done_out[out + rank] = some && (ended[i / width] || tokens[i] == a.end_token) ? 1 : 0;
  }
}

}  // namespace

size_t beam_ws_bytes(int32_t rows, int32_t vocab, int32_t width) {
  return static_cast<size_t>(beam_most_chunks(rows, vocab)) * beam_chunk_bytes(width);
}

hipError_t launch_beam_select(const BeamArgs& a, hipStream_t s) {
  const int each = beam_each(a.rows, a.vocab, a.width), chunks = beam_chunks(a.vocab, each);
  Stat* stats = static_cast<Stat*>(a.ws);
  Key* keys = reinterpret_cast<Key*>(stats + static_cast<size_t>(a.rows) * chunks);
  const dim3 grid(chunks, a.rows);
  if (each == 8)
    beam_chunk_kernel<8><<<grid, kThreads, 0, s>>>(a, keys, stats);
  else if (each == 16)
    beam_chunk_kernel<16><<<grid, kThreads, 0, s>>>(a, keys, stats);
  else
    beam_chunk_kernel<32><<<grid, kThreads, 0, s>>>(a, keys, stats);
  beam_join_kernel<<<a.rows / a.beams, kJoinThreads, (sizeof(double) + sizeof(int32_t)) * a.beams * a.width, s>>>(
      a, keys, stats, chunks);
  return hipGetLastError();
}

}  // namespace sq
