// The best continuations of groups of beams (sq_beam_select): for the rows b of
// a group
//     total(b, t) = score[b] + x[b][t] - log sum_u exp(x[b][u])
// and the `width` pairs (b, t) with the largest totals, in order.
//
// One pass over the logits.  A workgroup takes 4096 tokens of a row in
// registers and leaves its maximum, its sum of exponentials and its `width`
// best tokens, found by their keys: the logit's bits in the order of its value
// above the inverted token number, unique whole numbers whose order is that of
// the definition within a row.  A second kernel joins the chunks of each row of a
// group and its rows.  Totals are fp64: beams of one prompt lie next to each
// other.
#include "half_types.h"
#include "token_internal.h"

namespace sq {
namespace {

typedef unsigned long long Key;  // 0: none

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kEach = 16;                  // values of a thread
constexpr int kChunk = kThreads * kEach;   // tokens of a workgroup
constexpr int kMaxWidth = 64;
constexpr int kGroupOf = kWaves * kEach;   // values behind a maximum that the threshold is taken from
constexpr float kLog2e = 1.44269504088896340736f;

// Of one chunk of a row.
struct Stat {
  double sum;  // of 2^((x - top) log2 e)
  float top;
  int32_t unused;
};

__host__ __device__ constexpr int chunks_of(int vocab) { return (vocab + kChunk - 1) / kChunk; }

__device__ __forceinline__ Key key_of(float v, uint32_t token) {
  const uint32_t u = __float_as_uint(v + 0.0f);  // -0 counts as 0
  const uint32_t o = u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
  return (static_cast<Key>(o) << 32) | (0xFFFFFFFFu - token);
}
__device__ __forceinline__ uint32_t token_of(Key k) { return 0xFFFFFFFFu - static_cast<uint32_t>(k); }
__device__ __forceinline__ float value_of(Key k) {
  const uint32_t o = static_cast<uint32_t>(k >> 32);
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}

__device__ __forceinline__ Key max_key(Key a, Key b) { return a > b ? a : b; }
__device__ __forceinline__ Key lane_key(Key k, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(k), lane);
  const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(k >> 32), lane);
  return (static_cast<Key>(hi) << 32) | lo;
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

__global__ __launch_bounds__(kThreads) void beam_chunk_kernel(BeamArgs a, Key* keys, Stat* stats) {
  extern __shared__ Key list[];  // kGroupOf * width: no more keys reach the threshold
  __shared__ Key tops[kWaves][64];
  __shared__ float wave_top[kWaves];
  __shared__ double wave_total[kWaves];
  __shared__ int count;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int chunk = blockIdx.x, chunks = gridDim.x;
  const size_t row = blockIdx.y;
  if (a.done != nullptr && a.done[row] != 0) return;  // its logits do not count
  const int t0 = chunk * kChunk;
  float v[kEach / 8][8];
#pragma unroll
  for (int i = 0; i < kEach / 8; ++i) load_values(a, row, t0 + (i * kThreads + tid) * 8, v[i]);
  float top = -INFINITY;
  Key best = 0;
#pragma unroll
  for (int i = 0; i < kEach / 8; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int t = t0 + (i * kThreads + tid) * 8 + e;
      top = fmaxf(top, v[i][e]);
      if (t < a.vocab) best = max_key(best, key_of(v[i][e], t));
    }
  top = wave_max(top);
  tops[wave][lane] = best;
  if (lane == 0) wave_top[wave] = top;
  if (tid == 0) count = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    top = fmaxf(top, wave_top[w]);
    best = max_key(best, tops[w][lane]);
  }

  // exponentials; a NaN or an infinity leaves NaN
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < kEach / 8; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += v[i][e] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((v[i][e] - top) * kLog2e);
  const double total = wave_sum(sum);
  if (lane == 0) wave_total[wave] = total;

  // The width-th largest of the 64 maxima (every wave for itself): all of the
  // chunk's `width` best keys reach it.
  Key least = 1;
  int above = 0;
  for (int l = 0; l < 64; ++l) above += lane_key(best, l) > best ? 1 : 0;
  const uint64_t is_it = __ballot(best != 0 && above == a.width - 1);
  if (is_it != 0) least = lane_key(best, __ffsll(static_cast<unsigned long long>(is_it)) - 1);
#pragma unroll
  for (int i = 0; i < kEach / 8; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int t = t0 + (i * kThreads + tid) * 8 + e;
      const Key k = t < a.vocab ? key_of(v[i][e], t) : 0;
      if (k >= least) list[atomicAdd(&count, 1)] = k;
    }
  __syncthreads();
  const int n = count;
  Key* out = keys + (row * chunks + chunk) * a.width;
  for (int i = tid; i < max(n, a.width); i += kThreads) {
    if (i >= n) {
      out[i] = 0;
      continue;
    }
    const Key k = list[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += list[j] > k ? 1 : 0;
    if (rank < a.width) out[rank] = k;
  }
  if (tid == 0) {
    double s = wave_total[0];
    for (int w = 1; w < kWaves; ++w) s += wave_total[w];
    stats[row * chunks + chunk] = Stat{s, top, 0};
  }
}

// One workgroup per group of beams: a wave per row joins its chunks, then the
// rows' best are ordered.
constexpr int kJoinThreads = 512, kJoinWaves = kJoinThreads / 64;
constexpr int kLists = chunks_of(1 << 20) / 64;  // of a lane

__global__ __launch_bounds__(kJoinThreads) void beam_join_kernel(BeamArgs a, const Key* keys, const Stat* stats, int chunks) {
  extern __shared__ double totals[];  // [beams][width], then their tokens
  int32_t* tokens = reinterpret_cast<int32_t*>(totals + a.beams * a.width);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int group = blockIdx.x, width = a.width;
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
    float top = -INFINITY;
    for (int c = lane; c < chunks; c += 64) top = fmaxf(top, st[c].top);
    top = wave_max(top);
    double sum = 0.0;
    for (int c = lane; c < chunks; c += 64)
      if (st[c].sum != 0.0) sum += st[c].sum * exp(static_cast<double>(st[c].top) - top);
    sum = wave_sum(sum);
    const double lse = top + log(sum);
    // the chunks' lists are in order: the largest of their heads is next
    const Key* lists = keys + row * chunks * width;
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
      if (lane == 0) {
        const double total = score + (static_cast<double>(value_of(next)) - lse);
        totals[b * width + i] = next != 0 && live && total - total == 0.0 ? total : -INFINITY;
        tokens[b * width + i] = static_cast<int32_t>(token_of(next));
      }
    }
  }
  __syncthreads();
  // rows stand in order, and a row's tokens in the order of its totals
  const int n = a.beams * width;
  const size_t out = static_cast<size_t>(group) * width;
  for (int i = tid; i < n; i += kJoinThreads) {
    const double total = totals[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += totals[j] > total || (totals[j] == total && j < i) ? 1 : 0;
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
  return static_cast<size_t>(rows) * chunks_of(vocab) * (sizeof(Stat) + width * sizeof(Key));
}

hipError_t launch_beam_select(const BeamArgs& a, hipStream_t s) {
  const int chunks = chunks_of(a.vocab);
  Stat* stats = static_cast<Stat*>(a.ws);
  Key* keys = reinterpret_cast<Key*>(stats + static_cast<size_t>(a.rows) * chunks);
  beam_chunk_kernel<<<dim3(chunks, a.rows), kThreads, sizeof(Key) * kGroupOf * a.width, s>>>(a, keys, stats);
  beam_join_kernel<<<a.rows / a.beams, kJoinThreads, (sizeof(double) + sizeof(int32_t)) * a.beams * a.width, s>>>(
      a, keys, stats, chunks);
  return hipGetLastError();
}

}  // namespace sq
