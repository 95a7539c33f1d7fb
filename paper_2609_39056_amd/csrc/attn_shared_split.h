// How attention over a shared prefix is split over workgroups (host C++, no HIP).
//
// The prefix: query rows (requests of a group x query heads of a key-value head)
// go in tiles of 16 or 32 per workgroup, the prefix in chunks; every part costs
// its sums in memory, so there are as few chunks as fill the CUs beside the
// workgroups of the requests' own tokens, of at least 128 tokens.  Those are split as
// in the paged attention.
//
// Workgroups wanted, 384 up to head dimension 64, where a CU holds three of them, and 256
// past it: with 256 and 384, 24 groups of 56 rows of 64 by up to 4001 take 28.2 and 24.5 us;
// of 128, 64 rows of 5 heads on 8 by 8192 50.4 to 51.0 and 49.5, two groups of 16 rows on 8 by
// 32000 61.0 and 66.4, and 8 groups of 32 rows of 96 on 4 by 4096 22.7 and 27.3 (512: 24.8, 54.1,
// 68.9 and 30.7).  Tiles of 64 rows were slower in every form tried, then with two parts of a
// probability and 45 us for the second case: sums in accumulation registers (70 us), keys and
// values through LDS for four waves together (56 and 53).
#pragma once

#include <stdint.h>

#include <algorithm>

#include "attn_split.h"

namespace sq {

constexpr int64_t kSharedWanted = 384;      // workgroups that chunks are made for, at most
constexpr int64_t kSharedLeast = 128;       // tokens of a chunk, unless the prefix is shorter
constexpr int64_t kSharedMost = 8192;
constexpr int32_t kSharedRows = 32;         // the most query rows of a workgroup

struct SharedSplit {
  int32_t rows;                // query rows of a workgroup: 16 or 32
  int32_t slots;               // workgroups that the query rows of a key-value head can take
  int32_t chunk, count;        // of the prefix
  AttnSplit mine;              // of a request's own tokens
  uint32_t prefix_wgs, own_wgs;
};

// Workgroups of the prefixes (of whole rounds over the XCDs) and of the requests' own tokens.
inline int64_t prefix_wgs(int32_t groups, int32_t Hk, const SharedSplit& s) {
  return groups > 0 ? (static_cast<int64_t>(Hk) * s.count + 7) / 8 * 8 * s.slots : 0;
}
inline int64_t own_wgs(int32_t R, int32_t Hq, int32_t Hk, const SharedSplit& s) { return attn_heads(R, Hq, Hk) * s.mine.count; }
inline int64_t shared_wgs(int32_t R, int32_t groups, int32_t Hq, int32_t Hk, const SharedSplit& s) {
  return prefix_wgs(groups, Hk, s) + own_wgs(R, Hq, Hk, s);
}

// By the query rows that a group has on a key-value head.
inline int32_t shared_rows(int32_t R, int32_t groups, int32_t each, int32_t D) {
  const int64_t rows = static_cast<int64_t>(R) * each / std::max(1, groups);
  return rows > 16 && D <= 192 ? kSharedRows : 16;
}

inline SharedSplit shared_split(int32_t R, int32_t groups, int32_t Hq, int32_t Hk, int32_t D, int32_t max_shared,
                                int32_t max_own) {
  SharedSplit s;
  const int32_t each = Hq / Hk;
  s.rows = shared_rows(R, groups, each, D);
  const int64_t rows = static_cast<int64_t>(R) * each;
  s.slots = static_cast<int32_t>(rows / s.rows + groups);
  const int64_t busy = Hk * std::max<int64_t>(std::max(1, groups), (rows + s.rows - 1) / s.rows);
  const int64_t want = std::max<int64_t>(1, (D <= 64 ? kSharedWanted : 256) / busy);
  const int64_t even = ((max_shared + want - 1) / want + 31) / 32 * 32;
  const int64_t chunk = std::min(kSharedMost, std::max(kSharedLeast, even));
  s.chunk = static_cast<int32_t>(chunk);
  s.count = static_cast<int32_t>((max_shared + chunk - 1) / chunk);
  s.mine = attn_split(attn_heads(R, Hq, Hk), static_cast<int64_t>(max_own) + kAttnTile - 1);
  s.prefix_wgs = static_cast<uint32_t>(prefix_wgs(groups, Hk, s));  // (the caller refuses 2^31 or more in all)
  s.own_wgs = static_cast<uint32_t>(own_wgs(R, Hq, Hk, s));
  return s;
}

// Parts (requests x chunks) that no batch of at most R requests with prefixes up to
// max_shared has more of: busy is at least the requests' rows over 32.
inline int64_t shared_most_parts(int64_t R, int64_t Hq, int64_t max_shared) {
  const int64_t wanted = std::min(R * ((max_shared + kSharedLeast - 1) / kSharedLeast), kSharedWanted * kSharedRows / Hq + 2 * R);
  return std::max(wanted, R * ((max_shared + kSharedMost - 1) / kSharedMost));
}
inline int64_t own_most_parts(int64_t R, int64_t each, int64_t max_own) {
  return std::max(R, attn_most_parts(R, each, max_own + kAttnTile - 1));
}

// Bytes: the parts of both kinds (head_dim values, a maximum and a sum each), and a
// range of tokens per request.
inline size_t shared_ws_bytes(int32_t R, int32_t Hq, int32_t Hk, int32_t D, int32_t max_shared, int32_t max_own) {
  const int64_t parts = shared_most_parts(R, Hq, max_shared) + own_most_parts(R, attn_heads(1, Hq, Hk), max_own);
  return static_cast<size_t>(parts) * Hq * (D + 2) * 4 + static_cast<size_t>(R) * 8;
}

}  // namespace sq
