// How the paged attention splits histories over workgroups (host C++, no HIP).
//
// A workgroup costs about 5 us from its launch to its last store (three
// dependent loads, the join of its waves) and 1.2 us per 128 tokens; a split
// adds a second kernel, 3 to 6 us.  So short spans stay whole: up to 384
// tokens, up to 640 from 192 (request, head) pairs on (200 with up to 600, 32
// query heads: 22.5 us whole, 25 in parts), and up to 1280 where the pairs alone
// fill the CUs (768 with 1055 tokens: 37 us whole, 42 in parts; 512 with up to 700:
// 25 and 26; 2000 with up to 1200: 104 and 106; but 1024 with up to 1000: 56 and 52).
// Longer ones take chunks that make 2048 workgroups in all, eight per CU, but of at
// least 128 tokens (256 past 4096) and at most 512, which is what decides where there
// is much to read and evens out ragged batches: 512 heads with 1024 to 8192 tokens
// (8192 workgroups of 512) take 171 us, 178 in chunks of 384, 169 in 640 or 768, but
// 512 with up to 4096 93, 95, 95 and 97.  Spans past 65536 may take chunks of 1024
// (two histories of 131072, 8 heads: 136 us, 142 in chunks of 512: half the parts to
// join).
#pragma once

#include <stdint.h>

#include <algorithm>

namespace sq {

constexpr int32_t kAttnWhole = 1280;      // the longest span that is ever left whole
constexpr int32_t kAttnLone = 64;         // the longest span that one wave ever takes alone
constexpr int32_t kAttnQTile = 16;        // query heads of a workgroup
constexpr int32_t kAttnTile = 32;         // tokens a wave takes at a time; spans start at a multiple of it

struct AttnSplit {
  int32_t chunk;  // tokens of a workgroup
  int32_t count;  // workgroups of a history of the whole span
};

// Workgroups per split: requests x key-value heads x tiles of query heads.
inline int64_t attn_heads(int32_t R, int32_t Hq, int32_t Hk) {
  return static_cast<int64_t>(R) * Hk * ((Hq / Hk + kAttnQTile - 1) / kAttnQTile);
}
inline int64_t attn_wanted(int64_t heads) { return std::max<int64_t>(1, 2048 / std::max<int64_t>(1, heads)); }
// So many heads or more leave a span whole (INT64_MAX: no number of them).
inline int64_t attn_whole_from(int64_t span) {
  return span <= 384 ? 0 : span <= 640 ? 192 : span <= kAttnWhole ? 512 : INT64_MAX;
}
inline bool attn_whole(int64_t heads, int64_t span) { return heads >= attn_whole_from(span); }
// Whether a workgroup is a single wave: for one tile, and for two where the
// heads fill the CUs several times over (2160 heads of up to 24 tokens 9.3 us,
// with four waves 14.5; 4000 of 64 17.7 and 26.2; but 160 of 64 7.4 and 6.5, and
// 800 of 128 13.0 and 11.0).
inline bool attn_lone(int64_t heads, int64_t span) { return span <= (heads > 768 ? kAttnLone : kAttnTile); }
constexpr int64_t kAttnLeastShort = 128, kAttnLeast = 256, kAttnMost = 512, kAttnMostLong = 1024;
constexpr int64_t kAttnShort = 4096, kAttnLong = 65536;

inline AttnSplit attn_split(int64_t heads, int64_t span) {
  if (attn_whole(heads, span)) return {kAttnWhole, 1};
  const int64_t want = attn_wanted(heads);
  const int64_t even = ((span + want - 1) / want + 127) / 128 * 128;
  const int64_t least = span <= kAttnShort ? kAttnLeastShort : kAttnLeast;
  const int64_t chunk = std::min(span <= kAttnLong ? kAttnMost : kAttnMostLong, std::max(least, even));
  return {static_cast<int32_t>(chunk), static_cast<int32_t>((span + chunk - 1) / chunk)};
}

// Splits into the shortest chunks.
inline int64_t attn_shortest_splits(int64_t longest) {
  return std::max((longest + kAttnLeast - 1) / kAttnLeast,
                  (std::min(longest, kAttnShort) + kAttnLeastShort - 1) / kAttnLeastShort);
}
// No span up to `longest` is split into more parts.
inline int64_t attn_most_splits(int64_t heads, int64_t longest) {
  if (attn_whole(heads, longest)) return 1;
  return std::max(std::min(attn_wanted(heads), attn_shortest_splits(longest)), (longest + kAttnMost - 1) / kAttnMost);
}
// Parts (requests x splits) that no batch of at most R requests, of `each`
// heads, with spans up to `longest` has more of.  Fewer requests are split into
// more: up to the largest batch that is split at all, r requests have the most
// splits of r, or wanted splits that come to 2048 heads at most in all.
inline int64_t attn_most_parts(int64_t R, int64_t each, int64_t longest) {
  const int64_t from = attn_whole_from(longest);
  if (from == 0 || R == 0) return 0;
  const int64_t r = std::min(R, (from - 1) / each);
  return std::max(r * attn_most_splits(r * each, longest), std::min(2048 / each, r * attn_shortest_splits(longest)));
}

// Bytes of the parts: head_dim values, a maximum and a sum each.
inline size_t attn_part_bytes(int32_t R, int32_t Hq, int32_t D, int64_t splits) {
  return splits <= 1 ? 0 : static_cast<size_t>(R) * Hq * static_cast<size_t>(splits) * (D + 2) * 4;
}

// Tokens a call may attend per request, from a multiple of kAttnTile on.
inline int64_t attn_span(int32_t max_kv_len, int32_t window) {
  return window > 0 ? std::min<int64_t>(max_kv_len, static_cast<int64_t>(window) + kAttnTile - 1) : max_kv_len;
}

}  // namespace sq
