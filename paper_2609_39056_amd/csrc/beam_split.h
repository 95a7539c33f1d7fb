// How the choice of continuations splits rows of logits over workgroups (host C++, no HIP).
//
// A thread takes 8, 16 or 32 values, a workgroup a chunk of 2048, 4096 or 8192
// tokens.  Short chunks fill the chip where there is little to read, but leave more
// keys to join: 2048 tokens up to 1024 chunks in all, 4096 up to 8192 chunks' worth
// of 2048 (about 4096 of their own), and longer ones where a row would leave more than 256
// keys or is longer than 2^18 (128 rows of 131071, 8 each: 24.1, 20.9 and 20.0 us with
// 2048, 4096 and 8192 tokens; 8 rows, 16 each: 24.6, 19.3, 15.9; 64 rows of 32000, 4
// each: 10.1, 10.1, 10.9).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace sq {

constexpr int kBeamThreads = 256;
constexpr int kBeamMostEach = 32;
constexpr int64_t kBeamShort = 1024, kBeamMiddle = 8192;  // chunks of 2048 tokens up to which a thread takes 8 or 16
constexpr int64_t kBeamKeys = 256;                        // keys of a row, with chunks shorter than the longest

inline int beam_chunks(int32_t vocab, int each) { return (vocab + kBeamThreads * each - 1) / (kBeamThreads * each); }

// Values of a thread.
inline int beam_each(int32_t rows, int32_t vocab, int32_t width) {
  const int64_t shortest = static_cast<int64_t>(rows) * beam_chunks(vocab, 8);
  int each = vocab > (1 << 18) ? kBeamMostEach : 8;
  if (each == 8 && (shortest > kBeamShort || beam_chunks(vocab, 8) * int64_t{width} > kBeamKeys)) each = 16;
  if (each == 16 && (shortest > kBeamMiddle || beam_chunks(vocab, 16) * int64_t{width} > kBeamKeys)) each = 32;
  return each;
}

// Chunks that no call with as many rows and tokens or fewer has more of: of 2048 tokens
// kBeamShort at most, else of 4096 or longer.
inline int64_t beam_most_chunks(int64_t rows, int32_t vocab) {
  return std::max(std::min(kBeamShort, rows * beam_chunks(vocab, 8)), rows * beam_chunks(vocab, 16));
}

// Bytes of the workspace for a chunk: its sum, its maximum, and its best keys.
constexpr size_t beam_chunk_bytes(int32_t width) { return 16 + 8 * static_cast<size_t>(width); }

}  // namespace sq
