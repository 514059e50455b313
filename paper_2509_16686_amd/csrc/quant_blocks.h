// Blocks of query rows of the 8-bit cache's attention, numbered through the sequences: constexpr functions, so that the
// host can run them too.
#pragma once

#include <cstdint>

namespace egmla {

// Blocks there is room for: more than any rising offsets of T tokens make.
constexpr int q8_most_blocks(int T, int H, int block_rows, int B) {
  return static_cast<int>(static_cast<int64_t>(T) * H / block_rows) + B;
}
constexpr int q8_sequence_blocks(int first, int next, int H, int block_rows) {
  const int64_t rows = static_cast<int64_t>(next > first ? next - first : 0) * H;
  return static_cast<int>((rows + block_rows - 1) / block_rows);
}
// The first block behind `blocks` and `more`, which those of 256 sequences are at most (below 2^31: between two sequences
// that take all tokens the offset falls back).  Offsets that fall, which the call does not allow, could count a token many
// times: the count stops at the most.
constexpr int q8_blocks_behind(int blocks, int more, int most) { return more < most - blocks ? blocks + more : most; }

}  // namespace egmla
