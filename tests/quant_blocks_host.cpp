// Host run of the numbering of query blocks (quant_blocks.h) as q8_schedule takes it, 256 sequences at a time.
//
//   T H BLOCK_ROWS B   offsets 0, T, 0, T, ..: "last block, steps of the numbering that fall, numbers out of range"
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "quant_blocks.h"

using namespace egmla;

int main(int argc, char** argv) {
  if (argc != 5) return 2;
  const int T = std::atoi(argv[1]), H = std::atoi(argv[2]), rows = std::atoi(argv[3]), B = std::atoi(argv[4]);
  const int most = q8_most_blocks(T, H, rows, B);
  std::vector<int> first(B + 1);
  int blocks = 0;
  for (int b0 = 0; b0 < B; b0 += 256) {
    int64_t total = 0;
    for (int b = b0; b < B && b < b0 + 256; ++b) {
      first[b] = q8_blocks_behind(blocks, static_cast<int>(total), most);
      total += q8_sequence_blocks(b % 2 ? T : 0, b % 2 ? 0 : T, H, rows);
    }
    if (total > INT32_MAX) return 1;
    blocks = q8_blocks_behind(blocks, static_cast<int>(total), most);
  }
  first[B] = blocks;
  int falls = 0, outside = 0;
  for (int b = 0; b < B; ++b) falls += first[b + 1] < first[b];
  for (int f : first) outside += f < 0 || f > most;
  std::printf("%d %d %d\n", blocks, falls, outside);
  return 0;
}
