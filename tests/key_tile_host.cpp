// Host run of the stores that fill a key tile of the 8-bit cache's attention in blocks of 128 query rows (key_tile.h).
//
//   D_C   d_c 64, 128, 320 or 512: "stores into the other buffer, tile bytes of latents not stored to, or stored to
//         twice" over both buffers; every store lies within the buffers and the spare bytes (the program fails otherwise)
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "key_tile.h"

using namespace egmla;

namespace {

template <int DC>
int run() {
  using C = Q8Tile<DC>;
  int other = 0, wrong = 0;
  for (int base : {0, C::TILE}) {
    std::vector<int> stores(C::TILE, 0);
    for (int w = 0; w < 4; ++w)
      for (int p = 0; p < 64 * C::NLI; ++p)
        for (int half = 0; half < 2; ++half) {
          const int at = q8_latent_store<C>(base, w, p, half);
          if (at < 0 || at % 16 != 0 || at > C::SPARE) return 1;
          if (at == C::SPARE) continue;
          if (at / C::TILE != base / C::TILE) ++other;
          else ++stores[at % C::TILE];
        }
    for (int key = 0; key < C::KEYS; ++key)
      for (int piece = 0; piece < DC / 8; ++piece)
        wrong += stores[key * C::LROW + prefix_latent_byte(key, piece)] != 1;
  }
  std::printf("%d %d\n", other, wrong);
  return 0;
}

}  // namespace

int main(int argc, char** argv) {
  switch (argc == 2 ? std::atoi(argv[1]) : 0) {
    case 64: return run<64>();
    case 128: return run<128>();
    case 320: return run<320>();
    case 512: return run<512>();
  }
  return 2;
}
