// A tile of keys in LDS, as the attention kernels of 32 query rows a wave have it: constexpr functions, so that the host
// can run them too.
#pragma once

#include "host_plan.h"

namespace egmla {

// Byte of piece p (16 bytes: dims 8p ..) of a key's latent row, and of its
// RoPE row: the low bits of the piece are swizzled by the key so that the 16
// lanes of a 16-byte read cycle (keys) and the 32 lanes of a transposed 8-byte
// read cycle hit distinct banks.
constexpr int prefix_latent_byte(int key, int p) {
  return 256 * (p >> 4) + 16 * ((p & 15) ^ (((key & 3) << 2) | ((key >> 2) & 3)));
}
constexpr int prefix_rope_byte(int key, int p) { return 16 * (p ^ ((key >> 1) & 7)); }

// Tiles of the 8-bit cache's attention in blocks of 128 query rows (quant_rows.h): two buffers in turn, behind them 16
// spare bytes.
template <int DC_>
struct Q8Tile {
  static constexpr int DC = DC_, KEYS = DC <= 128 ? 64 : 32, KW = KEYS / 4;  // keys of a tile, of a wave's copies
  static constexpr int LROW = prefix_latent_row(DC), RROW = 128;             // bytes of a key: latent, RoPE key
  static constexpr int ROPE = KEYS * LROW, TILE = KEYS * (LROW + RROW);
  static constexpr int SPARE = 2 * TILE;
  static constexpr int PL = DC / 16;                     // pieces (16 codes) of a key
  static constexpr int NLI = (KW * PL + 63) / 64, NRI = KW * 8 / 64;
};

// Byte of the buffers that takes half `half` (8 fp16 values) of piece p of wave w's keys, for a tile that starts at byte
// `base`.  Lanes behind the wave's last piece store to the spare bytes, whichever buffer is filled: the other one is
// being attended to.
template <class C>
constexpr int q8_latent_store(int base, int w, int p, int half) {
  const int last = C::KW * C::PL - 1, q = p < last ? p : last, key = C::KW * w + q / C::PL;
  if (p > last) return C::SPARE;
  return base + key * C::LROW + prefix_latent_byte(key, 2 * (q % C::PL) + half);
}

}  // namespace egmla
