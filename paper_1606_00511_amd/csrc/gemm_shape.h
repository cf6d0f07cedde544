// Tiles and split-K factors of the MFMA products, by their estimated time.
#pragma once

#include <algorithm>
#include <cstdint>

#include "call_context.h"
#include "vocab_internal.h"

namespace hfk {

// Tiles of 32 and 64 rows up to here (the statistics have an entry a tile): for
// few columns of logits they fill the card (fp32, 299 rows, 1,360 x 1,728: 121
// -> 50 us; 1,000 rows: 124 -> 79; no difference from 16,000 columns on).
constexpr int FEW_ROWS = 1024;
constexpr size_t SPLIT_FLOATS = (size_t)32 << 20;   // partials of a split-K product

// Tiles and split-K factor of a product by its estimated time, in us, the
// longest of three and then some:
//   products  a 256 x 256 tile has a compute unit to itself, two of the others
//             share one; RATE: multiply-adds a us of a unit with them, measured
//             at 8,192 x 8,192 x 2,048 (bf16) and 8,192 x 2,048 x 2,048 (fp32), of
//             codes taken as twice bf16's, as the matrix cores have it (4.3e6 is
//             reached: 8,192 x 16,384 x 4,096 in 504 us); filling the LDS and
//             storing a tile take about 6 and 4 us more
//   memory    A once at 4.7 TB/s, which takes 5.5 MB on their way: AHEAD bytes
//             of A per workgroup (32,000 x 1,024 of bf16 for 5 rows: 18.6 us
//             with 250 tiles of 128 x 128, 13.6 with 250 of 128 x 64), and
//             somewhat less with fewer than two workgroups a unit
//   L2        every tile's operands at 15 TB/s
// Partials are written and read again, few of them in the last-level cache.
struct Shape {
  int tile, splits;
  double us;
};
constexpr double RATE[3][4] = {{0.24e6, 0.27e6, 0.22e6, 0.21e6},
                               {1.78e6, 2.4e6, 1.45e6, 1.1e6},
                               {3.5e6, 4.8e6, 2.9e6, 2.2e6}};
constexpr double BYTES_US = 4.7e6, L2_US = 15e6;
constexpr double AHEAD[4] = {16384, 32768, 32768, 49152};
// shapes: how many of the tiles TILE_* there are (2 .. 4; those of few rows from 3 on)
inline Shape shape_for(int type, int64_t M, int64_t N, int64_t K, bool split, int shapes) {
  Shape best = {0, 1, 1e300};
  const int es = type == VT_F32 ? 4 : type == VT_BF16 ? 2 : 1;
  for (int tile = 0; tile < (N <= FEW_ROWS ? shapes : 2); ++tile) {
    const int64_t RM = tile_m(tile), RN = tile_n(tile);
    const int64_t tm = (M + RM - 1) / RM, tn = (N + RN - 1) / RN, tiles = tm * tn;
    const int64_t slots = tile == TILE_BIG ? 256 : 512;
    for (int s = 1; s <= VMAX_SPLITS; ++s) {
      if (s > 1 && (!split || K / s < 256 ||
                    (size_t)s * up(N, VTILE) * up(M, VPAD) > SPLIT_FLOATS))
        break;
      const int64_t rounds = (tiles * s + slots - 1) / slots;
      // the workgroups of a unit share it; one alone does not fill it
      const double share = tile == TILE_BIG ? 1.0 : tiles * s > 256 ? 2.0 : 1.4;
      const double t = rounds * (share * RM * RN * (double)((K + s - 1) / s) /
                                     RATE[type][tile] + (tile == TILE_BIG ? 6.0 : 4.0));
      const double groups = (double)std::min(tiles * s, slots);
      const double mem = (double)M * K * es / BYTES_US *
                             std::max(1.0, 5.5e6 / (groups * AHEAD[tile])) *
                             std::max(1.0, 0.85 + 0.15 * 512 / groups) + 4.0;
      const double part = 8.0 * s * (double)M * N;
      const double l2 = ((double)tn * M + (double)tm * N) * K * es / L2_US + 4.0;
      const double est = std::max({t, mem, l2}) +
                         (s > 1 ? 4.0 + part / (part < 64e6 ? 2 * BYTES_US : BYTES_US) : 0.0);
      if (est < best.us) best = {tile, s, est};
    }
  }
  return best;
}

}  // namespace hfk
