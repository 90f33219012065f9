// The launch of added weights of few rows, out of the built library: a division that
// no kernel is made for is an error and launches nothing, for any type.  (Divisions
// that are fine are not launched here.)
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "evict.h"

using namespace starkv;

int main() {
  int checked = 0;
  for (int d : {64, 128})
    for (int type = 0; type < 3; ++type)
      for (int G : {1, 3, 4, 33, 64}) {
        PagedView v{};
        v.n_layers = 1;
        v.H = v.G = G;
        v.d = d;
        v.fp4 = type == 0;
        v.esz = type == 2 ? 4 : 2;
        v.row = v.fp4 ? d / 2 : d * v.esz;
        const int part = mass_part(v.fp4, v.row);
        MassCall c{};
        c.r.n = 1;
        const auto refused = [&](int tile, int row_blocks) {
          c.s = MassShape{};
          c.s.n_rows = c.s.tiles = c.s.blocks = c.s.n_split = 1;
          c.s.tile = tile;
          c.s.row_blocks = row_blocks;
          const int got = launch_mass_add(v, c, nullptr);
          if (got != 1) {          // hipErrorInvalidValue
            std::printf("d %d type %d G %d tile %d rows %d: %d\n", d, type, G, tile, row_blocks, got);
            std::exit(1);
          }
          ++checked;
        };
        for (int tile : {0, part / 2, 2 * part, 3 * part, kMassTile + part, 512}) refused(tile, 1);
        refused(part, 3);
        refused(part, 0);
        // the groups' sums of a tile would not fit LDS
        if (G * kMassTile * 8 > 64 * 1024) refused(kMassTile, 1);
      }
  std::printf("%d refused\n", checked);
  return 0;
}
