// Which tile and parts each product or weight gradient takes (built by
// tests/test_linear_choice.py with g++; no GPU, no HIP).  Reads lines
// "product|exact|grad rows cols long workspace_bytes" (long: the columns of the
// operands, or the tokens) and prints "tile_rows tile_cols whole parts" for each,
// on 256 CUs; "few" for a product of too few rows for a tile.
#include <cstdio>
#include <cstring>

#include "linear_plan.h"

using namespace muonbp;

int main() {
  char kind[16];
  long long rows, cols, along, bytes;
  while (std::scanf("%15s %lld %lld %lld %lld", kind, &rows, &cols, &along, &bytes) == 5) {
    const bool grad = !std::strcmp(kind, "grad"), exact = !std::strcmp(kind, "exact");
    if (!grad && rows <= kFewRows) {
      std::printf("few\n");
      continue;
    }
    const Choice c = grad ? weight_grad_choice(rows, cols, along, bytes / 4, 256)
                          : product_choice(exact, rows, cols, along, bytes / 4, 256);
    const TileCost& t = grad ? kWeightGradTiles[c.tile] : exact ? kProductExactTiles[c.tile] : kProductTiles[c.tile];
    std::printf("%d %d %d %d\n", t.bm, t.bn, c.shares.whole, c.shares.parts);
  }
}
