// Which tile a matrix product of the 8-bit linear layers runs on, and into how
// many parts its long axis is split.  Host code without HIP.
#pragma once
#include <cstdint>

namespace muonbp {

// Columns that share a scale, and those whose scales share a 32-bit word.
constexpr int kBlockCols = 128;
constexpr int kGroupCols = 4 * kBlockCols;

// Rows of a product up to which no tile is taken (k_product_few).
constexpr int kFewRows = 16;

constexpr int kMaxParts = 8;        // of a tile's long axis
constexpr int kSplitCounts = 4096;  // tiles in parts

// How a grid of tall x wide tiles is shared out: the first `whole` tiles to one
// workgroup each, the others, their long axis in `parts`, to `parts` workgroups
// each.
struct Shares {
  int whole, parts;
};

// A tile shape's cost in us, measured on 256 CUs: starting and storing a tile,
// and one slice of its long axis where a CU has one tile, or `full` of them or
// more (slower where the matrix cores then clock down, faster where tiles hide
// each other's waits).  Joining parts writes and reads all their sums, at 5 TB/s.
struct TileCost {
  int bm, bn;
  double start, slice, slice_full;
  int full;
  // Of `groups` workgroups that run `slices` each, all on the chip together or
  // in rounds.
  double rounds(int64_t groups, double slices, int cus) const {
    const double load = double(groups) / cus - (full - 1);
    const double at = load < 0.0 ? 0.0 : load > 1.0 ? 1.0 : load;
    return double((groups + cus - 1) / cus) * (start + (slice + (slice_full - slice) * at) * slices);
  }
  double us(const Shares& s, int64_t tiles, int64_t slices, int cus) const {
    const int64_t groups = (tiles - s.whole) * s.parts;
    double t = rounds(groups, double((slices + s.parts - 1) / s.parts), cus);
    if (s.whole) t += rounds(s.whole, double(slices), cus);
    return s.parts > 1 ? t + 1.0 + 0.4 * s.parts + 8.0 * double(groups) * bm * bn / 5e6 : t;
  }
};

struct Choice {
  int tile;  // in its table
  Shares shares;
  unsigned groups;
};

// The tile shape and the shares that cost least: no tile, every tile, or the
// tiles of the last, unfilled round in parts, whose sums fit sum_floats.
template <int N>
Choice choose(const TileCost (&tiles)[N], int64_t rows, int64_t cols, int64_t slices, int64_t most_parts,
              int64_t sum_floats, int cus) {
  Choice best{};
  double least = -1.0;
  for (int t = 0; t < N; ++t) {
    const int64_t bm = tiles[t].bm, bn = tiles[t].bn;
    const int64_t count = (rows + bm - 1) / bm * ((cols + bn - 1) / bn);
    for (int parts = 1; parts <= kMaxParts && parts <= most_parts; ++parts)
      for (int tail = 0; tail < 2; ++tail) {
        const int64_t whole = tail ? count / cus * cus : 0, cut = count - whole;
        if (tail && (parts == 1 || whole == 0 || cut == 0)) continue;
        if (parts > 1 && (cut > kSplitCounts || cut * parts * bm * bn > sum_floats)) continue;
        const Shares s{int(whole), parts};
        const double us = tiles[t].us(s, count, slices, cus);
        if (least < 0.0 || us < least) {
          least = us;
          best = Choice{t, s, unsigned(whole + cut * parts)};
        }
      }
  }
  return best;
}

// Slices of 64 columns, in 8 bits; widened (exact): half the rate, so the 256 x 256
// tile, whose widened fragments do not fit its registers, is left out.
constexpr TileCost kProductTiles[] = {{256, 256, 8.0, 0.50, 0.78, 1},
                                      {128, 128, 2.5, 0.25, 0.28, 2},
                                      {64, 128, 1.0, 0.18, 0.20, 2},
                                      {128, 256, 5.0, 0.32, 0.46, 1}};
constexpr TileCost kProductExactTiles[] = {{128, 128, 3.0, 0.37, 0.43, 2}, {64, 128, 1.0, 0.27, 0.29, 2}};

// For more than kFewRows rows.
inline Choice product_choice(bool exact, int64_t rows, int64_t cols, int64_t k, int64_t sum_floats, int cus) {
  const int64_t blocks = (k + kBlockCols - 1) / kBlockCols;
  return exact ? choose(kProductExactTiles, rows, cols, 2 * blocks, blocks, sum_floats, cus)
               : choose(kProductTiles, rows, cols, 2 * blocks, blocks, sum_floats, cus);
}

// Slices of 32 tokens.
constexpr TileCost kWeightGradTiles[] = {{256, 256, 8.0, 0.64, 0.82, 1},
                                         {128, 128, 4.0, 0.36, 0.29, 2},
                                         {64, 64, 3.0, 0.09, 0.09, 2}};

inline Choice weight_grad_choice(int64_t rows, int64_t cols, int64_t tokens, int64_t sum_floats, int cus) {
  const int64_t slices = (tokens + 31) / 32;
  return choose(kWeightGradTiles, rows, cols, slices, slices > 0 ? slices : 1, sum_floats, cus);
}

}  // namespace muonbp
