// Partition of a weight gradient's work and the bytes that its blocks may read.
// Plain code, compiled into the kernels and, by the CPU tests, with a host
// compiler on its own.
#pragma once

#include <stdint.h>

#include "emb.h"
#include "ws_words.h"

namespace emb {

constexpr int kStep = 64;    // rows a step takes
constexpr int kGroup = 128;  // columns of an LDS group

// rows of the step from r0 on (0 or less past the last)
EMB_HD inline int step_rows(int64_t N, int64_t r0) { return (int)(N - r0 < kStep ? N - r0 : kStep); }
// groups of 32 codes of a row from column k0 on (a row of codes is whole groups)
EMB_HD inline int groups_left(int32_t K, int k0) { return (K - k0 + EMB_SAVED_GROUP - 1) / EMB_SAVED_GROUP; }
// bytes of a row of dy from column c0 on; with `words` its rows are aligned to 4 bytes and read by words, of which an
// odd last value's is read whole (two bytes past it, within the aligned word that holds it)
EMB_HD inline int dy_row_bytes(int32_t F, int c0, int size, bool words) {
  return words ? ((F - c0) * size + 3) & ~3 : (F - c0) * size;
}
// Bytes readable from a step's first row on, at one column, where `left` rows lie ld bytes apart and `row` bytes of
// the last one follow the column: none where the column is past the matrix (row 0 or less).  A tile's second group of
// columns may be.
EMB_HD inline int rows_bytes(int left, int ld, int row) {
  // (in this form 32768 x 2048 x 6144 takes 803 us, with one condition of both 809)
  const int rows = row > 0 ? left : 0;
  return rows > 0 ? (rows - 1) * ld + row : 0;
}

// Tiles of 128 x 128 with the rows cut into as many parts as give each compute
// unit a block, of at least four steps: 2048 x 256 x 256 11.7 us (13.9 with eight),
// 2048 x 512 x 1536 18.6 and 18.6.
// Tiles of 256 x 256 (one block a compute unit: 256 sums a lane, 128 KB of LDS)
// with as many parts of at least 16 steps as fill one to four rounds of blocks.
// The way that is estimated to take least is taken; the figures (us) are fitted to
// some forty measurements: a block's beginning and end; a step of a small tile with one block a
// compute unit; a step of a large one, more the more compute units are busy; the
// writing and adding of a million parts' sums.  Measured, large against small tiles:
// 32768 x 1024 x 1024 87 (126), 1024 x 2048 x 6144 42 (55), 4096 x 1500 x 2500 60 (65),
// 8192 x 500 x 2500 53 (51), 2048 x 2048 x 2048 48 (38), 20000 x 300 x 800 50 (36); four
// parts of 192 large tiles in three full rounds against one part 785 (811), of 96
// tiles 416 (434).  (Repeated calls on one set of inputs.)
constexpr int kBlocks = 256, kSmallSteps = 4, kBigSteps = 16, kMostRounds = 4;
constexpr double kSmallUs = 6., kSmallStepUs = 0.9, kBigUs = 11., kBigStepUs = 0.85, kBusyUs = 1., kPartUs = 1.5e-6;
struct Plan {
  int groups, parts, steps;  // groups of 128 columns a tile has each way; parts of so many steps
  double us;
};
inline Plan plan_for(int64_t N, int32_t K, int32_t F, bool small) {
  const int64_t steps = (N + kStep - 1) / kStep;
  auto cut = [&](int groups, int rounds, int64_t least) {
    const int64_t tile = groups * kGroup, tiles = ((K + tile - 1) / tile) * ((F + tile - 1) / tile);
    int64_t p = rounds * kBlocks / tiles;
    if (p > steps / least) p = steps / least;
    if (p < 1) p = 1;
    Plan q{groups, 1, (int)((steps + p - 1) / p), 0.};
    if (q.steps > 0) q.parts = (int)((steps + q.steps - 1) / q.steps);
    const double blocks = (double)q.parts * (double)tiles / kBlocks, full = (double)(int64_t)(blocks + 1. - 0.5 / kBlocks);
    q.us = groups == 1 ? kSmallUs + q.steps * kSmallStepUs * (blocks > 1. ? blocks : 1.)
                       : kBigUs + q.steps * (kBigStepUs + kBusyUs * blocks / full) * full;
    if (q.parts > 1) q.us += (double)q.parts * K * F * kPartUs;
    return q;
  };
  Plan best = cut(1, 1, kSmallSteps);
  for (int r = 1; !small && r <= kMostRounds; ++r) {
    const Plan q = cut(2, r, kBigSteps);
    if (q.us < best.us) best = q;
  }
  return best;
}

}  // namespace emb
