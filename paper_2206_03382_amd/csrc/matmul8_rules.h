// Which tile an 8-bit product takes: plain host arithmetic on sizes, kept apart from the kernels so that a test can ask it without a GPU.
#pragma once
#include <stdint.h>

namespace moe {

// Whether 256 x 256 tiles, one to a unit, are expected to be done before 128 x 128 ones, two to a unit; rows: what an expert holds on average.  Both in microseconds, from launches of
// full rounds: a round of large tiles takes 9 + 1.33 a K-step of 128, one of small tiles 5 + 0.95, and small ones that have a unit to themselves 6 + 0.68.  Measured (small, large): 8 experts x
// 256 rows, 2048 x 2048 18.0 and 26.4 us, x 512 22.1 and 27.9, x 1024 41.3 and 34.1, x 2048 78.2 and 62.8; 64 x 128, 1024 x 1024 18.4 and 19.4, x 256 27.6 and 23.8, x 1024 99.3
// and 77.5; one of 1024 x 4096 x 4096 27.3 and 42.7, 2048 36.0 and 44.4, 4096 68.9 and 55.4; 17 x 453 rows, 776 x 1544 21.5 and 19.9.
static inline bool matmul8_takes_large_tile(int64_t E, double rows, int64_t K, int64_t N) {
  const double steps = (double)((K + 127) / 128);
  auto tiles = [&](int64_t side) { return (double)(E * ((N + side - 1) / side)) * (double)(((int64_t)rows + side - 1) / side); };
  auto rounds = [](double n, double places) { return (double)(int64_t)((n + places - 1) / places); };
  const double large = rounds(tiles(256), 256) * (9.0 + 1.33 * steps);
  const double small = tiles(128) <= 256 ? 6.0 + 0.68 * steps : rounds(tiles(128), 512) * (5.0 + 0.95 * steps);
  return large < small;
}

}  // namespace moe
