// How the products of the few-token layer are cut into blocks, and whether their plan has a launch of its own: plain host arithmetic on sizes, kept apart from the
// kernels so that a test can ask it without a GPU.
#pragma once
#include <stdint.h>

namespace moe {

// Units of work of both products: an expert each, or, where there are fewer choices than experts, a choice each.
static inline int64_t few_units_of(int64_t T, int64_t E, int k) { return E < T * k ? E : T * k; }

// Columns of a block.  Blocks of 64 where there are enough of them for three quarters of their places (two to a CU with one tile of rows, one with four), else of 32: more blocks, and more
// places taken, for more reads of the rows.  Rows of 32 columns of bf16 weights are half a line of 128 bytes: always 64.
// A layer of 8-bit weights, us with 64 and with 32 columns (blocks of a product with 64): 1 token x 2 experts of 4096 x 4096 (128) 36.2, 33.3; top-2 of 16 x 8 of 2048 x 2048 (256)
// 35.3, 31.9, of 16 x 32 of 1024 x 1024 (512) 37.5, 36.2, of 64 x 16 of 4096 x 1024 (256 and 1024) 70.8, 78.4, of 24 x 4 of 768 x 512 (32 and 48) 22.5, 19.6; top-8 of 16 x 32 of 1024 x 1024
// 41.7, 41.0, of 64 x 16 of 4096 x 1024 101.8, 116.1.
static inline int few_columns(int64_t T, int64_t units, int64_t width, bool bf16_weights) {
  return bf16_weights || (width + 63) / 64 * units >= (T <= 16 ? 384 : 192) ? 64 : 32;
}

// The plan by every block of the first product for itself, or, where they do not all run at once (two to a CU, or one of more than 16 tokens), in a launch of its own.
// us, first and then: 16 tokens x 8 experts of 2048 x 2048 (256 blocks) 41.1, 42.8; 1 x 8 of 128 of 4096 x 1024, 8 bits (128) 42.3, 44.1; 4 x 8 of 64 of 1024 x 4096 (512)
// 44.2, 46.3; 16 x 64 of 128 of 1024 x 1024, 8 bits (1024) 61.2, 58.5; 64 x 64 of 1024 x 4096 (4096) 264.7, 213.8.  Blocks of 32 columns, 8 bits: 1 x 8 of 128 of 2048 x 2560 (640)
// 42.7, 39.9; 4 x 8 of 64 of 4096 x 640 (640) 71.0, 69.4; 64 x 16 of 4096 x 640 (320) 65.4, 64.1; 8 x 16 of 512 x 1152 (576) 22.8, 23.5.
static inline bool few_planned(int64_t T, int64_t H, int64_t E, int k, bool bf16_weights) {
  const int64_t units = few_units_of(T, E, k), columns = few_columns(T, units, H, bf16_weights);
  return (H + columns - 1) / columns * units > (T <= 16 ? 512 : 256);
}

}  // namespace moe
