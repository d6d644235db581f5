// How many workgroups the dense operators' kernels take, and their split into launches that HIP
// accepts.  Host only, without HIP itself.
#pragma once

#include <stdint.h>

namespace embd {

// HIP refuses 2^32 threads or more along a dimension of a launch; sizes that fit the device pass that (a matrix
// of 2^27 rows and one column by k_quantize).  A power of two, so that every launch starts at a multiple of 8
// workgroups where workgroups are of one.
constexpr int64_t kLaunchThreads = (int64_t)1 << 31;

// launch(first, n) for the consecutive parts of `workgroups` workgroups of `threads`, until one fails.
template <class F>
auto in_launches(int64_t workgroups, int threads, F launch) -> decltype(launch((int64_t)0, 0u)) {
  const int64_t most = kLaunchThreads / threads;
  int64_t first = 0;
  for (;;) {
    const int64_t left = workgroups - first, n = left < most ? left : most;
    const auto e = launch(first, (unsigned)n);
    if (e != decltype(e){} || n == left) return e;
    first += n;
  }
}

constexpr int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Workgroups of k_quantize, of 32 rows x 128 columns: squares of kSquareCols tiles by one (or, where it goes by
// columns, 512 rows), from kSquaresFrom of them on spread over the XCDs and their number a multiple of 8.
constexpr int kQuantizeRows = 32, kQuantizeCols = 128;
constexpr int kSquareCols = 4, kSquareRowsByColumns = 512 / kQuantizeRows;
constexpr int kSquaresFrom = 64;
constexpr int square_rows(bool by_columns) { return by_columns ? kSquareRowsByColumns : 1; }
inline int64_t quantize_workgroups(int64_t rows, int64_t cols, bool by_columns) {
  const int64_t squares = ceil_div(rows, kQuantizeRows * square_rows(by_columns)) * ceil_div(cols, kQuantizeCols * kSquareCols);
  return (squares >= kSquaresFrom ? ceil_div(squares, 8) * 8 : squares) * square_rows(by_columns) * kSquareCols;
}

// Row tiles of a wave's side in k_product, the side of a workgroup's tile being 32 of them (256, 128 or 64 rows and
// columns): the least time, in units of a round of 256 workgroups of 256 x 256.  us a full round
// (16384x8192x12800): 92 at 8, 28.7 at 4, 10.9 at 2; one round alone (1024x1024x12800, 256 CUs not full at 8 and 4): 63,
// 25 and 18.3.  A launch of the smaller tiles is one workgroup a tile and must be one that HIP takes.
inline int64_t product_tiles(int64_t row_tiles_a, int64_t row_tiles_b, int f) {
  return ceil_div(row_tiles_a, 2 * f) * ceil_div(row_tiles_b, 2 * f);
}
inline int product_side(int64_t row_tiles_a, int64_t row_tiles_b) {
  const auto rounds = [&](int f) { return (double)ceil_div(product_tiles(row_tiles_a, row_tiles_b, f), 256); };
  const auto fits = [&](int f) { return product_tiles(row_tiles_a, row_tiles_b, f) * 256 < (int64_t)1 << 32; };
  const double t8 = rounds(8), t4 = 0.31 * rounds(4) + 0.09, t2 = 0.12 * (rounds(2) + 1);
  if (!fits(4) || (t8 <= t4 && (t8 <= t2 || !fits(2)))) return 8;
  return t4 <= t2 || !fits(2) ? 4 : 2;
}

}  // namespace embd
