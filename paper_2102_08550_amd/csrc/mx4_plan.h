// How the rows of a 4-bit product go to launches (device code in mx4_kernels.hip).
// Host only, no HIP: CPU tests include it too.
#pragma once

#include <cmath>
#include <cstdint>
#include <initializer_list>

namespace oscars {

// The tile of a product and its estimated time by what the kernels take on this card, in us
// (a K block: 256 inputs; n tiles):
//   32    3, and 2250 blocks a us over all CUs, ten more counted for each tile
//   64    2.9 and a block 0.31 while no CU has two tiles, 0.55 up to two; else 1.5 and a
//         block 0.58 for 512 at a time
//   128   3.2 and a block 0.69 up to 128 tiles, 0.86 up to 256; else 1.0, and 4.2 and a block
//         1.2 for 512 at a time
//   256   10 and a block 1.1 up to 64 tiles, 1.34 up to 128, 1.87 up to 256; else 8 and a
//         block 1.9 for 256 at a time
// Rows x inputs x outputs, measured with 32 / 64 / 128 / 256 (half of x zeros, bf16 outputs):
// 256 x 4096 x 1000: 6.2 / 7.4 / 11.8 / 26, 256 x 4096 x 4096: 15.2 / 7.9 / 14.2 / 27, 1024 x
// 2048 x 2048: 20 / 7.4 / 8.3 / 16.5, 2048 x 4096 x 2048: 49 / 20 / 16.5 / 27, 2048 x 4096 x
// 4096: 93 / 36 / 22.9 / 29, 4096 x 8191 x 2048: 151 / 68 / 39 / 51, 4096 x 4096 x 4096: 184 /
// 72 / 43 / 36.5, 8192 x 2048 x 4096: 275 / 80 / 48 / 43, 8192 x 4096 x 4096: 362 / 143 / 84 /
// 70.5.  The estimates of the large tiles, from an earlier form of the kernel, are up to 10%
// above these; of these shapes and 4096 x 256 x 4096 only the last gets another than its
// fastest tile (94 / 18 / 11.8 / 10.9: it takes 128).
struct Mx4Plan {
  int tile;
  double us;
};
inline double mx4_small_us(int64_t rows, int in, int outs) {
  return 3.0 + std::ceil(outs / 32.0) * std::ceil(static_cast<double>(rows) / 32.0) *
                   (std::ceil(in / 256.0) + 10.0) / 2250.0;
}
inline Mx4Plan mx4_plan(int64_t rows, int in, int outs) {
  const double k = (in + 255) / 256;
  Mx4Plan best{0, 0.0};
  for (int t : {32, 64, 128, 256}) {
    const double n = std::ceil(static_cast<double>(outs) / t) *
                     std::ceil(static_cast<double>(rows) / t);
    double us;
    if (t == 32)
      us = mx4_small_us(rows, in, outs);
    else if (t == 64)
      us = n <= 256.0 ? 2.9 + 0.31 * k
                      : n <= 512.0 ? 2.9 + 0.55 * k : std::ceil(n / 512.0) * (1.5 + 0.58 * k);
    else if (t == 128)
      us = n <= 128.0 ? 3.2 + 0.69 * k
                      : n <= 256.0 ? 3.2 + 0.86 * k : 1.0 + std::ceil(n / 512.0) * (4.2 + 1.2 * k);
    else
      us = n <= 64.0 ? 10.0 + 1.1 * k
                     : n <= 128.0 ? 10.0 + 1.34 * k
                                  : n <= 256.0 ? 10.0 + 1.87 * k
                                               : std::ceil(n / 256.0) * (8.0 + 1.9 * k);
    if (best.tile == 0 || us < best.us) best = {t, us};
  }
  return best;
}

constexpr int mx4_threads(int tile) { return tile == 256 ? 512 : 256; }

// launch(tile, at, n) for every launch of a product, rows at .. at + n - 1, until one
// does not return true.  A grid has less than 2^32 threads.
template <typename Launch>
bool mx4_launches(int64_t rows, int in, int outs, Launch&& launch) {
  const int tile = mx4_plan(rows, in, outs).tile;
  const int64_t most = 0xFFFFFFFFll / mx4_threads(tile) / ((outs + tile - 1) / tile) * tile;
  for (int64_t at = 0; at < rows;) {
    const int64_t n = rows - at < most ? rows - at : most;
    if (!launch(tile, at, n)) return false;
    at += n;
  }
  return true;
}

}  // namespace oscars
