// How the rows of a 4-bit product go to launches (device code in mx4_kernels.hip).
// Host only, no HIP: CPU tests include it too.
#pragma once

#include <cmath>
#include <cstdint>
#include <initializer_list>

namespace oscars {

// The first `rows` rows of a product in tiles of `tile`, and its estimated time in us
// (a K block: 256 inputs).
struct Mx4Plan {
  int tile;
  int64_t rows;
  double us;
};
inline Mx4Plan mx4_plan(int64_t rows, int in, int outs) {
  const double k = (in + 255) / 256;
  Mx4Plan best{0, rows, 0.0};
  for (int t : {32, 128, 256}) {
    const double n =
        static_cast<double>((outs + t - 1) / t) * static_cast<double>((rows + t - 1) / t);
    const double turns = std::floor(n / 512.0), last = n - 512.0 * turns;
    double us;
    if (t == 32)
      us = 3.5 + n * k / 2000.0;
    else if (t == 128)
      us = 8.0 + k * (n <= 256.0 ? 0.55
                                 : 1.2 * turns + (last > 256.0 ? 1.2 : last > 0.0 ? 0.75 : 0.0));
    else
      us = 20.0 + k * (n <= 144.0 ? 1.15 : n <= 256.0 ? 1.55 : 1.75 * std::ceil(n / 256.0));
    if (best.tile == 0 || us < best.us) {
      best.tile = t;
      best.us = us;
    }
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
