// How the rows of an 8-bit product go to launches (device code in
// int8_kernels.hip).  Host only, no HIP: CPU tests include it too.
#pragma once

#include <cmath>
#include <cstdint>
#include <initializer_list>

namespace oscars {

// The first `rows` rows of a product in tiles of `tile`, and its time by what the
// kernels take on this card, in us (a K block: 128 inputs):
//   32    3.5, and 2100 blocks a us over all CUs
//   128   8, and a block 0.55 while no CU has two tiles, else 1.2 for 512 at a time,
//         of which the last up to 256 take 0.75
//   256   20, and a block 1.15 while half of the CUs have a tile, 1.55 up to all
//         of them, else 1.75 for 256 at a time
// Rows x inputs x outputs, measured with 32 / 128 / 256: 256 x 4096 x 1000: 7.1 /
// 24.3 / 47.1, 1024 x 2048 x 2048: 20.4 / 17.9 / 31.7, 3000 x 3000 x 3000: 108 / 52 /
// 45.5, 10000 x 2048 x 2048: 168 / 64.5 / 72, 4096 x 4096 x 4096: 229 / 82.5 / 69.2.
struct I8Plan {
  int tile;
  int64_t rows;
  double us;
};
inline I8Plan i8_plan(int64_t rows, int in, int outs) {
  const double k = (in + 127) / 128;
  I8Plan best{0, rows, 0.0};
  for (int t : {32, 128, 256}) {
    const double n =
        static_cast<double>((outs + t - 1) / t) * static_cast<double>((rows + t - 1) / t);
    const double turns = std::floor(n / 512.0), last = n - 512.0 * turns;
    double us;
    if (t == 32)
      us = 3.5 + n * k / 2100.0;
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

// Rows that fill the CUs with tiles of 128 or 256 a whole number of times, where
// the others and a second launch (1 us) then take less than one more turn would:
// 4352 x 2048 x 2048 went from 38.3 to 32.0 us, 9000 x 4096 x 4096 from 171 to 160;
// 9216 x 2048 x 2048, which stays as it is at 57.8, would take 59.8.
inline I8Plan i8_first_rows(int64_t all, int in, int outs) {
  I8Plan best = i8_plan(all, in, outs);
  for (int t : {128, 256}) {
    const int64_t across = (outs + t - 1) / t, slots = t == 128 ? 512 : 256;
    const int64_t turns = across * ((all + t - 1) / t) / slots;
    const int64_t rows = turns * slots / across * t;
    if (rows == 0 || rows >= all) continue;
    const I8Plan first = i8_plan(rows, in, outs);
    const double us = first.us + 1.0 + i8_plan(all - rows, in, outs).us;
    if (us < best.us) best = {first.tile, rows, us};
  }
  return best;
}

constexpr int i8_threads(int tile) { return tile == 256 ? 512 : 256; }

// launch(tile, at, n) for every launch of a product, rows at .. at + n - 1, until one
// does not return true.  A grid has less than 2^32 threads: from 2^29 rows on those of
// 32 outputs or fewer, in tiles of 32, go to more than one.
template <typename Launch>
bool i8_launches(int64_t rows, int in, int outs, Launch&& launch) {
  const I8Plan first = i8_first_rows(rows, in, outs);
  for (int64_t at = 0; at < rows;) {
    const bool head = at < first.rows;
    const int64_t end = head ? first.rows : rows;
    const int tile = head ? first.tile : i8_plan(rows - first.rows, in, outs).tile;
    const int64_t most = 0xFFFFFFFFll / i8_threads(tile) / ((outs + tile - 1) / tile) * tile;
    const int64_t n = end - at < most ? end - at : most;
    if (!launch(tile, at, n)) return false;
    at += n;
  }
  return true;
}

}  // namespace oscars
