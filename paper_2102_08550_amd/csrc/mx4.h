// Launchers of the layer in microscaled 4-bit floating point (device code in
// mx4_kernels.hip).
//
// A row in 4 bits: 32 consecutive entries share a scale, the least power of two s
// (2^-127 to 2^125) with max |x| < 7 s, held as a byte e, s = 2^(e - 127); an entry is x / s rounded
// to the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives, ties to the even
// code, two a byte, the first in the low half.  Bytes are zero behind the row's last
// entry, to a whole 128 (256 entries), scales to a whole 16 (512 entries).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "philox.h"

namespace oscars {

constexpr int64_t MX4_MAX_COLS = int64_t{1} << 24;  // entries of a quantised row

constexpr int64_t mx4_bytes(int64_t cols) { return (cols + 255) / 256 * 128; }
constexpr int64_t mx4_scales(int64_t cols) { return (cols + 511) / 512 * 16; }

struct Mx4Rows {
  uint8_t* q;
  int64_t q_ld;
  uint8_t* scale;
  int64_t s_ld;
};

// What is quantised: x, or for the gradients what is behind a layer's epilogue:
// 0 where y <= 0 or the generator dropped the entry (only asked without y), else
// fl(x factor).
struct Mx4Source {
  const void* x;
  int64_t x_ld;
  bool bf16;
  int64_t rows;
  int cols;
  const void* y;  // of x's type, or nullptr; gradients only, like drop
  int64_t y_ld;
  DropArgs drop;
};
hipError_t launch_mx4_rows(const Mx4Source& a, const Mx4Rows& to, hipStream_t s);
// The rows of x' in 4 bits; fewer than 2^23 tiles.
int64_t mx4_column_tiles(int64_t rows, int cols);
hipError_t launch_mx4_columns(const Mx4Source& a, const Mx4Rows& to, hipStream_t s);

// What the gradients multiply: dz by columns and, with z_rows.q, by rows; x by columns;
// and dz's columns' sums, or nullptr: where mx4_sum_parts(rows) is not 0, so many parts of
// them, for a product to add up.
struct Mx4Gradient {
  Mx4Source z, x;
  Mx4Rows z_rows, z_columns, x_columns;
  float* sums;
  double* part;
};
int64_t mx4_sum_parts(int64_t rows);
hipError_t launch_mx4_gradient(const Mx4Gradient& g, hipStream_t s);

struct Mx4Values {
  const uint8_t* q;
  int64_t q_ld;
  const uint8_t* scale;
  int64_t s_ld;
  int64_t rows;
  int cols;
  void* out;
  int64_t out_ld;
  bool out_bf16;
};
hipError_t launch_mx4_values(const Mx4Values& a, hipStream_t s);

// out[c] = sum_i part[i][c], which workgroups behind a product's do.
struct Mx4Sums {
  const double* part;  // [parts][cols]; parts 0: nothing
  int64_t parts;
  int cols;
  float* out;
};

// out[r][o] = drop(relu?(sum_k x[r][k] w[o][k] + bias[o]))
struct Mx4Product {
  const uint8_t* xq;
  int64_t x_ld;
  const uint8_t* xs;
  int64_t xs_ld;
  const uint8_t* wq;
  int64_t w_ld;
  const uint8_t* ws;
  int64_t ws_ld;
  const float* bias;  // or nullptr
  bool relu;
  int64_t rows;
  int in, outs;
  void* out;
  int64_t out_ld;
  bool out_bf16;
  DropArgs drop;
  Mx4Sums sums;
  uint32_t row0;  // of dropout's rows, the first one's number
};
hipError_t launch_mx4_product(const Mx4Product& a, hipStream_t s);
// One or two products that wait for nothing of each other, in one launch if they are small.
hipError_t launch_mx4_products(const Mx4Product* p, int n, hipStream_t s);

// A few rows: quantisation and product in one launch (x of the caller's type; xq,
// x_ld, xs and xs_ld of `a` unused).
bool mx4_one_launch(int64_t rows, int in);
hipError_t launch_mx4_few(const Mx4Product& a, const void* x, int64_t x_ld, bool x_bf16,
                          hipStream_t s);

// `rows` rows of `cols` floats, ld apart: zeros.
hipError_t launch_mx4_zero(float* p, int64_t ld, int64_t rows, int cols, hipStream_t s);

}  // namespace oscars
