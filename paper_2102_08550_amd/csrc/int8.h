// Launchers of the 8-bit linear layer (device code in int8_kernels.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace oscars {

// q[r][c] = round-half-even(x[r][c] / scale[r]), scale[r] = max |x[r]| / 127;
// columns cols .. up to the next multiple of 128 (within ldq) are zero.
struct QuantArgs {
  const void* x;
  int64_t x_ld;
  bool bf16;
  int64_t rows;
  int cols;
  int8_t* q;
  int64_t q_ld;
  float* scale;
};
hipError_t launch_quantize_rows(const QuantArgs& a, hipStream_t s);

// out[r][o] = relu?(xscale[r] wscale[o] sum_k xq[r][k] wq[o][k] + bias[o])
struct MatmulI8Args {
  const int8_t* xq;  // rows of whole 128-byte blocks, zero from `in` on
  int64_t x_ld;
  const float* xscale;
  const int8_t* wq;
  int64_t w_ld;  // a multiple of 16
  const float* wscale;
  const float* bias;  // or nullptr
  bool relu;
  int64_t rows;
  int in, outs;
  void* out;
  int64_t out_ld;
  bool out_bf16;
};
hipError_t launch_matmul_i8(const MatmulI8Args& a, hipStream_t s);

// A few rows: quantisation and product in one launch (x of the caller's type;
// xq, x_ld and xscale of `a` unused).
bool linear_i8_one_launch(int64_t rows, int in);
hipError_t launch_linear_i8_few(const MatmulI8Args& a, const void* x, int64_t x_ld, bool x_bf16,
                                hipStream_t s);

}  // namespace oscars
