// Launchers of the orthogonalisation and of the server's step
// (device code in orthogonalize.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace oscars {

constexpr int ORTH_MAX_MATS = 32;
constexpr int ORTH_MAX_STEPS = 16;
constexpr int ORTH_MAX_DIM = 65536;

// One matrix of a call.  rows x cols with row stride ld (elements).
struct OrthMat {
  int rows, cols;
  const void* src;
  int64_t src_ld;
  void* dst;
  int64_t dst_ld;
  // With base: dst = keep base - rate orth(src) (base has dst's layout), all
  // fp32; else dst = orth(src).
  const float* base;
  float keep, rate;
};

struct OrthCoeffs {
  int steps;
  float a[ORTH_MAX_STEPS], b[ORTH_MAX_STEPS], c[ORTH_MAX_STEPS];
};

// Whether the polynomials keep every intermediate, from singular values in [0, 1]
// on, within the range of the fp16 planes, at both of its ends.
bool orth_coeffs_ok(const OrthCoeffs& c);
// Device bytes of a call's temporaries (their base 16-byte aligned).
int64_t orth_workspace(const OrthMat* mats, int count);
// norms_done: the sums of squares of every matrix are in the workspace already
// (launch_server_pass).
hipError_t launch_orthogonalize(const OrthMat* mats, int count, bool bf16, const OrthCoeffs& c,
                                void* ws, hipStream_t s, bool norms_done = false);

// The element-wise pass of the server's step over one flat model.
constexpr int SERVER_MAX_SEGS = 32;
struct ServerArgs {
  const float* global;
  const float* replicas;
  const float* momentum;
  float* global_out;
  float* momentum_out;
  float* update;  // u of the matrix segments, flat layout (workspace)
  int K;
  int64_t n;  // elements and stride of a replica, a multiple of 64
  float beta, plain_lr;
  int nesterov;
  int n_segs;
  int64_t start[SERVER_MAX_SEGS], end[SERVER_MAX_SEGS];
  int64_t size[SERVER_MAX_SEGS];  // elements that are matrix entries; the rest is plain
  int mat[SERVER_MAX_SEGS];       // index of the matrix, or -1
  float w[64];
};
hipError_t launch_server_pass(const ServerArgs& a, void* orth_ws, hipStream_t s);

}  // namespace oscars
