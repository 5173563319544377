// Orthogonalisation of updates by Newton-Schulz products, and the server's
// step around it.
//
//   X_0 = G / |G|_F;   for each step (a, b, c):
//     A = X X',  P = a I + b A + c A A,  X <- P X.
//
// G is taken m x n with m <= n (its transpose where it is tall: the iteration
// commutes with transposition), so A and P are the small square ones.  Every
// product is C = L R' of two K-contiguous operands (nt_mma.h): A from X with
// itself, A A from A with itself (symmetric), P X from P and X' kept beside X.
// A and P are symmetric: the tiles on and below the diagonal are computed, and
// each is stored to both places.  One launch runs a product for all matrices of
// a call.
//
// Number format.  The iterates live in the workspace as fp16 planes, scaled by
// powers of two so that neither end of fp16's range matters: NT_SPLIT (hi and
// lo, 22 bits, three matrix instructions a product) for fp32 and for bf16
// matrices, because a rounding is amplified by later steps: one multiplies the
// small singular directions by up to |a|.  With 11 bits in the last two steps of
// five a bf16 result had 16 to 28% of its entries one step or more off what the
// products in 32 bits give, with 22 bits 0.02 to 0.35% (4096 x 4096: 2607 us then,
// 3442 so).  X_0 is G times a power of two, exact and one plane for bf16 (one
// instruction a product); the rest of 1 / |G|_F is a factor on the first products,
// so nothing is rounded before the first step.
// Products sum in fp32 in a fixed order; norms in double.
#include "orthogonalize.h"

#include <cmath>

#include "nt_mma.h"

namespace oscars {
namespace {

typedef NtShape<256, 256, 2, 4> OrthL;
typedef NtShape<128, 128, 2, 2, true> OrthM;

enum OrthKind { ORTH_GRAM = 0, ORTH_POLY = 1, ORTH_APPLY = 2, ORTH_LAST = 3 };

constexpr float kScaleA = 128.0f;  // of A and P in their planes
constexpr float kMaxSigma = 16.0f;
constexpr float kMaxPoly = 400.0f;
// Least Frobenius norm of an iterate in its planes.  They hold 2^-25 / orth_scale of
// an entry, whatever its size: fp32 results stay where roundings to 22 bits put
// them down to 0.01 (two steps; 3e-6), at 1e-4 they are 2e-4 to 4e-4 off.
constexpr double kMinNorm = 1.0 / 16.0;
constexpr int kNormParts = 512;  // partial sums of squares per matrix

struct MatDesc {
  OrthMat u;
  int64_t at;  // of the matrix's planes in the workspace
};

struct OrthArgs {
  MatDesc mat[ORTH_MAX_MATS];
  int count;
  // A launch's workgroups go matrix after matrix: position i is matrix order[i],
  // its first workgroup first[i], a multiple of 8.  (Whole words: beside an array
  // of bytes with the same index the compiler addressed first[i] as (base + i) +
  // 3 i, and scalar loads drop the low bits of each summand.)
  int first[ORTH_MAX_MATS + 1];
  int order[ORTH_MAX_MATS];
  // Products in tiles of 128 or 256: position i's before cut[i] are done as such, the
  // others (of 128) as tiles of 32, in a launch with `rest` set.
  int cut[ORTH_MAX_MATS];
  int rest;
  char* ws;
  float a, b, c;
  int in_scaled;       // 1: the planes hold X times orth_scale; 0: X_0 (factor in the workspace)
  int parity;          // which of the two X' buffers is read
  int bf16;            // convert / LAST: the caller's type
};

__host__ __device__ __forceinline__ int pad64(int v) { return (v + 63) & ~63; }
__host__ __device__ __forceinline__ int mat_m(const OrthMat& u) {
  return u.rows < u.cols ? u.rows : u.cols;
}
__host__ __device__ __forceinline__ int mat_n(const OrthMat& u) {
  return u.rows < u.cols ? u.cols : u.rows;
}
__host__ __device__ __forceinline__ bool mat_tall(const OrthMat& u) { return u.rows > u.cols; }

// Head of the workspace: the factor on X_0 per matrix, then the partial sums.
constexpr int64_t kScaleBytes = 256;
constexpr int64_t kHeadBytes = kScaleBytes + int64_t{ORTH_MAX_MATS} * kNormParts * 8;
__device__ __forceinline__ float* ws_scale(char* ws) { return reinterpret_cast<float*>(ws); }
__device__ __forceinline__ double* ws_parts(char* ws, int mat) {
  return reinterpret_cast<double*>(ws + kScaleBytes) + mat * kNormParts;
}

struct Planes {
  char *x, *xt[2], *a, *p;
};
__host__ __device__ __forceinline__ int64_t plane_bytes(int rows, int k) {
  return (static_cast<int64_t>(rows) * (pad64(k) / 32 + 1) * NT_BLOCK + 255) / 256 * 256;
}
__host__ __device__ __forceinline__ Planes mat_planes(char* ws, const MatDesc& d) {
  const int m = mat_m(d.u), n = mat_n(d.u);
  Planes q;
  q.x = ws + d.at;
  q.xt[0] = q.x + plane_bytes(m, n);
  q.xt[1] = q.xt[0] + plane_bytes(n, m);
  q.a = q.xt[1] + plane_bytes(n, m);
  q.p = q.a + plane_bytes(m, m);
  return q;
}
__host__ __device__ int64_t mat_bytes(const OrthMat& u) {
  const int m = mat_m(u), n = mat_n(u);
  return plane_bytes(m, n) + 2 * plane_bytes(n, m) + 2 * plane_bytes(m, m);
}
// K blocks of a row of k values (k padded to 64 with zeros), and the bytes from one
// row to the next: an odd number of blocks.  Every tile reads and writes the same
// columns of many rows at a time; rows a power of two apart would put them all
// on a few memory channels.
__host__ __device__ __forceinline__ int row_blocks(int k, int fmt) {
  return pad64(k) / (fmt == NT_F16 ? 64 : 32);
}
__host__ __device__ __forceinline__ int64_t row_bytes(int k, int fmt) {
  return static_cast<int64_t>(row_blocks(k, fmt) | 1) * NT_BLOCK;
}

// Power of two on the iterates in their planes.  The rms of an m x n matrix
// with singular values near 1 is 1 / sqrt(n): 16 sqrt(n) brings it to about 16,
// its lo plane to 2^-8; an entry is at most kMaxSigma, 2^15 with the cap.
__host__ __device__ __forceinline__ float orth_scale(int n) {
  int e = 4;
  while (e < 11 && (int64_t{1} << (2 * (e - 4) + 1)) < n) ++e;
  return static_cast<float>(1 << e);
}

// The position of entry `at` of a launch's list: how many positions end at or
// before it.  A lane looks at each (ORTH_MAX_MATS <= 64), one load in all.
__device__ __forceinline__ int find_position(const int* first, int count, int at) {
  const int lane = threadIdx.x & 63;
  const bool past = lane < count - 1 && at >= first[lane + 1];
  return __builtin_popcountll(__ballot(past));
}
// Workgroups or tiles of one XCD (index mod 8) take neighbouring work.
__device__ __forceinline__ int xcd_index(int id, int total) {
  const int per = total >> 3, rem = total & 7, x = id & 7, q = id >> 3;
  return x * per + (x < rem ? x : rem) + q;
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typedef _Float16 h2 __attribute__((ext_vector_type(2)));
  const h2 v = {static_cast<_Float16>(a), static_cast<_Float16>(b)};
  return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ float lo_of(float v) {
  return v - static_cast<float>(static_cast<_Float16>(v));
}

// One 16-byte piece of a plane row: eight values from k (a multiple of 8), as hi
// or as lo.  The pieces of a 128-byte line are stored by neighbouring lanes in
// one instruction (store_lines): the L2 takes one request a line instead of one
// a piece, which had made the stores of 4096 x 4096 planes 70 us of 380.
__device__ __forceinline__ void put8(char* row, int k, int fmt, bool lo, const float* v) {
  nt_u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = lo ? lo_of(v[2 * i]) : v[2 * i], b = lo ? lo_of(v[2 * i + 1]) : v[2 * i + 1];
    w[i] = pack2(a, b);
  }
  char* p = fmt == NT_F16 ? row + 2 * static_cast<int64_t>(k)
                          : row + 4 * static_cast<int64_t>(k & ~31) + 2 * (k & 31) + (lo ? 64 : 0);
  *reinterpret_cast<nt_u32x4*>(p) = w;
}
// Rows first .. first + 31 below `rows` of planes at `base`, entries k0 .. k0 + 31:
// value(i, k, v) gives eight values of row first + i from entry k0 + k on.  A wave.
template <typename Value>
__device__ __forceinline__ void store_lines(char* base, int64_t ld, int first, int rows, int k0,
                                            int fmt, int lane, Value&& value) {
  const bool f16 = fmt == NT_F16;
  // SPLIT: 8 rows of 4 hi and 4 lo pieces; F16: 16 rows of 4 pieces
  const int per = f16 ? 16 : 8, mine = f16 ? lane >> 2 : lane >> 3, k = 8 * (lane & 3);
  const bool lo = !f16 && (lane & 4);
  for (int i = mine; i < 32; i += per) {
    float v[8];
    value(i, k, v);
    if (first + i < rows) put8(base + (first + i) * ld, k0 + k, fmt, lo, v);
  }
}

// N values from k (both multiples of 4, within 16) of an NT_SPLIT plane row, as they
// are stored: read by get, added up by value where they are used.
template <int N>
struct Stored {
  typedef _Float16 h4 __attribute__((ext_vector_type(4)));
  h4 hi[N / 4], lo[N / 4];
  __device__ __forceinline__ void get(const char* row, int k) {
    const h4* p =
        reinterpret_cast<const h4*>(row + 4 * static_cast<int64_t>(k & ~31) + 2 * (k & 31));
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      hi[i] = p[i];
      lo[i] = p[8 + i];
    }
  }
  __device__ __forceinline__ float value(int e) const {
    return static_cast<float>(hi[e / 4][e & 3]) + static_cast<float>(lo[e / 4][e & 3]);
  }
};

__device__ __forceinline__ float bf16_to_f32(uint16_t v) {
  return __builtin_bit_cast(float, static_cast<uint32_t>(v) << 16);
}
__device__ __forceinline__ uint16_t f32_to_bf16(float v) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return static_cast<uint16_t>(u >> 16) | 0x40;
  return static_cast<uint16_t>((u + 0x7FFF + ((u >> 16) & 1)) >> 16);
}

// Sum over the 256 threads of a workgroup, the same in every thread.
__device__ __forceinline__ double block_sum(double v, double* lds4) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) lds4[threadIdx.x >> 6] = v;
  __syncthreads();
  return (lds4[0] + lds4[1]) + (lds4[2] + lds4[3]);
}

// Workgroups (= partial sums) that a matrix's sum of squares takes: runs of 1024.
__host__ __device__ __forceinline__ int norm_parts(int64_t size) {
  const int64_t p = (size + 1023) / 1024;
  return static_cast<int>(p < kNormParts ? p : kNormParts);
}

template <bool BF16>
__device__ __forceinline__ float load_elem(const void* p, int64_t i) {
  if constexpr (BF16) return bf16_to_f32(static_cast<const uint16_t*>(p)[i]);
  else return static_cast<const float*>(p)[i];
}
// Four elements from i; zeros from `end` on.  vec: i a multiple of 4 behind an
// address of whole vectors.
template <bool BF16>
__device__ __forceinline__ void load4(const void* p, int64_t i, int64_t end, bool vec, float* v) {
  if (vec && i + 4 <= end) {
    if constexpr (BF16) {
      const nt_u32x2 w = *reinterpret_cast<const nt_u32x2*>(static_cast<const uint16_t*>(p) + i);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        v[2 * t] = bf16_to_f32(static_cast<uint16_t>(w[t]));
        v[2 * t + 1] = bf16_to_f32(static_cast<uint16_t>(w[t] >> 16));
      }
    } else {
      const nt_f32x4 w = *reinterpret_cast<const nt_f32x4*>(static_cast<const float*>(p) + i);
#pragma unroll
      for (int t = 0; t < 4; ++t) v[t] = w[t];
    }
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t) v[t] = i + t < end ? load_elem<BF16>(p, i + t) : 0.0f;
  }
}
template <bool BF16>
__device__ __forceinline__ bool whole_vectors(const OrthMat& u) {
  return ((reinterpret_cast<uintptr_t>(u.src) | static_cast<uintptr_t>(u.src_ld * (BF16 ? 2 : 4))) &
          (BF16 ? 7 : 15)) == 0;
}

// Partial sums of squares: workgroup p of a matrix takes its rows p, p + parts, ...
// (of a contiguous matrix, runs of 1024 elements, four at a time).  Reads the
// matrices once: 218 MB in 51 us, 4.3 TB/s; 4 us where a launch's latency is all.
template <bool BF16>
__global__ __launch_bounds__(256) void orth_norm_kernel(OrthArgs g) {
  __shared__ double lds4[4];
  const int i = find_position(g.first, g.count, blockIdx.x), local = blockIdx.x - g.first[i];
  const OrthMat& u = g.mat[i].u;
  const int64_t size = static_cast<int64_t>(u.rows) * u.cols;
  const int parts = norm_parts(size);
  if (local >= parts) return;
  const bool vec = whole_vectors<BF16>(u);
  double acc = 0.0;
  if (u.src_ld == u.cols) {
    const int64_t step = static_cast<int64_t>(parts) * 1024;
    for (int64_t base = static_cast<int64_t>(local) * 1024; base < size; base += 4 * step) {
      float v[4][4];
#pragma unroll
      for (int t = 0; t < 4; ++t)
        load4<BF16>(u.src, base + t * step + threadIdx.x * 4, size, vec, v[t]);
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc += static_cast<double>(v[t][e]) * v[t][e];
    }
  } else {
    for (int r = local; r < u.rows; r += parts)
      for (int c = 4 * threadIdx.x; c < u.cols; c += 1024) {
        float v[4];
        load4<BF16>(u.src, r * u.src_ld + c, r * u.src_ld + u.cols, vec, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc += static_cast<double>(v[e]) * v[e];
      }
  }
  acc = block_sum(acc, lds4);
  if (threadIdx.x == 0) ws_parts(g.ws, i)[local] = acc;
}

// X_0 = G 2^e into both planes, 2^e |G|_F in [2^13, 2^14); the factor
// 1 / (2^e |G|_F) goes to the workspace.  A workgroup takes 64 x 64 entries and
// turns them in LDS, so that both planes are stored by whole lines: 218 MB read and
// 436 MB written in 113 us, 5.8 TB/s.
template <bool BF16>
__global__ __launch_bounds__(256) void orth_convert_kernel(OrthArgs g) {
  __shared__ double lds4[4];
  __shared__ float tile[64][65];
  const int i = find_position(g.first, g.count, blockIdx.x), local = blockIdx.x - g.first[i];
  const OrthMat& u = g.mat[i].u;
  const int gc = (u.cols + 63) / 64;
  if (local >= gc * ((u.rows + 63) / 64)) return;
  // the tile's loads are on their way while the norm is added up
  const int r0 = (local / gc) * 64, c0 = (local % gc) * 64;
  const bool vec = whole_vectors<BF16>(u);
  float v[4][4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int r = r0 + 16 * t + (threadIdx.x >> 4), c = c0 + 4 * (threadIdx.x & 15);
    const int64_t row = (r < u.rows ? r : u.rows - 1) * u.src_ld;
    load4<BF16>(u.src, row + c, r < u.rows ? row + u.cols : row, vec, v[t]);
  }
  const int64_t size = static_cast<int64_t>(u.rows) * u.cols;
  const int parts = norm_parts(size);
  const double* part = ws_parts(g.ws, i);
  double sum = 0.0;
  for (int t = threadIdx.x; t < parts; t += 256) sum += part[t];
  sum = block_sum(sum, lds4);
  const double norm = sqrt(sum);
  int e = 0;
  const double f = frexp(norm, &e);  // norm = f 2^e
  const bool usable = norm > 0.0 && norm <= 1.7976931348623157e308;
  if (local == 0 && threadIdx.x == 0)
    ws_scale(g.ws)[i] = usable ? static_cast<float>(1.0 / (f * 16384.0))
                               : (norm == 0.0 ? 0.0f : __builtin_nanf(""));
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int k = 0; k < 4; ++k)
      tile[16 * t + (threadIdx.x >> 4)][4 * (threadIdx.x & 15) + k] =
          usable ? __builtin_ldexpf(v[t][k], 14 - e) : 0.0f;
  __syncthreads();
  const bool tall = mat_tall(u);
  const Planes q = mat_planes(g.ws, g.mat[i]);
  // G's rows and those of G': X is the one with m rows.  Wave w: quarter w of the tile.
  const int lane = threadIdx.x & 63, i0 = (threadIdx.x >> 7) * 32;
  const int j0 = (threadIdx.x >> 6 & 1) * 32;
  const int x_fmt = BF16 ? NT_F16 : NT_SPLIT;  // exact in one plane
  const int fmt1 = tall ? NT_SPLIT : x_fmt, fmt2 = tall ? x_fmt : NT_SPLIT;
  store_lines(tall ? q.xt[0] : q.x, row_bytes(u.cols, fmt1), r0 + i0, u.rows, c0 + j0, fmt1, lane,
              [&](int i, int k, float* v) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = tile[i0 + i][j0 + k + e];
              });
  store_lines(tall ? q.x : q.xt[0], row_bytes(u.rows, fmt2), c0 + i0, u.cols, r0 + j0, fmt2, lane,
              [&](int i, int k, float* v) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = tile[j0 + k + e][i0 + i];
              });
}

// One product for every matrix of the call.
//   GRAM   A = X X' (lower tiles, stored to both sides)
//   POLY   P = a I + b A + c A A (same)
//   APPLY  X <- P X, into X and the other X' buffer
//   LAST   the same into the caller's matrix

// A product's operands, and where a matrix's tile `local` lies.
template <int KIND>
struct Product {
  static constexpr bool SYM = KIND == ORTH_GRAM || KIND == ORTH_POLY;
  char *x, *a, *p;           // planes
  char *xt, *xt_next;        // X' that is read, and the other one
  const char *left, *right;  // operands
  int im, m, n, R, C, K;     // R x C results, K summed over
  void* dst;
  const float* base;
  int64_t dst_ld;
  float keep, rate;
  __device__ __forceinline__ Product(const OrthArgs& g, int mat) {
    const OrthMat& u = g.mat[mat].u;
    dst = u.dst;
    base = u.base;
    dst_ld = u.dst_ld;
    keep = u.keep;
    rate = u.rate;
    im = mat;
    m = mat_m(u);
    n = mat_n(u);
    const Planes q = mat_planes(g.ws, g.mat[mat]);
    x = q.x;
    a = q.a;
    p = q.p;
    // (arithmetic, not a choice between two members: that would put this in memory)
    const int64_t apart = q.xt[1] - q.xt[0];
    xt = q.xt[0] + (g.parity ? apart : 0);
    xt_next = q.xt[0] + (g.parity ? 0 : apart);
    const bool swap = KIND == ORTH_LAST && !mat_tall(u);  // a wide matrix's rows are columns here
    R = SYM ? m : (swap ? n : m);
    C = SYM ? m : (swap ? m : n);
    K = KIND == ORTH_GRAM ? n : m;
    left = KIND == ORTH_GRAM ? x : KIND == ORTH_POLY ? a : swap ? xt : p;
    right = KIND == ORTH_GRAM ? x : KIND == ORTH_POLY ? a : swap ? p : xt;
  }
  template <int B>
  __device__ __forceinline__ int tiles() const {
    const int tr = (R + B - 1) / B, tc = (C + B - 1) / B;
    return SYM ? tr * (tr + 1) / 2 : tr * tc;
  }
  // `id`: of the matrix's tiles of B x B
  template <int B>
  __device__ __forceinline__ void tile(int id, int* ti, int* tj) const {
    // bands of four tile rows, column by column: a band's operands stay in L2
    constexpr int BAND = 4;
    const int tr = (R + B - 1) / B, tc = (C + B - 1) / B;
    if (SYM) {
      // a band has the columns left of its first row, then a triangle
      int i = static_cast<int>((sqrtf(8.0f * id + 1.0f) - 1.0f) * 0.5f);
      while (i * (i + 1) / 2 > id) --i;
      while ((i + 1) * (i + 2) / 2 <= id) ++i;
      const int top = i / BAND * BAND, rows = tr - top < BAND ? tr - top : BAND;
      int at = id - top * (top + 1) / 2;
      if (at < rows * top) {
        *ti = top + at % rows;
        *tj = at / rows;
      } else {
        at -= rows * top;
        const int r = at < 1 ? 0 : at < 3 ? 1 : at < 6 ? 2 : 3;
        *ti = top + r;
        *tj = top + at - r * (r + 1) / 2;
      }
    } else {
      const int band = id / (BAND * tc), rows = tr - band * BAND < BAND ? tr - band * BAND : BAND;
      const int at = id - band * BAND * tc;
      *ti = band * BAND + at % rows;
      *tj = at / rows;
    }
  }
  // What a sum is multiplied with: the planes' scales, and POLY's c.
  __device__ __forceinline__ float factor(const OrthArgs& g) const {
    const float in = g.in_scaled ? 1.0f / orth_scale(n) : ws_scale(g.ws)[im];  // on one X
    return KIND == ORTH_GRAM    ? in * in * kScaleA
           : KIND == ORTH_POLY  ? g.c / kScaleA
           : KIND == ORTH_APPLY ? in / kScaleA * orth_scale(n)
                                : in / kScaleA;
  }
  // Planes that a result goes to: rows C with entries R, and rows R with entries C.
  __device__ __forceinline__ char* turned() const {
    return KIND == ORTH_GRAM ? a : KIND == ORTH_POLY ? p : xt_next;
  }
  __device__ __forceinline__ char* straight() const {
    return KIND == ORTH_GRAM ? a : KIND == ORTH_POLY ? p : x;
  }
  // POLY: rows r .. r + N - 1 of column c of A.
  template <int N>
  __device__ __forceinline__ void load_a(int r, int c, Stored<N>* t) const {
    // A(r, c) = A(c, r), consecutive
    if (KIND == ORTH_POLY) t->get(a + (c < C ? c : C - 1) * row_bytes(m, NT_SPLIT), r);
  }
  // Rows r .. r + N - 1 of column c: POLY's other terms (t of load_a), zeros in
  // the planes' padding.
  template <int N>
  __device__ __forceinline__ void finish(const OrthArgs& g, int r, int c, const Stored<N>& t,
                                         float* v) const {
    if constexpr (KIND == ORTH_POLY) {
#pragma unroll
      for (int e = 0; e < N; ++e)
        v[e] += g.b * t.value(e) + (r + e == c ? g.a * kScaleA : 0.0f);
    }
    if constexpr (KIND != ORTH_LAST) {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (r + e >= R || c >= C) v[e] = 0.0f;
    }
  }
  // LAST: N consecutive entries from `r` of the caller's row `c`.
  template <int N>
  __device__ __forceinline__ void out(const OrthArgs& g, int r, int c, const float* v) const {
    if (c >= C || r >= R) return;
    const int64_t at = c * dst_ld + r;
    const bool whole = r + N <= R;
    if (g.bf16) {
      uint16_t* p = static_cast<uint16_t*>(dst) + at;
      if (whole && (reinterpret_cast<uintptr_t>(p) & 7) == 0) {
#pragma unroll
        for (int e = 0; e < N; e += 4)
          *reinterpret_cast<nt_u32x2*>(p + e) =
              nt_u32x2{f32_to_bf16(v[e]) | static_cast<uint32_t>(f32_to_bf16(v[e + 1])) << 16,
                       f32_to_bf16(v[e + 2]) | static_cast<uint32_t>(f32_to_bf16(v[e + 3])) << 16};
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (r + e < R) p[e] = f32_to_bf16(v[e]);
      }
      return;
    }
    float* p = static_cast<float*>(dst) + at;
    const float* from = base + at;  // where there is one
    const uintptr_t low =
        reinterpret_cast<uintptr_t>(p) | (base ? reinterpret_cast<uintptr_t>(from) : 0);
    if (whole && (low & 15) == 0) {
      nt_f32x4 b[N / 4];
      if (base) {
#pragma unroll
        for (int e = 0; e < N / 4; ++e) b[e] = reinterpret_cast<const nt_f32x4*>(from)[e];
      }
#pragma unroll
      for (int e = 0; e < N / 4; ++e) {
        nt_f32x4 o = {v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]};
        if (base) o = keep * b[e] - rate * o;
        reinterpret_cast<nt_f32x4*>(p)[e] = o;
      }
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (r + e < R) p[e] = base ? keep * from[e] - rate * v[e] : v[e];
    }
  }
};

// One tile a workgroup.  A 32 x 32 block of the accumulator has, in lane (h, l),
// column l and rows 8 q + 4 h + t: four consecutive rows, which are four
// consecutive entries of the turned result.
// The matrix instructions bound it: three 4096 x 4096 and one 1000 x 4096 matrix
// (fp32) take GRAM and POLY 587 us each (418 tiles of 256, two turns of the CUs, the
// second 63% full; matrix units busy 57%), APPLY 1029 us (1226 TFLOP/s of matrix
// work, 65%).
// (LDS of exactly S::LDS_BYTES: one more variable beside the 128 KB of the 256 x
// 256 tile cost it 45 us of 335.)
template <class S, int KIND, int F>
__global__ __launch_bounds__(S::NT, 2) void orth_product_kernel(OrthArgs g) {
#if defined(__HIP_DEVICE_COMPILE__)  // buffer resources: no host form
  constexpr int TURN = 36;  // floats of an LDS row of the turned block
  typedef Product<KIND> Prod;
  static_assert(S::BM == S::BN, "symmetric tiles");
  static_assert(S::LDS_BYTES >= S::WM * S::WN * 32 * TURN * 4, "room to turn blocks");
  constexpr int PF = F == NT_SPLIT_B0 ? static_cast<int>(NT_SPLIT) : F;
  __shared__ __attribute__((aligned(16))) char lds[S::LDS_BYTES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = lane >> 5;
  const int pos = find_position(g.first, g.count, blockIdx.x);
  const Prod p(g, g.order[pos]);
  const int local = blockIdx.x - g.first[pos], tiles = g.cut[pos];
  if (local >= tiles) return;
  int ti, tj;
  p.template tile<S::BM>(xcd_index(local, tiles), &ti, &tj);
  const int r0 = ti * S::BM, c0 = tj * S::BN;
  const int64_t ld = row_bytes(p.K, PF);
  NtRows<S::NT, S::BM> ra;
  NtRows<S::NT, S::BN> rb;
  ra.init(p.left, ld, ld * p.R, r0, p.R, tid);
  rb.init(p.right, ld, ld * p.C, c0, p.C, tid);
  typename NtAcc<F>::type acc[S::MI][S::NJ];
#pragma unroll
  for (int i = 0; i < S::MI; ++i)
#pragma unroll
    for (int j = 0; j < S::NJ; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
  nt_tile<S, F>(ra, rb, row_blocks(p.K, PF), lds, tid, acc);

  // Block by block through LDS of the wave's own, turned[column][row]: a lane's
  // four consecutive rows lie together, and both the columns (the turned
  // result) and the rows (the straight one) are read 16 entries a lane.  One
  // copy of this code for all blocks (unrolled over the accumulators it is 30 KB).
  const float f = p.factor(g);
  const int rw = r0 + (wave / S::WN) * 32 * S::MI, cw = c0 + (wave % S::WN) * 32 * S::NJ;
  float* turn = reinterpret_cast<float*>(lds) + wave * 32 * TURN;
  const int64_t ld1 = row_bytes(p.R, NT_SPLIT), ld2 = row_bytes(p.C, NT_SPLIT);
  const int line = lane >> 1, k16 = 16 * (lane & 1);
  nt_barrier();  // the stages are read: LDS is free
#pragma nounroll
  for (int block = 0; block < S::MI * S::NJ; ++block) {
    const int rb0 = rw + 32 * (block / S::NJ), cb0 = cw + 32 * (block % S::NJ);
    if (rb0 >= pad64(p.R) || cb0 >= pad64(p.C)) continue;  // uniform over the wave
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
      for (int j = 0; j < S::NJ; ++j)
        if (block == i * S::NJ + j) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<nt_f32x4*>(turn + (lane & 31) * TURN + 8 * e + 4 * h) =
                nt_f32x4{acc[i][j][4 * e] * f, acc[i][j][4 * e + 1] * f,
                         acc[i][j][4 * e + 2] * f, acc[i][j][4 * e + 3] * f};
        }
    nt_wave_sync();
    if constexpr (KIND == ORTH_LAST) {
      // eight lanes store the 32 entries of a caller's row
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = 8 * e + (lane >> 3), k = 4 * (lane & 7);
        const nt_f32x4 t = *reinterpret_cast<const nt_f32x4*>(turn + row * TURN + k);
        const float v[4] = {t[0], t[1], t[2], t[3]};
        p.template out<4>(g, rb0 + k, cb0 + row, v);
      }
    } else {
      if constexpr (KIND == ORTH_POLY) {
        float v[16];
        float* mine = turn + line * TURN + k16;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const nt_f32x4 t = *reinterpret_cast<const nt_f32x4*>(mine + 4 * e);
#pragma unroll
          for (int o = 0; o < 4; ++o) v[4 * e + o] = t[o];
        }
        Stored<16> t;
        p.load_a(rb0 + k16, cb0 + line, &t);
        p.finish(g, rb0 + k16, cb0 + line, t, v);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          *reinterpret_cast<nt_f32x4*>(mine + 4 * e) =
              nt_f32x4{v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]};
        nt_wave_sync();
      }
      // turned: rows c, entries r (zeros in the padding)
      store_lines(p.turned(), ld1, cb0, p.C, rb0, NT_SPLIT, lane, [&](int i, int k, float* v) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const nt_f32x4 t = *reinterpret_cast<const nt_f32x4*>(turn + i * TURN + k + 4 * e);
#pragma unroll
          for (int o = 0; o < 4; ++o) v[4 * e + o] = rb0 + k + 4 * e + o < p.R ? t[o] : 0.0f;
        }
      });
      // straight: rows r, entries c (a diagonal tile holds both already)
      if (!Prod::SYM || ti != tj)
        store_lines(p.straight(), ld2, rb0, p.R, cb0, NT_SPLIT, lane, [&](int i, int k, float* v) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            v[e] = cb0 + k + e < p.C ? turn[(k + e) * TURN + i] : 0.0f;
        });
    }
    nt_wave_sync();
  }
#endif
}

// Small products, where a launch's latency is all there is: 32 x 32 results a
// workgroup, K dealt to its waves block by block.  A wave streams its blocks
// through LDS of its own (RING of them), into registers, and waits for no other
// wave until the sums meet.  The small planes' products have accumulators of
// their own (see NtShape::EXACT) and lo lo is kept: five steps of 10 x 256 matrices
// are off by 6.3e-7 of the result, 9.0e-7 in the worst of 24.
//   RING 2 (64 KB): up to two workgroups a CU, all there at once;
//   RING 1 (32 KB): more of them, five a CU cover for each other.
// (Calls of 17 launches: 512 x 512 106 us with RING 2, 113 with 1; 16 of 256 x 256
// 183 and 161; 536 workgroups, two turns of RING 2, 147 and 138.  RING 4: 6 us more
// a call at 64 x 64, 4 more at 256 x 8192, where what a CU can take from the L2 is
// the bound.  Eight waves, K in eight: 8 us more at 64 x 64, 14 less at 256 x 8192.)
constexpr int SMALL_WAVES = 4;
template <int KIND, int F, int RING>
__global__ __launch_bounds__(64 * SMALL_WAVES) void orth_small_kernel(OrthArgs g) {
#if defined(__HIP_DEVICE_COMPILE__)  // buffer resources: no host form
  constexpr int STAGE = 64 * NT_BLOCK, TURN = 33;
  constexpr int PF = F == NT_SPLIT_B0 ? static_cast<int>(NT_SPLIT) : F;
  typedef Product<KIND> Prod;
  __shared__ __attribute__((aligned(16))) char lds[SMALL_WAVES * RING * STAGE];
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);  // scalar addresses below
  const int pos = find_position(g.first, g.count, blockIdx.x);
  const Prod p(g, g.order[pos]);
  const int local = blockIdx.x - g.first[pos];
  int ti, tj;
  if (g.rest) {  // sixteenths of the tiles of 128 from cut[pos] on
    const int from = g.cut[pos], parts = (p.template tiles<128>() - from) * 16;
    if (local >= parts) return;
    const int id = xcd_index(local, parts);
    p.template tile<128>(from + id / 16, &ti, &tj);
    ti = 4 * ti + (id & 3);
    tj = 4 * tj + (id >> 2 & 3);
    if (ti * 32 >= p.R || tj * 32 >= p.C || (Prod::SYM && ti < tj)) return;
  } else {
    const int tiles = p.template tiles<32>();
    if (local >= tiles) return;
    p.template tile<32>(xcd_index(local, tiles), &ti, &tj);
  }
  const int r0 = ti * 32, c0 = tj * 32;
  const int64_t ld = row_bytes(p.K, PF);
  const int blocks = row_blocks(p.K, PF);
  NtRows<64, 32> ra, rb;
  ra.init(p.left, ld, ld * p.R, r0, p.R, lane);
  rb.init(p.right, ld, ld * p.C, c0, p.C, lane);
  char* ring = lds + wave * RING * STAGE;
  auto issue = [&](int i) {  // the wave's block i
    const int k = wave + SMALL_WAVES * i;
    char* t = ring + (i % RING) * STAGE;
    const int at = (k < blocks ? k : blocks - 1) * NT_BLOCK;
    ra.issue(t, at, lane);
    rb.issue(t + STAGE / 2, at, lane);
  };
  // the wave finishes rows 8 w + 4 h .. + 3 of column (lane & 31)
  const int r = r0 + 8 * wave + 4 * h, c = c0 + (lane & 31);
  Stored<4> terms;
  p.load_a(r, c, &terms);         // on its way during the products
  asm volatile("" ::: "memory");  // ahead of the blocks, whose waits count what follows
  nt_f32x16 acc, cross;
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = cross[e] = 0.0f;
  constexpr int PER = NtRows<64, 32>::P * 2;
  for (int i = 0; i < RING; ++i) issue(i);
  for (int i = 0; wave + SMALL_WAVES * i < blocks; ++i) {
    nt_wait_vm<(RING - 1) * PER>();
    const char* ta = ring + (i % RING) * STAGE;
    const char* tb = ta + STAGE / 2;
    nt_u32x4 fa[4], fb[4];
    const int row = lane & 31;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      fa[c] = nt_read(ta, row, 2 * c + h);
      fb[c] = nt_read(tb, row, 2 * c + h);
    }
    // the stage is in registers: refill it
    __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4));  // lgkmcnt(0)
    asm volatile("" ::: "memory");
    issue(i + RING);
    if constexpr (PF == NT_SPLIT) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        acc = nt_mfma<F>(fa[k], fb[k], acc);
        cross = nt_mfma<F>(fa[2 + k], fb[k], cross);
        if constexpr (F == NT_SPLIT) {
          cross = nt_mfma<F>(fa[k], fb[2 + k], cross);
          cross = nt_mfma<F>(fa[2 + k], fb[2 + k], cross);
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) acc = nt_mfma<F>(fa[k], fb[k], acc);
    }
  }
  nt_wait_vm<0>();
  __syncthreads();  // every wave is through with LDS: now the four sums
  float* sums = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int e = 0; e < 16; ++e) sums[(wave * 16 + e) * 64 + lane] = acc[e] + cross[e];
  __syncthreads();
  const float f = p.factor(g);
  float v[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < SMALL_WAVES; ++w) s += sums[(w * 16 + 4 * wave + t) * 64 + lane];
    v[t] = s * f;
  }
  p.finish(g, r, c, terms, v);
  // Through LDS, turned[column][row], so that eight lanes store a whole line: of
  // the caller's row, or 32 entries of a plane's.
  float* turn = sums + SMALL_WAVES * 16 * 64;
#pragma unroll
  for (int t = 0; t < 4; ++t) turn[(lane & 31) * TURN + 8 * wave + 4 * h + t] = v[t];
  __syncthreads();
  const int i = 8 * wave + (lane >> 3);
  if constexpr (KIND == ORTH_LAST) {
    const int k = 4 * (lane & 7);
#pragma unroll
    for (int t = 0; t < 4; ++t) v[t] = turn[i * TURN + k + t];
    p.template out<4>(g, r0 + k, c0 + i, v);
  } else {
    const int k = 8 * (lane & 3);
    const bool lo = lane & 4;
    // rows are padded to 64 entries: the last tile zeros what no tile covers
    const float none[8] = {};
    float w[8];
    if (c0 + i < p.C) {
      char* row = p.turned() + (c0 + i) * row_bytes(p.R, NT_SPLIT);
#pragma unroll
      for (int t = 0; t < 8; ++t) w[t] = turn[i * TURN + k + t];
      put8(row, r0 + k, NT_SPLIT, lo, w);
      if (r0 + 32 >= p.R && r0 + 32 < pad64(p.R)) put8(row, r0 + 32 + k, NT_SPLIT, lo, none);
    }
    if (Prod::SYM && ti == tj) return;
    if (r0 + i < p.R) {
      char* row = p.straight() + (r0 + i) * row_bytes(p.C, NT_SPLIT);
#pragma unroll
      for (int t = 0; t < 8; ++t) w[t] = turn[(k + t) * TURN + i];
      put8(row, c0 + k, NT_SPLIT, lo, w);
      if (c0 + 32 >= p.C && c0 + 32 < pad64(p.C)) put8(row, c0 + 32 + k, NT_SPLIT, lo, none);
    }
  }
#endif
}

// ------------------------------------------------------------------ launches

int tiles_of(const OrthMat& u, int kind, int bt) {
  const int tm = (mat_m(u) + bt - 1) / bt, tn = (mat_n(u) + bt - 1) / bt;
  return kind == ORTH_GRAM || kind == ORTH_POLY ? tm * (tm + 1) / 2 : tm * tn;
}
int blocks_of(const OrthMat& u, int kind, int fmt) {
  return row_blocks(kind == ORTH_GRAM ? mat_n(u) : mat_m(u), fmt);
}

// first[] for `work(i)` workgroups per matrix, matrices in order[]; the grid, or
// -1 where there is none of that size.
template <typename Work>
int layout_grid(OrthArgs* g, Work&& work) {
  int64_t at = 0;
  for (int i = 0; i < g->count; ++i) {
    g->first[i] = static_cast<int>(at);
    at += (static_cast<int64_t>(work(g->order[i])) + 7) / 8 * 8;
    if (at > 0x7FFFFFF0) return -1;
  }
  g->first[g->count] = static_cast<int>(at);
  return static_cast<int>(at);
}
void matrices_in_order(OrthArgs* g) {
  for (int i = 0; i < g->count; ++i) g->order[i] = i;
}

constexpr int kCus = 256;

template <class S, int KIND, int F>
hipError_t launch_product_shape(OrthArgs& g, hipStream_t s, int64_t most) {
  int at = 0;
  const int grid = layout_grid(&g, [&](int i) {
    const int64_t tiles = tiles_of(g.mat[i].u, KIND, S::BM);
    g.cut[at] = static_cast<int>(tiles < most ? tiles : most);
    most -= g.cut[at];
    return g.cut[at++];
  });
  if (grid < 0) return hipErrorInvalidValue;
  hipLaunchKernelGGL((orth_product_kernel<S, KIND, F>), dim3(grid), dim3(S::NT), 0, s, g);
  return hipGetLastError();
}

template <int KIND, int F>
hipError_t launch_product_small(OrthArgs& g, hipStream_t s, int rest) {
  int at = 0;
  g.rest = rest;
  const int grid = layout_grid(&g, [&](int i) {
    if (!rest) return tiles_of(g.mat[i].u, KIND, 32);
    return (tiles_of(g.mat[i].u, KIND, 128) - g.cut[at++]) * 16;
  });
  if (grid < 0) return hipErrorInvalidValue;
  const dim3 wg(64 * SMALL_WAVES);
  if (grid <= 2 * kCus)
    hipLaunchKernelGGL((orth_small_kernel<KIND, F, 2>), dim3(grid), wg, 0, s, g);
  else
    hipLaunchKernelGGL((orth_small_kernel<KIND, F, 1>), dim3(grid), wg, 0, s, g);
  return hipGetLastError();
}

// A product's time in us with tiles of 32, 128 or 256, from what the kernels take
// on this card (NT_SPLIT; a K block of 32 values; the first GRAM and APPLY of bf16
// matrices go by the same figures: with every other tile forced for either, calls
// of 256 x 256 to the 4096-wide ones below were at best 0.3% faster):
//   32    4 us, and 2400 blocks a us over all CUs
//   128   9 us, and a block 0.75 us while no CU has two tiles, else 1.45 us for
//         512 at a time
//   256   20 us, and a block 2.1 us while half of the CUs have a tile, else 2.45 us
//         for 256 at a time
// and, with more tiles than fit at once, some of a tile for the CUs that run dry.
// Where a few tiles of 128 are left after full turns of one or two to a CU, they
// are done in tiles of 32 by a second launch, 9 us and 1870 blocks a us: one matrix
// of 4096 (two turns of 256 and 16 left) went from 4329 to 3883 us, 2900 from 2170 to
// 1919, two of 2048 from 1432 to 1338; eight of 1024 (32 blocks of K, 32 tiles left)
// would have gone from 886 to 1000.
// Whole calls, fp32 (32 / 128 / 256, us): 512: 107 / 344 / 753, 1280: 357 / 583 /
// 1329, 2048: 1087 / 847 / 1908, 3328: 4245 / 2445 / 2932, 4096: 7895 / 4422 / 3984;
// three 4096 x 4096 and 1000 x 4096: 24179 / 11673 / 10962.  (Tiles cut along K,
// their sums joined by the last workgroup to arrive, were slower everywhere but
// there by 3%: the sums' way through memory and the caches' write-back.)
// `most`: of the tiles of 128, those done as such; the others are done in tiles of 32.
int best_tile(const OrthArgs& g, int kind, int fmt, int64_t* most) {
  int best = 0;
  double best_t = 0.0;
  for (int bt : {32, 128, 256}) {
    double tiles = 0.0, blocks = 0.0, longest = 0.0;
    for (int i = 0; i < g.count; ++i) {
      const double t = tiles_of(g.mat[i].u, kind, bt), k = blocks_of(g.mat[i].u, kind, fmt);
      tiles += t;
      blocks += t * k;
      longest = std::fmax(longest, k);
    }
    double us;
    if (bt == 32)
      us = 4.0 + blocks / 2400.0;
    else if (bt == 128)
      us = 9.0 + (tiles <= 256.0 ? 0.75 * longest : 1.45 * (blocks / 512.0 + 0.3 * longest));
    else
      us = 20.0 + (tiles <= 144.0   ? 2.1 * longest
                   : tiles <= 256.0 ? 2.45 * longest
                                    : 2.45 * (blocks / 256.0 + 0.3 * longest));
    if (best == 0 || us < best_t) {
      best = bt;
      best_t = us;
      *most = INT64_MAX;
    }
    if (bt == 128 && tiles > 256.0) {
      const double turns = std::floor(tiles / 256.0), rest = tiles - 256.0 * turns;
      double left = rest, over = 0.0;  // blocks of the last tiles
      for (int i = g.count - 1; i >= 0 && left > 0.0; --i) {
        const int at = g.order[i];
        const double n = std::fmin(left, tiles_of(g.mat[at].u, kind, bt));
        left -= n;
        over += n * blocks_of(g.mat[at].u, kind, fmt);
      }
      us = 9.0 + 0.725 * (blocks - over) / 256.0;
      if (rest > 0.0) us += 9.0 + 16.0 * over / 1870.0;
      if (std::fmod(turns, 2.0) != 0.0) us += 0.025 * longest;
      if (us < best_t) {
        best = bt;
        best_t = us;
        *most = rest > 0.0 ? static_cast<int64_t>(256.0 * turns) : INT64_MAX;
      }
    }
  }
  return best;
}

template <int KIND, int F>
hipError_t launch_product(OrthArgs& g, hipStream_t s) {
  constexpr int PF = F == NT_SPLIT_B0 ? static_cast<int>(NT_SPLIT) : F;
  // longest K first: the short tiles fill the gaps at the end
  matrices_in_order(&g);
  for (int i = 1; i < g.count; ++i)
    for (int j = i; j > 0 && blocks_of(g.mat[g.order[j]].u, KIND, PF) >
                                 blocks_of(g.mat[g.order[j - 1]].u, KIND, PF); --j) {
      const int t = g.order[j];
      g.order[j] = g.order[j - 1];
      g.order[j - 1] = t;
    }
  int64_t most;
  const int tile = best_tile(g, KIND, PF, &most);
  if (tile == 32) return launch_product_small<KIND, F>(g, s, 0);
  if (tile == 256) return launch_product_shape<OrthL, KIND, F>(g, s, most);
  const hipError_t e = launch_product_shape<OrthM, KIND, F>(g, s, most);
  return e != hipSuccess || most == INT64_MAX ? e : launch_product_small<KIND, F>(g, s, 1);
}

}  // namespace

bool orth_coeffs_ok(const OrthCoeffs& c) {
  if (c.steps < 1 || c.steps > ORTH_MAX_STEPS) return false;
  double top = 1.0;  // singular values lie in [0, top]
  for (int t = 0; t < c.steps; ++t) {
    const double a = c.a[t], b = c.b[t], d = c.c[t], u = top * top;
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(d)) return false;
    // of v = s^2 in [0, u]: p(v) = a + b v + d v^2, and s p whose derivative is
    // a + 3 b v + 5 d v^2; the largest are at an end or where a derivative is zero
    auto p = [&](double v) { return std::fabs(a + (b + d * v) * v); };
    double most = std::fmax(p(0.0), p(u)), next = top * p(u);
    auto inside = [&](double v) { return v > 0.0 && v < u; };
    const double flat = -b / (2.0 * d);
    if (inside(flat)) most = std::fmax(most, p(flat));
    const double disc = 9.0 * b * b - 20.0 * a * d;
    if (disc >= 0.0) {
      const double q = -0.5 * (3.0 * b + std::copysign(std::sqrt(disc), b));
      for (double v : {q / (5.0 * d), a / q})
        if (inside(v)) next = std::fmax(next, std::sqrt(v) * p(v));
    }
    if (!(most <= kMaxPoly) || !(next <= kMaxSigma)) return false;
    top = next * 1.01;  // roundings
  }
  // |X_t|_F^2 is the sum over the singular values s of X_0, whose squares add up to
  // 1, of s^2 times the square of the product of p's that it has met: no less than
  // the least such product.  Where its sign changes from one s to the next it is 0
  // between them.
  uint32_t negative = 0;
  for (int i = 0; i <= 256; ++i) {
    double s = (i / 256.0) * (i / 256.0), left = 1.0;
    uint32_t signs = 0;
    for (int t = 0; t + 1 < c.steps; ++t) {
      const double p = c.a[t] + (c.b[t] + c.c[t] * s * s) * s * s;
      left *= p;
      s *= p;
      signs |= (left < 0.0 ? 1u : 0u) << t;
      if (std::fabs(left) < kMinNorm) return false;
    }
    if (i > 0 && signs != negative) return false;
    negative = signs;
  }
  return true;
}

int64_t orth_workspace(const OrthMat* mats, int count) {
  int64_t at = kHeadBytes;
  for (int i = 0; i < count; ++i) at += mat_bytes(mats[i]);
  return at;
}

hipError_t launch_orthogonalize(const OrthMat* mats, int count, bool bf16, const OrthCoeffs& c,
                                void* ws, hipStream_t s, bool norms_done) {
  OrthArgs g{};
  g.count = count;
  g.ws = static_cast<char*>(ws);
  g.bf16 = bf16;
  int64_t at = kHeadBytes;
  for (int i = 0; i < count; ++i) {
    g.mat[i].u = mats[i];
    g.mat[i].at = at;
    at += mat_bytes(mats[i]);
  }
  hipError_t e = hipSuccess;
  matrices_in_order(&g);
  if (!norms_done) {
    const int grid = layout_grid(&g, [&](int i) {
      return norm_parts(static_cast<int64_t>(mats[i].rows) * mats[i].cols);
    });
    if (bf16) hipLaunchKernelGGL((orth_norm_kernel<true>), dim3(grid), dim3(256), 0, s, g);
    else hipLaunchKernelGGL((orth_norm_kernel<false>), dim3(grid), dim3(256), 0, s, g);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  {
    const int grid = layout_grid(&g, [&](int i) {
      return ((mats[i].rows + 63) / 64) * ((mats[i].cols + 63) / 64);
    });
    if (grid < 0) return hipErrorInvalidValue;
    if (bf16) hipLaunchKernelGGL((orth_convert_kernel<true>), dim3(grid), dim3(256), 0, s, g);
    else hipLaunchKernelGGL((orth_convert_kernel<false>), dim3(grid), dim3(256), 0, s, g);
    e = hipGetLastError();
  }
  for (int t = 0; t < c.steps && e == hipSuccess; ++t) {
    g.a = c.a[t];
    g.b = c.b[t];
    g.c = c.c[t];
    g.in_scaled = t > 0;
    g.parity = t & 1;
    // X_0 of a bf16 matrix is exact in one plane: its Gram product takes one
    // instruction, its product with P (hi, lo) two.
    const bool one_plane = t == 0 && bf16;
    e = one_plane ? launch_product<ORTH_GRAM, NT_F16>(g, s)
                  : launch_product<ORTH_GRAM, NT_SPLIT>(g, s);
    if (e != hipSuccess) break;
    e = launch_product<ORTH_POLY, NT_SPLIT>(g, s);
    if (e != hipSuccess) break;
    if (t + 1 == c.steps)
      e = launch_product<ORTH_LAST, NT_SPLIT>(g, s);
    else
      e = one_plane ? launch_product<ORTH_APPLY, NT_SPLIT_B0>(g, s)
                    : launch_product<ORTH_APPLY, NT_SPLIT>(g, s);
  }
  return e;
}

// ------------------------------------------------------------------ server's step
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

struct ServerGrid {
  int first[SERVER_MAX_SEGS + 1];
};

constexpr int kServerChunk = 1024;  // elements of a workgroup's pass

// The balanced tree of oscars_aggregate over P leaves w_k r_k (+0 from K on).
template <int P>
__device__ __forceinline__ f32x4 server_tree(const ServerArgs& a, const float* r, int k) {
  if constexpr (P == 1) {
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (k < a.K)
      v = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(r + k * a.n)) * a.w[k];
    return v;
  } else {
    return server_tree<P / 2>(a, r, k) + server_tree<P / 2>(a, r, k + P / 2);
  }
}

// Average, momentum and update of every element, one pass: K + 2 reads and two
// writes of the model, the momentum and, of matrix entries, u (with their sum of
// squares for the orthogonalisation), of everything else the new value.
template <int P>
__global__ __launch_bounds__(256) void server_pass_kernel(ServerArgs a, ServerGrid grid, char* ws) {
  __shared__ double lds4[4];
  int s = 0;
  while (s + 1 < a.n_segs && static_cast<int>(blockIdx.x) >= grid.first[s + 1]) ++s;
  const int local = blockIdx.x - grid.first[s];
  const int parts = grid.first[s + 1] - grid.first[s];
  const int mat = a.mat[s];
  const int64_t mat_end = a.start[s] + (mat >= 0 ? a.size[s] : 0);
  double sum = 0.0;
  for (int64_t i = a.start[s] + static_cast<int64_t>(local) * kServerChunk + threadIdx.x * 4;
       i < a.end[s]; i += static_cast<int64_t>(parts) * kServerChunk) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(a.global + i);
    const f32x4 m0 = *reinterpret_cast<const f32x4*>(a.momentum + i);
    const f32x4 d = x - server_tree<P>(a, a.replicas + i, 0);
    const f32x4 m = a.beta * m0 + d;
    const f32x4 u = a.nesterov ? d + a.beta * m : m;
    *reinterpret_cast<f32x4*>(a.momentum_out + i) = m;
    if (i + 4 <= mat_end) {
      *reinterpret_cast<f32x4*>(a.update + i) = u;
#pragma unroll
      for (int t = 0; t < 4; ++t) sum += static_cast<double>(u[t]) * u[t];
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if (i + t < mat_end) {
          a.update[i + t] = u[t];
          sum += static_cast<double>(u[t]) * u[t];
        } else {
          a.global_out[i + t] = x[t] - a.plain_lr * u[t];
        }
      }
    }
  }
  if (mat < 0) return;
  sum = block_sum(sum, lds4);
  if (threadIdx.x == 0) ws_parts(ws, mat)[local] = sum;
}

template <int P>
hipError_t launch_server_tree(const ServerArgs& a, const ServerGrid& grid, char* ws, int blocks,
                              hipStream_t s) {
  hipLaunchKernelGGL((server_pass_kernel<P>), dim3(blocks), dim3(256), 0, s, a, grid, ws);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_server_pass(const ServerArgs& a, void* orth_ws, hipStream_t s) {
  ServerGrid grid{};
  int at = 0;
  for (int i = 0; i < a.n_segs; ++i) {
    grid.first[i] = at;
    const int64_t len = a.end[i] - a.start[i];
    // a matrix has as many workgroups as the orthogonalisation reads partial sums
    at += a.mat[i] >= 0 ? norm_parts(a.size[i])
                        : static_cast<int>((len + kServerChunk - 1) / kServerChunk);
  }
  grid.first[a.n_segs] = at;
  char* ws = static_cast<char*>(orth_ws);
  if (a.K <= 1) return launch_server_tree<1>(a, grid, ws, at, s);
  if (a.K <= 2) return launch_server_tree<2>(a, grid, ws, at, s);
  if (a.K <= 4) return launch_server_tree<4>(a, grid, ws, at, s);
  if (a.K <= 8) return launch_server_tree<8>(a, grid, ws, at, s);
  if (a.K <= 16) return launch_server_tree<16>(a, grid, ws, at, s);
  if (a.K <= 32) return launch_server_tree<32>(a, grid, ws, at, s);
  return launch_server_tree<64>(a, grid, ws, at, s);
}

}  // namespace oscars
