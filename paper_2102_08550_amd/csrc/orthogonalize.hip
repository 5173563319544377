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
// lo, 22 bits, three matrix instructions a product) for fp32 matrices, and for
// bf16 matrices where a rounding would still be amplified by later steps: a
// step multiplies the small singular directions by up to |a|, so a rounding
// error of 2^-12 before a steps' product of 40 ends at 1e-2 of an entry, many
// bf16 roundings; the last steps run in plain fp16 (one instruction a product).
// X_0 is G times a power of two, exact for bf16; the rest of 1 / |G|_F is a
// factor on the first products, so nothing is rounded before the first step.
// Products sum in fp32 in a fixed order; norms in double.
#include "orthogonalize.h"

#include <cmath>

#include "nt_mma.h"

namespace oscars {
namespace {

typedef NtShape<256, 256, 2, 4, 2> OrthL;
typedef NtShape<128, 128, 2, 2, 2, 1> OrthM;
typedef NtShape<64, 64, 2, 2, 3, 2> OrthS;

enum OrthKind { ORTH_GRAM = 0, ORTH_POLY = 1, ORTH_APPLY = 2, ORTH_LAST = 3 };

constexpr float kScaleA = 128.0f;  // of A and P in their planes
constexpr float kMaxSigma = 16.0f;
constexpr float kMaxPoly = 400.0f;
constexpr int kNormParts = 512;  // partial sums of squares per matrix

struct MatDesc {
  OrthMat u;
  int64_t at;  // of the matrix's planes in the workspace
};

struct OrthArgs {
  MatDesc mat[ORTH_MAX_MATS];
  int first[ORTH_MAX_MATS + 1];  // first workgroup of each matrix (multiples of 8)
  int count;
  char* ws;
  float a, b, c;
  int in_scaled;       // 1: the planes hold X times orth_scale; 0: X_0 (factor in the workspace)
  int parity;          // which of the two X' buffers is read
  int x_fmt, xt_fmt;   // APPLY, convert: formats written
  int p_fmt;           // GRAM: format of A
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
  return (static_cast<int64_t>(rows) * pad64(k) * 4 + 255) / 256 * 256;
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
// Bytes of a row of k values (k padded to 64 with zeros).
__host__ __device__ __forceinline__ int64_t row_bytes(int k, int fmt) {
  return static_cast<int64_t>(pad64(k)) * (fmt == NT_F16 ? 2 : 4);
}

// Power of two on the iterates in their planes.  The rms of an m x n matrix
// with singular values near 1 is 1 / sqrt(n): 16 sqrt(n) brings it to about 16,
// its lo plane to 2^-8; an entry is at most kMaxSigma, 2^15 with the cap.
__host__ __device__ __forceinline__ float orth_scale(int n) {
  int e = 4;
  while (e < 11 && (int64_t{1} << (2 * (e - 4) + 1)) < n) ++e;
  return static_cast<float>(1 << e);
}

// Which matrix a workgroup works for, and its index among the matrix's
// workgroups such that those on one XCD (index mod 8) take neighbouring tiles.
__device__ __forceinline__ int find_mat(const OrthArgs& g, int block, int tiles_of_all,
                                        int* local) {
  int i = 0;
  while (i + 1 < g.count && block >= g.first[i + 1]) ++i;
  *local = block - g.first[i];
  return i;
}
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

// Four values k .. k + 3 (k a multiple of 4) of a plane row.
__device__ __forceinline__ void put4(char* row, int k, int fmt, const float* v) {
  const nt_u32x2 hi = {pack2(v[0], v[1]), pack2(v[2], v[3])};
  if (fmt == NT_F16) {
    *reinterpret_cast<nt_u32x2*>(row + 2 * static_cast<int64_t>(k)) = hi;
  } else {
    char* p = row + 4 * static_cast<int64_t>(k & ~31) + 2 * (k & 31);
    *reinterpret_cast<nt_u32x2*>(p) = hi;
    const nt_u32x2 lo = {pack2(lo_of(v[0]), lo_of(v[1])), pack2(lo_of(v[2]), lo_of(v[3]))};
    *reinterpret_cast<nt_u32x2*>(p + 64) = lo;
  }
}
// Sixteen values from k (a multiple of 16).
__device__ __forceinline__ void put16(char* row, int k, int fmt, const float* v) {
  const nt_u32x4 h0 = {pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
  const nt_u32x4 h1 = {pack2(v[8], v[9]), pack2(v[10], v[11]), pack2(v[12], v[13]),
                       pack2(v[14], v[15])};
  if (fmt == NT_F16) {
    nt_u32x4* p = reinterpret_cast<nt_u32x4*>(row + 2 * static_cast<int64_t>(k));
    p[0] = h0;
    p[1] = h1;
  } else {
    nt_u32x4* p =
        reinterpret_cast<nt_u32x4*>(row + 4 * static_cast<int64_t>(k & ~31) + 2 * (k & 31));
    p[0] = h0;
    p[1] = h1;
    float l[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) l[i] = lo_of(v[i]);
    p[4] = nt_u32x4{pack2(l[0], l[1]), pack2(l[2], l[3]), pack2(l[4], l[5]), pack2(l[6], l[7])};
    p[5] = nt_u32x4{pack2(l[8], l[9]), pack2(l[10], l[11]), pack2(l[12], l[13]),
                    pack2(l[14], l[15])};
  }
}
__device__ __forceinline__ void get4(const char* row, int k, int fmt, float* v) {
  typedef _Float16 h4 __attribute__((ext_vector_type(4)));
  if (fmt == NT_F16) {
    const h4 h = *reinterpret_cast<const h4*>(row + 2 * static_cast<int64_t>(k));
#pragma unroll
    for (int t = 0; t < 4; ++t) v[t] = static_cast<float>(h[t]);
  } else {
    const char* p = row + 4 * static_cast<int64_t>(k & ~31) + 2 * (k & 31);
    const h4 h = *reinterpret_cast<const h4*>(p), l = *reinterpret_cast<const h4*>(p + 64);
#pragma unroll
    for (int t = 0; t < 4; ++t) v[t] = static_cast<float>(h[t]) + static_cast<float>(l[t]);
  }
}

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

// Workgroups (= partial sums) that a matrix's sum of squares takes.
__host__ __device__ __forceinline__ int norm_parts(int64_t size) {
  const int64_t p = (size + 4095) / 4096;
  return static_cast<int>(p < kNormParts ? p : kNormParts);
}

template <bool BF16>
__device__ __forceinline__ float load_elem(const void* p, int64_t i) {
  if constexpr (BF16) return bf16_to_f32(static_cast<const uint16_t*>(p)[i]);
  else return static_cast<const float*>(p)[i];
}

// Partial sums of squares: workgroup p of a matrix takes its rows p, p + parts, ...
// (of a contiguous matrix, chunks of 1024 elements).
template <bool BF16>
__global__ __launch_bounds__(256) void orth_norm_kernel(OrthArgs g) {
  __shared__ double lds4[4];
  int local;
  const int i = find_mat(g, blockIdx.x, 0, &local);
  const OrthMat& u = g.mat[i].u;
  const int64_t size = static_cast<int64_t>(u.rows) * u.cols;
  const int parts = norm_parts(size);
  if (local >= parts) return;
  double acc = 0.0;
  if (u.src_ld == u.cols) {
    for (int64_t base = static_cast<int64_t>(local) * 1024; base < size;
         base += static_cast<int64_t>(parts) * 1024) {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int64_t e = base + t * 256 + threadIdx.x;
        const double v = e < size ? load_elem<BF16>(u.src, e) : 0.0f;
        acc += v * v;
      }
    }
  } else {
    for (int r = local; r < u.rows; r += parts)
      for (int c = threadIdx.x; c < u.cols; c += 256) {
        const double v = load_elem<BF16>(u.src, r * u.src_ld + c);
        acc += v * v;
      }
  }
  acc = block_sum(acc, lds4);
  if (threadIdx.x == 0) ws_parts(g.ws, i)[local] = acc;
}

// X_0 = G 2^e into both planes, 2^e |G|_F in [2^13, 2^14); the factor
// 1 / (2^e |G|_F) goes to the workspace.  A workgroup takes 64 x 64 entries.
template <bool BF16>
__global__ __launch_bounds__(256) void orth_convert_kernel(OrthArgs g) {
  __shared__ double lds4[4];
  __shared__ float tile[64][65];
  int local;
  const int i = find_mat(g, blockIdx.x, 0, &local);
  const OrthMat& u = g.mat[i].u;
  const int gc = (u.cols + 63) / 64, gr = (u.rows + 63) / 64;
  if (local >= gc * gr) return;
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
  const double mul = usable ? ldexp(1.0, 14 - e) : 0.0;
  if (local == 0 && threadIdx.x == 0)
    ws_scale(g.ws)[i] = usable ? static_cast<float>(1.0 / (f * 16384.0))
                               : (norm == 0.0 ? 0.0f : __builtin_nanf(""));
  const int r0 = (local / gc) * 64, c0 = (local % gc) * 64;
  for (int t = threadIdx.x; t < 4096; t += 256) {
    const int r = t >> 6, c = t & 63;
    float v = 0.0f;
    if (usable && r0 + r < u.rows && c0 + c < u.cols)
      v = static_cast<float>(load_elem<BF16>(u.src, (r0 + r) * u.src_ld + c0 + c) * mul);
    tile[r][c] = v;
  }
  __syncthreads();
  const bool tall = mat_tall(u);
  const Planes q = mat_planes(g.ws, g.mat[i]);
  // "straight": rows of G; "turned": rows of G'.  X is the one with m rows.
  const int row = threadIdx.x >> 2, k = (threadIdx.x & 3) * 16;
  float v[16];
  if (r0 + row < u.rows) {
#pragma unroll
    for (int t = 0; t < 16; ++t) v[t] = tile[row][k + t];
    const int fmt = tall ? g.xt_fmt : g.x_fmt;
    put16((tall ? q.xt[0] : q.x) + (r0 + row) * row_bytes(u.cols, fmt), c0 + k, fmt, v);
  }
  if (c0 + row < u.cols) {
#pragma unroll
    for (int t = 0; t < 16; ++t) v[t] = tile[k + t][row];
    const int fmt = tall ? g.x_fmt : g.xt_fmt;
    put16((tall ? q.x : q.xt[0]) + (c0 + row) * row_bytes(u.rows, fmt), r0 + k, fmt, v);
  }
}

// One product for every matrix of the call.
//   GRAM   A = X X' (lower tiles, stored to both sides)
//   POLY   P = a I + b A + c A A (same)
//   APPLY  X <- P X, into X and the other X' buffer
//   LAST   the same into the caller's matrix
// A 32 x 32 block of the accumulator has, in lane (h, l), column l and rows
// 8 q + 4 h + t: four consecutive rows, which are four consecutive entries of
// the transposed result; the straight one goes through LDS.
template <class S, int KIND, int F>
__global__ __launch_bounds__(S::NT, 2) void orth_product_kernel(OrthArgs g) {
#if defined(__HIP_DEVICE_COMPILE__)  // buffer resources: no host form
  constexpr int TURN = 36;  // floats of an LDS row of the turned block
  constexpr bool SYM = KIND == ORTH_GRAM || KIND == ORTH_POLY;
  static_assert(S::BM == S::BN, "symmetric tiles");
  static_assert(S::LDS_BYTES >= S::WM * S::WN * 32 * TURN * 4, "room to turn blocks");
  __shared__ __attribute__((aligned(16))) char lds[S::LDS_BYTES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = lane >> 5;
  int local;
  const int im = find_mat(g, blockIdx.x, 0, &local);
  const MatDesc& d = g.mat[im];
  const int m = mat_m(d.u), n = mat_n(d.u);
  const bool tall = mat_tall(d.u);
  const Planes q = mat_planes(g.ws, d);
  // rows of the left (R) and right (C) operand
  const bool swap = KIND == ORTH_LAST && !tall;
  const int R = SYM ? m : (swap ? n : m), C = SYM ? m : (swap ? m : n);
  const int tr = (R + S::BM - 1) / S::BM, tc = (C + S::BN - 1) / S::BN;
  const int total = SYM ? tr * (tr + 1) / 2 : tr * tc;
  if (local >= total) return;
  const int id = xcd_index(local, total);
  int ti, tj;
  if (SYM) {
    ti = static_cast<int>((sqrtf(8.0f * id + 1.0f) - 1.0f) * 0.5f);
    while (ti * (ti + 1) / 2 > id) --ti;
    while ((ti + 1) * (ti + 2) / 2 <= id) ++ti;
    tj = id - ti * (ti + 1) / 2;
  } else {
    // bands of four tile rows, column by column: a band's operands stay in L2
    constexpr int BAND = 4;
    const int band = id / (BAND * tc), rows = tr - band * BAND < BAND ? tr - band * BAND : BAND;
    const int at = id - band * BAND * tc;
    ti = band * BAND + at % rows;
    tj = at / rows;
  }
  const int r0 = ti * S::BM, c0 = tj * S::BN;

  const int K = KIND == ORTH_GRAM ? n : m;
  const int64_t ld = row_bytes(K, F == NT_SPLIT_B0 ? NT_SPLIT : F);
  const char* xt = g.parity ? q.xt[1] : q.xt[0];
  const char* left = KIND == ORTH_GRAM ? q.x : KIND == ORTH_POLY ? q.a : (swap ? xt : q.p);
  const char* right = KIND == ORTH_GRAM ? q.x : KIND == ORTH_POLY ? q.a : (swap ? q.p : xt);
  NtRows<S::NT, S::BM> ra;
  NtRows<S::NT, S::BN> rb;
  ra.init(left, ld, ld * R, r0, R, tid);
  rb.init(right, ld, ld * C, c0, C, tid);
  typename NtAcc<F>::type acc[S::MI][S::NJ];
#pragma unroll
  for (int i = 0; i < S::MI; ++i)
#pragma unroll
    for (int j = 0; j < S::NJ; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
  nt_tile<S, F>(ra, rb, 0, static_cast<int>(ld / NT_BLOCK), lds, tid, acc);

  const float x_scale = orth_scale(n);
  const float in = g.in_scaled ? 1.0f / x_scale : ws_scale(g.ws)[im];  // on one X of a product
  const float f_acc = KIND == ORTH_GRAM   ? in * in * kScaleA
                      : KIND == ORTH_POLY ? g.c / kScaleA
                      : KIND == ORTH_APPLY ? in / kScaleA * x_scale
                                           : in / kScaleA;
  const int rw = r0 + (wave / S::WN) * 32 * S::MI, cw = c0 + (wave % S::WN) * 32 * S::NJ;
  float* turn = reinterpret_cast<float*>(lds) + wave * 32 * TURN;
  constexpr int PF = F == NT_SPLIT_B0 ? static_cast<int>(NT_SPLIT) : F;  // POLY: planes of A and P
  nt_barrier();  // the stages are read: LDS is free
#pragma unroll
  for (int i = 0; i < S::MI; ++i)
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) {
      const int rb0 = rw + 32 * i, cb0 = cw + 32 * j, c = cb0 + (lane & 31);
      if (rb0 >= pad64(R) || cb0 >= pad64(C)) continue;  // uniform over the wave
      float v[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] = acc[i][j][e] * f_acc;
      if constexpr (KIND == ORTH_POLY) {
        if (c < C) {
#pragma unroll
          for (int s4 = 0; s4 < 4; ++s4) {
            // A(r, c) = A(c, r), four consecutive
            const int r = rb0 + 8 * s4 + 4 * h;
            float t[4];
            get4(q.a + c * row_bytes(m, PF), r, PF, t);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              v[4 * s4 + e] += g.b * t[e] + (r + e == c ? g.a * kScaleA : 0.0f);
          }
        }
      }
      if constexpr (KIND == ORTH_LAST) {
        if (c < C) {
#pragma unroll
          for (int s4 = 0; s4 < 4; ++s4) {
            const int r = rb0 + 8 * s4 + 4 * h;
            const int64_t at = c * d.u.dst_ld + r;
            if (g.bf16) {
              uint16_t* p = static_cast<uint16_t*>(d.u.dst) + at;
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (r + e < R) p[e] = f32_to_bf16(v[4 * s4 + e]);
            } else {
              float* p = static_cast<float*>(d.u.dst) + at;
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (r + e < R) {
                  float o = v[4 * s4 + e];
                  if (d.u.base) o = d.u.keep * d.u.base[at + e] - d.u.rate * o;
                  p[e] = o;
                }
            }
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int r = rb0 + 8 * (e >> 2) + 4 * h + (e & 3);
          if (r >= R || c >= C) v[e] = 0.0f;  // the planes are padded with zeros
        }
        const int fmt1 = KIND == ORTH_GRAM ? g.p_fmt : KIND == ORTH_POLY ? PF : g.xt_fmt;
        const int fmt2 = KIND == ORTH_APPLY ? g.x_fmt : fmt1;
        char* d1 = KIND == ORTH_GRAM ? q.a : KIND == ORTH_POLY ? q.p : g.parity ? q.xt[0] : q.xt[1];
        char* d2 = KIND == ORTH_APPLY ? q.x : d1;
        // transposed: rows c, entries r
        if (c < C) {
#pragma unroll
          for (int s4 = 0; s4 < 4; ++s4)
            put4(d1 + c * row_bytes(R, fmt1), rb0 + 8 * s4 + 4 * h, fmt1, v + 4 * s4);
        }
        // straight: rows r, entries c (a diagonal tile holds both already)
        if (!SYM || ti != tj) {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            turn[(8 * (e >> 2) + 4 * h + (e & 3)) * TURN + (lane & 31)] = v[e];
          __builtin_amdgcn_wave_barrier();
          const int r = rb0 + (lane >> 1), k = 16 * (lane & 1);
          float w[16];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const nt_f32x4 t =
                *reinterpret_cast<const nt_f32x4*>(turn + (lane >> 1) * TURN + k + 4 * e);
#pragma unroll
            for (int o = 0; o < 4; ++o) w[4 * e + o] = t[o];
          }
          __builtin_amdgcn_wave_barrier();
          if (r < R) put16(d2 + r * row_bytes(C, fmt2), cb0 + k, fmt2, w);
        }
      }
    }
#endif
}

// ------------------------------------------------------------------ launches

int tiles_of(const OrthMat& u, int kind, int bt) {
  const int tm = (mat_m(u) + bt - 1) / bt, tn = (mat_n(u) + bt - 1) / bt;
  return kind == ORTH_GRAM || kind == ORTH_POLY ? tm * (tm + 1) / 2 : tm * tn;
}

// first[] for `work(i)` workgroups per matrix; returns the grid.
template <typename Work>
int layout_grid(OrthArgs* g, Work&& work) {
  int64_t at = 0;
  for (int i = 0; i < g->count; ++i) {
    g->first[i] = static_cast<int>(at);
    at += (work(i) + 7) / 8 * 8;
    if (at > 0x7FFFFFF0) return -1;
  }
  g->first[g->count] = static_cast<int>(at);
  return static_cast<int>(at);
}

template <class S, int KIND, int F>
hipError_t launch_product_shape(OrthArgs& g, hipStream_t s) {
  const int grid = layout_grid(&g, [&](int i) { return tiles_of(g.mat[i].u, KIND, S::BM); });
  if (grid < 0) return hipErrorInvalidValue;
  hipLaunchKernelGGL((orth_product_kernel<S, KIND, F>), dim3(grid), dim3(S::NT), 0, s, g);
  return hipGetLastError();
}

template <int KIND, int F>
hipError_t launch_product(OrthArgs& g, hipStream_t s) {
  int64_t big = 0, mid = 0;
  for (int i = 0; i < g.count; ++i) {
    big += tiles_of(g.mat[i].u, KIND, OrthL::BM);
    mid += tiles_of(g.mat[i].u, KIND, OrthM::BM);
  }
  // the largest tile that still gives most of the 256 CUs a workgroup
  if (big >= 192) return launch_product_shape<OrthL, KIND, F>(g, s);
  if (mid >= 192) return launch_product_shape<OrthM, KIND, F>(g, s);
  return launch_product_shape<OrthS, KIND, F>(g, s);
}

}  // namespace

bool orth_coeffs_ok(const OrthCoeffs& c) {
  if (c.steps < 1 || c.steps > ORTH_MAX_STEPS) return false;
  double top = 1.0;  // singular values lie in [0, top]
  for (int t = 0; t < c.steps; ++t) {
    const double a = c.a[t], b = c.b[t], d = c.c[t];
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(d)) return false;
    double next = 0.0;
    for (int i = 0; i <= 4096; ++i) {
      const double x = top * i / 4096.0, s = x * x;
      const double p = a + b * s + d * s * s;
      if (!(std::fabs(p) <= kMaxPoly)) return false;
      next = std::fmax(next, std::fabs(x * p));
    }
    if (!(next <= kMaxSigma)) return false;
    top = next * 1.01;  // between the samples, and roundings
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
  // Step t in plain fp16 (bf16 matrices): where a rounding in it is amplified
  // by no more than 16 by the end.
  bool plain[ORTH_MAX_STEPS + 1];
  double amp = 1.0;
  plain[c.steps] = bf16;
  for (int t = c.steps - 1; t >= 0; --t) {
    amp *= std::fmax(1.0, std::fabs(static_cast<double>(c.a[t])));
    plain[t] = bf16 && amp <= 16.0;
  }
  auto fmt = [&](int t) { return plain[t] ? static_cast<int>(NT_F16) : static_cast<int>(NT_SPLIT); };
  hipError_t e = hipSuccess;
  if (!norms_done) {
    const int grid = layout_grid(&g, [&](int i) {
      return norm_parts(static_cast<int64_t>(mats[i].rows) * mats[i].cols);
    });
    if (bf16) hipLaunchKernelGGL((orth_norm_kernel<true>), dim3(grid), dim3(256), 0, s, g);
    else hipLaunchKernelGGL((orth_norm_kernel<false>), dim3(grid), dim3(256), 0, s, g);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  // X_0 of a bf16 matrix is exact in one plane: its Gram product takes one
  // instruction, its product with P (hi, lo) two.
  g.x_fmt = bf16 ? static_cast<int>(NT_F16) : static_cast<int>(NT_SPLIT);
  g.xt_fmt = fmt(0);
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
    g.p_fmt = fmt(t);
    const bool gram1 = t == 0 ? bf16 : plain[t];  // X in one plane
    e = gram1 ? launch_product<ORTH_GRAM, NT_F16>(g, s) : launch_product<ORTH_GRAM, NT_SPLIT>(g, s);
    if (e != hipSuccess) break;
    e = plain[t] ? launch_product<ORTH_POLY, NT_F16>(g, s)
                 : launch_product<ORTH_POLY, NT_SPLIT>(g, s);
    if (e != hipSuccess) break;
    if (t + 1 < c.steps) {
      g.x_fmt = g.xt_fmt = fmt(t + 1);
      if (plain[t]) e = launch_product<ORTH_APPLY, NT_F16>(g, s);
      else if (t == 0 && bf16) e = launch_product<ORTH_APPLY, NT_SPLIT_B0>(g, s);
      else e = launch_product<ORTH_APPLY, NT_SPLIT>(g, s);
    } else {
      e = plain[t] ? launch_product<ORTH_LAST, NT_F16>(g, s)
                   : launch_product<ORTH_LAST, NT_SPLIT>(g, s);
    }
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
// or three writes of the model.  Matrix entries leave u and their sum of
// squares for the orthogonalisation, everything else is updated here.
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
