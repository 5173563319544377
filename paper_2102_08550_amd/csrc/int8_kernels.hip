// The linear layer in 8-bit integers: each row of the input (token, sample) and
// each output channel has a scale of its own,
//   y[r][o] = sx[r] sw[o] sum_k xq[r][k] wq[o][k] + b[o].
// The sums are exact (int32; K <= 65536 terms of at most 127^2 stay below 2^31),
// so nothing depends on how K is cut.  The scaling is fl(fl(sum) fl(sx sw)) in
// fp32, then the bias, then the rounding to the output's type.
//
//   quantize_rows   one pass over the rows, a wave or a workgroup a row;
//   matmul_i8       tiles on 32x32x32 matrix instructions (nt_mma.h);
//   linear_i8_few   up to 16 rows: a stream of the weights, with the rows'
//                   quantisation in front of it in every workgroup.
#include "int8.h"

#include "nt_mma.h"

namespace oscars {
namespace {

__device__ __forceinline__ float i8_bf16(uint32_t v) {
  return __builtin_bit_cast(float, v << 16);
}
__device__ __forceinline__ uint16_t i8_to_bf16(float v) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return static_cast<uint16_t>(u >> 16) | 0x40;
  return static_cast<uint16_t>((u + 0x7FFF + ((u >> 16) & 1)) >> 16);
}
__device__ __forceinline__ uint32_t abs_bits(float v) {
  return __builtin_bit_cast(uint32_t, v) & 0x7FFFFFFFu;
}

// The scale of a row from the largest |x| as bits (a NaN's are above infinity's,
// and those above every number's): 0 where it is not a normal number (the row
// counts as zeros), NaN where the row has one or an infinity.
__device__ __forceinline__ float row_scale(uint32_t top) {
  if (top >= 0x7F800000u) return __builtin_nanf("");
  const float s = __builtin_bit_cast(float, top) / 127.0f;
  return s >= 1.17549435e-38f ? s : 0.0f;
}

// round-half-even(x / s) of the quotient itself.  x (1 / s) is off by less than
// one, the remainder x - q s is exact (a multiple of the smaller ulp, of at most
// 24 bits) and says where the quotient lies: past the half, or on it.
__device__ __forceinline__ int quant(float x, float s, float inv) {
  float q = __builtin_rintf(x * inv);
  const float r = __builtin_fmaf(-q, s, x), t = 2.0f * __builtin_fabsf(r);
  const bool odd = static_cast<int>(q) & 1;
  if (t > s || (t == s && odd)) q += __builtin_copysignf(1.0f, r);
  return static_cast<int>(q);
}
__device__ __forceinline__ uint32_t quant4(const float* v, float s, float inv) {
  uint32_t w = 0;
#pragma unroll
  for (int t = 0; t < 4; ++t)
    w |= (static_cast<uint32_t>(quant(v[t], s, inv)) & 0xFFu) << (8 * t);
  return w;
}
// For scale 0 or NaN every integer is 0: 1 / s is replaced by 0 and s by 1.
struct Divisor {
  float s, inv;
};
__device__ __forceinline__ Divisor divisor(float scale) {
  const bool ok = scale > 0.0f;
  return Divisor{ok ? scale : 1.0f, ok ? 1.0f / scale : 0.0f};
}

// Eight consecutive entries from column c (a multiple of 8); zeros from `cols` on.
template <bool BF16, bool VEC>
__device__ __forceinline__ void load8(const void* row, int c, int cols, float* v) {
  if (VEC && c + 8 <= cols) {
    if constexpr (BF16) {
      const nt_u32x4 w =
          *reinterpret_cast<const nt_u32x4*>(static_cast<const uint16_t*>(row) + c);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        v[2 * t] = i8_bf16(w[t] & 0xFFFFu);
        v[2 * t + 1] = i8_bf16(w[t] >> 16);
      }
    } else {
      const nt_f32x4* p = reinterpret_cast<const nt_f32x4*>(static_cast<const float*>(row) + c);
      const nt_f32x4 a = p[0], b = p[1];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        v[t] = a[t];
        v[4 + t] = b[t];
      }
    }
  } else {
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      v[t] = 0.0f;
      if (c + t < cols) {
        if constexpr (BF16) v[t] = i8_bf16(static_cast<const uint16_t*>(row)[c + t]);
        else v[t] = static_cast<const float*>(row)[c + t];
      }
    }
  }
}

// A not finite entry's integer is 0 (the row's scale is NaN): the divisor's inv
// is 0, and the entry itself is dropped here.
__device__ __forceinline__ void drop_if(bool drop, float* v) {
#pragma unroll
  for (int t = 0; t < 8; ++t) v[t] = drop ? 0.0f : v[t];
}

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t o = __shfl_xor(v, d);
    v = o > v ? o : v;
  }
  return v;
}

// THR threads a row (64: four rows a workgroup), KEEP chunks of 8 columns a
// thread held in registers between the maximum and the rounding (rows of up to
// 8 THR KEEP columns; KEEP = 0: longer ones, read again from the L2).
template <bool BF16, bool VEC, int THR, int KEEP>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantArgs a) {
  __shared__ uint32_t top4[4];
  const int tid = threadIdx.x & (THR - 1);
  const int64_t r = static_cast<int64_t>(blockIdx.x) * (256 / THR) + threadIdx.x / THR;
  if (THR == 64 && r >= a.rows) return;  // whole waves: no barrier follows
  const char* row = static_cast<const char*>(a.x) + r * a.x_ld * (BF16 ? 2 : 4);
  float v[KEEP > 0 ? KEEP : 1][8];
  uint32_t top = 0;
  if constexpr (KEEP > 0) {
#pragma unroll
    for (int i = 0; i < KEEP; ++i) load8<BF16, VEC>(row, 8 * (tid + THR * i), a.cols, v[i]);
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
#pragma unroll
      for (int t = 0; t < 8; ++t) top = max(top, abs_bits(v[i][t]));
  } else {
    for (int c = 8 * tid; c < a.cols; c += 8 * THR) {
      load8<BF16, VEC>(row, c, a.cols, v[0]);
#pragma unroll
      for (int t = 0; t < 8; ++t) top = max(top, abs_bits(v[0][t]));
    }
  }
  top = wave_max(top);
  if constexpr (THR == 256) {
    if ((threadIdx.x & 63) == 0) top4[threadIdx.x >> 6] = top;
    __syncthreads();
    top = max(max(top4[0], top4[1]), max(top4[2], top4[3]));
  }
  const float scale = row_scale(top);
  const Divisor d = divisor(scale);
  const bool drop = !(scale > 0.0f);
  if (tid == 0) a.scale[r] = scale;
  // pad to a whole 128-byte block, as far as the row goes
  const int64_t end64 = (static_cast<int64_t>(a.cols) + 127) / 128 * 128;
  const int end = static_cast<int>(end64 < a.q_ld ? end64 : a.q_ld);
  int8_t* q = a.q + r * a.q_ld;
  auto put = [&](int c, float* x) {
    if (c >= end) return;
    drop_if(drop, x);
    *reinterpret_cast<nt_u32x2*>(q + c) =
        nt_u32x2{quant4(x, d.s, d.inv), quant4(x + 4, d.s, d.inv)};
  };
  if constexpr (KEEP > 0) {
#pragma unroll
    for (int i = 0; i < KEEP; ++i) put(8 * (tid + THR * i), v[i]);
  } else {
    for (int c = 8 * tid; c < end; c += 8 * THR) {
      load8<BF16, VEC>(row, c, a.cols, v[0]);
      put(c, v[0]);
    }
  }
}

template <bool BF16, bool VEC>
hipError_t quantize_launch(const QuantArgs& a, hipStream_t s) {
  if (a.cols <= 1024) {  // a wave a row
    const int64_t blocks = (a.rows + 3) / 4;
    if (blocks > 0x7FFFFFFF) return hipErrorInvalidValue;
    const dim3 grid(static_cast<unsigned>(blocks));
    if (a.cols <= 512)
      hipLaunchKernelGGL((quantize_rows_kernel<BF16, VEC, 64, 1>), grid, dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((quantize_rows_kernel<BF16, VEC, 64, 2>), grid, dim3(256), 0, s, a);
  } else {
    if (a.rows > 0x7FFFFFFF) return hipErrorInvalidValue;
    const dim3 grid(static_cast<unsigned>(a.rows));
    if (a.cols <= 2048)
      hipLaunchKernelGGL((quantize_rows_kernel<BF16, VEC, 256, 1>), grid, dim3(256), 0, s, a);
    else if (a.cols <= 4096)
      hipLaunchKernelGGL((quantize_rows_kernel<BF16, VEC, 256, 2>), grid, dim3(256), 0, s, a);
    else if (a.cols <= 8192)
      hipLaunchKernelGGL((quantize_rows_kernel<BF16, VEC, 256, 4>), grid, dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((quantize_rows_kernel<BF16, VEC, 256, 0>), grid, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

bool aligned_rows(const void* p, int64_t row_bytes, int to) {
  return reinterpret_cast<uintptr_t>(p) % to == 0 && row_bytes % to == 0;
}

// ------------------------------------------------------------------ tiles

typedef NtShape<256, 256, 2, 4, 2> I8L;
typedef NtShape<128, 128, 2, 2, 2> I8M;
typedef NtShape<64, 64, 2, 2, 3> I8S;

__device__ __forceinline__ float i8_finish(int32_t acc, float sx, float sw, float b, bool relu) {
  float y = static_cast<float>(acc) * (sx * sw) + b;
  if (relu) y = y < 0.0f ? 0.0f : y;  // keeps a NaN
  return y;
}

// Output rows are input rows; the tile's own rows (R) are output channels, four
// consecutive ones a lane.  A block of 32 x 32 goes through LDS so that a row's
// 32 outputs are stored together.  VEC: 16-byte stores.
template <class S, bool OUT_BF16, bool VEC>
__global__ __launch_bounds__(S::NT, 2) void matmul_i8_kernel(MatmulI8Args a) {
#if defined(__HIP_DEVICE_COMPILE__)  // buffer resources: no host form
  constexpr int TURN = 36;
  static_assert(S::LDS_BYTES >= S::WM * S::WN * 32 * TURN * 4, "room to turn blocks");
  __shared__ __attribute__((aligned(16))) char lds[S::LDS_BYTES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = lane >> 5;
  const int tr = (a.outs + S::BM - 1) / S::BM;
  const int tc = static_cast<int>((a.rows + S::BN - 1) / S::BN);
  const int total = tr * tc;
  int id;
  {  // the workgroups of one XCD (index mod 8) take neighbouring tiles
    const int per = total >> 3, rem = total & 7, x = blockIdx.x & 7, q = blockIdx.x >> 3;
    id = x * per + (x < rem ? x : rem) + q;
  }
  // bands of four tile columns (rows of the input), channel tile by channel tile
  constexpr int BAND = 4;
  const int band = id / (BAND * tr), cols = tc - band * BAND < BAND ? tc - band * BAND : BAND;
  const int at = id - band * BAND * tr;
  const int r0 = (at / cols) * S::BM;
  const int64_t c0 = static_cast<int64_t>(band * BAND + at % cols) * S::BN;

  const int blocks = (a.in + NT_BLOCK - 1) / NT_BLOCK;
  NtRows<S::NT, S::BM> ra;
  NtRows<S::NT, S::BN> rb;
  // weights end at their last row's last 16 bytes; what a block reads past a
  // row's end (its neighbour, or nothing past the last) meets zeros of xq
  ra.init(a.wq, a.w_ld, (a.outs - 1) * a.w_ld + (a.in + 15) / 16 * 16, r0, a.outs, tid);
  const int64_t left = a.rows - c0;
  rb.init(a.xq + c0 * a.x_ld, a.x_ld, left * a.x_ld, 0,
          static_cast<int>(left < S::BN ? left : S::BN), tid);
  nt_i32x16 acc[S::MI][S::NJ];
#pragma unroll
  for (int i = 0; i < S::MI; ++i)
#pragma unroll
    for (int j = 0; j < S::NJ; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
  nt_tile<S, NT_I8>(ra, rb, 0, blocks, lds, tid, acc);

  const int rw = r0 + (wave / S::WN) * 32 * S::MI;
  const int64_t cw = c0 + (wave % S::WN) * 32 * S::NJ;
  float* turn = reinterpret_cast<float*>(lds) + wave * 32 * TURN;
  nt_barrier();  // the stages are read: LDS is free
#pragma unroll
  for (int i = 0; i < S::MI; ++i) {
    if (rw + 32 * i >= a.outs) continue;
    float sw[16], bias[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int o = rw + 32 * i + 8 * (e >> 2) + 4 * h + (e & 3);
      const int oc = o < a.outs ? o : a.outs - 1;
      sw[e] = a.wscale[oc];
      bias[e] = a.bias ? a.bias[oc] : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) {
      const int64_t c = cw + 32 * j + (lane & 31);
      if (cw + 32 * j >= a.rows) continue;  // uniform over the wave
      const float sx = a.xscale[c < a.rows ? c : a.rows - 1];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        nt_f32x4 t;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          t[e] = i8_finish(acc[i][j][4 * q + e], sx, sw[4 * q + e], bias[4 * q + e], a.relu);
        *reinterpret_cast<nt_f32x4*>(turn + (lane & 31) * TURN + 8 * q + 4 * h) = t;
      }
      __builtin_amdgcn_wave_barrier();
      const int64_t row = cw + 32 * j + (lane >> 1);
      const int k = 16 * (lane & 1), o = rw + 32 * i + k;
      float v[16];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const nt_f32x4 t =
            *reinterpret_cast<const nt_f32x4*>(turn + (lane >> 1) * TURN + k + 4 * e);
#pragma unroll
        for (int f = 0; f < 4; ++f) v[4 * e + f] = t[f];
      }
      __builtin_amdgcn_wave_barrier();
      if (row >= a.rows || o >= a.outs) continue;
      const int n = a.outs - o < 16 ? a.outs - o : 16;
      if constexpr (OUT_BF16) {
        uint16_t* p = static_cast<uint16_t*>(a.out) + row * a.out_ld + o;
        if (VEC && n == 16) {
          nt_u32x4 w[2];
#pragma unroll
          for (int e = 0; e < 8; ++e)
            w[e >> 2][e & 3] = i8_to_bf16(v[2 * e]) |
                               static_cast<uint32_t>(i8_to_bf16(v[2 * e + 1])) << 16;
          reinterpret_cast<nt_u32x4*>(p)[0] = w[0];
          reinterpret_cast<nt_u32x4*>(p)[1] = w[1];
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (e < n) p[e] = i8_to_bf16(v[e]);
        }
      } else {
        float* p = static_cast<float*>(a.out) + row * a.out_ld + o;
        if (VEC && n == 16) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            reinterpret_cast<nt_f32x4*>(p)[e] =
                nt_f32x4{v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]};
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (e < n) p[e] = v[e];
        }
      }
    }
  }
#endif
}

template <class S>
hipError_t matmul_launch(const MatmulI8Args& a, hipStream_t s) {
  const int64_t tiles = ((a.outs + S::BM - 1) / S::BM) * ((a.rows + S::BN - 1) / S::BN);
  if (tiles > 0x7FFFFFFF) return hipErrorInvalidValue;
  const dim3 grid(static_cast<unsigned>(tiles));
  const bool vec = aligned_rows(a.out, a.out_ld * (a.out_bf16 ? 2 : 4), 16);
  if (a.out_bf16) {
    if (vec) hipLaunchKernelGGL((matmul_i8_kernel<S, true, true>), grid, dim3(S::NT), 0, s, a);
    else hipLaunchKernelGGL((matmul_i8_kernel<S, true, false>), grid, dim3(S::NT), 0, s, a);
  } else {
    if (vec) hipLaunchKernelGGL((matmul_i8_kernel<S, false, true>), grid, dim3(S::NT), 0, s, a);
    else hipLaunchKernelGGL((matmul_i8_kernel<S, false, false>), grid, dim3(S::NT), 0, s, a);
  }
  return hipGetLastError();
}

// ------------------------------------------------------------------ a few rows

// Up to 16 rows.  A workgroup takes 16 output channels, its eight waves K slices
// of 64 in turn (16x16x64: lane l has channel or row l & 15, bytes 16 (l >> 4)).
// The weights' loads are in flight before anything else; meanwhile every
// workgroup quantises all rows into LDS for itself (they come from the L2).
// The eight partial sums meet in LDS: integers, in any order the same.
constexpr int FEW_ROWS = 16;
constexpr int FEW_WAVES = 8;
constexpr int FEW_AHEAD = 8;           // K slices of a wave loaded ahead
// Bytes of quantised rows: the smaller one where it holds them, so that more than
// one workgroup fits a CU.
constexpr int FEW_LDS_S = 32 << 10, FEW_LDS_L = 136 << 10;

__host__ __device__ __forceinline__ int few_row_bytes(int in) {
  return (in + 63) / 64 * 64 + 16;  // 16 more: consecutive rows start in other banks
}

template <int LDS, bool X_BF16, bool VEC, bool OUT_BF16>
__global__ __launch_bounds__(64 * FEW_WAVES) void linear_i8_few_kernel(MatmulI8Args a, const void* x,
                                                                       int64_t x_ld) {
  __shared__ __attribute__((aligned(16))) char few_lds[LDS];  // quantised rows
  __shared__ int part[FEW_WAVES][64][4];
  __shared__ float scales[FEW_ROWS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int rows = static_cast<int>(a.rows), in = a.in, ld = few_row_bytes(in);
  const int slices = (in + 63) / 64;
  const int ch = blockIdx.x * 16 + (lane & 15), chc = ch < a.outs ? ch : a.outs - 1;
  const int8_t* w = a.wq + chc * a.w_ld;
  const int end = (in + 15) / 16 * 16;  // of a row of weights
  auto load_w = [&](int slice) {
    const int k = slice * 64 + 16 * (lane >> 4);
    // past the row's end: its first bytes, against zeros of the quantised rows
    return *reinterpret_cast<const nt_i32x4*>(w + (k < end ? k : 0));
  };
  nt_i32x4 ahead[FEW_AHEAD];
#pragma unroll
  for (int i = 0; i < FEW_AHEAD; ++i) {
    const int sl = wave + FEW_WAVES * i;
    ahead[i] = load_w(sl < slices ? sl : 0);
  }
  // rows wave, wave + 8: a wave quantises a row
  for (int r = wave; r < rows; r += FEW_WAVES) {
    const char* row = static_cast<const char*>(x) + r * x_ld * (X_BF16 ? 2 : 4);
    uint32_t top = 0;
    float v[8];
    for (int c = 8 * lane; c < in; c += 512) {
      load8<X_BF16, VEC>(row, c, in, v);
#pragma unroll
      for (int t = 0; t < 8; ++t) top = max(top, abs_bits(v[t]));
    }
    const float scale = row_scale(wave_max(top));
    const Divisor d = divisor(scale);
    const bool drop = !(scale > 0.0f);
    if (lane == 0) scales[r] = scale;
    for (int c = 8 * lane; c < slices * 64; c += 512) {
      load8<X_BF16, VEC>(row, c, in, v);
      drop_if(drop, v);
      *reinterpret_cast<nt_u32x2*>(few_lds + r * ld + c) =
          nt_u32x2{quant4(v, d.s, d.inv), quant4(v + 4, d.s, d.inv)};
    }
  }
  __syncthreads();
  nt_i32x4 acc = {0, 0, 0, 0};
  // lanes of rows that are not there read the last one; their sums are not used
  const char* b = few_lds + ((lane & 15) < rows ? (lane & 15) : rows - 1) * ld + 16 * (lane >> 4);
  for (int i0 = 0; wave + FEW_WAVES * i0 < slices; i0 += FEW_AHEAD) {
#pragma unroll
    for (int i = 0; i < FEW_AHEAD; ++i) {
      const int sl = wave + FEW_WAVES * (i0 + i), next = sl + FEW_WAVES * FEW_AHEAD;
      const nt_i32x4 cur = ahead[i];
      if (next < slices) ahead[i] = load_w(next);  // uniform over the wave
      if (sl < slices)
        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(
            cur, *reinterpret_cast<const nt_i32x4*>(b + sl * 64), acc, 0, 0, 0);
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) part[wave][lane][e] = acc[e];
  __syncthreads();
  // lane l, element e: channel 4 (l >> 4) + e, row l & 15
  if (tid < 256) {
    const int e = tid & 3, l = tid >> 2;
    int sum = 0;
#pragma unroll
    for (int i = 0; i < FEW_WAVES; ++i) sum += part[i][l][e];
    const int r = l & 15, o = blockIdx.x * 16 + 4 * (l >> 4) + e;
    if (r < rows && o < a.outs) {
      const float y = i8_finish(sum, scales[r], a.wscale[o], a.bias ? a.bias[o] : 0.0f, a.relu);
      if constexpr (OUT_BF16) static_cast<uint16_t*>(a.out)[r * a.out_ld + o] = i8_to_bf16(y);
      else static_cast<float*>(a.out)[r * a.out_ld + o] = y;
    }
  }
}

template <int LDS, bool X_BF16, bool VEC>
hipError_t few_launch(const MatmulI8Args& a, const void* x, int64_t x_ld, hipStream_t s) {
  const dim3 grid((a.outs + 15) / 16), wg(64 * FEW_WAVES);
  if (a.out_bf16)
    hipLaunchKernelGGL((linear_i8_few_kernel<LDS, X_BF16, VEC, true>), grid, wg, 0, s, a, x, x_ld);
  else
    hipLaunchKernelGGL((linear_i8_few_kernel<LDS, X_BF16, VEC, false>), grid, wg, 0, s, a, x, x_ld);
  return hipGetLastError();
}

template <bool X_BF16, bool VEC>
hipError_t few_launch(const MatmulI8Args& a, const void* x, int64_t x_ld, hipStream_t s) {
  return a.rows * few_row_bytes(a.in) <= FEW_LDS_S
             ? few_launch<FEW_LDS_S, X_BF16, VEC>(a, x, x_ld, s)
             : few_launch<FEW_LDS_L, X_BF16, VEC>(a, x, x_ld, s);
}

}  // namespace

hipError_t launch_quantize_rows(const QuantArgs& a, hipStream_t s) {
  const bool vec = aligned_rows(a.x, a.x_ld * (a.bf16 ? 2 : 4), 16);
  if (a.bf16) return vec ? quantize_launch<true, true>(a, s) : quantize_launch<true, false>(a, s);
  return vec ? quantize_launch<false, true>(a, s) : quantize_launch<false, false>(a, s);
}

hipError_t launch_matmul_i8(const MatmulI8Args& a, hipStream_t s) {
  auto tiles = [&](int t) { return ((a.outs + t - 1) / t) * ((a.rows + t - 1) / t); };
  // the largest tile that still gives most of the 256 CUs a workgroup
  if (tiles(I8L::BM) >= 192) return matmul_launch<I8L>(a, s);
  if (tiles(I8M::BM) >= 192) return matmul_launch<I8M>(a, s);
  return matmul_launch<I8S>(a, s);
}

bool linear_i8_one_launch(int64_t rows, int in) {
  return rows <= FEW_ROWS && rows * few_row_bytes(in) <= FEW_LDS_L;
}

hipError_t launch_linear_i8_few(const MatmulI8Args& a, const void* x, int64_t x_ld, bool x_bf16,
                                hipStream_t s) {
  const bool vec = aligned_rows(x, x_ld * (x_bf16 ? 2 : 4), 16);
  if (x_bf16)
    return vec ? few_launch<true, true>(a, x, x_ld, s) : few_launch<true, false>(a, x, x_ld, s);
  return vec ? few_launch<false, true>(a, x, x_ld, s) : few_launch<false, false>(a, x, x_ld, s);
}

}  // namespace oscars
