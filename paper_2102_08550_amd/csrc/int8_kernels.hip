// The linear layer in 8-bit integers: each row of the input (token, sample) and
// each output channel has a scale of its own,
//   y[r][o] = sx[r] sw[o] sum_k xq[r][k] wq[o][k] + b[o].
// The sums are exact (int32; K <= 65536 terms of at most 127^2 stay below 2^31),
// so nothing depends on how K is cut.  The scaling is fl(fl(sum) fl(sx sw)) in
// fp32, then the bias, then the rounding to the output's type.
//
//   quantize_rows   one pass over the rows, a wave or a workgroup a row;
//   matmul_i8       tiles on 32x32x32 matrix instructions (nt_mma.h);
//   linear_i8_few   one row, or up to 16 short ones: a stream of the weights, with
//                   the rows' quantisation in front of it in every workgroup.
#include "int8.h"

#include "int8_plan.h"
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
// Eight of them, a byte each.  Added to 1.5 2^23 the quotient is rounded to an
// integer, whose low byte is the result's; remainders below the half say that it
// is right.  Where one of the eight is not (next to a half: about one in 10^6 of
// ordinary entries) they are done again, one by one.  (8191 x 4096 in bf16: 23.3 us
// with all one by one, mostly their instructions; 19.2 us, 5.3 TB/s, like this.)
__device__ __forceinline__ nt_u32x2 quant8(const float* v, float s, float inv) {
  constexpr float BIG = 12582912.0f;
  uint32_t f[8];
  float worst = 0.0f;
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    const float y = __builtin_fmaf(v[t], inv, BIG);
    worst = __builtin_fmaxf(worst, __builtin_fabsf(__builtin_fmaf(BIG - y, s, v[t])));
    f[t] = __builtin_bit_cast(uint32_t, y);
  }
  if (2.0f * worst >= s) {
#pragma unroll
    for (int t = 0; t < 8; ++t) f[t] = static_cast<uint32_t>(quant(v[t], s, inv));
  }
  nt_u32x2 w;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const uint32_t lo = __builtin_amdgcn_perm(f[4 * t + 1], f[4 * t], 0x0C0C0400u);
    const uint32_t hi = __builtin_amdgcn_perm(f[4 * t + 3], f[4 * t + 2], 0x0C0C0400u);
    w[t] = lo | hi << 16;
  }
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
    *reinterpret_cast<nt_u32x2*>(q + c) = quant8(x, d.s, d.inv);
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
  const bool waves = a.cols <= 1024;  // a wave a row
  const dim3 grid(static_cast<unsigned>(waves ? (a.rows + 3) / 4 : a.rows));
  if (a.cols <= 512)
    hipLaunchKernelGGL((quantize_rows_kernel<BF16, VEC, 64, 1>), grid, dim3(256), 0, s, a);
  else if (waves)
    hipLaunchKernelGGL((quantize_rows_kernel<BF16, VEC, 64, 2>), grid, dim3(256), 0, s, a);
  else if (a.cols <= 2048)
    hipLaunchKernelGGL((quantize_rows_kernel<BF16, VEC, 256, 1>), grid, dim3(256), 0, s, a);
  else if (a.cols <= 4096)
    hipLaunchKernelGGL((quantize_rows_kernel<BF16, VEC, 256, 2>), grid, dim3(256), 0, s, a);
  else if (a.cols <= 8192)
    hipLaunchKernelGGL((quantize_rows_kernel<BF16, VEC, 256, 4>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((quantize_rows_kernel<BF16, VEC, 256, 0>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

bool aligned_rows(const void* p, int64_t row_bytes, int to) {
  return reinterpret_cast<uintptr_t>(p) % to == 0 && row_bytes % to == 0;
}

// ------------------------------------------------------------------ tiles

typedef NtShape<256, 256, 2, 4> I8L;
typedef NtShape<128, 128, 2, 2> I8M;
static_assert(i8_threads(I8L::BM) == I8L::NT && i8_threads(I8M::BM) == I8M::NT, "int8_plan.h");

__device__ __forceinline__ float i8_finish(int32_t acc, float sx, float sw, float b, bool relu) {
  float y = static_cast<float>(acc) * (sx * sw) + b;
  if (relu) y = y < 0.0f ? 0.0f : y;  // keeps a NaN
  return y;
}

// N channels from o on of an output row.
template <int N, bool OUT_BF16, bool VEC>
__device__ __forceinline__ void store_outs(const MatmulI8Args& a, int64_t row, int o,
                                           const float* v) {
  if constexpr (OUT_BF16) {
    uint16_t* p = static_cast<uint16_t*>(a.out) + row * a.out_ld + o;
    if (VEC && o + N <= a.outs) {
      uint32_t w[N / 2];
#pragma unroll
      for (int e = 0; e < N / 2; ++e)
        w[e] = i8_to_bf16(v[2 * e]) | static_cast<uint32_t>(i8_to_bf16(v[2 * e + 1])) << 16;
      if constexpr (N == 8)
        *reinterpret_cast<nt_u32x4*>(p) = nt_u32x4{w[0], w[1], w[2], w[3]};
      else
        *reinterpret_cast<nt_u32x2*>(p) = nt_u32x2{w[0], w[1]};
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (o + e < a.outs) p[e] = i8_to_bf16(v[e]);
    }
  } else {
    float* p = static_cast<float*>(a.out) + row * a.out_ld + o;
    if (VEC && o + N <= a.outs) {
#pragma unroll
      for (int e = 0; e < N; e += 4)
        *reinterpret_cast<nt_f32x4*>(p + e) = nt_f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (o + e < a.outs) p[e] = v[e];
    }
  }
}

// Output rows are input rows; the tile's own rows (R) are output channels, four
// consecutive ones a lane.  Two blocks of 32 channels go through LDS so that
// neighbouring lanes store whole 128-byte lines of an output row.  VEC: 16-byte
// stores.
template <class S, bool OUT_BF16, bool VEC>
__global__ __launch_bounds__(S::NT, 2) void matmul_i8_kernel(MatmulI8Args a) {
#if defined(__HIP_DEVICE_COMPILE__)  // buffer resources: no host form
  constexpr int TURN = 68;  // 64 channels of a row
  static_assert(S::LDS_BYTES >= S::WM * S::WN * 32 * TURN * 4 && S::MI % 2 == 0, "turned blocks");
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
  nt_tile<S, NT_I8>(ra, rb, blocks, lds, tid, acc);

  const int rw = r0 + (wave / S::WN) * 32 * S::MI;
  const int64_t cw = c0 + (wave % S::WN) * 32 * S::NJ;
  int* turn = reinterpret_cast<int*>(lds) + wave * 32 * TURN;
  constexpr int PER = OUT_BF16 ? 8 : 4, LANES = 64 / PER;  // 16 bytes a lane
  const int k = PER * (lane % LANES);
  nt_barrier();  // the stages are read: LDS is free
#pragma nounroll
  for (int i = 0; i < S::MI; i += 2) {
    const int o = rw + 32 * i + k;  // the lane's channels
    if (rw + 32 * i >= a.outs) continue;
    float sw[PER], bias[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int oc = o + e < a.outs ? o + e : a.outs - 1;
      sw[e] = a.wscale[oc];
      bias[e] = a.bias ? a.bias[oc] : 0.0f;
    }
#pragma nounroll
    for (int j = 0; j < S::NJ; ++j) {
      const int64_t row0 = cw + 32 * j;
      if (row0 >= a.rows) continue;  // uniform over the wave
#pragma unroll
      for (int ii = 0; ii < S::MI; ++ii)
#pragma unroll
        for (int jj = 0; jj < S::NJ; ++jj)
          if ((ii & ~1) == i && jj == j) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
              *reinterpret_cast<nt_i32x4*>(turn + (lane & 31) * TURN + 32 * (ii & 1) + 8 * q +
                                           4 * h) =
                  nt_i32x4{acc[ii][jj][4 * q], acc[ii][jj][4 * q + 1], acc[ii][jj][4 * q + 2],
                           acc[ii][jj][4 * q + 3]};
          }
      nt_wave_sync();
      for (int r = lane / LANES; r < 32; r += 64 / LANES) {
        const int64_t row = row0 + r;
        const float sx = a.xscale[row < a.rows ? row : a.rows - 1];
        float v[PER];
#pragma unroll
        for (int e = 0; e < PER; e += 4) {
          const nt_i32x4 t = *reinterpret_cast<const nt_i32x4*>(turn + r * TURN + k + e);
#pragma unroll
          for (int f = 0; f < 4; ++f)
            v[e + f] = i8_finish(t[f], sx, sw[e + f], bias[e + f], a.relu);
        }
        if (row < a.rows && o < a.outs) store_outs<PER, OUT_BF16, VEC>(a, row, o, v);
      }
      nt_wave_sync();
    }
  }
#endif
}

// Few tiles: 32 x 32 outputs a workgroup, K dealt to its four waves block by block.
// A wave streams its blocks through LDS of its own (RING of them), into registers,
// and waits for no other wave until the four sums meet.
constexpr int I8_SMALL_RING = 2;

template <bool OUT_BF16, bool VEC>
__global__ __launch_bounds__(256) void matmul_i8_small_kernel(MatmulI8Args a) {
#if defined(__HIP_DEVICE_COMPILE__)  // buffer resources: no host form
  constexpr int STAGE = 64 * NT_BLOCK, RING = I8_SMALL_RING;
  __shared__ __attribute__((aligned(16))) char lds[4 * RING * STAGE];
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);  // scalar addresses below
  const int tr = (a.outs + 31) / 32;
  const int r0 = static_cast<int>(blockIdx.x % tr) * 32;
  const int64_t c0 = static_cast<int64_t>(blockIdx.x / tr) * 32;
  const int blocks = (a.in + NT_BLOCK - 1) / NT_BLOCK;
  NtRows<64, 32> ra, rb;
  // as in matmul_i8_kernel
  ra.init(a.wq, a.w_ld, (a.outs - 1) * a.w_ld + (a.in + 15) / 16 * 16, r0, a.outs, lane);
  const int64_t left = a.rows - c0;
  rb.init(a.xq + c0 * a.x_ld, a.x_ld, left * a.x_ld, 0, static_cast<int>(left < 32 ? left : 32),
          lane);
  char* ring = lds + wave * RING * STAGE;
  auto issue = [&](int i) {  // the wave's block i
    const int k = wave + 4 * i;
    char* t = ring + (i % RING) * STAGE;
    const int at = (k < blocks ? k : blocks - 1) * NT_BLOCK;
    ra.issue(t, at, lane);
    rb.issue(t + STAGE / 2, at, lane);
  };
  nt_i32x16 acc;
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = 0;
  constexpr int PER = NtRows<64, 32>::P * 2;
  for (int i = 0; i < RING; ++i) issue(i);
  for (int i = 0; wave + 4 * i < blocks; ++i) {
    nt_wait_vm<(RING - 1) * PER>();
    const char* ta = ring + (i % RING) * STAGE;
    const char* tb = ta + STAGE / 2;
    nt_u32x4 fa[4], fb[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      fa[c] = nt_read(ta, lane & 31, 2 * c + h);
      fb[c] = nt_read(tb, lane & 31, 2 * c + h);
    }
    // the stage is in registers: refill it
    __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4));  // lgkmcnt(0)
    asm volatile("" ::: "memory");
    issue(i + RING);
#pragma unroll
    for (int c = 0; c < 4; ++c) acc = nt_mfma<NT_I8>(fa[c], fb[c], acc);
  }
  nt_wait_vm<0>();
  __syncthreads();  // every wave is through with LDS: now the four sums
  int* sums = reinterpret_cast<int*>(lds);
#pragma unroll
  for (int e = 0; e < 16; ++e) sums[(wave * 16 + e) * 64 + lane] = acc[e];
  __syncthreads();
  // wave w finishes channels 8 w + 4 h .. + 3 of row (lane & 31)
  const int o = r0 + 8 * wave + 4 * h;
  const int64_t row = c0 + (lane & 31);
  if (row >= a.rows || o >= a.outs) return;
  const float sx = a.xscale[row];
  float v[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    int s = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) s += sums[(w * 16 + 4 * wave + t) * 64 + lane];
    const int oc = o + t < a.outs ? o + t : a.outs - 1;
    v[t] = i8_finish(s, sx, a.wscale[oc], a.bias ? a.bias[oc] : 0.0f, a.relu);
  }
  store_outs<4, OUT_BF16, VEC>(a, row, o, v);
#endif
}

template <bool OUT_BF16, bool VEC>
hipError_t matmul_launch(const MatmulI8Args& a, int tile, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>((a.outs + tile - 1) / tile * ((a.rows + tile - 1) / tile)));
  if (tile == I8L::BM)
    hipLaunchKernelGGL((matmul_i8_kernel<I8L, OUT_BF16, VEC>), grid, dim3(I8L::NT), 0, s, a);
  else if (tile == I8M::BM)
    hipLaunchKernelGGL((matmul_i8_kernel<I8M, OUT_BF16, VEC>), grid, dim3(I8M::NT), 0, s, a);
  else
    hipLaunchKernelGGL((matmul_i8_small_kernel<OUT_BF16, VEC>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

// ------------------------------------------------------------------ a few rows

// Up to 16 rows.  A workgroup takes 16 output channels, its eight waves K slices
// of 64 in turn (16x16x64: lane l has channel or row l & 15, bytes 16 (l >> 4)).
// While the weights are on their way every workgroup quantises all rows into LDS
// for itself (they come from the L2).
// The eight partial sums meet in LDS: integers, in any order the same.
constexpr int FEW_ROWS = 16;
constexpr int FEW_WAVES = 8;
constexpr int FEW_AHEAD = 8;           // K slices of a wave loaded ahead
// Every workgroup quantises all rows: up to so many entries that is less than a
// launch of its own takes (bf16, 4096 x 4096: 4 rows 10.5 us, 8 rows 13.6 and in two
// launches 12.3, 16 rows 18.9 and 12.8; 16 rows of 1024 x 1024 8.5, of 2048 x 2048
// 11.3 and 7.9).  One row is taken at any length.
constexpr int FEW_ENTRIES = 16384;
// Bytes of quantised rows: the smaller one where it holds them, so that more
// workgroups fit a CU.
constexpr int FEW_LDS_S = 18 << 10, FEW_LDS_L = 65 << 10;

__host__ __device__ __forceinline__ int few_row_bytes(int in) {
  return (in + 63) / 64 * 64 + 16;  // 16 more: consecutive rows start in other banks
}

template <int LDS, bool X_BF16, bool VEC, bool OUT_BF16>
__global__ __launch_bounds__(64 * FEW_WAVES) void linear_i8_few_kernel(MatmulI8Args a,
                                                                       const void* x,
                                                                       int64_t x_ld) {
  __shared__ __attribute__((aligned(16))) char few_lds[LDS];  // quantised rows
  __shared__ int part[FEW_WAVES][64][4];
  __shared__ float scales[FEW_ROWS];
  __shared__ uint32_t tops[2 * FEW_WAVES];
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
  // All threads on the rows: 512 / R of them a row, R the power of two that holds
  // the rows (one row: all 512).  Loads come back in order, so the rows' first
  // ones go out in front of the weights'.
  int shift = 9;
  while (shift > 5 && (512 >> shift) < rows) --shift;
  const int per = 1 << shift, r = tid >> shift, at = tid & (per - 1);
  const char* row = static_cast<const char*>(x) + (r < rows ? r : 0) * x_ld * (X_BF16 ? 2 : 4);
  const bool once = in <= 8 * per;  // the row stays in registers
  float v[8] = {};
  uint32_t top = 0;
  if (once) {
    load8<X_BF16, VEC>(row, 8 * at, in, v);
  } else {
    for (int c = 8 * at; c < in; c += 8 * per) {
      load8<X_BF16, VEC>(row, c, in, v);
#pragma unroll
      for (int t = 0; t < 8; ++t) top = max(top, abs_bits(v[t]));
    }
  }
  nt_i32x4 ahead[FEW_AHEAD];
#pragma unroll
  for (int i = 0; i < FEW_AHEAD; ++i) {
    const int sl = wave + FEW_WAVES * i;
    ahead[i] = load_w(sl < slices ? sl : 0);
  }
  if (once) {
#pragma unroll
    for (int t = 0; t < 8; ++t) top = max(top, abs_bits(v[t]));
  }
  for (int d = 1; d < (per < 64 ? per : 64); d *= 2) {
    const uint32_t o = __shfl_xor(top, d);
    top = o > top ? o : top;
  }
  if ((lane & 31) == 0) tops[tid >> 5] = top;  // by halves of a wave
  __syncthreads();
  for (int h = (r << shift) >> 5; h < ((r + 1) << shift) >> 5; ++h) top = max(top, tops[h]);
  const float scale = row_scale(top);
  const Divisor d = divisor(scale);
  const bool drop = !(scale > 0.0f);
  if (at == 0) scales[r] = scale;
  if (r < rows)
    for (int c = 8 * at; c < slices * 64; c += 8 * per) {
      if (!once) load8<X_BF16, VEC>(row, c, in, v);
      drop_if(drop, v);
      *reinterpret_cast<nt_u32x2*>(few_lds + r * ld + c) = quant8(v, d.s, d.inv);
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
    const int q = l & 15, o = blockIdx.x * 16 + 4 * (l >> 4) + e;
    if (q < rows && o < a.outs) {
      const float y = i8_finish(sum, scales[q], a.wscale[o], a.bias ? a.bias[o] : 0.0f, a.relu);
      if constexpr (OUT_BF16) static_cast<uint16_t*>(a.out)[q * a.out_ld + o] = i8_to_bf16(y);
      else static_cast<float*>(a.out)[q * a.out_ld + o] = y;
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

hipError_t launch_quantize_rows(const QuantArgs& args, hipStream_t s) {
  const int64_t es = args.bf16 ? 2 : 4;
  const bool vec = aligned_rows(args.x, args.x_ld * es, 16);
  constexpr int64_t MOST = int64_t{1} << 23;  // rows a launch: a grid has less than 2^32 threads
  for (int64_t r = 0; r < args.rows; r += MOST) {
    QuantArgs a = args;
    a.x = static_cast<const char*>(args.x) + r * args.x_ld * es;
    a.q += r * a.q_ld;
    a.scale += r;
    a.rows = args.rows - r < MOST ? args.rows - r : MOST;
    hipError_t e;
    if (a.bf16) e = vec ? quantize_launch<true, true>(a, s) : quantize_launch<true, false>(a, s);
    else e = vec ? quantize_launch<false, true>(a, s) : quantize_launch<false, false>(a, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_matmul_i8(const MatmulI8Args& args, hipStream_t s) {
  const bool vec = aligned_rows(args.out, args.out_ld * (args.out_bf16 ? 2 : 4), 16);
  auto launch = [&](const MatmulI8Args& a, int tile) {
    if (a.out_bf16)
      return vec ? matmul_launch<true, true>(a, tile, s) : matmul_launch<true, false>(a, tile, s);
    return vec ? matmul_launch<false, true>(a, tile, s) : matmul_launch<false, false>(a, tile, s);
  };
  hipError_t e = hipSuccess;
  i8_launches(args.rows, args.in, args.outs, [&](int tile, int64_t at, int64_t rows) {
    MatmulI8Args a = args;
    a.rows = rows;
    a.xq += at * a.x_ld;
    a.xscale += at;
    a.out = static_cast<char*>(a.out) + at * a.out_ld * (a.out_bf16 ? 2 : 4);
    e = launch(a, tile);
    return e == hipSuccess;
  });
  return e;
}

bool linear_i8_one_launch(int64_t rows, int in) {
  static_assert(FEW_LDS_S >= FEW_ENTRIES + FEW_ROWS * (63 + 16) && FEW_LDS_L >= 65536 + 63 + 16,
                "room for the rows");
  return rows == 1 || (rows <= FEW_ROWS && rows * in <= FEW_ENTRIES);
}

hipError_t launch_linear_i8_few(const MatmulI8Args& a, const void* x, int64_t x_ld, bool x_bf16,
                                hipStream_t s) {
  const bool vec = aligned_rows(x, x_ld * (x_bf16 ? 2 : 4), 16);
  if (x_bf16)
    return vec ? few_launch<true, true>(a, x, x_ld, s) : few_launch<true, false>(a, x, x_ld, s);
  return vec ? few_launch<false, true>(a, x, x_ld, s) : few_launch<false, false>(a, x, x_ld, s);
}

}  // namespace oscars
