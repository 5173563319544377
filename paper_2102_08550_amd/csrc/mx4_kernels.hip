// The linear layer in microscaled 4-bit floating point (mx4.h has the format):
//   y[r][o] = drop(relu(sum_k Q(x)[r][k] Q(w)[o][k] + b[o])),
// and what its gradients take.  A product of two entries is exact, and so is its
// scale; the matrix units add them into fp32.
//
//   mx4_rows      rows into 4 bits, one pass;
//   mx4_columns   columns into 4 bits (the rows of x');
//   mx4_gradient  the output's gradient by columns, and rows, and its sums, and x by
//                 columns: all that the gradients multiply;
//   mx4_values    4 bits back into values;
//   mx4_product   tiles on 32x32x64 block-scaled matrix instructions: a lane's 16
//                 bytes of an operand are one block of 32 with one scale;
//   mx4_few       one row, or up to 32 short ones: a stream of the weights, with the
//                 rows' quantisation in front of it in every workgroup.
#include "mx4.h"

#include "mx4_plan.h"
#include "nt_mma.h"

namespace oscars {
namespace {

typedef int mx_i32x8 __attribute__((ext_vector_type(8)));
typedef float mx_f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float mx_bf16(uint32_t v) {
  return __builtin_bit_cast(float, v << 16);
}
__device__ __forceinline__ uint16_t mx_to_bf16(float v) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return static_cast<uint16_t>(u >> 16) | 0x40;
  return static_cast<uint16_t>((u + 0x7FFF + ((u >> 16) & 1)) >> 16);
}

// A block's scale from its largest |x| as bits.  Adding a quarter of the significand's
// range carries into the exponent from 7/4 on: then the largest entry would be
// rounded to 8, which is not there, and the scale is twice as large.  (Scales by the
// exponent alone, with what is above 6 cut to 6, have 1.06 times the squared error for
// normal entries, 1.04 where channels differ, 2.1 for uniform ones; scales that bring
// the largest to 6 or below 1.06, 1.10 and 1.00 times.)  Scales end at 2^125: what is
// left above 6 is cut to 6, where 2^126 would make it 2^128.
// s: what the conversion divides by (its exponent counts, 2^-127 among them).  A block that is
// not alive has only zeros: one without a normal number (s such that all round to
// zero), or with a NaN or an infinity (byte 255: NaN).
struct MxScale {
  uint32_t byte;
  float s;
  bool alive;
};
__device__ __forceinline__ MxScale mx_scale(uint32_t top) {
  const uint32_t e = (top + 0x00200000u) >> 23;
  const uint32_t byte = e > 254 ? 252 : e > 2 ? e - 2 : 0;
  MxScale r{byte, __builtin_bit_cast(float, byte << 23),
            top >= 0x00800000u && top < 0x7F800000u};
  if (top >= 0x7F800000u) r.byte = 255u;
  if (top < 0x00800000u) r = MxScale{0u, 1.0f, false};
  return r;
}
// The larger magnitude; a NaN's bits are above infinity's, and those above every number's.
__device__ __forceinline__ float mx_larger(float top, float v) {
  return __builtin_elementwise_maximum(top, __builtin_fabsf(v));  // keeps a NaN
}
__device__ __forceinline__ uint32_t mx_bits(float top) {
  return __builtin_bit_cast(uint32_t, top) & 0x7FFFFFFFu;
}
// Two entries in units of the scale into byte B of w, the first in its low half: rounded to
// nearest, ties to even.
template <int B>
__device__ __forceinline__ uint32_t mx_pack2(uint32_t w, float a, float b, float s) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a, b, s, B);
}
template <int B>
__device__ __forceinline__ uint32_t mx_pack2(uint32_t w, uint32_t pair, float s) {  // of bf16
  typedef __bf16 two __attribute__((ext_vector_type(2)));
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(two, pair), s, B);
}
__device__ __forceinline__ uint32_t mx_pack8(const float* v, const MxScale& m) {
  uint32_t w = mx_pack2<0>(0u, v[0], v[1], m.s);
  w = mx_pack2<1>(w, v[2], v[3], m.s);
  w = mx_pack2<2>(w, v[4], v[5], m.s);
  w = mx_pack2<3>(w, v[6], v[7], m.s);
  return m.alive ? w : 0u;
}
__device__ __forceinline__ uint32_t mx_pack8(const uint32_t* pairs, const MxScale& m) {
  uint32_t w = mx_pack2<0>(0u, pairs[0], m.s);
  w = mx_pack2<1>(w, pairs[1], m.s);
  w = mx_pack2<2>(w, pairs[2], m.s);
  w = mx_pack2<3>(w, pairs[3], m.s);
  return m.alive ? w : 0u;
}
// The larger magnitudes of two pairs in bf16, as bits.
__device__ __forceinline__ uint32_t mx_larger2(uint32_t top, uint32_t pair) {
  typedef uint16_t two __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(
      uint32_t, __builtin_elementwise_max(__builtin_bit_cast(two, top),
                                          __builtin_bit_cast(two, pair & 0x7FFF7FFFu)));
}

// Eight consecutive entries from column c (a multiple of 8).  VEC: cols % 8 == 0, 16-byte loads.
// Columns behind the last read the last ones again, so that no load waits behind a branch;
// mx_clip8 makes them zeros.
template <bool BF16, bool VEC>
__device__ __forceinline__ void mx_load8(const void* row, int c, int cols, float* v) {
  if constexpr (VEC) {
    const int at = c < cols ? c : cols - 8;
    if constexpr (BF16) {
      const nt_u32x4 w =
          *reinterpret_cast<const nt_u32x4*>(static_cast<const uint16_t*>(row) + at);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        v[2 * t] = mx_bf16(w[t] & 0xFFFFu);
        v[2 * t + 1] = mx_bf16(w[t] >> 16);
      }
    } else {
      const nt_f32x4* p = reinterpret_cast<const nt_f32x4*>(static_cast<const float*>(row) + at);
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
      const int at = c + t < cols ? c + t : cols - 1;
      if constexpr (BF16) v[t] = mx_bf16(static_cast<const uint16_t*>(row)[at]);
      else v[t] = static_cast<const float*>(row)[at];
    }
  }
}
template <bool VEC>
__device__ __forceinline__ void mx_clip8(int c, int cols, float* v) {
#pragma unroll
  for (int t = 0; t < 8; ++t) v[t] = (VEC ? c : c + t) < cols ? v[t] : 0.0f;
}

__device__ __forceinline__ uint32_t mx_top8(const float* v) {
  float top = 0.0f;
#pragma unroll
  for (int t = 0; t < 8; ++t) top = mx_larger(top, v[t]);
  return mx_bits(top);
}

// The gradient behind the layer's epilogue (mx4.h), factor 1 without dropout.  A NaN in y passes
// it on.
__device__ __forceinline__ float mx_pass(float dy, float y, float factor) {
  return y <= 0.0f ? 0.0f : dy * factor;
}

// A wave takes 512 columns of a row, a lane eight of them, four lanes a block; neighbouring
// waves have neighbouring pieces.  4096 x 4096 in fp32 12.9 us, 8191 x 4096 in bf16 14.3:
// 5.9 TB/s; 10000 x 784 in bf16, two pieces a row, 6.5 to 7.9.  Tried against an earlier
// form (12.5 and 16.3 us): four pieces a wave with all loads on their way 13.9 and 17.2; 16
// rows of the same columns a workgroup, which in rows a power of two apart meet in the
// same channels, 17 and 17.4.
template <bool BF16, bool VEC>
__global__ __launch_bounds__(256) void mx4_rows_kernel(Mx4Source a, Mx4Rows to, int pieces) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t units = a.rows * pieces, step = static_cast<int64_t>(gridDim.x) * 4;
  const int end = static_cast<int>(mx4_bytes(a.cols)) * 2;
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * 4 + wave; u < units; u += step) {
    const int64_t row = u / pieces;
    const int c = static_cast<int>(u - row * pieces) * 512 + 8 * lane;
    const char* from = static_cast<const char*>(a.x) + row * a.x_ld * (BF16 ? 2 : 4);
    uint32_t top, pairs[4];
    float v[8];
    if constexpr (BF16 && VEC) {
      const nt_u32x4 w = *reinterpret_cast<const nt_u32x4*>(
          reinterpret_cast<const uint16_t*>(from) + (c < a.cols ? c : a.cols - 8));
      uint32_t two = 0;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        pairs[t] = c < a.cols ? w[t] : 0u;
        two = mx_larger2(two, pairs[t]);
      }
      top = max(two << 16, two & 0xFFFF0000u);
    } else {
      mx_load8<BF16, VEC>(from, c, a.cols, v);
      mx_clip8<VEC>(c, a.cols, v);
      top = mx_top8(v);
    }
    top = max(top, static_cast<uint32_t>(__shfl_xor(top, 1)));
    top = max(top, static_cast<uint32_t>(__shfl_xor(top, 2)));
    const MxScale s = mx_scale(top);
    if (c < end) {
      uint32_t w;
      if constexpr (BF16 && VEC) w = mx_pack8(pairs, s);
      else w = mx_pack8(v, s);
      *reinterpret_cast<uint32_t*>(to.q + row * to.q_ld + c / 2) = w;
    }
    if ((lane & 3) == 0) to.scale[row * to.s_ld + c / 32] = static_cast<uint8_t>(s.byte);
  }
}

// 256 rows x 64 columns a workgroup, eight waves of 32 rows; a lane has two neighbouring
// columns of half of its wave's rows.  A column's block of 32 rows is two lanes', its
// bytes are turned by LDS so that eight neighbouring lanes store a column's 128.
// BOTH: by rows as well, a block of 32 columns 16 lanes', for which the gradient is
// read once.  4096 x 4096 in fp32 12.7 us, 6.0 TB/s; dz of 8191 x 2048 both ways, from dy and
// y in bf16, with x of 8191 x 4096 41 us, 4.3 TB/s (98 in an early form with loads behind
// branches and every lane reducing every row).
constexpr int MXC_ROWS = 256, MXC_COLS = 64;

struct Mx4Columns {
  Mx4Source from;
  Mx4Rows to;
  Mx4Rows rows;  // BOTH
  float* sums;   // of the columns, held in 64 bits, or nullptr:
  double* part;  // where they go for each 256 rows, if there are more
};
template <bool BOTH>
struct MxColumnsLds {
  static constexpr int LD = 128 + 16;  // 16 more: neighbouring columns start in other banks
  __attribute__((aligned(16))) uint8_t q[MXC_COLS * LD];
  __attribute__((aligned(16))) uint8_t scale[MXC_COLS][8];
  double part[8][MXC_COLS];
  __attribute__((aligned(16))) uint8_t row_q[BOTH ? MXC_ROWS : 1][32];
  __attribute__((aligned(16))) uint8_t row_scale[BOTH ? MXC_ROWS : 1][2];
};

template <int CTRL>
__device__ __forceinline__ uint32_t mx_dpp(uint32_t v) {
  return static_cast<uint32_t>(
      __builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xF, 0xF, false));
}
// Of N values a lane, one per row, and 16 lanes: the first N / 2 rows' largest in the lanes whose
// bit N / 2 is clear, the others' in their partners.
template <int CTRL, int N>
__device__ __forceinline__ void mx_fold(uint32_t (&m)[16], int lane) {
  const bool up = lane & (N / 2);
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    const uint32_t keep = up ? m[i + N / 2] : m[i], give = up ? m[i] : m[i + N / 2];
    m[i] = max(keep, mx_dpp<CTRL>(give));
  }
}
// What the lane that is K-th of four has; every lane has to ask.
template <int K>
__device__ __forceinline__ uint32_t mx_from_quad(uint32_t v) {
  return mx_dpp<K * 0x55>(v);
}
// ... of sixteen.
template <int K>
__device__ __forceinline__ float mx_from_row(float v) {
  return __builtin_bit_cast(float, mx_dpp<0x150 + K>(__builtin_bit_cast(uint32_t, v)));
}

// SUMS: the columns' sums too, if p.sums is there.
template <bool BF16, bool VEC, int MODE, bool BOTH, bool SUMS>
__device__ __forceinline__ void mx_columns(const Mx4Columns& p, int64_t tile_row, int tile_col,
                                           MxColumnsLds<BOTH>& lds) {
  const Mx4Source& a = p.from;
  const int tid = threadIdx.x, lane = tid & 63, pair = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c0 = tile_col * MXC_COLS, c = c0 + 2 * pair;
  const int64_t r0 = tile_row * MXC_ROWS, r_wave = r0 + 32 * wave, mine = r_wave + 16 * h;
  constexpr int ES = BF16 ? 2 : 4;
  typedef MxColumnsLds<BOTH> Lds;
  // Rows and columns behind the last read the last one again, so that no load waits behind
  // a branch, and count as zeros.  VEC: an even number of columns, pairs aligned.
  const int64_t left = a.rows - mine;
  const int seen = static_cast<int>(left < 16 ? left : 16);  // of the lane's rows, may be < 0
  const int c_in = c < a.cols ? c : (VEC ? a.cols - 2 : a.cols - 1);
  const int c_next = c + 1 < a.cols ? 1 : 0;
  const bool clip = __any(seen < 16 || c + 1 >= a.cols);
  // each(i, address of row i's pair)
  auto rows = [&](const void* from, int64_t ld, auto&& each) {
    if (r_wave + 32 <= a.rows && ld < (int64_t{1} << 24)) {
      // the wave's rows from one address, the lane's place in them in 32 bits
      const char* at = static_cast<const char*>(from) + r_wave * ld * ES;
      const uint32_t place = (static_cast<uint32_t>(16 * h) * static_cast<uint32_t>(ld) +
                              static_cast<uint32_t>(c_in)) * ES;
#pragma unroll
      for (int i = 0; i < 16; ++i) each(i, at + i * ld * ES + place);
    } else {
      const char* at = static_cast<const char*>(from) +
                       ((left > 0 ? mine : a.rows - 1) * ld + c_in) * ES;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        each(i, at);
        at += i + 1 < seen ? ld * ES : 0;
      }
    }
  };
  auto put = [&](int t, const MxScale& s, nt_u32x2 w) {  // of column t of the pair
    const int col = 2 * pair + t;
    *reinterpret_cast<nt_u32x2*>(lds.q + col * Lds::LD + 16 * wave + 8 * h) = w;
    if (h == 0) lds.scale[col][wave] = static_cast<uint8_t>(s.byte);
  };
  auto add = [&](int t, auto&& value) {  // value(i), i < 16: of column t of the pair
    if constexpr (SUMS) {
      if (p.sums) {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum += static_cast<double>(value(i));
        sum += __shfl_xor(sum, 32);
        if (h == 0) lds.part[wave][2 * pair + t] = sum;
      }
    }
  };
  if constexpr (BF16 && VEC && MODE == 0 && !BOTH) {
    // as it is: both columns' magnitudes at once, pairs of rows put together for the conversion
    uint32_t w[16], two = 0;
    rows(a.x, a.x_ld,
         [&](int i, const char* at) { w[i] = *reinterpret_cast<const uint32_t*>(at); });
    if (clip) {
#pragma unroll
      for (int i = 0; i < 16; ++i) w[i] = i < seen && c < a.cols ? w[i] : 0u;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) two = mx_larger2(two, w[i]);
    two = mx_larger2(two, __shfl_xor(two, 32));
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const MxScale s = mx_scale(t ? two & 0xFFFF0000u : two << 16);
      uint32_t rows2[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        rows2[i] =
            __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], t ? 0x07060302u : 0x05040100u);
      put(t, s, nt_u32x2{mx_pack8(rows2, s), mx_pack8(rows2 + 4, s)});
      add(t, [&](int i) { return mx_bf16(t ? w[i] >> 16 : w[i] & 0xFFFFu); });
    }
  } else {
    auto load = [&](const void* from, int64_t ld, float(&v)[2][16]) {
      rows(from, ld, [&](int i, const char* at) {
        if constexpr (VEC && BF16) {
          const uint32_t w = *reinterpret_cast<const uint32_t*>(at);
          v[0][i] = mx_bf16(w & 0xFFFFu);
          v[1][i] = __builtin_bit_cast(float, w & 0xFFFF0000u);
        } else if constexpr (VEC) {
          const mx_f32x2 w = *reinterpret_cast<const mx_f32x2*>(at);
          v[0][i] = w[0];
          v[1][i] = w[1];
        } else if constexpr (BF16) {
          v[0][i] = mx_bf16(reinterpret_cast<const uint16_t*>(at)[0]);
          v[1][i] = mx_bf16(reinterpret_cast<const uint16_t*>(at)[c_next]);
        } else {
          v[0][i] = reinterpret_cast<const float*>(at)[0];
          v[1][i] = reinterpret_cast<const float*>(at)[c_next];
        }
      });
    };
    float v[2][16];
    load(a.x, a.x_ld, v);
    if constexpr (MODE == 1) {
      float y[2][16];
      load(a.y, a.y_ld, y);
      const float factor = a.drop.below ? a.drop.factor : 1.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        v[0][i] = mx_pass(v[0][i], y[0][i], factor);
        v[1][i] = mx_pass(v[1][i], y[1][i], factor);
      }
    }
    if (clip) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        v[0][i] = i < seen && c < a.cols ? v[0][i] : 0.0f;
        v[1][i] = i < seen && c + 1 < a.cols ? v[1][i] : 0.0f;
      }
    }
    if constexpr (MODE == 2) {
      // four lanes share a call of the generator for a row: each makes one of four rows'
      const uint64_t offset = drop_offset(a.drop);
      const int k = lane & 3;
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const Words4 w = drop_words(a.drop, offset, static_cast<uint32_t>(mine + i + k), c / 8);
#define OSCARS_KEEP(K)                                                                       \
  {                                                                                          \
    const uint32_t u0 = mx_from_quad<K>(w.w[0]), u1 = mx_from_quad<K>(w.w[1]);               \
    const uint32_t u2 = mx_from_quad<K>(w.w[2]), u3 = mx_from_quad<K>(w.w[3]);               \
    const uint32_t u = k & 2 ? (k & 1 ? u3 : u2) : (k & 1 ? u1 : u0);                        \
    v[0][i + K] = (u & 0xFFFFu) >= a.drop.below ? v[0][i + K] * a.drop.factor : 0.0f;        \
    v[1][i + K] = u >> 16 >= a.drop.below ? v[1][i + K] * a.drop.factor : 0.0f;              \
  }
        OSCARS_KEEP(0)
        OSCARS_KEEP(1)
        OSCARS_KEEP(2)
        OSCARS_KEEP(3)
#undef OSCARS_KEEP
      }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float most = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) most = mx_larger(most, v[t][i]);
      uint32_t top = mx_bits(most);
      top = max(top, static_cast<uint32_t>(__shfl_xor(top, 32)));
      const MxScale s = mx_scale(top);
      put(t, s, nt_u32x2{mx_pack8(v[t], s), mx_pack8(v[t] + 8, s)});
      add(t, [&](int i) { return v[t][i]; });
    }
    if constexpr (BOTH) {
      // 16 lanes have a block of each of 16 rows: lane l comes to hold row l's largest
      uint32_t m[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) m[i] = mx_bits(mx_larger(__builtin_fabsf(v[0][i]), v[1][i]));
      mx_fold<0x140, 16>(m, lane);  // with lane 15 - l,
      mx_fold<0x141, 8>(m, lane);   // 7 - l of eight,
      mx_fold<0x1B, 4>(m, lane);    // 3 - l of four,
      mx_fold<0xB1, 2>(m, lane);    // 1 - l of two
      const MxScale s = mx_scale(m[0]);
      const int row0 = 32 * wave + 16 * h;
      lds.row_scale[row0 + (lane & 15)][pair >> 4] = static_cast<uint8_t>(s.byte);
      // bytes of four rows in a lane turn into four lanes' bytes of a row (a block with a NaN
      // may have codes other than 0: it is its scale that counts)
      const uint32_t turn1 = lane & 1 ? 0x03070105u : 0x06020400u;
      const uint32_t turn2 = lane & 2 ? 0x03020706u : 0x05040100u;
#define OSCARS_ROWS(I)                                                                           \
  {                                                                                              \
    uint32_t w = mx_pack2<0>(0u, v[0][I], v[1][I], mx_from_row<I>(s.s));                         \
    w = mx_pack2<1>(w, v[0][I + 1], v[1][I + 1], mx_from_row<I + 1>(s.s));                       \
    w = mx_pack2<2>(w, v[0][I + 2], v[1][I + 2], mx_from_row<I + 2>(s.s));                       \
    w = mx_pack2<3>(w, v[0][I + 3], v[1][I + 3], mx_from_row<I + 3>(s.s));                       \
    w = __builtin_amdgcn_perm(mx_dpp<0xB1>(w), w, turn1);                                        \
    w = __builtin_amdgcn_perm(mx_dpp<0x4E>(w), w, turn2);                                        \
    *reinterpret_cast<uint32_t*>(&lds.row_q[row0 + I + (lane & 3)][pair & ~3]) = w;              \
  }
      OSCARS_ROWS(0)
      OSCARS_ROWS(4)
      OSCARS_ROWS(8)
      OSCARS_ROWS(12)
#undef OSCARS_ROWS
    }
  }
  __syncthreads();
  {
    const int col = tid >> 3, k = tid & 7;
    if (c0 + col < a.cols)
      *reinterpret_cast<nt_u32x4*>(p.to.q + (c0 + col) * p.to.q_ld + tile_row * 128 + 16 * k) =
          *reinterpret_cast<const nt_u32x4*>(lds.q + col * Lds::LD + 16 * k);
  }
  if (tid < MXC_COLS && c0 + tid < a.cols) {
    uint8_t* s = p.to.scale + (c0 + tid) * p.to.s_ld + tile_row * 8;
    *reinterpret_cast<nt_u32x2*>(s) = *reinterpret_cast<const nt_u32x2*>(lds.scale[tid]);
    // the last tile fills the scales to a whole 16
    if ((tile_row & 1) == 0 && r0 + MXC_ROWS >= a.rows)
      *reinterpret_cast<nt_u32x2*>(s + 8) = nt_u32x2{0, 0};
    if constexpr (SUMS) {
      if (p.sums) {
        double sum = 0.0;
#pragma unroll
        for (int w = 0; w < 8; ++w) sum += lds.part[w][tid];
        if (p.part) p.part[tile_row * a.cols + c0 + tid] = sum;
        else p.sums[c0 + tid] = static_cast<float>(sum);
      }
    }
  }
  if constexpr (BOTH) {
    const int row = tid >> 1, k = tid & 1;
    if (r0 + row < a.rows) {
      if (c0 < mx4_bytes(a.cols) * 2)
        *reinterpret_cast<nt_u32x4*>(p.rows.q + (r0 + row) * p.rows.q_ld + c0 / 2 + 16 * k) =
            *reinterpret_cast<const nt_u32x4*>(&lds.row_q[row][16 * k]);
      if (k == 0)
        *reinterpret_cast<uint16_t*>(p.rows.scale + (r0 + row) * p.rows.s_ld + c0 / 32) =
            *reinterpret_cast<const uint16_t*>(lds.row_scale[row]);
    }
  }
}

// Tiles of 64 columns: with BOTH to a whole 512, whose scales are all written.
__host__ __device__ __forceinline__ int mx_column_tiles(int cols, bool both) {
  return static_cast<int>(both ? (static_cast<int64_t>(cols) + 511) / 512 * 8
                               : (static_cast<int64_t>(cols) + MXC_COLS - 1) / MXC_COLS);
}
__host__ __device__ __forceinline__ int64_t mx_row_tiles(int64_t rows) {
  return (rows + MXC_ROWS - 1) / MXC_ROWS;
}

template <bool BF16, bool VEC>
__global__ __launch_bounds__(512) void mx4_columns_kernel(Mx4Columns p) {
  __shared__ __attribute__((aligned(16))) MxColumnsLds<false> lds;
  const int across = mx_column_tiles(p.from.cols, false);
  mx_columns<BF16, VEC, 0, false, false>(p, blockIdx.x / across,
                                         static_cast<int>(blockIdx.x % across), lds);
}

// What the gradients quantise in one launch: dz by columns, and for dx by rows, and x by
// columns.  The workgroups of one XCD (index mod 8) take neighbouring tiles: they
// share lines of dz's rows.
template <bool BF16, bool VEC, int MODE, bool BOTH>
__global__ __launch_bounds__(512) void mx4_gradient_kernel(Mx4Columns z, Mx4Columns x,
                                                           int z_tiles) {
  __shared__ __attribute__((aligned(16))) MxColumnsLds<BOTH> lds;
  const int total = gridDim.x, per = total >> 3, rem = total & 7;
  const int n = blockIdx.x & 7, q = blockIdx.x >> 3;
  int id = n * per + (n < rem ? n : rem) + q;
  if (id < z_tiles) {
    const int across = mx_column_tiles(z.from.cols, BOTH);
    mx_columns<BF16, VEC, MODE, BOTH, true>(z, id / across, id % across, lds);
  } else {
    id -= z_tiles;
    const int across = mx_column_tiles(x.from.cols, false);
    auto& own = reinterpret_cast<MxColumnsLds<false>&>(lds);
    if (x.from.bf16) mx_columns<true, VEC, 0, false, false>(x, id / across, id % across, own);
    else mx_columns<false, VEC, 0, false, false>(x, id / across, id % across, own);
  }
}

// Values: eight a thread.  A row's scale of 2^-127 is no normal number: entries are
// converted at scale 1 and multiplied, exactly.
template <bool OUT_BF16, bool VEC>
__global__ __launch_bounds__(256) void mx4_values_kernel(Mx4Values a, uint32_t groups) {
  const int64_t units = a.rows * groups, step = static_cast<int64_t>(gridDim.x) * 256;
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; u < units; u += step) {
    const int64_t row = u / groups;
    const int c = static_cast<int>(u - row * groups) * 8;
    const uint32_t w = *reinterpret_cast<const uint32_t*>(a.q + row * a.q_ld + c / 2);
    const uint32_t e = a.scale[row * a.s_ld + c / 32];
    const float s = __builtin_bit_cast(float, e == 0     ? 0x00400000u
                                              : e == 255 ? 0x7FC00000u
                                                         : e << 23);
    const auto v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0);
    const auto v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
    const auto v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2);
    const auto v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
    const float v[8] = {v0[0] * s, v0[1] * s, v1[0] * s, v1[1] * s,
                        v2[0] * s, v2[1] * s, v3[0] * s, v3[1] * s};
    if constexpr (OUT_BF16) {
      uint16_t* p = static_cast<uint16_t*>(a.out) + row * a.out_ld + c;
      if (VEC && c + 8 <= a.cols) {
        nt_u32x4 o;
#pragma unroll
        for (int t = 0; t < 4; ++t)
          o[t] = mx_to_bf16(v[2 * t]) | static_cast<uint32_t>(mx_to_bf16(v[2 * t + 1])) << 16;
        *reinterpret_cast<nt_u32x4*>(p) = o;
      } else {
#pragma unroll
        for (int t = 0; t < 8; ++t)
          if (c + t < a.cols) p[t] = mx_to_bf16(v[t]);
      }
    } else {
      float* p = static_cast<float*>(a.out) + row * a.out_ld + c;
      if (VEC && c + 8 <= a.cols) {
        reinterpret_cast<nt_f32x4*>(p)[0] = nt_f32x4{v[0], v[1], v[2], v[3]};
        reinterpret_cast<nt_f32x4*>(p)[1] = nt_f32x4{v[4], v[5], v[6], v[7]};
      } else {
#pragma unroll
        for (int t = 0; t < 8; ++t)
          if (c + t < a.cols) p[t] = v[t];
      }
    }
  }
}

__global__ __launch_bounds__(256) void mx4_zero_kernel(float* p, int64_t ld, int64_t rows,
                                                       int cols) {
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
    for (int c = threadIdx.x; c < cols; c += 256) p[r * ld + c] = 0.0f;
}

// ------------------------------------------------------------------ products

__device__ __forceinline__ float mx_finish(const Mx4Product& a, float acc, float b) {
  const float y = acc + b;
  return a.relu ? __builtin_elementwise_maximum(y, 0.0f) : y;  // keeps a NaN
}
// Four outputs of a row from o (a multiple of 4) on.
__device__ __forceinline__ void mx_drop4(const Mx4Product& a, uint64_t offset, int64_t row, int o,
                                         float* v) {
  const Words4 w = drop_words(a.drop, offset, a.row0 + static_cast<uint32_t>(row), o / 8);
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const bool keep = o & 4 ? drop_keeps(a.drop, w, t + 4) : drop_keeps(a.drop, w, t);
    v[t] = keep ? v[t] * a.drop.factor : 0.0f;
  }
}

// Four channels from o on of an output row.
template <bool OUT_BF16, bool VEC>
__device__ __forceinline__ void mx_store4(const Mx4Product& a, int64_t row, int o, const float* v) {
  if constexpr (OUT_BF16) {
    uint16_t* p = static_cast<uint16_t*>(a.out) + row * a.out_ld + o;
    if (VEC && o + 4 <= a.outs) {
      uint32_t w[2];
#pragma unroll
      for (int e = 0; e < 2; ++e)
        w[e] = mx_to_bf16(v[2 * e]) | static_cast<uint32_t>(mx_to_bf16(v[2 * e + 1])) << 16;
      *reinterpret_cast<nt_u32x2*>(p) = nt_u32x2{w[0], w[1]};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (o + e < a.outs) p[e] = mx_to_bf16(v[e]);
    }
  } else {
    float* p = static_cast<float*>(a.out) + row * a.out_ld + o;
    if (VEC && o + 4 <= a.outs) {
      *reinterpret_cast<nt_f32x4*>(p) = nt_f32x4{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (o + e < a.outs) p[e] = v[e];
    }
  }
}

// Two values in bf16, rounded to nearest even, by the one instruction there is for it.
__device__ __forceinline__ uint32_t mx_bf16_pair(float lo, float hi) {
  typedef __bf16 pair __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((mx_f32x2{lo, hi}), pair));
}
// 16 bytes of an output row in its type, from channel o on.
template <bool OUT_BF16, bool VEC>
__device__ __forceinline__ void mx_store16(const Mx4Product& a, int64_t row, int o, nt_u32x4 w) {
  constexpr int N = OUT_BF16 ? 8 : 4;
  if constexpr (OUT_BF16) {
    uint16_t* p = static_cast<uint16_t*>(a.out) + row * a.out_ld + o;
    if (VEC && o + N <= a.outs) {
      __builtin_nontemporal_store(w, reinterpret_cast<nt_u32x4*>(p));
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (o + e < a.outs) p[e] = static_cast<uint16_t>(w[e >> 1] >> (16 * (e & 1)));
    }
  } else {
    uint32_t* p = static_cast<uint32_t*>(a.out) + row * a.out_ld + o;
    if (VEC && o + N <= a.outs) {
      __builtin_nontemporal_store(w, reinterpret_cast<nt_u32x4*>(p));
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (o + e < a.outs) p[e] = w[e];
    }
  }
}

template <int BYTE>
__device__ __forceinline__ nt_f32x16 mx_mfma(nt_u32x4 a, nt_u32x4 b, nt_f32x16 c, uint32_t sa,
                                             uint32_t sb) {
  const mx_i32x8 x = {static_cast<int>(a[0]), static_cast<int>(a[1]), static_cast<int>(a[2]),
                      static_cast<int>(a[3]), 0, 0, 0, 0};
  const mx_i32x8 y = {static_cast<int>(b[0]), static_cast<int>(b[1]), static_cast<int>(b[2]),
                      static_cast<int>(b[3]), 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, BYTE,
                                                         static_cast<int>(sa), BYTE,
                                                         static_cast<int>(sb));
}

// Workgroup tile: BM x BN outputs, WM x WN waves.  A stage is 128 bytes of a row, 256
// entries of K; RING stages in LDS, and scales for two stages each.
template <int BM_, int BN_, int WM_, int WN_, int RING_>
struct MxShape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, RING = RING_;
  static constexpr int NT = 64 * WM * WN, MI = BM / WM / 32, NJ = BN / WN / 32;
  static constexpr int STAGE = (BM + BN) * NT_BLOCK, SCALES = (BM + BN) * 16;
  static constexpr int PARTS = RING / 2 + 1;  // of scales, in LDS
  static constexpr int LDS_BYTES = RING * STAGE + PARTS * SCALES;
  static constexpr int LOADS = STAGE / 16 / NT;                           // of a wave and stage
  static constexpr int EU = NT / 256 * (LDS_BYTES > (80 << 10) ? 1 : 2);  // waves of a SIMD
  static_assert(BM % (32 * WM) == 0 && BN % (32 * WN) == 0, "whole blocks");
  static_assert(BM % 64 == 0 && BN % 64 == 0 && BM + BN <= NT, "a row of scales a lane");
};
typedef MxShape<256, 256, 2, 4, 2> MxL;
typedef MxShape<128, 128, 2, 2, 2> MxM;
typedef MxShape<64, 64, 2, 2, 4> MxS;
static_assert(mx4_threads(256) == MxL::NT && mx4_threads(128) == MxM::NT &&
                  mx4_threads(64) == MxS::NT,
              "mx4_plan.h");

// p and bytes are the same for the wave; where the compiler computes them on the vector unit
// (64-bit comparisons are its), it would loop over the lanes' buffers around every load.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t mx_buffer(const uint8_t* p, int64_t bytes) {
  const int n = static_cast<int>(bytes < 0xFFFFFFFFll ? bytes : 0xFFFFFFFFll);
  const uint64_t at = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(at));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(at >> 32));
  return __builtin_amdgcn_make_buffer_rsrc(
      reinterpret_cast<void*>(static_cast<uint64_t>(hi) << 32 | lo), 0,
      __builtin_amdgcn_readfirstlane(n), 0x00020000u);
}
typedef __attribute__((address_space(3))) void* mx_lds;

// Rows and scales of a tile's operands as buffers that end behind the last row: what
// lies behind it reads as zeros.  A row's place is in the vector offset, which is checked
// against the buffer's end; the scalar offset, the place in the row, need not be.
struct MxTile {
  __amdgpu_buffer_rsrc_t a, b, scales;
};
// The part of the addresses that is the same for every tile.  A lane's 16 bytes of a
// stage: row r, chunk p at LDS byte 128 r + 16 p holds chunk p ^ turn(r) of the row:
// 16 consecutive rows' chunks lie in different banks.
__device__ __forceinline__ int mx_turn(int r) { return (r ^ ((r >> 3) & 3)) & 7; }
template <class S>
struct MxPlace {
  static constexpr int PA = S::BM * 8 / S::NT, PB = S::BN * 8 / S::NT, STEP = S::NT / 8;
  static_assert(STEP % 32 == 0, "the same turn in every part");
  int a, a_step, b, b_step, scales;
  __device__ __forceinline__ MxPlace(const Mx4Product& p, int tid, int wave) {
    const int r = tid / 8, c = 16 * ((tid % 8) ^ mx_turn(r));
    a = static_cast<int>(r * p.w_ld) + c;
    b = static_cast<int>(r * p.x_ld) + c;
    a_step = static_cast<int>(STEP * p.w_ld);
    b_step = static_cast<int>(STEP * p.x_ld);
    // a row a lane, A's rows and then B's
    scales = static_cast<int>(64 * wave < S::BM ? tid * p.ws_ld : (tid - S::BM) * p.xs_ld);
  }
};
__device__ __forceinline__ nt_u32x4 mx_read(const char* tile, int row, int chunk) {
  return *reinterpret_cast<const nt_u32x4*>(tile + row * NT_BLOCK + 16 * (chunk ^ mx_turn(row)));
}

// Sums of parts, workgroup `index` of NT threads: NT / 8 columns, every eighth part a thread.
template <int NT>
__device__ __forceinline__ void mx_sums(const Mx4Sums& a, int index, char* lds) {
  constexpr int COLS = NT / 8;
  double* some = reinterpret_cast<double*>(lds);
  const int l = threadIdx.x % COLS, k = threadIdx.x / COLS, c = index * COLS + l;
  double s = 0.0;
  if (c < a.cols)
#pragma unroll 4
    for (int64_t i = k; i < a.parts; i += 8) s += a.part[i * a.cols + c];
  some[k * COLS + l] = s;
  __syncthreads();
  if (k == 0 && c < a.cols) {
    double all = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) all += some[i * COLS + l];
    a.out[c] = static_cast<float>(all);
  }
}
unsigned sums_grid(const Mx4Sums& a, int threads) {
  return a.parts > 0 ? static_cast<unsigned>((a.cols + threads / 8 - 1) / (threads / 8)) : 0u;
}

// A wave's 32 x 32 block of sums into outputs: acc[4 q + t] is channel o + 8 q + 4 h + t
// (h: the lane's half of the wave) of row `row`.
__device__ __forceinline__ void mx_epilogue(const Mx4Product& a, uint64_t offset, int64_t row,
                                            int o, int h, const nt_f32x4 (&bias)[4],
                                            const nt_f32x16& acc, float (&v)[16]) {
#pragma unroll
  for (int e = 0; e < 16; ++e) v[e] = mx_finish(a, acc[e], bias[e >> 2][e & 3]);
  if (a.drop.below) {
    // eight channels share a call of the generator, and four of them are the other half's:
    // each half makes one of two calls, and they swap words
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const Words4 w = drop_words(a.drop, offset, a.row0 + static_cast<uint32_t>(row), o / 8 + 2 * p + h);
      const auto x = __builtin_amdgcn_permlane32_swap(w.w[0], w.w[2], false, false);
      const auto y = __builtin_amdgcn_permlane32_swap(w.w[1], w.w[3], false, false);
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const uint32_t lo = x[q], hi = y[q];
        float* u = v + 4 * (2 * p + q);
        u[0] = (lo & 0xFFFFu) >= a.drop.below ? u[0] * a.drop.factor : 0.0f;
        u[1] = lo >> 16 >= a.drop.below ? u[1] * a.drop.factor : 0.0f;
        u[2] = (hi & 0xFFFFu) >= a.drop.below ? u[2] * a.drop.factor : 0.0f;
        u[3] = hi >> 16 >= a.drop.below ? u[3] * a.drop.factor : 0.0f;
      }
    }
  }
}

// Four channels 8 q + 4 h .. + 3 of each of a block's four q.
__device__ __forceinline__ void mx_bias(const Mx4Product& a, int o, int h, nt_f32x4 (&bias)[4]) {
  if (a.bias && o + 32 <= a.outs) {
    // the same for the wave but for its halves: loaded by the scalar unit
    const auto* p = (const __attribute__((address_space(4))) float*)(a.bias + o);
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float lo = p[8 * q + t], hi = p[8 * q + 4 + t];
        bias[q][t] = h ? hi : lo;
      }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int c = o + 8 * q + 4 * h + t;
        bias[q][t] = a.bias ? a.bias[c < a.outs ? c : a.outs - 1] : 0.0f;
      }
  }
}

// Output rows are input rows; the tile's own rows (A's) are output channels, four
// consecutive ones a lane.
// The last products of a stage are issued behind the barrier that ends it, with the
// next stage's first operands on their way; then the loads into the stage that is
// free go out, a whole stage ahead.  The empty asm keeps each group's products where
// they are written: without it they sink below the loads of the groups behind
// them, whose operands then do not fit the registers (8192 x 4096 x 4096: 139 us instead
// of 78).  A 256 x 256 tile's stage takes 2900 cycles, where two waves' 32 products are
// 2048, and a tile 2.4 us until its first stage is there and 4.6 for its outputs.  The
// clock goes by the operands' bits: 1.6 to 1.8 GHz on random ones, 2.37 on zeros, which
// take as many cycles (76 and 58 us; instructions from registers alone 6.5 and 9.7 PFLOP/s
// at 1.63 and 2.38 GHz); 70.5 us where half of x is zeros.  Tried when the kernel took 78:
// stages of 64 bytes, four of them in LDS, 88 us; four waves of 128 x 128 outputs 87;
// workgroups that take one tile after the other, the next one's loads ahead of the stores,
// 76, but 55 instead of 51 where there is one tile a CU.
// Of a stage's eight chunks a lane takes 4 h + c in group c (h: its half of the wave), so
// that its four scales are neighbouring bytes and the instruction picks byte c.  The order
// of K within a stage is free, both operands have the same.  Scales come in parts of
// 16 bytes a row, two stages'.
// VEC: 16-byte stores.
template <class S, bool OUT_BF16, bool VEC>
__global__ __launch_bounds__(S::NT, S::EU) void mx4_product_kernel(Mx4Product a) {
#if defined(__HIP_DEVICE_COMPILE__)  // buffer resources: no host form
  constexpr int ABYTES = S::BM * NT_BLOCK, ES = OUT_BF16 ? 2 : 4;
  __shared__ __attribute__((aligned(16))) char lds[S::LDS_BYTES];
  char* const scales = lds + S::RING * S::STAGE;
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, r = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int am = (wave / S::WN) * 32 * S::MI, bm = (wave % S::WN) * 32 * S::NJ;
  const int tr = (a.outs + S::BM - 1) / S::BM;
  const int tc = static_cast<int>((a.rows + S::BN - 1) / S::BN);
  if (static_cast<int>(blockIdx.x) >= tr * tc) {
    mx_sums<S::NT>(a.sums, blockIdx.x - tr * tc, lds);
    return;
  }
  int r0;
  int64_t c0;
  {  // the workgroups of one XCD (index mod 8) take neighbouring tiles
    const int total = tr * tc, per = total >> 3, rem = total & 7;
    const int x = blockIdx.x & 7, q = blockIdx.x >> 3;
    const int id = x * per + (x < rem ? x : rem) + q;
    // bands of four tile columns (rows of the input), channel tile by channel tile
    constexpr int BAND = 4;
    const int band = id / (BAND * tr), cols = tc - band * BAND < BAND ? tc - band * BAND : BAND;
    const int in_band = id - band * BAND * tr;
    r0 = (in_band / cols) * S::BM;
    c0 = static_cast<int64_t>(band * BAND + in_band % cols) * S::BN;
  }
  const int blocks = (a.in + 255) / 256;
  const MxPlace<S> at(a, tid, wave);
  MxTile t;
  {
    const int64_t left = a.rows - c0, qb = mx4_bytes(a.in), sb = mx4_scales(a.in);
    const int nb = __builtin_amdgcn_readfirstlane(static_cast<int>(left < S::BN ? left : S::BN));
    const int na = a.outs - r0 < S::BM ? a.outs - r0 : S::BM;
    const bool first = 64 * wave < S::BM;
    t.a = mx_buffer(a.wq + r0 * a.w_ld, (na - 1) * a.w_ld + qb);
    t.b = mx_buffer(a.xq + c0 * a.x_ld, (nb - 1) * a.x_ld + qb);
    t.scales = mx_buffer(first ? a.ws + r0 * a.ws_ld : a.xs + c0 * a.xs_ld,
                         first ? (na - 1) * a.ws_ld + sb : (nb - 1) * a.xs_ld + sb);
  }
  // stage s, and with an even one its part of the scales
  auto issue = [&](int s) {
    if (s >= blocks) return;
    char* to = lds + s % S::RING * S::STAGE + wave * 1024;
    const int k = s * NT_BLOCK;
#pragma unroll
    for (int p = 0; p < MxPlace<S>::PA; ++p)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(t.a, (mx_lds)(to + S::NT * 16 * p), 16,
                                               at.a + p * at.a_step, k, 0, 0);
#pragma unroll
    for (int p = 0; p < MxPlace<S>::PB; ++p)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(t.b, (mx_lds)(to + ABYTES + S::NT * 16 * p), 16,
                                               at.b + p * at.b_step, k, 0, 0);
    if ((s & 1) == 0 && 64 * wave < S::BM + S::BN)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          t.scales, (mx_lds)(scales + (s >> 1) % S::PARTS * S::SCALES + wave * 1024), 16,
          at.scales, 8 * s, 0, 0);
  };
  auto load = [&](int s, int c, nt_u32x4(&fa)[S::MI], nt_u32x4(&fb)[S::NJ]) {
    const char* from = lds + s % S::RING * S::STAGE;
#pragma unroll
    for (int i = 0; i < S::MI; ++i) fa[i] = mx_read(from + (am + 32 * i) * NT_BLOCK, r, 4 * h + c);
#pragma unroll
    for (int j = 0; j < S::NJ; ++j)
      fb[j] = mx_read(from + ABYTES + (bm + 32 * j) * NT_BLOCK, r, 4 * h + c);
  };
  auto load_scales = [&](int s, uint32_t(&sa)[S::MI], uint32_t(&sb)[S::NJ]) {
    const char* from = scales + (s >> 1) % S::PARTS * S::SCALES + 16 * r + 8 * (s & 1) + 4 * h;
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
      sa[i] = *reinterpret_cast<const uint32_t*>(from + (am + 32 * i) * 16);
#pragma unroll
    for (int j = 0; j < S::NJ; ++j)
      sb[j] = *reinterpret_cast<const uint32_t*>(from + (S::BM + bm + 32 * j) * 16);
  };
  uint32_t sa[2][S::MI], sb[2][S::NJ];
  nt_u32x4 fa[2][S::MI], fb[2][S::NJ];
  nt_f32x16 acc[S::MI][S::NJ];
#pragma unroll
  for (int i = 0; i < S::MI; ++i)
#pragma unroll
    for (int j = 0; j < S::NJ; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
#pragma unroll
  for (int s = 0; s < S::RING; ++s) issue(s);
  if (S::RING <= blocks) nt_wait_vm<(S::RING - 1) * S::LOADS>();
  else nt_wait_vm<0>();
  nt_barrier();
  load(0, 0, fa[0], fb[0]);
  load_scales(0, sa[0], sb[0]);
  // a stage; its scales are sa[E], sb[E], the next one's go to the others
#define OSCARS_STAGE(STAGE, E)                                                                  \
  {                                                                                             \
    const int now = STAGE;                                                                      \
    _Pragma("unroll") for (int c = 0; c < 4; ++c) {                                             \
      if (c < 3) {                                                                              \
        load(now, c + 1, fa[(c + 1) & 1], fb[(c + 1) & 1]);                                     \
      } else {                                                                                  \
        /* the next stage is there, and this one read by every wave */                          \
        if (S::RING > 2 && now + S::RING <= blocks) nt_wait_vm<(S::RING - 2) * S::LOADS>();     \
        else nt_wait_vm<0>();                                                                   \
        nt_barrier();                                                                           \
        load(now + 1, 0, fa[0], fb[0]);                                                         \
        load_scales(now + 1, sa[1 - (E)], sb[1 - (E)]);                                         \
        issue(now + S::RING);                                                                   \
      }                                                                                         \
      __builtin_amdgcn_sched_barrier(0);                                                        \
      _Pragma("unroll") for (int i = 0; i < S::MI; ++i)                                         \
          _Pragma("unroll") for (int j = 0; j < S::NJ; ++j) {                                   \
        if (c == 0) acc[i][j] = mx_mfma<0>(fa[0][i], fb[0][j], acc[i][j], sa[E][i], sb[E][j]);  \
        if (c == 1) acc[i][j] = mx_mfma<1>(fa[1][i], fb[1][j], acc[i][j], sa[E][i], sb[E][j]);  \
        if (c == 2) acc[i][j] = mx_mfma<2>(fa[0][i], fb[0][j], acc[i][j], sa[E][i], sb[E][j]);  \
        if (c == 3) acc[i][j] = mx_mfma<3>(fa[1][i], fb[1][j], acc[i][j], sa[E][i], sb[E][j]);  \
      }                                                                                         \
      _Pragma("unroll") for (int i = 0; i < S::MI; ++i)                                         \
          _Pragma("unroll") for (int j = 0; j < S::NJ; ++j) asm volatile("" : "+v"(acc[i][j])); \
      __builtin_amdgcn_sched_barrier(0);                                                        \
    }                                                                                           \
  }
  int stage = 0;
  for (; stage + 1 < blocks; stage += 2) {
    OSCARS_STAGE(stage, 0)
    OSCARS_STAGE(stage + 1, 1)
  }
  if (stage < blocks) OSCARS_STAGE(stage, 0)
#undef OSCARS_STAGE

  // The outputs of 32 rows, two blocks of 32 channels of them where a wave has two, go through
  // LDS in their type, so that neighbouring lanes store whole lines of an output row.
  constexpr int WIDE = S::MI % 2 == 0 ? 2 : 1, TURN = 32 * WIDE * ES + 16;  // bytes of a row
  constexpr int PER = 16 / ES, LANES = 32 * WIDE / PER;  // channels of a lane, lanes of a row
  static_assert(S::LDS_BYTES >= S::WM * S::WN * 32 * TURN, "turned blocks");
  char* const turn = lds + wave * 32 * TURN;
  const uint64_t offset = a.drop.below ? drop_offset(a.drop) : 0;
  nt_barrier();  // the stages are read: LDS is free
#pragma unroll
  for (int i = 0; i < S::MI; i += WIDE) {
    const int o = r0 + am + 32 * i;
    if (o >= a.outs) continue;  // uniform over the wave
    nt_f32x4 bias[WIDE][4];
#pragma unroll
    for (int k = 0; k < WIDE; ++k) mx_bias(a, o + 32 * k, h, bias[k]);
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) {
      const int64_t row0 = c0 + bm + 32 * j;
      if (row0 >= a.rows) continue;  // uniform over the wave
#pragma unroll
      for (int k = 0; k < WIDE; ++k) {
        float v[16];
        mx_epilogue(a, offset, row0 + r, o + 32 * k, h, bias[k], acc[i + k][j], v);
        char* to = turn + r * TURN + (32 * k + 4 * h) * ES;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if constexpr (OUT_BF16)
            *reinterpret_cast<nt_u32x2*>(to + 8 * q * ES) =
                nt_u32x2{mx_bf16_pair(v[4 * q], v[4 * q + 1]),
                         mx_bf16_pair(v[4 * q + 2], v[4 * q + 3])};
          else
            *reinterpret_cast<nt_f32x4*>(to + 8 * q * ES) =
                nt_f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
        }
      }
      nt_wave_sync();
      const int mine = o + PER * (lane % LANES);
#pragma unroll
      for (int n = 0; n < 32; n += 64 / LANES) {
        const int64_t row = row0 + n + lane / LANES;
        const nt_u32x4 w = *reinterpret_cast<const nt_u32x4*>(
            turn + (n + lane / LANES) * TURN + 16 * (lane % LANES));
        if (row < a.rows && mine < a.outs) mx_store16<OUT_BF16, VEC>(a, row, mine, w);
      }
      nt_wave_sync();
    }
  }
#endif
}

// Few tiles: 32 x 32 outputs a workgroup, K dealt to its four waves block by block.
// A wave streams its blocks and their scales through LDS of its own (RING of them),
// into registers, and waits for no other wave until the four sums meet, in order.
constexpr int MX_SMALL_RING = 2;

// Up to two products in one launch, the second's workgroups behind the first's.
struct Mx4Pair {
  Mx4Product p[2];
  bool vec[2];
  int first, all;  // workgroups; p[0]'s sums are behind them
};
__global__ __launch_bounds__(256) void mx4_small_kernel(Mx4Pair both) {
#if defined(__HIP_DEVICE_COMPILE__)  // buffer resources: no host form
  constexpr int DATA = 64 * NT_BLOCK, STAGE = DATA + 512, RING = MX_SMALL_RING;
  __shared__ __attribute__((aligned(16))) char lds[4 * RING * STAGE];
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);  // scalar addresses below
  if (static_cast<int>(blockIdx.x) >= both.all) {
    mx_sums<256>(both.p[0].sums, blockIdx.x - both.all, lds);
    return;
  }
  const bool second = static_cast<int>(blockIdx.x) >= both.first;
  const Mx4Product& a = both.p[second];
  const int index = blockIdx.x - (second ? both.first : 0);
  const int tr = (a.outs + 31) / 32;
  const int r0 = index % tr * 32;
  const int64_t c0 = static_cast<int64_t>(index / tr) * 32;
  const int blocks = (a.in + 255) / 256;
  const int64_t left = a.rows - c0;
  const int here = static_cast<int>(left < 32 ? left : 32);
  NtRows<64, 32> ra, rb;
  const int64_t qb = mx4_bytes(a.in), sb = mx4_scales(a.in);
  ra.init(a.wq, a.w_ld, (a.outs - 1) * a.w_ld + qb, r0, a.outs, lane);
  rb.init(a.xq + c0 * a.x_ld, a.x_ld, (here - 1) * a.x_ld + qb, 0, here, lane);
  // a block's scales: 8 bytes a row, four of them a lane
  const int na = a.outs - r0 < 32 ? a.outs - r0 : 32;
  const __amdgpu_buffer_rsrc_t rsa = mx_buffer(a.ws + r0 * a.ws_ld, (na - 1) * a.ws_ld + sb);
  const __amdgpu_buffer_rsrc_t rsb = mx_buffer(a.xs + c0 * a.xs_ld, (here - 1) * a.xs_ld + sb);
  const int row = lane & 31;
  const int va = static_cast<int>((row < na ? row : na - 1) * a.ws_ld) + 4 * h;
  const int vb = static_cast<int>((row < here ? row : here - 1) * a.xs_ld) + 4 * h;
  char* ring = lds + wave * RING * STAGE;
  auto issue = [&](int i) {  // the wave's block i
    const int k = wave + 4 * i;
    char* t = ring + (i % RING) * STAGE;
    const int block = k < blocks ? k : blocks - 1;
    ra.issue(t, block * NT_BLOCK, lane);
    rb.issue(t + DATA / 2, block * NT_BLOCK, lane);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsa, (mx_lds)(t + DATA), 4, va, block * 8, 0, 0);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsb, (mx_lds)(t + DATA + 256), 4, vb, block * 8, 0,
                                             0);
  };
  nt_f32x16 acc;
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
  constexpr int PER = NtRows<64, 32>::P * 2 + 2;
  for (int i = 0; i < RING; ++i) issue(i);
  for (int i = 0; wave + 4 * i < blocks; ++i) {
    nt_wait_vm<(RING - 1) * PER>();
    const char* ta = ring + (i % RING) * STAGE;
    const char* tb = ta + DATA / 2;
    nt_u32x4 fa[4], fb[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      fa[c] = nt_read(ta, lane & 31, 4 * h + c);
      fb[c] = nt_read(tb, lane & 31, 4 * h + c);
    }
    const uint32_t sa = *reinterpret_cast<const uint32_t*>(ta + DATA + 4 * lane);
    const uint32_t sb4 = *reinterpret_cast<const uint32_t*>(ta + DATA + 256 + 4 * lane);
    // the stage is in registers: refill it
    __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4));  // lgkmcnt(0)
    asm volatile("" ::: "memory");
    issue(i + RING);
    acc = mx_mfma<0>(fa[0], fb[0], acc, sa, sb4);
    acc = mx_mfma<1>(fa[1], fb[1], acc, sa, sb4);
    acc = mx_mfma<2>(fa[2], fb[2], acc, sa, sb4);
    acc = mx_mfma<3>(fa[3], fb[3], acc, sa, sb4);
  }
  nt_wait_vm<0>();
  __syncthreads();  // every wave is through with LDS: now the four sums
  float* sums = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int e = 0; e < 16; ++e) sums[(wave * 16 + e) * 64 + lane] = acc[e];
  __syncthreads();
  // wave w finishes channels 8 w + 4 h .. + 3 of row (lane & 31)
  const int o = r0 + 8 * wave + 4 * h;
  const int64_t r = c0 + row;
  if (r >= a.rows || o >= a.outs) return;
  float v[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) s += sums[(w * 16 + 4 * wave + t) * 64 + lane];
    const int oc = o + t < a.outs ? o + t : a.outs - 1;
    v[t] = mx_finish(a, s, a.bias ? a.bias[oc] : 0.0f);
  }
  if (a.drop.below) mx_drop4(a, drop_offset(a.drop), r, o, v);
  const bool vec = both.vec[second];
  if (a.out_bf16) {
    if (vec) mx_store4<true, true>(a, r, o, v);
    else mx_store4<true, false>(a, r, o, v);
  } else {
    if (vec) mx_store4<false, true>(a, r, o, v);
    else mx_store4<false, false>(a, r, o, v);
  }
#endif
}

bool aligned_rows(const void* p, int64_t row_bytes, int to) {
  return reinterpret_cast<uintptr_t>(p) % to == 0 && row_bytes % to == 0;
}
bool out_aligned(const Mx4Product& a) {
  return aligned_rows(a.out, a.out_ld * (a.out_bf16 ? 2 : 4), 16);
}
unsigned product_grid(const Mx4Product& a, int tile) {
  return static_cast<unsigned>((a.outs + tile - 1) / tile * ((a.rows + tile - 1) / tile));
}

hipError_t small_launch(const Mx4Product* p, int n, hipStream_t s) {
  Mx4Pair both{};
  unsigned grid = 0;
  for (int i = 0; i < n; ++i) {
    both.p[i] = p[i];
    both.vec[i] = out_aligned(p[i]);
    if (i == 0) both.first = static_cast<int>(product_grid(p[0], 32));
    grid += product_grid(p[i], 32);
  }
  both.all = static_cast<int>(grid);
  hipLaunchKernelGGL(mx4_small_kernel, dim3(grid + sums_grid(p[0].sums, 256)), dim3(256), 0, s,
                     both);
  return hipGetLastError();
}

template <bool OUT_BF16, bool VEC>
hipError_t product_launch(const Mx4Product& a, int tile, hipStream_t s) {
  if (tile == 32) return small_launch(&a, 1, s);
  const dim3 grid(product_grid(a, tile) + sums_grid(a.sums, mx4_threads(tile)));
  if (tile == 256)
    hipLaunchKernelGGL((mx4_product_kernel<MxL, OUT_BF16, VEC>), grid, dim3(MxL::NT), 0, s, a);
  else if (tile == 128)
    hipLaunchKernelGGL((mx4_product_kernel<MxM, OUT_BF16, VEC>), grid, dim3(MxM::NT), 0, s, a);
  else
    hipLaunchKernelGGL((mx4_product_kernel<MxS, OUT_BF16, VEC>), grid, dim3(MxS::NT), 0, s, a);
  return hipGetLastError();
}

// ------------------------------------------------------------------ a few rows

// Up to 32 rows.  A workgroup takes 16 output channels, its eight waves slices of 512
// of K in turn: four 16x16x128 instructions for each 16 rows, lane l channel or row l & 15,
// block l >> 4 of 128 entries.  While the weights are on their way every workgroup
// quantises all rows into LDS for itself (they come from the L2).  The eight partial
// sums meet in LDS, in order.  One row of 4096 by 4096 outputs: 4.8 us.
constexpr int FEW_ROWS = 32;
constexpr int FEW_WAVES = 8;
// Every workgroup quantises all rows: up to so many entries that is less than a launch of
// its own takes.  One row is taken at any length.
constexpr int FEW_ENTRIES = 16384;

__host__ __device__ __forceinline__ int few_row_bytes(int in) {
  return (in + 511) / 512 * 256 + 16;  // 16 more: consecutive rows start in other banks
}
__host__ __device__ __forceinline__ int few_row_scales(int in) { return (in + 511) / 512 * 16; }
// quantised rows and scales: FEW_ENTRIES of FEW_ROWS rows, or 65536 of one
constexpr int FEW_LDS_S = 18 << 10, FEW_LDS_L = 35 << 10;

template <int LDS, bool X_BF16, bool VEC, bool OUT_BF16, bool TWO>
__global__ __launch_bounds__(64 * FEW_WAVES) void mx4_few_kernel(Mx4Product a, const void* x,
                                                                 int64_t x_ld) {
  constexpr int HALVES = TWO ? 2 : 1;  // of 16 rows
  __shared__ __attribute__((aligned(16))) char few_lds[LDS];
  __shared__ float part[HALVES][FEW_WAVES][64][4];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rows = static_cast<int>(a.rows), in = a.in, ld = few_row_bytes(in);
  const int sld = few_row_scales(in), slices = (in + 511) / 512;
  char* scales = few_lds + rows * ld;
  const int ch = blockIdx.x * 16 + (lane & 15), chc = ch < a.outs ? ch : a.outs - 1;
  const int g = lane >> 4;
  const uint8_t* w = a.wq + chc * a.w_ld + 16 * g;
  const uint8_t* ws = a.ws + chc * a.ws_ld;
  const int64_t qb = mx4_bytes(in);
  nt_u32x4 cur[4], cur_s;
  auto load_w = [&](int sl) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      // the second half of the last slice may not be there: zeros of x meet the first's
      const int at = sl * 256 + 64 * c;
      cur[c] = *reinterpret_cast<const nt_u32x4*>(w + (at + 64 <= qb ? at : at - 128));
    }
    cur_s = *reinterpret_cast<const nt_u32x4*>(ws + sl * 16);
  };
  if (wave < slices) load_w(wave);
  // the rows, eight entries a thread, four threads a block
  const int per = slices * 64;  // threads' work of a row
  for (int i = tid; i < rows * per; i += 64 * FEW_WAVES) {
    const int r = i / per, c = 8 * (i - r * per);
    float v[8];
    mx_load8<X_BF16, VEC>(static_cast<const char*>(x) + r * x_ld * (X_BF16 ? 2 : 4), c, in, v);
    mx_clip8<VEC>(c, in, v);
    uint32_t top = mx_top8(v);
    top = max(top, static_cast<uint32_t>(__shfl_xor(top, 1)));
    top = max(top, static_cast<uint32_t>(__shfl_xor(top, 2)));
    const MxScale s = mx_scale(top);
    *reinterpret_cast<uint32_t*>(few_lds + r * ld + c / 2) = mx_pack8(v, s);
    if ((lane & 3) == 0) scales[r * sld + c / 32] = static_cast<char>(s.byte);
  }
  __syncthreads();
  nt_f32x4 acc[HALVES];
  const char *b[HALVES], *bs[HALVES];
#pragma unroll
  for (int n = 0; n < HALVES; ++n) {
    acc[n] = nt_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // lanes of rows that are not there read the last one; their sums are not used
    const int r = 16 * n + (lane & 15) < rows ? 16 * n + (lane & 15) : rows - 1;
    b[n] = few_lds + r * ld + 16 * g;
    bs[n] = scales + r * sld;
  }
  for (int sl = wave; sl < slices; sl += FEW_WAVES) {
    const nt_u32x4 wv[4] = {cur[0], cur[1], cur[2], cur[3]}, wsc = cur_s;
    if (sl + FEW_WAVES < slices) load_w(sl + FEW_WAVES);
#pragma unroll
    for (int n = 0; n < HALVES; ++n) {
      const nt_u32x4 xsc = *reinterpret_cast<const nt_u32x4*>(bs[n] + sl * 16);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const nt_u32x4 xv = *reinterpret_cast<const nt_u32x4*>(b[n] + sl * 256 + 64 * c);
        const mx_i32x8 p = {static_cast<int>(wv[c][0]), static_cast<int>(wv[c][1]),
                            static_cast<int>(wv[c][2]), static_cast<int>(wv[c][3]), 0, 0, 0, 0};
        const mx_i32x8 q = {static_cast<int>(xv[0]), static_cast<int>(xv[1]),
                            static_cast<int>(xv[2]), static_cast<int>(xv[3]), 0, 0, 0, 0};
        // the lane's scale to the lowest byte
        acc[n] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
            p, q, acc[n], 4, 4, 0, static_cast<int>(wsc[c] >> (8 * g)), 0,
            static_cast<int>(xsc[c] >> (8 * g)));
      }
    }
  }
#pragma unroll
  for (int n = 0; n < HALVES; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) part[n][wave][lane][e] = acc[n][e];
  __syncthreads();
  // lane l, element e: channel 4 (l >> 4) + e, row l & 15; a thread finishes one output
  if (tid < 256 * HALVES) {
    const int n = tid >> 8, e = tid & 3, l = (tid >> 2) & 63;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < FEW_WAVES; ++i) sum += part[n][i][l][e];
    const int q = 16 * n + (l & 15), o = blockIdx.x * 16 + 4 * (l >> 4) + e;
    if (q < rows && o < a.outs) {
      float y = mx_finish(a, sum, a.bias ? a.bias[o] : 0.0f);
      if (a.drop.below) {
        const Words4 d = drop_words(a.drop, drop_offset(a.drop), q, o / 8);
        const uint32_t d01 = o & 2 ? d.w[1] : d.w[0], d23 = o & 2 ? d.w[3] : d.w[2];
        const uint32_t word = o & 4 ? d23 : d01;
        y = (o & 1 ? word >> 16 : word & 0xFFFFu) >= a.drop.below ? y * a.drop.factor : 0.0f;
      }
      if constexpr (OUT_BF16) static_cast<uint16_t*>(a.out)[q * a.out_ld + o] = mx_to_bf16(y);
      else static_cast<float*>(a.out)[q * a.out_ld + o] = y;
    }
  }
}

template <int LDS, bool X_BF16, bool VEC, bool TWO>
hipError_t few_launch(const Mx4Product& a, const void* x, int64_t x_ld, hipStream_t s) {
  const dim3 grid((a.outs + 15) / 16), wg(64 * FEW_WAVES);
  if (a.out_bf16)
    hipLaunchKernelGGL((mx4_few_kernel<LDS, X_BF16, VEC, true, TWO>), grid, wg, 0, s, a, x, x_ld);
  else
    hipLaunchKernelGGL((mx4_few_kernel<LDS, X_BF16, VEC, false, TWO>), grid, wg, 0, s, a, x, x_ld);
  return hipGetLastError();
}

template <bool X_BF16, bool VEC>
hipError_t few_launch(const Mx4Product& a, const void* x, int64_t x_ld, hipStream_t s) {
  if (a.rows > 16) return few_launch<FEW_LDS_S, X_BF16, VEC, true>(a, x, x_ld, s);
  return a.rows * (few_row_bytes(a.in) + few_row_scales(a.in)) <= FEW_LDS_S
             ? few_launch<FEW_LDS_S, X_BF16, VEC, false>(a, x, x_ld, s)
             : few_launch<FEW_LDS_L, X_BF16, VEC, false>(a, x, x_ld, s);
}

template <bool BF16, bool VEC>
hipError_t rows_launch(const Mx4Source& a, const Mx4Rows& to, hipStream_t s) {
  const int pieces = (a.cols + 511) / 512;
  const int64_t want = (a.rows * pieces + 3) / 4;
  const dim3 grid(static_cast<unsigned>(want < 4096 ? want : 4096)), wg(256);
  hipLaunchKernelGGL((mx4_rows_kernel<BF16, VEC>), grid, wg, 0, s, a, to, pieces);
  return hipGetLastError();
}

// How the gradient is made: 0 as it is, 1 with y, 2 with the generator.
int source_mode(const Mx4Source& a) { return a.y ? 1 : a.drop.below ? 2 : 0; }

template <bool BF16, bool VEC, int MODE>
hipError_t gradient_launch(const Mx4Columns& z, const Mx4Columns& x, bool both, unsigned grid,
                           int z_tiles, hipStream_t s) {
  if (both)
    hipLaunchKernelGGL((mx4_gradient_kernel<BF16, VEC, MODE, true>), dim3(grid), dim3(512), 0, s, z,
                       x, z_tiles);
  else
    hipLaunchKernelGGL((mx4_gradient_kernel<BF16, VEC, MODE, false>), dim3(grid), dim3(512), 0, s,
                       z, x, z_tiles);
  return hipGetLastError();
}
template <bool BF16, bool VEC>
hipError_t gradient_launch(const Mx4Columns& z, const Mx4Columns& x, bool both, unsigned grid,
                           int z_tiles, hipStream_t s) {
  const int mode = source_mode(z.from);
  if (mode == 0) return gradient_launch<BF16, VEC, 0>(z, x, both, grid, z_tiles, s);
  if (mode == 1) return gradient_launch<BF16, VEC, 1>(z, x, both, grid, z_tiles, s);
  return gradient_launch<BF16, VEC, 2>(z, x, both, grid, z_tiles, s);
}

bool source_aligned(const Mx4Source& a, int to) {
  const int64_t es = a.bf16 ? 2 : 4;
  return aligned_rows(a.x, a.x_ld * es, to) && (!a.y || aligned_rows(a.y, a.y_ld * es, to));
}
bool pairs_aligned(const Mx4Source& a) {
  return a.cols % 2 == 0 && source_aligned(a, a.bf16 ? 4 : 8);
}

}  // namespace

hipError_t launch_mx4_rows(const Mx4Source& a, const Mx4Rows& to, hipStream_t s) {
  const bool vec = a.cols % 8 == 0 && source_aligned(a, 16);
  if (a.bf16) return vec ? rows_launch<true, true>(a, to, s) : rows_launch<true, false>(a, to, s);
  return vec ? rows_launch<false, true>(a, to, s) : rows_launch<false, false>(a, to, s);
}

int64_t mx4_column_tiles(int64_t rows, int cols) {
  return mx_row_tiles(rows) * mx_column_tiles(cols, false);
}

hipError_t launch_mx4_columns(const Mx4Source& a, const Mx4Rows& to, hipStream_t s) {
  const bool vec = pairs_aligned(a);
  const dim3 grid(static_cast<unsigned>(mx4_column_tiles(a.rows, a.cols))), wg(512);
  const Mx4Columns p{a, to, Mx4Rows{}, nullptr, nullptr};
  if (a.bf16) {
    if (vec) hipLaunchKernelGGL((mx4_columns_kernel<true, true>), grid, wg, 0, s, p);
    else hipLaunchKernelGGL((mx4_columns_kernel<true, false>), grid, wg, 0, s, p);
  } else {
    if (vec) hipLaunchKernelGGL((mx4_columns_kernel<false, true>), grid, wg, 0, s, p);
    else hipLaunchKernelGGL((mx4_columns_kernel<false, false>), grid, wg, 0, s, p);
  }
  return hipGetLastError();
}

int64_t mx4_sum_parts(int64_t rows) {
  const int64_t n = mx_row_tiles(rows);
  return n > 1 ? n : 0;
}

hipError_t launch_mx4_gradient(const Mx4Gradient& g, hipStream_t s) {
  const bool both = g.z_rows.q != nullptr;
  const bool vec = pairs_aligned(g.z) && pairs_aligned(g.x);
  const int64_t parts = mx4_sum_parts(g.z.rows);
  const Mx4Columns z{g.z, g.z_columns, g.z_rows, g.sums, parts ? g.part : nullptr};
  const Mx4Columns x{g.x, g.x_columns, Mx4Rows{}, nullptr, nullptr};
  const int64_t nz = mx_row_tiles(g.z.rows) * mx_column_tiles(g.z.cols, both);
  const unsigned grid = static_cast<unsigned>(nz + mx4_column_tiles(g.x.rows, g.x.cols));
  const int z_tiles = static_cast<int>(nz);
  if (g.z.bf16)
    return vec ? gradient_launch<true, true>(z, x, both, grid, z_tiles, s)
               : gradient_launch<true, false>(z, x, both, grid, z_tiles, s);
  return vec ? gradient_launch<false, true>(z, x, both, grid, z_tiles, s)
             : gradient_launch<false, false>(z, x, both, grid, z_tiles, s);
}

hipError_t launch_mx4_values(const Mx4Values& a, hipStream_t s) {
  const uint32_t groups = static_cast<uint32_t>((static_cast<int64_t>(a.cols) + 7) / 8);
  const int64_t want = (a.rows * groups + 255) / 256;
  const dim3 grid(static_cast<unsigned>(want < 8192 ? want : 8192));
  const bool vec = aligned_rows(a.out, a.out_ld * (a.out_bf16 ? 2 : 4), 16);
#define OSCARS_VALUES(B, V) \
  hipLaunchKernelGGL((mx4_values_kernel<B, V>), grid, dim3(256), 0, s, a, groups)
  if (a.out_bf16) {
    if (vec) OSCARS_VALUES(true, true);
    else OSCARS_VALUES(true, false);
  } else {
    if (vec) OSCARS_VALUES(false, true);
    else OSCARS_VALUES(false, false);
  }
#undef OSCARS_VALUES
  return hipGetLastError();
}

hipError_t launch_mx4_product(const Mx4Product& args, hipStream_t s) {
  const bool vec = out_aligned(args);
  hipError_t e = hipSuccess;
  mx4_launches(args.rows, args.in, args.outs, [&](int tile, int64_t at, int64_t rows) {
    Mx4Product a = args;
    a.rows = rows;
    a.xq += at * a.x_ld;
    a.xs += at * a.xs_ld;
    a.out = static_cast<char*>(a.out) + at * a.out_ld * (a.out_bf16 ? 2 : 4);
    a.row0 = static_cast<uint32_t>(at);
    if (at > 0) a.sums.parts = 0;
    if (a.out_bf16)
      e = vec ? product_launch<true, true>(a, tile, s) : product_launch<true, false>(a, tile, s);
    else
      e = vec ? product_launch<false, true>(a, tile, s) : product_launch<false, false>(a, tile, s);
    return e == hipSuccess;
  });
  return e;
}

hipError_t launch_mx4_products(const Mx4Product* p, int n, hipStream_t s) {
  // in one launch of small tiles, where that is no slower than each as it would go alone
  double together = 3.0, alone = 0.0;
  int64_t tiles = 0;
  for (int i = 0; i < n; ++i) {
    const Mx4Plan best = mx4_plan(p[i].rows, p[i].in, p[i].outs);
    together += mx4_small_us(p[i].rows, p[i].in, p[i].outs) - 3.0;
    alone += best.us;
    tiles += (p[i].rows + 31) / 32 * ((p[i].outs + 31) / 32);
  }
  const bool small = together <= alone && tiles < (1 << 24);
  if (small) return small_launch(p, n, s);
  hipError_t e = hipSuccess;
  for (int i = 0; i < n && e == hipSuccess; ++i) e = launch_mx4_product(p[i], s);
  return e;
}

bool mx4_one_launch(int64_t rows, int in) {
  static_assert(FEW_LDS_S >= FEW_ENTRIES * 17 / 32 + FEW_ROWS * (256 + 32) &&
                    FEW_LDS_L >= 65536 / 512 * 272 + 16,
                "room for the rows");
  return rows == 1 || (rows <= FEW_ROWS && rows * in <= FEW_ENTRIES);
}

hipError_t launch_mx4_few(const Mx4Product& a, const void* x, int64_t x_ld, bool x_bf16,
                          hipStream_t s) {
  const bool vec = a.in % 8 == 0 && aligned_rows(x, x_ld * (x_bf16 ? 2 : 4), 16);
  if (x_bf16)
    return vec ? few_launch<true, true>(a, x, x_ld, s) : few_launch<true, false>(a, x, x_ld, s);
  return vec ? few_launch<false, true>(a, x, x_ld, s) : few_launch<false, false>(a, x, x_ld, s);
}

hipError_t launch_mx4_zero(float* p, int64_t ld, int64_t rows, int cols, hipStream_t s) {
  hipLaunchKernelGGL(mx4_zero_kernel, dim3(static_cast<unsigned>(rows < 4096 ? rows : 4096)),
                     dim3(256), 0, s, p, ld, rows, cols);
  return hipGetLastError();
}

}  // namespace oscars
