// Tile product C[r][c] = sum_k A[r][k] B[c][k] shared by the operators on the
// global model (orthogonalize.hip, int8_kernels.hip).
//
// Both operands are stored K-contiguous as rows of whole 128-byte blocks; a
// block is what one row takes of one K step, whatever the element type:
//   NT_I8      128 int8;
//   NT_F16     64 fp16;
//   NT_SPLIT   32 values as two fp16 each, hi = fp16(v) in the first 64 bytes,
//              lo = fp16(v - hi) in the last 64: 22 bits of mantissa.  A product
//              is hi hi + hi lo + lo hi (lo lo is below the 22 bits).
// The 16 bytes that a lane feeds a matrix instruction are 8 fp16 or 16 int8 and
// sit at the same place for all of them (row = lane & 31, 16-byte chunk 2 s +
// (lane >> 5) of K group s), so staging and LDS reads are the same code.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace oscars {

typedef float nt_f32x4 __attribute__((ext_vector_type(4)));
typedef float nt_f32x16 __attribute__((ext_vector_type(16)));
typedef int32_t nt_i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t nt_i32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t nt_u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t nt_u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 nt_f16x8 __attribute__((ext_vector_type(8)));

enum NtFormat { NT_I8 = 0, NT_F16 = 1, NT_SPLIT = 2, NT_SPLIT_B0 = 3 };  // B0: B's lo are zero

constexpr int NT_BLOCK = 128;  // bytes of a row per K step

template <int F> struct NtAcc { typedef nt_f32x16 type; };
template <> struct NtAcc<NT_I8> { typedef nt_i32x16 type; };

template <int F>
__device__ __forceinline__ typename NtAcc<F>::type nt_mfma(nt_u32x4 a, nt_u32x4 b,
                                                           typename NtAcc<F>::type c) {
  if constexpr (F == NT_I8)
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(nt_i32x4, a),
                                                 __builtin_bit_cast(nt_i32x4, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(nt_f16x8, a),
                                                  __builtin_bit_cast(nt_f16x8, b), c, 0, 0, 0);
}

// Workgroup tile: BM x BN outputs, WM x WN waves, two stages in LDS.  EXACT, where
// there are registers for it: NT_SPLIT's products with a lo plane have accumulators
// of their own, added at the end.  Every product rounds the sum it goes into, and
// the small ones would round the large sum two more times.  Five Newton-Schulz
// steps in 128 x 128 tiles, error in the Frobenius norm, without and with: 1024 x
// 4096 1.70e-6 and 1.07e-6, 2048 x 2048 2.68e-6 and 1.55e-6, 2900 x 2950 2.91e-6 and
// 1.67e-6; the calls take 0.3 to 0.5% longer.
template <int BM_, int BN_, int WM_, int WN_, bool EXACT_ = false>
struct NtShape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
  static constexpr bool EXACT = EXACT_;
  static constexpr int NT = 64 * WM * WN, MI = BM / WM / 32, NJ = BN / WN / 32;
  static constexpr int LDS_BYTES = 2 * (BM + BN) * NT_BLOCK;
  static_assert(BM % (32 * WM) == 0 && BN % (32 * WN) == 0, "whole matrix blocks per wave");
};

// One operand's rows as a buffer: the resource starts at the tile's first row.
// A lane's 16 bytes of a stage: row r, chunk p at LDS byte 128 r + 16 p holds
// chunk p ^ ((r ^ r >> 3) & 7) of the row, so that both the reads of 32
// consecutive rows and the writes spread over the banks.  Rows past the last
// one read the last one again (their outputs are not stored).
template <int NTHR, int ROWS>
struct NtRows {
  static constexpr int P = ROWS * 8 / NTHR;
  static_assert(ROWS * 8 % NTHR == 0, "whole wave instructions");
  __amdgpu_buffer_rsrc_t rsrc;
  int voff[P];
  // base: row 0 of the operand; bytes: from base to the operand's end
  __device__ __forceinline__ void init(const void* base, int64_t ld, int64_t bytes, int row0,
                                       int rows, int tid) {
    const int64_t at = row0 * ld, left = bytes - at;
    rsrc = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char*>(static_cast<const char*>(base) + at), 0,
        static_cast<int>(left < 0x7FFFFFFF ? left : 0x7FFFFFFF), 0x00020000u);
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int idx = tid + NTHR * p, r = idx >> 3;
      const int c = (idx & 7) ^ ((r ^ (r >> 3)) & 7);
      const int rr = row0 + r < rows ? r : rows - 1 - row0;
      voff[p] = static_cast<int>(rr * ld) + 16 * c;
    }
  }
  // wave w's instruction p fills tile rows (64 w + NTHR p) / 8 .. + 7
  __device__ __forceinline__ void issue(char* tile, int kbyte, int tid, int p) const {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        rsrc, (__attribute__((address_space(3))) void*)(tile + ((tid & ~63) + NTHR * p) * 16), 16,
        voff[p], kbyte, 0, 0);
  }
  __device__ __forceinline__ void issue(char* tile, int kbyte, int tid) const {
#pragma unroll
    for (int p = 0; p < P; ++p) issue(tile, kbyte, tid, p);
  }
};

template <int N>
__device__ __forceinline__ void nt_wait_vm() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}
__device__ __forceinline__ void nt_barrier() {
  __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4));  // lgkmcnt(0)
  asm volatile("s_barrier" ::: "memory");
}

// Between a wave's stores to LDS and other lanes' loads of them, or the next stores:
// LDS operations of one wave execute in order, so it is the compiler alone that has
// to keep it (no instruction comes of the fences).
__device__ __forceinline__ void nt_wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

__device__ __forceinline__ nt_u32x4 nt_read(const char* tile, int row, int chunk) {
  return *reinterpret_cast<const nt_u32x4*>(tile + row * NT_BLOCK +
                                            16 * (chunk ^ ((row ^ (row >> 3)) & 7)));
}

// acc[i][j] += the tile's products over `blocks` K blocks.  lds: S::LDS_BYTES,
// free.  Ends with nothing in flight.
//
// A stage begins with a barrier and the first operands' way from LDS, and its loads
// (eight a wave, 16 bytes a lane) hold the wave up while they are issued: the L2
// gives a CU 64 bytes a cycle, 512 cycles for the stage of a 128 x 128 tile.  So
// the stage's last products are issued behind the barrier that ends it, with the
// next stage's first operands on their way, each group of products has the next
// group's operands loaded in front of it, and a 256 x 256 tile's loads go out in
// four parts between the groups.  TFLOP/s of matrix work of NT_SPLIT at 4096 x 4096
// x 4096, fp16 at 8192, int8 at 8192 x 4096 x 4096: in one run 1266, 996, 2022
// without all that and 1330, 1188, 2139 with the loads in one burst (torch's
// products: fp16 1393, int8 2122); in another, the card's clock 10% lower, 1103,
// 1072, 1980 in one burst and 1176, 1140, 2105 in parts.
// The stage of a 128 x 128 tile is too short for that: its later parts come too
// late (a call with 2048 x 2048 11% slower); three stages, one workgroup a CU,
// lose more with 512 tiles than they gain with 256.  Two such workgroups overlap;
// one alone (four waves on a CU) takes 0.67 us a block of NT_SPLIT, 0.50 without
// its loads, 0.59 without its LDS reads, 0.38 without both.
template <class S, int F, class RowsA, class RowsB, class Acc>
__device__ __forceinline__ void nt_tile(const RowsA& a, const RowsB& b, int blocks, char* lds,
                                        int tid, Acc (&acc)[S::MI][S::NJ]) {
  constexpr int ABYTES = S::BM * NT_BLOCK, STAGE = (S::BM + S::BN) * NT_BLOCK;
  constexpr bool SPLIT = F == NT_SPLIT || F == NT_SPLIT_B0, CROSS = S::EXACT && SPLIT;
  const int lane = tid & 63, wave = tid >> 6;
  const int arow = (wave / S::WN) * 32 * S::MI + (lane & 31);
  const int brow = (wave % S::WN) * 32 * S::NJ + (lane & 31), h = lane >> 5;
  static_assert(RowsA::P == 4 && RowsB::P == 4, "stages in four parts");
  constexpr bool SPREAD = S::NT == 512;
  auto issue = [&](int s) {
    char* t = lds + (s & 1) * STAGE;
    a.issue(t, s * NT_BLOCK, tid);
    b.issue(t + ABYTES, s * NT_BLOCK, tid);
  };
  auto issue_part = [&](int s, int part) {
    if (!SPREAD || s >= blocks) return;
    char* t = lds + (s & 1) * STAGE;
    a.issue(t, s * NT_BLOCK, tid, part);
    b.issue(t + ABYTES, s * NT_BLOCK, tid, part);
  };
  auto load_a = [&](const char* t, int c, nt_u32x4(&fa)[S::MI]) {
#pragma unroll
    for (int i = 0; i < S::MI; ++i) fa[i] = nt_read(t, arow + 32 * i, 2 * c + h);
  };
  auto load_b = [&](const char* t, int c, nt_u32x4(&fb)[S::NJ]) {
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) fb[j] = nt_read(t + ABYTES, brow + 32 * j, 2 * c + h);
  };

  // NT_SPLIT's products with a lo plane
  Acc cross[CROSS ? S::MI : 1][CROSS ? S::NJ : 1];
  if constexpr (CROSS) {
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
      for (int j = 0; j < S::NJ; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) cross[i][j][e] = 0;
  }
  auto& low = [&]() -> Acc(&)[S::MI][S::NJ] {
    if constexpr (CROSS) return cross;
    else return acc;
  }();
  // the scheduler keeps loads and products in the order written
  auto mul = [&](nt_u32x4(&fa)[S::MI], nt_u32x4(&fb)[S::NJ], Acc(&to)[S::MI][S::NJ]) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) to[i][j] = nt_mfma<F>(fa[i], fb[j], to[i][j]);
    __builtin_amdgcn_sched_barrier(0);
  };
  nt_u32x4 a0[S::MI], a1[S::MI], b0[S::NJ], b1[S::NJ], b2[S::NJ];
  issue(0);
  nt_wait_vm<0>();
  nt_barrier();
  if constexpr (SPREAD) issue_part(1, 0);
  else if (blocks > 1) issue(1);
  load_a(lds, 0, a0);
  load_b(lds, 0, b0);
  for (int s = 0; s < blocks; ++s) {
    const char* t = lds + (s & 1) * STAGE;
    const char* next = lds + ((s + 1) & 1) * STAGE;
    // what the last group multiplies is a1 and, of b, b2 (SPLIT) or b1
    if constexpr (SPLIT) {
      issue_part(s + 1, 1);
      if constexpr (F == NT_SPLIT) {
        load_b(t, 2, b1);
        mul(a0, b0, acc);  // hi hi, the first 16 of K
        issue_part(s + 1, 2);
        load_a(t, 2, a1);
        mul(a0, b1, low);  // hi lo
      } else {
        issue_part(s + 1, 2);
        load_a(t, 2, a1);
        mul(a0, b0, acc);
      }
      issue_part(s + 1, 3);
      load_a(t, 1, a0);
      load_b(t, 1, b2);
      mul(a1, b0, low);  // lo hi
      if constexpr (F == NT_SPLIT) {
        load_b(t, 3, b1);
        mul(a0, b2, acc);  // the second 16
        load_a(t, 3, a1);
        mul(a0, b1, low);
      } else {
        load_a(t, 3, a1);
        mul(a0, b2, acc);
      }
    } else {
      issue_part(s + 1, 1);
      load_a(t, 1, a1);
      load_b(t, 1, b1);
      mul(a0, b0, acc);
      issue_part(s + 1, 2);
      issue_part(s + 1, 3);
      load_a(t, 2, a0);
      load_b(t, 2, b0);
      mul(a1, b1, acc);
      load_a(t, 3, a1);
      load_b(t, 3, b1);
      mul(a0, b0, acc);
    }
    nt_wait_vm<0>();  // the next stage is there,
    nt_barrier();     // and this one read by every wave
    if constexpr (SPREAD) issue_part(s + 2, 0);
    else if (s + 2 < blocks) issue(s + 2);
    load_a(next, 0, a0);
    load_b(next, 0, b0);
    if constexpr (SPLIT) mul(a1, b2, low);
    else mul(a1, b1, acc);
  }
  nt_wait_vm<0>();
  if constexpr (CROSS) {
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) acc[i][j] += cross[i][j];
  }
}

}  // namespace oscars
