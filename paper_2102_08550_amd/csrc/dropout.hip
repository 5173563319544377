// Dropout from a counter-based generator (philox.h): one pass over x, eight entries
// a thread and call of the generator.
#include "philox.h"

namespace oscars {
namespace {

typedef float dr_f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t dr_u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float dr_bf16(uint32_t v) { return __builtin_bit_cast(float, v << 16); }
__device__ __forceinline__ uint32_t dr_to_bf16(float v) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return u >> 16 | 0x40u;
  return (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}

template <bool BF16, bool VEC>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a, uint32_t groups,
                                                      uint64_t step_rows, uint32_t step_groups) {
  const uint64_t offset = drop_offset(a.drop);
  uint64_t at = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x;
  uint64_t row = at / groups;
  uint32_t g = static_cast<uint32_t>(at - row * groups);
  while (row < static_cast<uint64_t>(a.rows)) {
    const Words4 w = drop_words(a.drop, offset, static_cast<uint32_t>(row), g);
    const int64_t c = static_cast<int64_t>(g) * 8;
    const int64_t n = a.cols - c;
    if constexpr (BF16) {
      const uint16_t* x = static_cast<const uint16_t*>(a.x) + row * a.x_ld + c;
      uint16_t* y = static_cast<uint16_t*>(a.out) + row * a.out_ld + c;
      if (VEC && n >= 8) {
        dr_u32x4 v = *reinterpret_cast<const dr_u32x4*>(x);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const uint32_t lo = dr_to_bf16(dr_bf16(v[t] & 0xFFFFu) * a.drop.factor);
          const uint32_t hi = dr_to_bf16(dr_bf16(v[t] >> 16) * a.drop.factor);
          v[t] = (drop_keeps(a.drop, w, 2 * t) ? lo : 0u) |
                 (drop_keeps(a.drop, w, 2 * t + 1) ? hi << 16 : 0u);
        }
        *reinterpret_cast<dr_u32x4*>(y) = v;
      } else {
#pragma unroll
        for (int t = 0; t < 8; ++t)
          if (t < n)
            y[t] = drop_keeps(a.drop, w, t)
                       ? static_cast<uint16_t>(dr_to_bf16(dr_bf16(x[t]) * a.drop.factor))
                       : static_cast<uint16_t>(0);
      }
    } else {
      const float* x = static_cast<const float*>(a.x) + row * a.x_ld + c;
      float* y = static_cast<float*>(a.out) + row * a.out_ld + c;
      if (VEC && n >= 8) {
        dr_f32x4 v[2] = {reinterpret_cast<const dr_f32x4*>(x)[0],
                         reinterpret_cast<const dr_f32x4*>(x)[1]};
#pragma unroll
        for (int t = 0; t < 8; ++t)
          v[t >> 2][t & 3] = drop_keeps(a.drop, w, t) ? v[t >> 2][t & 3] * a.drop.factor : 0.0f;
        reinterpret_cast<dr_f32x4*>(y)[0] = v[0];
        reinterpret_cast<dr_f32x4*>(y)[1] = v[1];
      } else {
#pragma unroll
        for (int t = 0; t < 8; ++t)
          if (t < n) y[t] = drop_keeps(a.drop, w, t) ? x[t] * a.drop.factor : 0.0f;
      }
    }
    row += step_rows;
    g += step_groups;
    if (g >= groups) {
      g -= groups;
      ++row;
    }
  }
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t s) {
  const int64_t es = a.bf16 ? 2 : 4;
  auto rows16 = [&](const void* p, int64_t ld) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * es % 16 == 0;
  };
  const bool vec = rows16(a.x, a.x_ld) && rows16(a.out, a.out_ld);
  const uint32_t groups = static_cast<uint32_t>((static_cast<int64_t>(a.cols) + 7) / 8);
  const uint64_t units = static_cast<uint64_t>(a.rows) * groups;
  const uint64_t want = (units + 255) / 256, most = 256 * 16;
  const unsigned grid = static_cast<unsigned>(want < most ? want : most);
  const uint64_t stride = static_cast<uint64_t>(grid) * 256;
  const uint64_t step_rows = stride / groups;
  const uint32_t step_groups = static_cast<uint32_t>(stride % groups);
#define OSCARS_DROP(B, V) \
  hipLaunchKernelGGL((dropout_kernel<B, V>), dim3(grid), dim3(256), 0, s, a, groups, step_rows, \
                     step_groups)
  if (a.bf16) {
    if (vec) OSCARS_DROP(true, true);
    else OSCARS_DROP(true, false);
  } else {
    if (vec) OSCARS_DROP(false, true);
    else OSCARS_DROP(false, false);
  }
#undef OSCARS_DROP
  return hipGetLastError();
}

}  // namespace oscars
