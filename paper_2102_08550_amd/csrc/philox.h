// The counter-based generator behind dropout: Philox4x32-10 (Salmon, Moraes, Dror,
// Shaw: Parallel random numbers: as easy as 1, 2, 3; 2011).  A mask is a function
// of the seed, the offset and an entry's place, so it is never stored: whoever
// needs it again, the backward pass among them, computes it again.
//
// Entry (r, c): counter (c / 8, r, offset low, offset high), key the seed; the
// entry's 16 bits are half c mod 2 (low first) of word (c mod 8) / 2.  It is
// dropped where they are below `below` = round(65536 p).  16 bits and not 32: the
// generator's integer products, at a quarter of the other instructions' rate, take
// eight entries a call, and 65536 / (65536 - below) is the exact factor for what
// is kept.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace oscars {

struct DropArgs {
  uint32_t below;  // 0: no dropout
  float factor;    // of what is kept
  uint32_t key[2];
  uint64_t offset;
  const uint64_t* more;  // device, added to the offset, or nullptr
};

#if defined(__HIPCC__)
struct Words4 {
  uint32_t w[4];
};

__device__ __forceinline__ Words4 philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3,
                                         uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p = static_cast<uint64_t>(c0) * 0xD2511F53u;
    const uint64_t q = static_cast<uint64_t>(c2) * 0xCD9E8D57u;
    c0 = static_cast<uint32_t>(q >> 32) ^ c1 ^ k0;
    c1 = static_cast<uint32_t>(q);
    c2 = static_cast<uint32_t>(p >> 32) ^ c3 ^ k1;
    c3 = static_cast<uint32_t>(p);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return Words4{{c0, c1, c2, c3}};
}

__device__ __forceinline__ uint64_t drop_offset(const DropArgs& d) {
  return d.offset + (d.more ? *d.more : 0);
}
// The words of entries 8 group .. 8 group + 7 of a row.
__device__ __forceinline__ Words4 drop_words(const DropArgs& d, uint64_t offset, uint32_t row,
                                             uint32_t group) {
  return philox(group, row, static_cast<uint32_t>(offset), static_cast<uint32_t>(offset >> 32),
                d.key[0], d.key[1]);
}
__device__ __forceinline__ bool drop_keeps(const DropArgs& d, const Words4& w, int t) {
  const uint32_t h = t & 1 ? w.w[t >> 1] >> 16 : w.w[t >> 1] & 0xFFFFu;
  return h >= d.below;
}
#endif

// out[r][c] = kept ? fl(x[r][c] factor) : 0, rounded to the type once more.
struct DropoutArgs {
  const void* x;
  int64_t x_ld;
  void* out;
  int64_t out_ld;
  bool bf16;
  int64_t rows;
  int cols;
  DropArgs drop;
};
hipError_t launch_dropout(const DropoutArgs& a, hipStream_t s);

}  // namespace oscars
