// The paged 4-bit key/value cache: layout and helpers shared by the kernels that write it
// (paged_cache.hip) and read it (paged_cache.hip, paged_attention.hip).
//
// A page holds `P` positions of every key/value head.  Row (page, head, offset) is
// (page * Hkv + head) * P + offset; its D/2 code bytes of the key and of the value are two
// arrays, and its four 16-bit parameters (key scale as fp16 bits, key zero-point, value scale,
// value zero-point) one 8-byte word of a third: one load instead of four of two bytes, and
// 16 positions of a head, the smallest page, fill a 128-byte line.
#pragma once

#include "common.h"

namespace offq {

struct PagedCache {
  uint8_t* kc;    // [pages, Hkv, P, D/2]
  uint8_t* vc;    // [pages, Hkv, P, D/2]
  int16_t* par;   // [pages, Hkv, P, 4]
  int64_t pages;
  int log2p;      // P = 2^log2p, 16 .. 4096
  int Hkv;

  __device__ __forceinline__ int64_t row(int64_t page, int head, int off) const {
    return ((page * Hkv + head) << log2p) + off;
  }
  // the row of a slot (page * P + offset) at a head; the slot must lie in [0, pages * P)
  __device__ __forceinline__ int64_t slot_row(int64_t slot, int head) const {
    return row(slot >> log2p, head, (int)(slot & ((int64_t(1) << log2p) - 1)));
  }
  __device__ __forceinline__ bool holds(int64_t slot) const {
    return slot >= 0 && slot < (pages << log2p);
  }
};

// y = H x over the D = 8 * LPH channels that LPH adjacent lanes hold, eight a lane (H the
// Sylvester Hadamard matrix, unnormalised): channel bits 0..2 inside the lane, the others
// across the lanes.
template <int LPH>
__device__ __forceinline__ void fwht_lanes(float* x, int lane) {
#pragma unroll
  for (int st = 1; st < 8; st <<= 1)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (!(i & st)) {
        const float a = x[i], b = x[i + st];
        x[i] = a + b;
        x[i + st] = a - b;
      }
#pragma unroll
  for (int st = 1; st < LPH; st <<= 1) {
    const bool up = lane & st;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float o = __shfl_xor(x[i], st);
      x[i] = up ? o - x[i] : x[i] + o;
    }
  }
}

// fl32(1 / sqrt(D)), the factor of the normalised rotation
template <int D>
__host__ __device__ constexpr float hadamard_norm() {
  static_assert(D == 64 || D == 128, "head dimension");
  return D == 64 ? 0.125f : 0.08838834764831845f;
}

}  // namespace offq
