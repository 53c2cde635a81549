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

// The value of lane ^ X within a row of 16 lanes, without LDS: DPP has the exchanges by 1, 2, 8
// and 7 (a mirrored half row); by 4 is by 7, then by 3.
template <int X>
__device__ __forceinline__ int lane_xor(int v) {
  static_assert(X == 1 || X == 2 || X == 4 || X == 8, "lane exchange");
  if constexpr (X == 1) return __builtin_amdgcn_mov_dpp(v, 0xB1, 0xf, 0xf, true);
  if constexpr (X == 2) return __builtin_amdgcn_mov_dpp(v, 0x4E, 0xf, 0xf, true);
  if constexpr (X == 4)
    return __builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, true), 0x1B, 0xf, 0xf, true);
  return __builtin_amdgcn_mov_dpp(v, 0x128, 0xf, 0xf, true);
}
template <int X>
__device__ __forceinline__ float lane_xor(float v) {
  return __builtin_bit_cast(float, lane_xor<X>(__builtin_bit_cast(int, v)));
}

// One Hadamard butterfly across the lanes l and l ^ X of a wave: sums below, differences above.
template <int X>
__device__ __forceinline__ float lane_butterfly(float v, int lane) {
  const float sign = lane & X ? -1.0f : 1.0f;
  if constexpr (X < 16) {
    return __builtin_fmaf(sign, v, lane_xor<X>(v));
  } else {  // (the exchange of rows gives both lanes' values in both lanes)
    const uint32_t u = __float_as_uint(v);
    const auto r = X == 16 ? __builtin_amdgcn_permlane16_swap(u, u, false, false)
                           : __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __builtin_fmaf(sign, __uint_as_float(r[1]), __uint_as_float(r[0]));
  }
}

// Over a wave, the same in every lane.
__device__ __forceinline__ float wave_sum(float v) {
  v += lane_xor<1>(v);
  v += lane_xor<2>(v);
  v += lane_xor<4>(v);
  v += lane_xor<8>(v);
  const int i = __builtin_bit_cast(int, v);
  auto row = [&](int l) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(i, l)); };
  return (row(0) + row(16)) + (row(32) + row(48));
}
__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, lane_xor<1>(v));
  v = fmaxf(v, lane_xor<2>(v));
  v = fmaxf(v, lane_xor<4>(v));
  v = fmaxf(v, lane_xor<8>(v));
  const int i = __builtin_bit_cast(int, v);
  auto row = [&](int l) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(i, l)); };
  return fmaxf(fmaxf(row(0), row(16)), fmaxf(row(32), row(48)));
}
__device__ __forceinline__ int wave_add(int v) {
  v += lane_xor<1>(v);
  v += lane_xor<2>(v);
  v += lane_xor<4>(v);
  v += lane_xor<8>(v);
  return (__builtin_amdgcn_readlane(v, 0) + __builtin_amdgcn_readlane(v, 16)) +
         (__builtin_amdgcn_readlane(v, 32) + __builtin_amdgcn_readlane(v, 48));
}
// The sum over the lanes up to this one.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // within rows of 16 lanes
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // rows 0 and 2 into 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // the first half into the second
  return v;
}

// op over the LPH (8 or 16) lanes of a row's group, the same in each.
template <int LPH, class Op>
__device__ __forceinline__ float group_reduce(float v, Op op) {
  v = op(v, lane_xor<1>(v));
  v = op(v, lane_xor<2>(v));
  v = op(v, lane_xor<4>(v));
  if constexpr (LPH == 16) v = op(v, lane_xor<8>(v));
  return v;
}

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
  const float s1 = lane & 1 ? -1.0f : 1.0f, s2 = lane & 2 ? -1.0f : 1.0f;
  const float s4 = lane & 4 ? -1.0f : 1.0f, s8 = lane & 8 ? -1.0f : 1.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __builtin_fmaf(s1, x[i], lane_xor<1>(x[i]));
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __builtin_fmaf(s2, x[i], lane_xor<2>(x[i]));
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __builtin_fmaf(s4, x[i], lane_xor<4>(x[i]));
  if constexpr (LPH == 16) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __builtin_fmaf(s8, x[i], lane_xor<8>(x[i]));
  }
}

// fl32(1 / sqrt(D)), the factor of the normalised rotation
template <int D>
__host__ __device__ constexpr float hadamard_norm() {
  static_assert(D == 64 || D == 128, "head dimension");
  return D == 64 ? 0.125f : 0.08838834764831845f;
}

}  // namespace offq
