// Writing and reading back the paged 4-bit key/value cache (gfx950).
//
// Write, per token m and head (all in fp32; one rounding to bf16 of the query, one to a 4-bit
// code of a key or value channel):
//   x' = x / sqrt(mean_d x_d^2 + eps) * w      queries and keys, where a weight is given
//   (x'_a, x'_b) -> amplitude * (x'_a cos t - x'_b sin t, x'_b cos t + x'_a sin t),
//     t = pos * f_i, over the pairs i < rotary / 2 of channels (a, b) = (i, i + rotary / 2),
//     or (2 i, 2 i + 1); channels from `rotary` on pass
//   key, value: y = c H x' where asked, then the quantizer of Eq. 1 over the head
// The angle is taken in 64 bits and reduced there: at position 10^6 a 32-bit product is off by
// 0.03 of a radian.  The key is not rounded to bf16 on the way to its codes.
// Read: s (c - z), then c H of it where asked, rounded to bf16 once.
#include "internal.h"
#include "paged.h"

namespace offq {
namespace {

__device__ __forceinline__ void load8(const uint16_t* p, float* x) {
  const uint4 w4 = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    x[2 * k] = bf16_lo(w[k]);
    x[2 * k + 1] = bf16_hi(w[k]);
  }
}

__device__ __forceinline__ void store8(uint16_t* p, const float* x) {
  *reinterpret_cast<uint4*>(p) = make_uint4(bf16x2_rne(x[0], x[1]), bf16x2_rne(x[2], x[3]),
                                            bf16x2_rne(x[4], x[5]), bf16x2_rne(x[6], x[7]));
}

// amplitude * (cos, sin) of pos * f
__device__ __forceinline__ float2 turn(int pos, float f, float amplitude) {
  double rev = (double)pos * (double)f * 0.15915494309189535;  // revolutions: 1 / (2 pi)
  rev -= __builtin_rint(rev);
  float sn, cs;
  sincospif(2.0f * (float)rev, &sn, &cs);
  return make_float2(amplitude * cs, amplitude * sn);
}

// Row of 8 * LPH channels -> codes (one word a lane) and (scale | zero << 16).
template <int LPH>
__device__ __forceinline__ uint32_t quantize_row(const float* x, uint32_t& par) {
  float mx = x[0], mn = x[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    mx = fmaxf(mx, x[i]);
    mn = fminf(mn, x[i]);
  }
#pragma unroll
  for (int o = 1; o < LPH; o <<= 1) {
    mx = fmaxf(mx, __shfl_xor(mx, o));
    mn = fminf(mn, __shfl_xor(mn, o));
  }
  const QParams p = quant_params(mx, mn);
  const uint32_t lo = __float_as_uint(p.lo);
  uint32_t code = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) code |= (quant_bits(x[k], p) - lo) << (4 * k);
  par = (uint32_t)p.s16 | ((uint32_t)(uint16_t)p.z << 16);
  return code;
}

// One workgroup per token; a group of D / 8 lanes takes one query head, or the key and the
// value of one key/value head, at a time.
template <int D>
__global__ __launch_bounds__(256) void rope_kv_paged_kernel(RopeKvPagedArgs a, PagedCache c) {
  constexpr int LPH = D / 8, NG = 256 / LPH;
  __shared__ float2 s_cs[D / 2];
  const int tid = (int)__builtin_amdgcn_workitem_id_x();
  const int64_t m = __builtin_amdgcn_workgroup_id_x();
  const int l = tid & (LPH - 1), first = (tid & 63) & ~(LPH - 1);
  const int half = a.rotary / 2;
  if (tid < half) s_cs[tid] = turn(a.positions[m], a.inv_freq[tid], a.amplitude);
  __syncthreads();
  // this lane's part of the rotation: its partner lane (half layout) and its eight angles
  const int shift = half / 8;
  const bool turns = a.pairs ? 8 * l < a.rotary : l < 2 * shift;
  const bool upper = !a.pairs && l >= shift;
  const int partner = first + (turns && !a.pairs ? (upper ? l - shift : l + shift) : l);
  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int k = a.pairs ? 4 * l + i / 2 : 8 * (upper ? l - shift : l) + i;
    const float2 v = turns ? s_cs[k] : make_float2(1.0f, 0.0f);
    cs[i] = v.x;
    sn[i] = v.y;
  }
  auto prepared = [&](float* x, const uint16_t* w) {
    if (w) {
      float ss = 0.0f, wf[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(x[i], x[i], ss);
#pragma unroll
      for (int o = 1; o < LPH; o <<= 1) ss += __shfl_xor(ss, o);
      const float inv = 1.0f / __builtin_sqrtf(ss * (1.0f / D) + a.eps);
      load8(w + 8 * l, wf);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= inv * wf[i];
    }
    if (a.pairs) {
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float p = x[i], q = x[i + 1];
        x[i] = p * cs[i] - q * sn[i];
        x[i + 1] = q * cs[i] + p * sn[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float p = __shfl(x[i], partner);
        x[i] = upper ? x[i] * cs[i] + p * sn[i] : x[i] * cs[i] - p * sn[i];
      }
    }
  };
  const uint16_t* row = a.qkv + m * a.ldq + 8 * l;
  const int64_t slot = a.slots[m];
  for (int j = tid / LPH; j < a.Hq + c.Hkv; j += NG) {
    float x[8];
    load8(row + (int64_t)j * D, x);
    if (j < a.Hq) {
      prepared(x, a.q_weight);
      store8(a.q_out + m * a.ldo + (int64_t)j * D + 8 * l, x);
      continue;
    }
    const int h = j - a.Hq;
    uint32_t kp, vp;
    prepared(x, a.k_weight);
    if (a.k_had) {
      fwht_lanes<LPH>(x, l);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= hadamard_norm<D>();
    }
    const uint32_t kw = quantize_row<LPH>(x, kp);
    load8(row + (int64_t)(j + c.Hkv) * D, x);
    if (a.v_had) {
      fwht_lanes<LPH>(x, l);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= hadamard_norm<D>();
    }
    const uint32_t vw = quantize_row<LPH>(x, vp);
    if (!c.holds(slot)) continue;
    const int64_t r = c.slot_row(slot, h);
    reinterpret_cast<uint32_t*>(c.kc + r * (D / 2))[l] = kw;
    reinterpret_cast<uint32_t*>(c.vc + r * (D / 2))[l] = vw;
    if (l == 0) *reinterpret_cast<uint2*>(c.par + 4 * r) = make_uint2(kp, vp);
  }
}

// A group of D / 8 lanes per (row, head).
template <int D>
__global__ __launch_bounds__(256) void kv_dequantize_paged_kernel(
    PagedCache c, const int64_t* __restrict__ slots, int64_t M, int k_had, int v_had,
    uint16_t* __restrict__ k_out, int64_t ldk, uint16_t* __restrict__ v_out, int64_t ldv) {
  constexpr int LPH = D / 8, NG = 256 / LPH;
  const int tid = (int)__builtin_amdgcn_workitem_id_x();
  const int l = tid & (LPH - 1);
  const int64_t g = (int64_t)__builtin_amdgcn_workgroup_id_x() * NG + tid / LPH;
  const int64_t m = g / c.Hkv;
  const int h = (int)(g - m * c.Hkv);
  if (m >= M) return;  // whole groups leave together
  const int64_t slot = slots[m];
  if (!c.holds(slot)) return;
  const int64_t r = c.slot_row(slot, h);
  const uint2 par = *reinterpret_cast<const uint2*>(c.par + 4 * r);
  auto one = [&](const uint8_t* codes, uint32_t p, int had, uint16_t* out, int64_t ld) {
    const uint32_t w = reinterpret_cast<const uint32_t*>(codes + r * (D / 2))[l];
    const float s = fp16_bits_to_f32((uint16_t)p);
    const int z = (int16_t)(p >> 16);
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = s * (float)((int)((w >> (4 * i)) & 15u) - z);
    if (had) {
      fwht_lanes<LPH>(x, l);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= hadamard_norm<D>();
    }
    store8(out + m * ld + (int64_t)h * D + 8 * l, x);
  };
  if (k_out) one(c.kc, par.x, k_had, k_out, ldk);
  if (v_out) one(c.vc, par.y, v_had, v_out, ldv);
}

}  // namespace

hipError_t launch_rope_kv_paged(const RopeKvPagedArgs& a, const PagedCache& c, int head_dim,
                                hipStream_t stream) {
  if (head_dim == 128)
    hipLaunchKernelGGL(rope_kv_paged_kernel<128>, dim3((unsigned)a.M), dim3(256), 0, stream, a, c);
  else
    hipLaunchKernelGGL(rope_kv_paged_kernel<64>, dim3((unsigned)a.M), dim3(256), 0, stream, a, c);
  return hipGetLastError();
}

hipError_t launch_kv_dequantize_paged(const PagedCache& c, int head_dim, const int64_t* slots,
                                      int64_t M, bool k_had, bool v_had, uint16_t* k_out,
                                      int64_t ldk, uint16_t* v_out, int64_t ldv,
                                      hipStream_t stream) {
  const int ng = 256 / (head_dim / 8);
  const unsigned grid = (unsigned)((M * c.Hkv + ng - 1) / ng);
  hipLaunchKernelGGL(head_dim == 128 ? kv_dequantize_paged_kernel<128> : kv_dequantize_paged_kernel<64>,
                     dim3(grid), dim3(256), 0, stream, c, slots, M, k_had ? 1 : 0, v_had ? 1 : 0,
                     k_out, ldk, v_out, ldv);
  return hipGetLastError();
}

}  // namespace offq
