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
//
// Both are bound by memory where they are large (a large copy here: 4.9 TB/s).  Write, 8191 tokens
// of 48 heads with norms: 39 us for 176 MB, 4.5 TB/s, its vector work 75 % of that; angles from
// LDS for each round, a hardware reciprocal root, eight waves per SIMD and a second round on its
// way did not change it.  Read, 131072 rows of 8 heads: 152 us for 680 MB, 4.5 TB/s.  Below about
// 1000 rows a call is its launch, 4 us.
#include <type_traits>

#include "internal.h"
#include "paged.h"

namespace offq {
namespace {

typedef uint32_t u4_t __attribute__((ext_vector_type(4)));

template <bool NT>  // past the caches
__device__ __forceinline__ void store8(uint16_t* p, const float* x) {
  const u4_t v = {bf16x2_rne(x[0], x[1]), bf16x2_rne(x[2], x[3]), bf16x2_rne(x[4], x[5]),
                  bf16x2_rne(x[6], x[7])};
  if constexpr (NT) __builtin_nontemporal_store(v, reinterpret_cast<u4_t*>(p));
  else *reinterpret_cast<u4_t*>(p) = v;
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
  mx = group_reduce<LPH>(mx, [](float a, float b) { return fmaxf(a, b); });
  mn = group_reduce<LPH>(mn, [](float a, float b) { return fminf(a, b); });
  const QParams p = quant_params(mx, mn);
  const uint32_t lo = __float_as_uint(p.lo);
  uint32_t code = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) code |= (quant_bits(x[k], p) - lo) << (4 * k);
  par = (uint32_t)p.s16 | ((uint32_t)(uint16_t)p.z << 16);
  return code;
}

// A wave takes one token, or one of `parts` of its heads where tokens are few, in rounds of
// 64 / (D / 8) query heads, then of key/value heads, D / 8 lanes each (a group past the last head
// does that one again).  The token's angles are formed by the wave, one pair a lane, and handed
// round in LDS; the next round's channels are on their way while one is worked on.  The rounds of
// queries have no branch around a load or store, so that a wait counts the loads it needs and not
// the stores after them: 8191 tokens of 48 heads, with the reading back, 53 -> 49 us.
// FULL: the half layout over the whole head, whose partner channels sit half a group away.
// NT: what is read and the queries written go past the caches.
template <int D, bool FULL, bool NT>
__global__ __launch_bounds__(256) void rope_kv_paged_kernel(RopeKvPagedArgs a, PagedCache c, int parts) {
  constexpr int LPH = D / 8, NG = 64 / LPH;
  __shared__ alignas(16) float2 s_cs[4][D / 2];
  const int tid = (int)__builtin_amdgcn_workitem_id_x();
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t item = (int64_t)__builtin_amdgcn_workgroup_id_x() * 4 + wave;
  const int64_t m = __builtin_amdgcn_readfirstlane((int)(item / parts));
  const int part = (int)(item - m * parts);
  if (m >= a.M) return;
  const int l = lane & (LPH - 1), g = lane / LPH;
  const int rq = (a.Hq + NG - 1) / NG, rounds = rq + (c.Hkv + NG - 1) / NG;
  const uint16_t* row = a.qkv + m * a.ldq + 8 * l;
  auto load = [&](int head) {
    const u4_t* p = reinterpret_cast<const u4_t*>(row + (int64_t)head * D);
    return NT ? __builtin_nontemporal_load(p) : *p;
  };
  auto fetch = [&](int r) {  // a query's channels, or a key's
    r = min(r, rounds - 1);
    return load(r < rq ? min(NG * r + g, a.Hq - 1) : a.Hq + min(NG * (r - rq) + g, c.Hkv - 1));
  };
  u4_t next = fetch(part);
  // (without a weight, 16 bytes that are there and are not used)
  const u4_t qw = *reinterpret_cast<const u4_t*>(a.q_weight ? a.q_weight + 8 * l : row);
  const u4_t kw = *reinterpret_cast<const u4_t*>(a.k_weight ? a.k_weight + 8 * l : row);
  const int half = a.rotary / 2;
  if (lane < half) s_cs[wave][lane] = turn(a.positions[m], a.inv_freq[lane], a.amplitude);
  const int64_t slot = a.slots[m];
  __builtin_amdgcn_wave_barrier();
  // this lane's part of the rotation: its partner lane (half layout) and its eight angles
  const int shift = half / 8;
  const bool turns = FULL || (a.pairs ? 8 * l < a.rotary : l < 2 * shift);
  const bool upper = FULL ? l >= LPH / 2 : !a.pairs && l >= shift;
  const int partner = (lane & ~(LPH - 1)) + (turns && !a.pairs ? (upper ? l - shift : l + shift) : l);
  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int k = FULL ? 8 * (l & (LPH / 2 - 1)) + i : a.pairs ? 4 * l + i / 2 : 8 * (upper ? l - shift : l) + i;
    const float2 v = turns ? s_cs[wave][k] : make_float2(1.0f, 0.0f);
    cs[i] = v.x;
    sn[i] = upper ? v.y : -v.y;  // half layout: x cos + partner * this
  }
  auto unpack = [](const u4_t& v, float* x) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[2 * k] = bf16_lo(v[k]);
      x[2 * k + 1] = bf16_hi(v[k]);
    }
  };
  auto prepared = [&](float* x, bool normed, const u4_t& weight) {
    if (normed) {
      float w[8], ss = 0.0f;
      unpack(weight, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(x[i], x[i], ss);
      ss = group_reduce<LPH>(ss, [](float p, float q) { return p + q; });
      const float inv = 1.0f / __builtin_sqrtf(ss * (1.0f / D) + a.eps);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= inv * w[i];
    }
    if (!FULL && a.pairs) {
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float p = x[i], q = x[i + 1];
        x[i] = p * cs[i] + q * sn[i];
        x[i + 1] = q * cs[i] - p * sn[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float p = FULL ? lane_xor<LPH / 2>(x[i]) : __shfl(x[i], partner);
        x[i] = __builtin_fmaf(p, sn[i], x[i] * cs[i]);
      }
    }
  };
  auto rotate = [&](float* x) {
    fwht_lanes<LPH>(x, l);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= hadamard_norm<D>();
  };
  int r = part;
  for (; r < rq; r += parts) {
    float x[8];
    unpack(next, x);
    next = fetch(r + parts);
    prepared(x, a.q_weight, qw);
    store8<NT>(a.q_out + m * a.ldo + (int64_t)min(NG * r + g, a.Hq - 1) * D + 8 * l, x);
  }
  for (; r < rounds; r += parts) {
    const int h = min(NG * (r - rq) + g, c.Hkv - 1);
    float x[8], v[8];
    unpack(next, x);
    const u4_t value = load(a.Hq + c.Hkv + h);
    next = fetch(r + parts);
    uint32_t kp, vp;
    prepared(x, a.k_weight, kw);
    if (a.k_had) rotate(x);
    const uint32_t kc = quantize_row<LPH>(x, kp);
    unpack(value, v);
    if (a.v_had) rotate(v);
    const uint32_t vc = quantize_row<LPH>(v, vp);
    if (c.holds(slot)) {
      const int64_t at = c.slot_row(slot, h);
      reinterpret_cast<uint32_t*>(c.kc + at * (D / 2))[l] = kc;
      reinterpret_cast<uint32_t*>(c.vc + at * (D / 2))[l] = vc;
      if (l == 0) *reinterpret_cast<uint2*>(c.par + 4 * at) = make_uint2(kp, vp);
    }
  }
}

typedef _Float16 h2_t __attribute__((ext_vector_type(2)));

// A group of D / 8 lanes per row, a code word (8 channels) each, so that a store writes the row's
// 2 D bytes in one piece (with four lanes of 32 channels, which need half the exchanges, 64-byte
// pieces: 137 us against 132 without a rotation, 131072 rows of 8 heads).  A masked word holds two
// codes as fp16 subnormals c 2^-24, in which sums of up to 128 codes are exact: the rotation runs
// on them as packed halves; the zero-point, whose rotation is D z in channel 0 and nothing
// elsewhere, comes after it; and one multiplication by s turns a half into a value.
template <int D, bool HAD, bool NT>
__device__ __forceinline__ void dequantize_row(uint32_t w, uint32_t par, int l, uint16_t* out) {
  constexpr int LPH = D / 8;
  const float s = fp16_bits_to_f32((uint16_t)par), z = (float)(int16_t)(par >> 16);
  h2_t h[4];  // channels 8 l + i and + i + 4
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __builtin_bit_cast(h2_t, (w >> (4 * i)) & 0x000F000Fu);
  if constexpr (HAD) {
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = h2_t{h[i].x, h[i].x} + h2_t{h[i].y, -h[i].y};  // channel bit 2
#pragma unroll
    for (int st = 1; st < 4; st <<= 1)  // bits 0, 1
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!(i & st)) {
          const h2_t p = h[i], q = h[i + st];
          h[i] = p + q;
          h[i + st] = p - q;
        }
    auto across = [&](auto x) {  // a channel bit above them
      constexpr int X = decltype(x)::value;
      const _Float16 sign = l & X ? -1.0f : 1.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        h[i] = __builtin_elementwise_fma(
            h2_t{sign, sign}, h[i], __builtin_bit_cast(h2_t, lane_xor<X>(__builtin_bit_cast(int, h[i]))));
    };
    across(std::integral_constant<int, 1>{});
    across(std::integral_constant<int, 2>{});
    across(std::integral_constant<int, 4>{});
    if constexpr (LPH == 16) across(std::integral_constant<int, 8>{});
  }
  const float k = s * (HAD ? hadamard_norm<D>() : 1.0f);
  const float kk = k * 0x1p24f, sub = HAD ? 0.0f : -s * z;
  float y[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[i] = __builtin_fmaf((float)h[i].x, kk, sub);
    y[i + 4] = __builtin_fmaf((float)h[i].y, kk, sub);
  }
  if (HAD && l == 0) y[0] = __builtin_fmaf((float)h[0].x, 0x1p24f, -z * D) * k;
  store8<NT>(out, y);
}

template <int D, bool NT>
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
  const uint32_t kw = reinterpret_cast<const uint32_t*>(c.kc + r * (D / 2))[l];
  const uint32_t vw = reinterpret_cast<const uint32_t*>(c.vc + r * (D / 2))[l];
  const int64_t at = (int64_t)h * D + 8 * l;
  if (k_out) {
    if (k_had) dequantize_row<D, true, NT>(kw, par.x, l, k_out + m * ldk + at);
    else dequantize_row<D, false, NT>(kw, par.x, l, k_out + m * ldk + at);
  }
  if (v_out) {
    if (v_had) dequantize_row<D, true, NT>(vw, par.y, l, v_out + m * ldv + at);
    else dequantize_row<D, false, NT>(vw, par.y, l, v_out + m * ldv + at);
  }
}

}  // namespace

hipError_t launch_rope_kv_paged(const RopeKvPagedArgs& a, const PagedCache& c, int head_dim,
                                hipStream_t stream) {
  const int ng = 64 / (head_dim / 8);
  const int64_t rounds = (a.Hq + ng - 1) / ng + (c.Hkv + ng - 1) / ng;
  // a token's heads go to several waves until there are 4096 of them, 16 a CU
  int64_t parts = (4096 + a.M - 1) / a.M;
  parts = parts < 1 ? 1 : parts > rounds ? rounds : parts;
  const dim3 grid((unsigned)((a.M * parts + 3) / 4));
  const bool full = !a.pairs && a.rotary == head_dim;
  // Queries beyond the L2s' 32 MB, and what they come from, bypass the caches (8191 tokens of 48
  // heads: 47 -> 42 us); with 24 MB of input that costs more than it gives (2000 tokens of 48 heads
  // with their reading back: 17.5 us, bypassing 19.6).
  const bool nt = 2 * a.M * a.Hq * head_dim > (32 << 20);
#define OFFQ_ROPE(D_, F_)                                                                        \
  hipLaunchKernelGGL((nt ? rope_kv_paged_kernel<D_, F_, true> : rope_kv_paged_kernel<D_, F_, false>), \
                     grid, dim3(256), 0, stream, a, c, (int)parts)
  if (head_dim == 128) {
    if (full) OFFQ_ROPE(128, true);
    else OFFQ_ROPE(128, false);
  } else {
    if (full) OFFQ_ROPE(64, true);
    else OFFQ_ROPE(64, false);
  }
#undef OFFQ_ROPE
  return hipGetLastError();
}

hipError_t launch_kv_dequantize_paged(const PagedCache& c, int head_dim, const int64_t* slots,
                                      int64_t M, bool k_had, bool v_had, uint16_t* k_out,
                                      int64_t ldk, uint16_t* v_out, int64_t ldv,
                                      hipStream_t stream) {
  const int ng = 256 / (head_dim / 8);
  const unsigned grid = (unsigned)((M * c.Hkv + ng - 1) / ng);
  // Outputs beyond the L2s' 32 MB bypass them (131072 rows of 8 heads: 164 -> 154 us); smaller ones
  // stay for the next kernel (5000 rows: 8 us either way).
  const bool nt = 2 * M * c.Hkv * head_dim * ((k_out != nullptr) + (v_out != nullptr)) > (32 << 20);
  auto kernel = head_dim == 128 ? nt ? kv_dequantize_paged_kernel<128, true> : kv_dequantize_paged_kernel<128, false>
                                : nt ? kv_dequantize_paged_kernel<64, true> : kv_dequantize_paged_kernel<64, false>;
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, stream, c, slots, M, k_had ? 1 : 0,
                     v_had ? 1 : 0, k_out, ldk, v_out, ldv);
  return hipGetLastError();
}

}  // namespace offq
