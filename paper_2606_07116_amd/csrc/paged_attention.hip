// Causal attention of packed new tokens over the paged 4-bit key/value cache (gfx950).
//
// Sequence b of a call has the query rows q_starts[b] .. q_starts[b + 1] - 1 and seq_lens[b]
// positions in the pages that row b of the page table names, the new tokens' among them:
// query i of its n sits at position seq_lens[b] - n + i and sees the positions up to its own.
//   q_r  = c H q where the keys were rotated
//   s_j  = sm_scale * sk_j * sum_d q_r[d] (ck_j[d] - zk_j)
//   o[d] = sum_j e^(s_j - max s) sv_j (cv_j[d] - zv_j) / sum_j e^(s_j - max s)
//   (then c H o where the values were rotated); a row that sees no position gives 0
#include "internal.h"
#include "paged.h"

namespace offq {
namespace {

constexpr float LOG2E = 1.4426950408889634f;

// One wave per (query row, head): 64 positions at a time, a lane first holding one position's
// score, then D / 64 channels of the output.
template <int D>
__global__ __launch_bounds__(64) void kv_attention_paged_kernel(PagedAttentionArgs a, PagedCache c) {
  constexpr int E = D / 64;
  __shared__ float s_q[D];
  __shared__ float s_p[64];
  __shared__ int64_t s_row[64];
  const int lane = (int)__builtin_amdgcn_workitem_id_x();
  const int m = (int)__builtin_amdgcn_workgroup_id_x(), hq = (int)__builtin_amdgcn_workgroup_id_y();
  // the sequence of row m: the last b with q_starts[b] <= m
  int b = 0;
  for (int hi = a.B; hi - b > 1;) {
    const int mid = (b + hi) / 2;
    if (a.q_starts[mid] <= m) b = mid;
    else hi = mid;
  }
  const int q0 = a.q_starts[b], n = a.q_starts[b + 1] - q0;
  const int i = m - q0;
  if (i < 0 || i >= n || i >= a.max_new) return;  // in no sequence
  const int len = a.seq_lens[b];
  const int hk = hq / (a.Hq / c.Hkv);
  const int64_t seen = min((int64_t)len - n + i + 1, (int64_t)a.max_pages << c.log2p);
  const uint16_t* q = a.q + (int64_t)m * a.ldq + (int64_t)hq * D;
  for (int e = 0; e < E; ++e) s_q[e * 64 + lane] = bf16_lo(q[e * 64 + lane]);
  __syncthreads();
  if (a.k_had) {
    float y[E];
    for (int e = 0; e < E; ++e) {
      y[e] = 0.0f;
      const int d = e * 64 + lane;
      for (int k = 0; k < D; ++k) y[e] += (__builtin_popcount(k & d) & 1) ? -s_q[k] : s_q[k];
    }
    __syncthreads();
    for (int e = 0; e < E; ++e) s_q[e * 64 + lane] = y[e] * hadamard_norm<D>();
    __syncthreads();
  }
  const float NEG = -__builtin_inff();
  float mx = NEG, l = 0.0f, o[E] = {};
  for (int64_t j0 = 0; j0 < seen; j0 += 64) {
    const int64_t j = j0 + lane;
    float s = NEG;
    int64_t r = -1;
    if (j < seen) {
      const int page = a.page_table[(int64_t)b * a.max_pages + (j >> c.log2p)];
      if (page >= 0 && page < c.pages) {
        r = c.row(page, hk, (int)(j & ((1 << c.log2p) - 1)));
        const int z = c.par[4 * r + 1];
        float dot = 0.0f;
        for (int w = 0; w < D / 8; ++w) {
          const uint32_t u = reinterpret_cast<const uint32_t*>(c.kc + r * (D / 2))[w];
          for (int k = 0; k < 8; ++k)
            dot = __builtin_fmaf(s_q[8 * w + k], (float)((int)((u >> (4 * k)) & 15u) - z), dot);
        }
        s = a.sm_scale * LOG2E * fp16_bits_to_f32((uint16_t)c.par[4 * r]) * dot;
      }
    }
    float bm = s;
    for (int off = 32; off >= 1; off >>= 1) bm = fmaxf(bm, __shfl_xor(bm, off));
    if (bm == NEG) continue;
    const float mn = fmaxf(mx, bm);
    const float f = __builtin_amdgcn_exp2f(mx - mn);
    const float p = __builtin_amdgcn_exp2f(s - mn);
    mx = mn;
    l = l * f + p;  // this lane's positions
    s_p[lane] = p;
    s_row[lane] = r;
    __syncthreads();
    for (int e = 0; e < E; ++e) o[e] *= f;
    for (int k = 0; k < 64; ++k) {
      const int64_t rk = s_row[k];
      if (rk < 0) continue;
      const float w = s_p[k] * fp16_bits_to_f32((uint16_t)c.par[4 * rk + 2]);
      const int z = c.par[4 * rk + 3];
      for (int e = 0; e < E; ++e) {
        const int d = e * 64 + lane;
        const int code = (c.vc[rk * (D / 2) + d / 2] >> (4 * (d & 1))) & 15;
        o[e] = __builtin_fmaf(w, (float)(code - z), o[e]);
      }
    }
    __syncthreads();
  }
  for (int off = 32; off >= 1; off >>= 1) l += __shfl_xor(l, off);
  for (int e = 0; e < E; ++e) o[e] = l > 0.0f ? o[e] / l : 0.0f;
  if (a.v_had) {
    __syncthreads();
    for (int e = 0; e < E; ++e) s_q[e * 64 + lane] = o[e];
    __syncthreads();
    for (int e = 0; e < E; ++e) {
      const int d = e * 64 + lane;
      float y = 0.0f;
      for (int k = 0; k < D; ++k) y += (__builtin_popcount(k & d) & 1) ? -s_q[k] : s_q[k];
      o[e] = y * hadamard_norm<D>();
    }
  }
  uint16_t* out = a.out + (int64_t)m * a.ldo + (int64_t)hq * D;
  for (int e = 0; e < E; ++e) out[e * 64 + lane] = f32_to_bf16_rne(o[e]);
}

}  // namespace

int64_t kv_attention_paged_workspace_floats(int64_t, int64_t, int64_t, int64_t, int, int64_t) {
  return 0;
}

hipError_t launch_kv_attention_paged(const PagedAttentionArgs& a, const PagedCache& c, int head_dim,
                                     float*, hipStream_t stream) {
  const dim3 grid((unsigned)a.M, (unsigned)a.Hq);
  if (head_dim == 128)
    hipLaunchKernelGGL(kv_attention_paged_kernel<128>, grid, dim3(64), 0, stream, a, c);
  else
    hipLaunchKernelGGL(kv_attention_paged_kernel<64>, grid, dim3(64), 0, stream, a, c);
  return hipGetLastError();
}

}  // namespace offq
