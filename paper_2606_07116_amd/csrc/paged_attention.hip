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
constexpr int CHUNK_MIN = 512;   // positions of a chunk, at least

typedef _Float16 h8_t __attribute__((ext_vector_type(8)));
typedef _Float16 h2_t __attribute__((ext_vector_type(2)));
typedef float f4_t __attribute__((ext_vector_type(4)));

constexpr float TAU = 8.0f;     // a row's reference maximum may lag by up to 2^TAU
constexpr float LOWEST = -1e30f;  // a reference maximum below every score

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// What a sequence asks for, lengths made safe whatever the tables hold: `rows` query rows
// (token, head of the group) of a key/value head, the first of them token q0 at position pos0,
// and `keys` positions that the last of them sees.
struct Seq {
  int q0, rows, keys, pos0;
};
__device__ __forceinline__ Seq sequence(const PagedAttentionArgs& a, int log2p, int G, int b) {
  const int lo = min(max(a.q_starts[b], 0), a.M), hi = min(max(a.q_starts[b + 1], lo), a.M);
  const int n = hi - lo, t = min(n, a.max_new);
  Seq s;
  s.q0 = lo;
  s.rows = t * G;
  s.pos0 = max(a.seq_lens[b], -(1 << 30)) - n;
  s.keys = (int)min((int64_t)max(s.pos0, -t) + t, (int64_t)a.max_pages << log2p);
  return s;
}

// ---------------------------------------------------------------------------
// Few rows: sequences of up to 16 RT query rows (new tokens x heads of a group).  What bounds
// them is the cache's bytes, so the keys of all such sequences are cut into chunks of one length,
// chosen on the device so that about `target` workgroups get one each whatever the lengths are;
// a chunk's four waves take a quarter each, and a second kernel joins a row's chunks.
//
// A wave takes 32 positions at a time, two groups of 16 (a group lies in one page), straight from
// memory into the operands of 16x16x32 fp16 matrix products, the next block's loads in flight:
// * a masked code word holds the codes c as fp16 subnormals c 2^-24 (16 c 2^-24 the odd ones,
//   whose query channels are divided by 16): exact products, one AND per two codes;
// * scores S^T = K Q^T: lane (row pr = lane % 16, kq = lane / 16) gets positions 4 kq .. 4 kq + 3
//   of both groups for its query row, which are the eight positions that the value product
//   O = W V wants from it: the weights never leave the lane;
// * values: lane (column pr, kq) loads the code word of its eight positions, a byte permute puts
//   two positions side by side, and a mask per nibble leaves the operand of one product;
// * scale and zero-point of a position are prepared by one lane and read from LDS.
// The zero-point terms are kept out of the products (sum q, sum w z in fp32), so large offsets
// cost no accuracy.  The query and the weights p sv are rounded to fp16 (2^-11), scaled so that
// neither tiny nor huge scales leave its range: the weights by a power of two that follows the
// largest value scale met.
struct Chunking {
  int len;          // positions per chunk, a multiple of 128
  int b, head, chunk, nchunk, unit0;  // this unit's; unit0: the sequence's first unit
  bool found;
  Seq s;
};

// The chunk length, and what unit `unit` is.  Every wave works it out for itself, 64 sequences
// at a time.
__device__ __forceinline__ Chunking find_chunk(const PagedAttentionArgs& a, int log2p, int Hkv,
                                               int few_rows, int target, int max_chunks, int unit) {
  const int lane = (int)__builtin_amdgcn_workitem_id_x() & 63;
  const int G = a.Hq / Hkv;
  float total = 0.0f;
  int longest = 0;
  Seq s{};
  auto load = [&](int b) {
    s = Seq{};
    if (b < a.B) s = sequence(a, log2p, G, b);
    if (s.rows > few_rows) s.rows = 0;
  };
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    load(b0 + lane);
    if (s.rows) {
      total += (float)s.keys;
      longest = max(longest, s.keys);
    }
  }
  total = wave_sum(total);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) longest = max(longest, __shfl_xor(longest, o));
  Chunking c{};
  // (a rounding of the fp32 sum only shifts the chunk length, the same for every unit)
  const float want = fminf(fmaxf(total * (float)Hkv / (float)target, (float)longest / (float)max_chunks),
                           1073741824.0f);
  c.len = max(CHUNK_MIN, ((int)want + 128) & ~127);
  int base = 0;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    if (a.B > 64) load(b0 + lane);
    const int nc = s.rows ? max(1, (s.keys + c.len - 1) / c.len) : 0;
    int incl = nc;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int p = __shfl_up(incl, o);
      if (lane >= o) incl += p;
    }
    const int first = base + incl - nc;
    const uint64_t mine = __builtin_amdgcn_ballot_w64(nc > 0 && unit >= Hkv * first && unit < Hkv * (first + nc));
    if (mine) {
      const int o = __builtin_ctzll(mine);
      c.found = true;
      c.b = b0 + o;
      c.nchunk = __builtin_amdgcn_readlane(nc, o);
      c.unit0 = Hkv * __builtin_amdgcn_readlane(first, o);
      c.head = (unit - c.unit0) / c.nchunk;
      c.chunk = unit - c.unit0 - c.head * c.nchunk;
      c.s.q0 = __builtin_amdgcn_readlane(s.q0, o);
      c.s.rows = __builtin_amdgcn_readlane(s.rows, o);
      c.s.keys = __builtin_amdgcn_readlane(s.keys, o);
      c.s.pos0 = __builtin_amdgcn_readlane(s.pos0, o);
      return c;
    }
    base += __builtin_amdgcn_readlane(incl, 63);
  }
  return c;
}

// The rows of a chunk that the second kernel joins: per (sequence) where its units start.
struct alignas(16) Joint {
  int q0, rows, nchunk, unit0;
};

template <int D>
struct Block {
  uint32_t k[2][D / 32];  // a quarter row of key codes per group
  uint32_t v[2][4];       // a word of value codes of four positions per group
  uint2 par;              // lane < 32: the parameters of position `lane`
  uint32_t ok;            // bit g: group g is in the cache
};

// One row (D / 64 channels a lane) rotated by c H.
template <int D>
__device__ __forceinline__ void rotate_wave(float (&x)[D / 64], int lane) {
  if constexpr (D == 128) {
    const float p = x[0] + x[1], q = x[0] - x[1];
    x[0] = p;
    x[1] = q;
  }
#pragma unroll
  for (int st = 1; st < 64; st <<= 1) {
    const bool up = lane & st;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) {
      const float o = __shfl_xor(x[e], st);
      x[e] = up ? o - x[e] : x[e] + o;
    }
  }
#pragma unroll
  for (int e = 0; e < D / 64; ++e) x[e] *= hadamard_norm<D>();
}

// A finished row: o / l (0 where nothing was seen), rotated back if asked, rounded once.  The
// wave holds channels lane * D / 64 and on.
template <int D>
__device__ __forceinline__ void store_row(const PagedAttentionArgs& a, int row, int hq, float (&o)[D / 64],
                                          float l, int lane) {
#pragma unroll
  for (int e = 0; e < D / 64; ++e) o[e] = l > 0.0f ? o[e] / l : 0.0f;
  if (a.v_had) rotate_wave<D>(o, lane);
  uint16_t* dst = a.out + (int64_t)row * a.ldo + (int64_t)hq * D;
  if constexpr (D == 128) reinterpret_cast<uint32_t*>(dst)[lane] = bf16x2_rne(o[0], o[1]);
  else dst[lane] = f32_to_bf16_rne(o[0]);
}

template <int D, int RT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(RT == 1 ? 3 : 2))) void
kv_attention_paged_few_kernel(PagedAttentionArgs a, PagedCache c, int few_rows, int target,
                              int max_chunks, Joint* __restrict__ joints, float* __restrict__ rec) {
  constexpr int NW = D / 32;  // key code words of a lane
  constexpr int NM = D / 16;  // products of a value block: 16 columns of NM channels each
  constexpr int OROW = D + 4;
  __shared__ union {
    _Float16 q[16 * RT][D + 8];  // the queries in operand order
    float o[4][16][OROW];        // a row tile's outputs, one per wave
  } u;
  __shared__ float4 s_par[4][32];  // per wave and position: score slope, score offset / sum q, sv, zv
  __shared__ float s_qsum[16 * RT], s_qmax[4];
  __shared__ float s_m[4][16 * RT], s_l[4][16 * RT], s_z[4][16 * RT], s_scale[4];

  const int tid = (int)__builtin_amdgcn_workitem_id_x();
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int pr = lane & 15, kq = lane >> 4;
  const int unit = (int)__builtin_amdgcn_workgroup_id_x();
  const int G = a.Hq / c.Hkv;
  const Chunking w = find_chunk(a, c.log2p, c.Hkv, few_rows, target, max_chunks, unit);
  if (!w.found) return;
  const int rows = w.s.rows, hk = w.head;
  if (joints && w.chunk == 0 && hk == 0 && tid == 0)
    joints[w.b] = Joint{w.s.q0, rows, w.nchunk, w.unit0};
  // the wave's positions: a quarter of the chunk
  const int k_end = min(w.s.keys, (w.chunk + 1) * w.len);
  const int k_begin = w.chunk * w.len + wave * (w.len >> 2);
  const int k_stop = min(k_end, k_begin + (w.len >> 2));

  // ---- page ids: lane i holds that of the 16 positions from id0 + 16 i on
  const int32_t* table = a.page_table + (int64_t)w.b * a.max_pages;
  auto load_ids = [&](int from) {
    const int key = from + 16 * lane;
    return key < k_stop ? table[key >> c.log2p] : -1;
  };
  int id0 = k_begin;
  int ids = load_ids(id0);

  Block<D> blk[2];
  auto load_block = [&](int k0, Block<D>& x) {
    x.ok = 0;
    int64_t row[2];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int key = k0 + 16 * g;
      const int id = __builtin_amdgcn_readlane(ids, (key - id0) >> 4);
      const bool ok = id >= 0 && id < c.pages;
      x.ok |= ok ? 1u << g : 0u;
      row[g] = c.row(ok ? id : 0, hk, key & ((1 << c.log2p) - 1));
      const uint8_t* kp = c.kc + row[g] * (D / 2);
      const uint8_t* vp = c.vc + row[g] * (D / 2);
      const uint32_t ko = (uint32_t)(pr * (D / 2) + kq * (D / 8));
      if constexpr (D == 128) {
        const uint4 t = *reinterpret_cast<const uint4*>(kp + ko);
        x.k[g][0] = t.x;
        x.k[g][1] = t.y;
        x.k[g][2] = t.z;
        x.k[g][3] = t.w;
      } else {
        const uint2 t = *reinterpret_cast<const uint2*>(kp + ko);
        x.k[g][0] = t.x;
        x.k[g][1] = t.y;
      }
      const uint32_t vo = (uint32_t)(4 * kq * (D / 2) + 4 * (D == 128 ? pr : pr >> 1));
#pragma unroll
      for (int i = 0; i < 4; ++i)
        x.v[g][i] = *reinterpret_cast<const uint32_t*>(vp + vo + i * (D / 2));
    }
    const int64_t r = (lane & 16) ? row[1] : row[0];
    x.par = *reinterpret_cast<const uint2*>(c.par + 4 * (r + pr));
  };
  const bool any = k_begin < k_stop;
  if (any) load_block(k_begin, blk[0]);

  // ---- queries: rotated, scaled by one power of two into the fp16 range, in operand order
  {
    constexpr int PER = 4 * RT;  // rows of a wave
    float x[PER][D / 64];
    float qm = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int r = wave + 4 * i;
#pragma unroll
      for (int e = 0; e < D / 64; ++e) x[i][e] = 0.0f;
      if (r < rows) {
        const uint16_t* src = a.q + (int64_t)(w.s.q0 + r / G) * a.ldq + (int64_t)(hk * G + r % G) * D;
        if constexpr (D == 128) {
          const uint32_t t = reinterpret_cast<const uint32_t*>(src)[lane];
          x[i][0] = bf16_lo(t);
          x[i][1] = bf16_hi(t);
        } else {
          x[i][0] = bf16_lo(src[lane]);
        }
        if (a.k_had) rotate_wave<D>(x[i], lane);
      }
#pragma unroll
      for (int e = 0; e < D / 64; ++e) qm = fmaxf(qm, fabsf(x[i][e]));
    }
    qm = wave_max(qm);
    if (lane == 0) s_qmax[wave] = qm;
    __syncthreads();
    qm = fmaxf(fmaxf(s_qmax[0], s_qmax[1]), fmaxf(s_qmax[2], s_qmax[3]));
    const int e15 = 15 - __builtin_amdgcn_frexp_expf(qm);  // the largest query in [2^14, 2^15)
    if (tid < 4) s_scale[tid] = (float)e15;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int r = wave + 4 * i;
      float sum = 0.0f;
#pragma unroll
      for (int e = 0; e < D / 64; ++e) {
        const int d = lane * (D / 64) + e, f = d & 7;
        const _Float16 h = (_Float16)__builtin_amdgcn_ldexpf(x[i][e], f & 1 ? e15 - 4 : e15);
        u.q[r][(d & ~7) + (f < 4 ? 2 * f : 2 * f - 7)] = h;
        sum += f & 1 ? 16.0f * (float)h : (float)h;
      }
      sum = wave_sum(sum);
      if (lane == 0) s_qsum[r] = sum;
    }
    __syncthreads();
  }
  // scores in the log2 domain: dots carry 2^(e15 - 24), sums of q 2^e15
  const int e15 = (int)s_scale[0];
  const float slope = __builtin_amdgcn_ldexpf(a.sm_scale * LOG2E, 24 - e15);
  h8_t qb[RT][NW];
  float qs[RT], m[RT], l[RT], zs[RT];
  int pos[RT];
  f4_t o[RT][NM];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
#pragma unroll
    for (int j = 0; j < NW; ++j)
      qb[t][j] = *reinterpret_cast<const h8_t*>(&u.q[16 * t + pr][kq * (D / 4) + 8 * j]);
    qs[t] = __builtin_amdgcn_ldexpf(s_qsum[16 * t + pr], -24);
    pos[t] = w.s.pos0 + (16 * t + pr) / G;
    m[t] = LOWEST;
    l[t] = zs[t] = 0.0f;
#pragma unroll
    for (int k = 0; k < NM; ++k) o[t][k] = f4_t{0.0f, 0.0f, 0.0f, 0.0f};
  }
  float v_lim = 0.0f;   // the largest value scale met, rounded up to a power of two
  float v_mul = 1.0f;   // 2^7 / v_lim: weights stay below 2^(7 + TAU)

  auto compute = [&](int k0, const Block<D>& x) {
    // ---- the positions' parameters, by one lane each
    const int key = k0 + lane;
    const bool valid = lane < 32 && ((x.ok >> (lane >> 4)) & 1) && key < k_stop;
    const uint32_t vm = (uint32_t)__builtin_amdgcn_ballot_w64(valid);
    const float sk = valid ? slope * fp16_bits_to_f32((uint16_t)x.par.x) : 0.0f;
    const float zk = valid ? (float)(int16_t)(x.par.x >> 16) : 0.0f;
    const float sv = valid ? fp16_bits_to_f32((uint16_t)x.par.y) : 0.0f;
    const float zv = valid ? (float)(int16_t)(x.par.y >> 16) : 0.0f;
    if (__builtin_amdgcn_ballot_w64(sv > v_lim)) {
      const float top = wave_max(sv);
      const float lim = __builtin_amdgcn_ldexpf(1.0f, __builtin_amdgcn_frexp_expf(top));
      const float f = v_lim / lim;
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        zs[t] *= f;
#pragma unroll
        for (int k = 0; k < NM; ++k) o[t][k] *= f;
      }
      v_lim = lim;
      v_mul = 128.0f / lim;
    }
    if (lane < 32) s_par[wave][lane] = make_float4(sk, -sk * zk, sv * v_mul, zv);
    __builtin_amdgcn_wave_barrier();
    f4_t d[RT][2];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
#pragma unroll
      for (int t = 0; t < RT; ++t) d[t][g] = f4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < NW; ++j) {
        const uint32_t y = x.k[g][j], y8 = y >> 8;
        const uint4 kk = make_uint4(y & 0x000F000Fu, y & 0x00F000F0u, y8 & 0x000F000Fu, y8 & 0x00F000F0u);
#pragma unroll
        for (int t = 0; t < RT; ++t)
          d[t][g] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8_t, kk), qb[t][j],
                                                           d[t][g], 0, 0, 0);
      }
    }
    float4 p4[2][4];
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int r = 0; r < 4; ++r) p4[g][r] = s_par[wave][16 * g + 4 * kq + r];
    __builtin_amdgcn_wave_barrier();
    uint32_t wb[RT][4];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      float sc[2][4], top = -__builtin_inff();
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          sc[g][r] = __builtin_fmaf(p4[g][r].x, d[t][g][r], p4[g][r].y * qs[t]);
      if (vm != 0xFFFFFFFFu || k0 + 31 > w.s.pos0) {
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int j = 16 * g + 4 * kq + r;
            if (!((vm >> j) & 1) || k0 + j > pos[t]) sc[g][r] = -__builtin_inff();
          }
      }
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, sc[g][r]);
      // The row's reference maximum moves only when a block passes it by more than TAU.
      if (__builtin_amdgcn_ballot_w64(top > m[t] + TAU)) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float mn = fmaxf(m[t], top);
        const float f = __builtin_amdgcn_exp2f(m[t] - mn);
        m[t] = mn;
        l[t] *= f;
        zs[t] *= f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float fr = __shfl(f, 4 * kq + r);
#pragma unroll
          for (int k = 0; k < NM; ++k) o[t][k][r] *= fr;
        }
      }
      float wf[2][4];
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float p = __builtin_amdgcn_exp2f(sc[g][r] - m[t]);
          l[t] += p;
          wf[g][r] = p * p4[g][r].z;
        }
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const h2_t h = {(_Float16)wf[g][2 * r], (_Float16)wf[g][2 * r + 1]};
          wb[t][2 * g + r] = __builtin_bit_cast(uint32_t, h);
          zs[t] = __builtin_fmaf((float)h.x, p4[g][2 * r].w, zs[t]);
          zs[t] = __builtin_fmaf((float)h.y, p4[g][2 * r + 1].w, zs[t]);
        }
    }
    // ---- values: operand slots 4 kq .. 4 kq + 3 of both groups, two positions a word
    uint32_t xs[4][NM / 2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t p = x.v[i >> 1][2 * (i & 1)], q = x.v[i >> 1][2 * (i & 1) + 1];
      if constexpr (D == 128) {
        xs[i][0] = __builtin_amdgcn_perm(q, p, 0x05040100u);
        xs[i][2] = __builtin_amdgcn_perm(q, p, 0x07060302u);
        xs[i][3] = xs[i][2] >> 8;
      } else {  // columns of four channels: the lower or upper half of the word
        xs[i][0] = __builtin_amdgcn_perm(q, p, pr & 1 ? 0x07060302u : 0x05040100u);
      }
      xs[i][1] = xs[i][0] >> 8;
    }
#pragma unroll
    for (int k = 0; k < NM; ++k) {
      const uint32_t mask = (k & 1) ? 0x00F000F0u : 0x000F000Fu;
      const uint4 vv = make_uint4(xs[0][k >> 1] & mask, xs[1][k >> 1] & mask, xs[2][k >> 1] & mask,
                                  xs[3][k >> 1] & mask);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const uint4 ww = make_uint4(wb[t][0], wb[t][1], wb[t][2], wb[t][3]);
        o[t][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8_t, ww),
                                                         __builtin_bit_cast(h8_t, vv), o[t][k], 0, 0, 0);
      }
    }
  };

  for (int k0 = k_begin; k0 < k_stop; k0 += 64) {
    // (the ids of the block after this pair: a lane for each 16 positions, 1024 in all)
    auto next = [&](int k, Block<D>& x) {
      if (k >= k_stop) return;
      if (k - id0 >= 1024) {
        id0 = k;
        ids = load_ids(id0);
      }
      load_block(k, x);
    };
    next(k0 + 32, blk[1]);
    compute(k0, blk[0]);
    next(k0 + 64, blk[0]);
    if (k0 + 32 < k_stop) compute(k0 + 32, blk[1]);
  }

  // ---- join the waves, a row tile at a time
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    l[t] += __shfl_xor(l[t], 16);
    l[t] += __shfl_xor(l[t], 32);
    zs[t] += __shfl_xor(zs[t], 16);
    zs[t] += __shfl_xor(zs[t], 32);
    if (lane < 16) {
      s_m[wave][16 * t + pr] = m[t];
      s_l[wave][16 * t + pr] = l[t];
      s_z[wave][16 * t + pr] = zs[t];
    }
  }
  __syncthreads();
  const float v_back = 1.0f / v_mul;
  for (int t = 0; t < RT; ++t) {
    if (16 * t >= rows) break;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * t + 4 * kq + r;
      const float top = fmaxf(fmaxf(s_m[0][row], s_m[1][row]), fmaxf(s_m[2][row], s_m[3][row]));
      const float f = __builtin_amdgcn_exp2f(s_m[wave][row] - top) * v_back, z = s_z[wave][row];
#pragma unroll
      for (int k = 0; k < NM; ++k) {
        f4_t ov = o[0][k];
#pragma unroll
        for (int tt = 1; tt < RT; ++tt)
          if (tt == t) ov = o[tt][k];
        u.o[wave][4 * kq + r][NM * pr + k] =
            (__builtin_amdgcn_ldexpf(ov[r], k & 1 ? 20 : 24) - z) * f;
      }
    }
    __syncthreads();
    for (int i = wave; i < 16 && 16 * t + i < rows; i += 4) {
      const int row = 16 * t + i;
      float ov[D / 64];
#pragma unroll
      for (int e = 0; e < D / 64; ++e) {
        const int d = lane * (D / 64) + e;
        ov[e] = (u.o[0][i][d] + u.o[1][i][d]) + (u.o[2][i][d] + u.o[3][i][d]);
      }
      const float top = fmaxf(fmaxf(s_m[0][row], s_m[1][row]), fmaxf(s_m[2][row], s_m[3][row]));
      float lt = 0.0f;
#pragma unroll
      for (int k = 0; k < 4; ++k) lt = __builtin_fmaf(s_l[k][row], __builtin_amdgcn_exp2f(s_m[k][row] - top), lt);
      if (w.nchunk == 1) {
        store_row<D>(a, w.s.q0 + row / G, hk * G + row % G, ov, lt, lane);
      } else {
        float* dst = rec + (int64_t)unit * few_rows * (D + 2);
        if (lane == 0) *reinterpret_cast<float2*>(dst + 2 * row) = make_float2(top, lt);
        dst += 2 * few_rows + row * D;
        if constexpr (D == 128) reinterpret_cast<float2*>(dst)[lane] = make_float2(ov[0], ov[1]);
        else dst[lane] = ov[0];
      }
    }
    __syncthreads();
  }
}

// Joins the chunks of a row: one workgroup per (sequence, key/value head, row), four waves over
// the chunks.
template <int D>
__global__ __launch_bounds__(256) void kv_attention_paged_join_kernel(
    PagedAttentionArgs a, int Hkv, int cap, const Joint* __restrict__ joints,
    const float* __restrict__ rec, int log2p, int few_rows) {
  __shared__ float s_o[4][D], s_ml[2][4];
  const int lane = (int)__builtin_amdgcn_workitem_id_x() & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)__builtin_amdgcn_workitem_id_x() >> 6);
  const int G = a.Hq / Hkv;
  const int id = (int)__builtin_amdgcn_workgroup_id_x();
  const int hk = id % Hkv, row = id / Hkv % cap, b = id / Hkv / cap;
  const Seq s = sequence(a, log2p, G, b);
  if (row >= s.rows || s.rows > few_rows) return;
  const Joint j = joints[b];
  if (j.nchunk <= 1) return;
  const int64_t size = (int64_t)cap * (D + 2);
  const float* first = rec + (int64_t)(j.unit0 + hk * j.nchunk) * size;
  float top = LOWEST;
  for (int i = lane; i < j.nchunk; i += 64) top = fmaxf(top, first[i * size + 2 * row]);
  top = wave_max(top);
  float l = 0.0f, o[D / 64] = {};
  for (int i0 = 64 * wave; i0 < j.nchunk; i0 += 256) {
    float f = 0.0f;
    if (i0 + lane < j.nchunk) {
      const float2 ml = *reinterpret_cast<const float2*>(first + (i0 + lane) * size + 2 * row);
      f = __builtin_amdgcn_exp2f(ml.x - top);
      l = __builtin_fmaf(f, ml.y, l);
    }
    const int n = min(64, j.nchunk - i0);
    const float* src = first + i0 * size + 2 * cap + row * D + lane * (D / 64);
    for (int k = 0; k < n; k += 8) {  // (factors past the last chunk are 0)
      float v[8][D / 64];
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < D / 64; ++e) v[i][e] = src[min(k + i, n - 1) * size + e];
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < D / 64; ++e) o[e] = __builtin_fmaf(__shfl(f, k + i), v[i][e], o[e]);
    }
  }
  l = wave_sum(l);
  if (lane == 0) s_ml[0][wave] = l;
#pragma unroll
  for (int e = 0; e < D / 64; ++e) s_o[wave][lane * (D / 64) + e] = o[e];
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int e = 0; e < D / 64; ++e) {
    const int d = lane * (D / 64) + e;
    o[e] = (s_o[0][d] + s_o[1][d]) + (s_o[2][d] + s_o[3][d]);
  }
  l = (s_ml[0][0] + s_ml[0][1]) + (s_ml[0][2] + s_ml[0][3]);
  store_row<D>(a, j.q0 + row / G, hk * G + row % G, o, l, lane);
}

// One wave per (query row, head): 64 positions at a time, a lane first holding one position's
// score, then D / 64 channels of the output.
template <int D>
__global__ __launch_bounds__(64) void kv_attention_paged_kernel(PagedAttentionArgs a, PagedCache c,
                                                               int few_rows) {
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
  const int G = a.Hq / c.Hkv, hk = hq / G;
  if (min(n, a.max_new) * G <= few_rows) return;
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

namespace {

// How the few-row kernel is launched: the rows it takes, its row tiles, and its units.
struct Few {
  int rows, tiles, target, units, max_chunks;
  bool join;
};
Few few_shape(int64_t B, int64_t Hq, int64_t Hkv, int64_t max_new, int64_t cap) {
  const int64_t G = Hq / Hkv, most = max_new * G;
  Few f;
  f.tiles = most <= 16 ? 1 : most <= 32 ? 2 : most <= 64 ? 4 : 1;
  f.rows = (int)(most <= 64 ? most : 16);
  f.target = 1024;
  f.max_chunks = 256;
  f.join = cap > CHUNK_MIN;
  f.units = (int)(f.join ? f.target + B * Hkv : B * Hkv);
  return f;
}

}  // namespace

int64_t kv_attention_paged_workspace_floats(int64_t M, int64_t B, int64_t Hq, int64_t Hkv,
                                            int head_dim, int64_t max_new) {
  const Few f = few_shape(B, Hq, Hkv, max_new, int64_t(1) << 30);
  return 4 * B + (int64_t)f.units * f.rows * (head_dim + 2);
}

hipError_t launch_kv_attention_paged(const PagedAttentionArgs& a, const PagedCache& c, int head_dim,
                                     float* workspace, hipStream_t stream) {
  const Few f = few_shape(a.B, a.Hq, c.Hkv, a.max_new, (int64_t)a.max_pages << c.log2p);
  Joint* joints = f.join ? reinterpret_cast<Joint*>(workspace) : nullptr;
  float* rec = workspace + 4 * (int64_t)a.B;
#define OFFQ_FEW(D_, RT_)                                                                        \
  hipLaunchKernelGGL((kv_attention_paged_few_kernel<D_, RT_>), dim3((unsigned)f.units), dim3(256), \
                     0, stream, a, c, f.rows, f.target, f.max_chunks, joints, rec)
  if (head_dim == 128) {
    if (f.tiles == 1) OFFQ_FEW(128, 1);
    else if (f.tiles == 2) OFFQ_FEW(128, 2);
    else OFFQ_FEW(128, 4);
  } else {
    if (f.tiles == 1) OFFQ_FEW(64, 1);
    else if (f.tiles == 2) OFFQ_FEW(64, 2);
    else OFFQ_FEW(64, 4);
  }
#undef OFFQ_FEW
  if (f.join) {
    const dim3 grid((unsigned)(f.rows * c.Hkv * a.B));
    hipLaunchKernelGGL(head_dim == 128 ? kv_attention_paged_join_kernel<128> : kv_attention_paged_join_kernel<64>,
                       grid, dim3(256), 0, stream, a, c.Hkv, f.rows, joints, rec, c.log2p, f.rows);
  }
  if (a.max_new * (a.Hq / c.Hkv) > f.rows) {
    const dim3 grid((unsigned)a.M, (unsigned)a.Hq);
    hipLaunchKernelGGL(head_dim == 128 ? kv_attention_paged_kernel<128> : kv_attention_paged_kernel<64>,
                       grid, dim3(64), 0, stream, a, c, f.rows);
  }
  return hipGetLastError();
}

}  // namespace offq
