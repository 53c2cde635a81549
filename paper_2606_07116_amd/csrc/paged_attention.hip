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
// Positions of a chunk, at least: of one that is joined, and where no sequence is longer.  (A chunk
// that is joined at all may as well be short: one token after 4 x 2000 positions 12.9 us, with 512
// 14.2; one after 300 in a cache of 304: 12.2 us with 256 and the join, 9.9 without.)
constexpr int CHUNK_MIN = 256, CHUNK_ONE = 512;

typedef _Float16 h8_t __attribute__((ext_vector_type(8)));
typedef _Float16 h2_t __attribute__((ext_vector_type(2)));
typedef __bf16 b8_t __attribute__((ext_vector_type(8)));
typedef float f4_t __attribute__((ext_vector_type(4)));

constexpr float TAU = 8.0f;     // a row's reference maximum may lag by up to 2^TAU
constexpr float LOWEST = -1e30f;  // a reference maximum below every score

// (a uniform value that went through the vector units, a division for instance)
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// A position whose scales are not both finite (a row that was never written): its key's becomes
// NaN, and so what sees it; its value's 0, since a weight of 0 times NaN or infinity would reach
// the rows that do not.
__device__ __forceinline__ uint2 for_those_who_see(uint2 par) {
  const bool bad = ((par.x & 0x7C00u) == 0x7C00u) | ((par.y & 0x7C00u) == 0x7C00u);
  return make_uint2(bad ? 0x7E00u : par.x, bad ? 0u : par.y);
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
// chosen on the device so that the resident workgroups get one each whatever the lengths are; a
// chunk's four waves take a quarter each, and a second kernel joins a row's chunks.
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
// neither tiny nor huge scales leave its range: the query by a power of two of its row, the
// weights by one that follows the largest value scale met (values of scales 2^21 below it lose bits).
//
// Measured (a large copy here: 4.9 TB/s, reads alone 6.2): 8 x 32768 positions of 32 heads of their
// own 205 us, 5.6 TB/s; 24 ragged sequences of up to 30000, five query heads to each of 8, 70 us
// with the join's 5; 16 x 4097 21 us for 72 MB.  A workgroup costs 6 us besides its positions'
// bytes (who it is, page ids, first block, queries, the waves' join), which is what is left there
// and below: one token after 300 positions 8.3 us.
struct Chunking {
  int len;          // positions per chunk, a multiple of 128
  int b, head, chunk, nchunk, unit0;  // this unit's; unit0: the sequence's first unit
  bool found;
  Seq s;
};

// The chunk length.  `slots` workgroups are resident at once.  One round of units costs its longest
// chunk, so the shortest length whose units fit the slots is tried first; where it is far above
// the mean (a few long sequences among many), or there are more sequences than slots, chunks of
// half the mean in several rounds.  The cost of a unit besides its positions is that of about 400
// (6 us).  `blocks` of 128 positions; units(len): how many units that gives.
template <typename Units>
__device__ __forceinline__ int chunk_length(int64_t blocks, int Hkv, int slots, int chunk_min, Units units) {
  const int mean = uniform((int)min((blocks * Hkv * 128 + slots - 1) / slots, (int64_t)1 << 30));
  auto round_up = [&](int64_t v) { return (int)max((int64_t)chunk_min, (v + 127) & ~(int64_t)127); };
  const int several = round_up((mean + 1) / 2);  // at most 2 slots + a unit per sequence and head
  int len = round_up(mean);
  if (units(1 << 30) > slots) return several;  // (no sequence is longer)
  while (units(len) > slots) {
    if (len > mean + several / 2 + 400) return several;
    len = round_up(len + len / 16 + 1);
  }
  return len;
}

// The rows of a chunk that the second kernel joins: per (sequence) where its units start.
struct alignas(16) Joint {
  int q0, rows, nchunk, unit0;
};

// The plan of a call of more than 64 sequences, made by a kernel of its own: the sequences'
// joints and first tiles, and what they come from.
struct alignas(16) Plan {
  int len, tiles, pad[2];
};

// The last of `n` ascending numbers that is not above x; the first is not.
template <typename First>
__device__ __forceinline__ int last_not_above(int n, int x, First first) {
  const int lane = (int)__builtin_amdgcn_workitem_id_x() & 63;
  int lo = 0;
  while (n > 1) {
    const int step = (n + 63) >> 6, i = lane * step;
    const bool below = i < n && first(lo + min(i, n - 1)) <= x;
    const int k = __builtin_popcountll(__builtin_amdgcn_ballot_w64(below)) - 1;
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo;
}

// What unit `unit` is.  Without a plan (up to 64 sequences, one a lane) every wave works it out for
// itself.
__device__ __forceinline__ Chunking find_chunk(const PagedAttentionArgs& a, int log2p, int Hkv,
                                               int few_rows, int slots, int chunk_min,
                                               const Plan* plan, const Joint* joints, int unit) {
  const int lane = (int)__builtin_amdgcn_workitem_id_x() & 63;
  const int G = a.Hq / Hkv;
  Chunking c{};
  if (plan) {
    c.b = last_not_above(a.B, unit, [&](int b) { return joints[b].unit0; });
    const Joint j = joints[c.b];
    c.len = plan->len;
    c.nchunk = uniform(j.nchunk);
    c.unit0 = uniform(j.unit0);
    c.found = unit - c.unit0 < Hkv * c.nchunk;
    c.s = sequence(a, log2p, G, c.b);
  } else {
    Seq s{};
    if (lane < a.B) s = sequence(a, log2p, G, lane);
    if (s.rows > few_rows) s.rows = 0;
    auto chunks = [&](int len) { return s.rows ? max(1, (s.keys + len - 1) / len) : 0; };
    c.len = chunk_length(wave_add(s.rows ? (s.keys + 127) >> 7 : 0), Hkv, slots, chunk_min,
                         [&](int len) { return Hkv * wave_add(chunks(len)); });
    const int nc = chunks(c.len);
    const int first = wave_scan(nc) - nc;
    const uint64_t mine =
        __builtin_amdgcn_ballot_w64(nc > 0 && unit >= Hkv * first && unit < Hkv * (first + nc));
    if (!mine) return c;
    c.found = true;
    c.b = __builtin_ctzll(mine);
    c.nchunk = __builtin_amdgcn_readlane(nc, c.b);
    c.unit0 = Hkv * __builtin_amdgcn_readlane(first, c.b);
    c.s.q0 = __builtin_amdgcn_readlane(s.q0, c.b);
    c.s.rows = __builtin_amdgcn_readlane(s.rows, c.b);
    c.s.keys = __builtin_amdgcn_readlane(s.keys, c.b);
    c.s.pos0 = __builtin_amdgcn_readlane(s.pos0, c.b);
  }
  if (!c.found) return c;
  c.head = uniform((unit - c.unit0) / c.nchunk);
  c.chunk = unit - c.unit0 - c.head * c.nchunk;
  return c;
}

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
  for (int e = 0; e < D / 64; ++e) {
    x[e] = lane_butterfly<1>(x[e], lane);
    x[e] = lane_butterfly<2>(x[e], lane);
    x[e] = lane_butterfly<4>(x[e], lane);
    x[e] = lane_butterfly<8>(x[e], lane);
    x[e] = lane_butterfly<16>(x[e], lane);
    x[e] = lane_butterfly<32>(x[e], lane);
  }
#pragma unroll
  for (int e = 0; e < D / 64; ++e) x[e] *= hadamard_norm<D>();
}

// A finished row: o / l (0 where nothing was seen; NaN stays), rotated back if asked, rounded once.  The
// wave holds channels lane * D / 64 and on.
template <int D>
__device__ __forceinline__ void store_row(const PagedAttentionArgs& a, int row, int hq, float (&o)[D / 64],
                                          float l, int lane) {
#pragma unroll
  for (int e = 0; e < D / 64; ++e) o[e] = l == 0.0f ? 0.0f : o[e] / l;
  if (a.v_had) rotate_wave<D>(o, lane);
  uint16_t* dst = a.out + (int64_t)row * a.ldo + (int64_t)hq * D;
  if constexpr (D == 128) reinterpret_cast<uint32_t*>(dst)[lane] = bf16x2_rne(o[0], o[1]);
  else dst[lane] = f32_to_bf16_rne(o[0]);
}

template <int D, int RT>
__global__ __launch_bounds__(256, 2) void
kv_attention_paged_few_kernel(PagedAttentionArgs a, PagedCache c, int few_rows, int slots,
                              int chunk_min, const Plan* __restrict__ plan,
                              Joint* __restrict__ joints, float* __restrict__ rec) {
  constexpr int NW = D / 32;  // key code words of a lane
  constexpr int NM = D / 16;  // products of a value block: 16 columns of NM channels each
  constexpr int OROW = D + 4;
  __shared__ union {
    _Float16 q[16 * RT][D + 8];  // the queries in operand order
    float o[4][16][OROW];        // a row tile's outputs, one per wave
  } u;
  // per wave and position: (score slope, score offset / sum q), (sv, zv)
  __shared__ alignas(16) float2 s_kp[4][32], s_vp[4][32];
  __shared__ float s_qsum[16 * RT], s_slope[16 * RT];
  __shared__ float s_m[4][16 * RT], s_l[4][16 * RT], s_z[4][16 * RT];

  const int tid = (int)__builtin_amdgcn_workitem_id_x();
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int pr = lane & 15, kq = lane >> 4;
  const int unit = (int)__builtin_amdgcn_workgroup_id_x();
  const int G = a.Hq / c.Hkv;
  const Chunking w = find_chunk(a, c.log2p, c.Hkv, few_rows, slots, chunk_min, plan, joints, unit);
  if (!w.found) return;
  const int rows = w.s.rows, hk = w.head;
  if (joints && !plan && w.chunk == 0 && hk == 0 && tid == 0)
    joints[w.b] = Joint{w.s.q0, rows, w.nchunk, w.unit0};
  // the chunk, the sequence's chunks being alike, and the wave's quarter of it
  const int len = uniform(((w.s.keys + w.nchunk - 1) / w.nchunk + 127) & ~127);
  const int k_end = min(w.s.keys, (w.chunk + 1) * len);
  const int quarter = ((k_end - w.chunk * len + 127) >> 7) * 32;
  const int k_begin = w.chunk * len + wave * quarter;
  const int k_stop = min(k_end, k_begin + quarter);

  // ---- page ids: lane i holds that of the 16 positions from id0 + 16 i on
  const int32_t* table = a.page_table + (int64_t)w.b * a.max_pages;
  auto load_ids = [&](int from) {
    const int key = from + 16 * lane;
    int id = key < k_stop ? table[key >> c.log2p] : -1;
    // (waited for here, where it is rare: not after the branch, with all loads in flight)
    asm volatile("" : "+v"(id));
    return id;
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

  // ---- queries: rotated, scaled by a power of two into the fp16 range, in operand order.  D / 8
  // lanes a row.  (A loop that stays one: unrolled, its code costs more to fetch than its work.)
  constexpr int LPH = D / 8, NG = 64 / LPH;
  const int l8 = lane & (LPH - 1), g8 = lane / LPH;
  {
    uint4 next;
    auto fetch = [&](int r) {
      r = min(r, rows - 1);
      next = *reinterpret_cast<const uint4*>(a.q + (int64_t)(w.s.q0 + r / G) * a.ldq +
                                             (int64_t)(hk * G + r % G) * D + 8 * l8);
    };
    if (NG * wave < rows) fetch(NG * wave + g8);
#pragma unroll 1
    for (int r0 = NG * wave; r0 < rows; r0 += 4 * NG) {
      const int r = r0 + g8;
      float x[8] = {bf16_lo(next.x), bf16_hi(next.x), bf16_lo(next.y), bf16_hi(next.y),
                    bf16_lo(next.z), bf16_hi(next.z), bf16_lo(next.w), bf16_hi(next.w)};
      if (r0 + 4 * NG < rows) fetch(r + 4 * NG);
      if (a.k_had) {
        fwht_lanes<LPH>(x, l8);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= hadamard_norm<D>();
      }
      float qm = 0.0f, sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) qm = fmaxf(qm, fabsf(x[i]));
      qm = group_reduce<LPH>(qm, [](float p, float q) { return fmaxf(p, q); });
      const int e15 = 15 - __builtin_amdgcn_frexp_expf(qm);  // the row's largest in [2^14, 2^15)
      uint32_t word[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {  // channels k and k + 4, the odd ones / 16
        const int e = k & 1 ? e15 - 4 : e15;
        const h2_t h = {(_Float16)__builtin_amdgcn_ldexpf(x[k], e), (_Float16)__builtin_amdgcn_ldexpf(x[k + 4], e)};
        const float both = (float)h.x + (float)h.y;
        sum += k & 1 ? 16.0f * both : both;
        word[k] = __builtin_bit_cast(uint32_t, h);
      }
      sum = group_reduce<LPH>(sum, [](float p, float q) { return p + q; });
      if (r < rows) {
        *reinterpret_cast<uint4*>(&u.q[r][8 * l8]) = make_uint4(word[0], word[1], word[2], word[3]);
        // scores in the log2 domain: dots carry 2^(e15 - 24), sums of q 2^e15
        if (l8 == 0) {
          s_qsum[r] = __builtin_amdgcn_ldexpf(sum, -24);
          s_slope[r] = __builtin_amdgcn_ldexpf(a.sm_scale * LOG2E, 24 - e15);
        }
      }
    }
    for (int i = 64 * wave + lane; i < (16 * RT - rows) * (D / 8); i += 256)
      *reinterpret_cast<uint4*>(&u.q[rows + i / (D / 8)][i % (D / 8) * 8]) = make_uint4(0, 0, 0, 0);
    if (tid >= rows && tid < 16 * RT) {
      s_qsum[tid] = 0.0f;
      s_slope[tid] = 1.0f;  // (finite and not 0: -inf at a masked position stays that)
    }
    __syncthreads();
  }
  h8_t qb[RT][NW];
  float qs[RT], slope[RT], m[RT], l[RT], zs[RT];
  int pos[RT];
  f4_t o[RT][NM];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
#pragma unroll
    for (int j = 0; j < NW; ++j)
      qb[t][j] = *reinterpret_cast<const h8_t*>(&u.q[16 * t + pr][kq * (D / 4) + 8 * j]);
    qs[t] = s_qsum[16 * t + pr];
    slope[t] = s_slope[16 * t + pr];
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
    // (no branch here: behind one, the wait for the parameters takes in the next block's loads)
    const bool valid = (lane < 32) & ((x.ok >> (lane >> 4 & 1)) & 1) & (key < k_stop);
    const uint32_t vm = (uint32_t)__builtin_amdgcn_ballot_w64(valid);
    const uint2 par = for_those_who_see(x.par);
    const float sk = valid ? fp16_bits_to_f32((uint16_t)par.x) : 0.0f;
    const float zk = valid ? (float)(int16_t)(par.x >> 16) : 0.0f;
    const float sv = valid ? fp16_bits_to_f32((uint16_t)par.y) : 0.0f;
    const float zv = valid ? (float)(int16_t)(par.y >> 16) : 0.0f;
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
    if (lane < 32) {
      s_kp[wave][lane] = make_float2(sk, -sk * zk);
      s_vp[wave][lane] = make_float2(sv * v_mul, zv);
    }
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
    // this lane's positions, two to a 16-byte read
    float4 kp[4], vp[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      kp[i] = *reinterpret_cast<const float4*>(&s_kp[wave][16 * (i >> 1) + 4 * kq + 2 * (i & 1)]);
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f4_t& x = d[t][i >> 1];
        const int r = 2 * (i & 1);
        x[r] = __builtin_fmaf(kp[i].x, x[r], kp[i].y * qs[t]);
        x[r + 1] = __builtin_fmaf(kp[i].z, x[r + 1], kp[i].w * qs[t]);
      }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      vp[i] = *reinterpret_cast<const float4*>(&s_vp[wave][16 * (i >> 1) + 4 * kq + 2 * (i & 1)]);
    uint32_t wb[RT][4];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      f4_t (&sc)[2] = d[t];
      float top = -__builtin_inff();
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
      if (__builtin_amdgcn_ballot_w64(__builtin_fmaf(top, slope[t], -m[t]) > TAU)) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float mn = fmaxf(m[t], top * slope[t]);
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
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i >> 1][2 * (i & 1)], slope[t], -m[t]));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i >> 1][2 * (i & 1) + 1], slope[t], -m[t]));
        l[t] += p0 + p1;
        const h2_t h = {(_Float16)(p0 * vp[i].x), (_Float16)(p1 * vp[i].z)};
        wb[t][i] = __builtin_bit_cast(uint32_t, h);
        zs[t] = __builtin_fmaf((float)h.x, vp[i].y, zs[t]);
        zs[t] = __builtin_fmaf((float)h.y, vp[i].w, zs[t]);
      }
    }
    __builtin_amdgcn_wave_barrier();
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

  const int k_last = k_begin + ((k_stop - 1 - k_begin) & ~31);
  for (int k0 = k_begin; k0 < k_stop; k0 += 64) {
    // (Past the end the last block again: behind a branch around the loads, the waits for the block
    // before would take them in.  Page ids: a lane for each 16 positions, 1024 in all.)
    auto next = [&](int k, Block<D>& x) {
      k = min(k, k_last);
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
    if (16 * t + 4 * kq < rows) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * t + 4 * kq + r;
        const float top = fmaxf(fmaxf(s_m[0][row], s_m[1][row]), fmaxf(s_m[2][row], s_m[3][row]));
        const float f = __builtin_amdgcn_exp2f(s_m[wave][row] - top) * v_back, z = s_z[wave][row];
        float y[NM];
#pragma unroll
        for (int k = 0; k < NM; ++k) {
          f4_t ov = o[0][k];
#pragma unroll
          for (int tt = 1; tt < RT; ++tt)
            if (tt == t) ov = o[tt][k];
          y[k] = (__builtin_amdgcn_ldexpf(ov[r], k & 1 ? 20 : 24) - z) * f;
        }
#pragma unroll
        for (int k = 0; k < NM; k += 4)
          *reinterpret_cast<float4*>(&u.o[wave][4 * kq + r][NM * pr + k]) =
              make_float4(y[k], y[k + 1], y[k + 2], y[k + 3]);
      }
    }
    __syncthreads();
    const int i = NG * wave + g8, row = 16 * t + i;
    if (i < 16 && row < rows) {
      float y[8] = {};
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int c = 0; c < 8; c += 4) {
          const float4 v = *reinterpret_cast<const float4*>(&u.o[k][i][8 * l8 + c]);
          y[c] += v.x;
          y[c + 1] += v.y;
          y[c + 2] += v.z;
          y[c + 3] += v.w;
        }
      const float top = fmaxf(fmaxf(s_m[0][row], s_m[1][row]), fmaxf(s_m[2][row], s_m[3][row]));
      float lt = 0.0f;
#pragma unroll
      for (int k = 0; k < 4; ++k) lt = __builtin_fmaf(s_l[k][row], __builtin_amdgcn_exp2f(s_m[k][row] - top), lt);
      if (w.nchunk == 1) {  // (as in store_row)
        const float f = lt == 0.0f ? 0.0f : 1.0f / lt;
#pragma unroll
        for (int c = 0; c < 8; ++c) y[c] *= f;
        if (a.v_had) {
          fwht_lanes<LPH>(y, l8);
#pragma unroll
          for (int c = 0; c < 8; ++c) y[c] *= hadamard_norm<D>();
        }
        *reinterpret_cast<uint4*>(a.out + (int64_t)(w.s.q0 + row / G) * a.ldo + (int64_t)(hk * G + row % G) * D +
                                  8 * l8) = make_uint4(bf16x2_rne(y[0], y[1]), bf16x2_rne(y[2], y[3]),
                                                       bf16x2_rne(y[4], y[5]), bf16x2_rne(y[6], y[7]));
      } else {
        float* dst = rec + (int64_t)unit * few_rows * (D + 2);
        if (l8 == 0) *reinterpret_cast<float2*>(dst + 2 * row) = make_float2(top, lt);
        dst += 2 * few_rows + row * D + 8 * l8;
#pragma unroll
        for (int c = 0; c < 8; c += 2) *reinterpret_cast<float2*>(dst + c) = make_float2(y[c], y[c + 1]);
      }
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// Many rows: tiles of 256 query rows (new tokens x heads of a group) of a sequence and
// key/value head, eight waves of 32 rows, over blocks of 64 positions.  With many queries per
// key the products bound it, so both run as 32x32x16 fp16 matrix products and everything that
// can leave the score loop does:
// * a block's codes become fp16 values once per workgroup, on their way to LDS: keys A c with
//   A = sk 2^-E, values A (c - z') with A = sv 2^-F and z' the zero-point held in 0 .. 15, one
//   rounding each (2^-11; a value's zero-point term another).  E and F are the workgroup's and
//   follow the largest sk (8192 + |z|) and sv met, rarely; the query carries sm_scale log2(e) 2^E;
// * what a value's zero-point has beyond its codes, A (z - z'), is one number a row and stays in
//   fp32: blocks that have any, a flag of theirs, sum the weights times it, in the branch that
//   moves references (in fp16, offsets of 300 and 3000 steps left noise of 1.3 and 12 % of their
//   norm in the other channels of values that are rotated back);
// * the keys' zero-point term -z_j sum q, which can be far larger than the score, is a k-step of
//   its own: A z_j and sum q as three fp16 pieces each, their six leading products.  Half of its 16
//   products have z 2^12 times larger and the sum as much smaller, where the sum never leaves fp16's
//   range; the other half have what A z_j leaves beyond the range there, of the largest keys;
// * the score product starts from -m, the row's reference, so what it leaves are the exponents of
//   the weights: per weight one exp2, half a conversion to fp16 and half a dot product for the
//   sum.  A row takes its reference from the scores of the first tile that it sees, wherever they
//   lie (left at 0, rows 2^-16 to 2^-25 below it lost their weights' bits to fp16's subnormals):
//   before the loop where that is its workgroup's first tile.  That it has to move later shows in
//   the sum, infinite where a weight left the fp16 range and, so far, for a row that saw nothing;
// * S^T = K Q^T: a lane holds 16 positions of one query row per tile of 32, so maximum and sum
//   stay in the lane, and the tile is in the operand layout of O^T = V^T P^T; V^T lies in LDS with
//   the positions in the order of the accumulator and the channels as (nibble, code word), so
//   that a lane ends with eight consecutive channels of each of its words;
// * a reference puts the row's largest weight of its tile at 2^3: 2^13 below the range's end, and
//   what lies 2^27 below it still counts.  (At 2^7 the same instructions took 2 % longer, 674 us for
//   656: small weights become subnormal and 0, and the clock is as high as the bits allow.)  The
//   sum is taken of the rounded weights.
// Longest tiles start first.  Where the tiles do not fill the CUs, the keys of a tile are split
// over workgroups and the rows joined by a second kernel.
//
// Measured: 2.2 us per tile and block, 920 TFLOP/s inside, where a large library product reaches
// 1150; three prompts of up to 8000 tokens 648 to 683 us (by the card's clock) with the tiles' 8 us
// each besides their blocks, 7 % more where the values' zero-points lie beyond their codes.
// What bounds it are a block's phases, which two waves per SIMD do not hide from each other: matrix
// cores busy 44 % of the time, vector units 43 %, LDS 35 %.  Not faster: 64 rows a wave and one
// wave per SIMD (twice the time: accumulators moved about), the keys' zero-points in their codes
// and no k-step for them (2 %, and a branch for far ones takes that back), half a block between
// the waves of a SIMD, priorities, scheduling groups, two chains of accumulators.
constexpr int ROWS = 256;      // query rows of a tile
constexpr int KB = 64;         // positions of a block
constexpr int VROW = 2 * KB + 16;
constexpr float MID = 3.0f;    // a reference puts its row's largest weight of a tile at 2^MID
constexpr float HUGE_SUM = 3e38f;

typedef float f16_t __attribute__((ext_vector_type(16)));

template <int D>
struct alignas(16) Stage {
  uint8_t k[3][KB * (2 * D + 16)];  // per position: A c 2^-9, 8 fp16 per code word, in operand order
  uint8_t v[2][D * VROW];           // per channel (nibble * D / 8 + word): A (c - z) 2^-9 of the 64 positions
  struct Par {                      // what a block's codes are staged with
    uint4 z[2][KB];                 // per position: the pieces of the keys' A z: [1] of A z / 2 up
                                    // to 2^15, [0] of the rest / 2^13
    uint32_t a[KB];                 // the keys' A and A / 16
    uint32_t ab[KB];                // the values' A and -A z' 2^-9
    float rest[KB];                 // the values' A (z - z') 2^-9
    int E, F;                       // (F of values, twice, and whether any `rest` is not 0)
    uint32_t valid[2];              // bit j: position j is there
  } par[4];
};

// Workgroup barrier for LDS traffic only: global loads in flight stay in flight.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

__device__ __forceinline__ uint32_t pk_f16(float a, float b) {
  const h2_t h = {(_Float16)a, (_Float16)b};
  return __builtin_bit_cast(uint32_t, h);
}
__device__ __forceinline__ uint32_t pk_mul(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2_t, a) * __builtin_bit_cast(h2_t, b));
}
__device__ __forceinline__ uint32_t pk_fma(uint32_t a, uint32_t b, uint32_t c) {
  return __builtin_bit_cast(uint32_t,
                            __builtin_elementwise_fma(__builtin_bit_cast(h2_t, a), __builtin_bit_cast(h2_t, b),
                                                      __builtin_bit_cast(h2_t, c)));
}

// x = h1 + h2 + h3 + O(2^-33 x): fp16 pieces
struct Pieces {
  float h1, h2, h3;
};
__device__ __forceinline__ Pieces pieces(float x) {
  Pieces p;
  p.h1 = (float)(_Float16)x;
  p.h2 = (float)(_Float16)(x - p.h1);
  p.h3 = (float)(_Float16)(x - p.h1 - p.h2);
  return p;
}

struct Tile {
  int b, i;  // sequence and tile within it
  int index, count;
  bool found;
  Seq s;
};
// Tile number `t` of all sequences' tiles, counted from the last: the longest of a sequence first.
// Without a plan (up to 64 sequences, one a lane) every wave works it out for itself.  `tiles`: what
// there is room for, all of them where the starts ascend.
__device__ __forceinline__ int tiles_of(const Seq& s, int few_rows) {
  return s.rows > few_rows ? (s.rows + ROWS - 1) / ROWS : 0;
}
__device__ __forceinline__ Tile find_tile(const PagedAttentionArgs& a, int log2p, int G, int few_rows,
                                          int tiles, const Plan* plan, const int* starts, int t) {
  const int lane = (int)__builtin_amdgcn_workitem_id_x() & 63;
  Tile r{};
  if (plan) {
    r.count = min(plan->tiles, tiles);
    r.found = t < r.count;
    if (!r.found) return r;
    r.index = r.count - 1 - t;
    r.b = last_not_above(a.B, r.index, [&](int b) { return starts[b]; });
    r.i = r.index - uniform(starts[r.b]);
    r.s = sequence(a, log2p, G, r.b);
    return r;
  }
  Seq s{};
  if (lane < a.B) s = sequence(a, log2p, G, lane);
  const int mine = tiles_of(s, few_rows);
  const int incl = wave_scan(mine);
  r.count = min(__builtin_amdgcn_readlane(incl, 63), tiles);
  r.found = t < r.count;
  if (!r.found) return r;
  r.index = r.count - 1 - t;
  const uint64_t hit =
      __builtin_amdgcn_ballot_w64(r.index >= incl - mine && r.index < incl);
  r.b = __builtin_ctzll(hit);
  r.i = r.index - __builtin_amdgcn_readlane(incl - mine, r.b);
  r.s.q0 = __builtin_amdgcn_readlane(s.q0, r.b);
  r.s.rows = __builtin_amdgcn_readlane(s.rows, r.b);
  r.s.keys = __builtin_amdgcn_readlane(s.keys, r.b);
  r.s.pos0 = __builtin_amdgcn_readlane(s.pos0, r.b);
  return r;
}

// The plan of a call of more than 64 sequences, by one workgroup.  (Worked out by every wave, 64
// sequences at a time, one token after 512 x 500 positions took 361 us, after 1024 x 300 722.)
__global__ __launch_bounds__(1024) void kv_attention_paged_plan_kernel(
    PagedAttentionArgs a, int log2p, int Hkv, int few_rows, int slots, int chunk_min,
    Plan* __restrict__ plan, Joint* __restrict__ joints, int* __restrict__ starts) {
  __shared__ int64_t s_sum[16];
  __shared__ int2 s_scan[16];
  const int tid = (int)__builtin_amdgcn_workitem_id_x();
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = a.Hq / Hkv;
  auto at = [&](int b) {
    Seq s{};
    if (b < a.B) s = sequence(a, log2p, G, b);
    return s;
  };
  auto few = [&](const Seq& s) { return s.rows > 0 && s.rows <= few_rows; };
  auto chunks = [&](const Seq& s, int len) { return few(s) ? max(1, (s.keys + len - 1) / len) : 0; };
  auto total = [&](auto value) {  // over all sequences
    int64_t sum = 0;
    for (int b0 = 0; b0 < a.B; b0 += 1024) sum += wave_add(value(at(b0 + tid)));
    __syncthreads();
    if (lane == 0) s_sum[wave] = sum;
    __syncthreads();
    sum = 0;
    for (int k = 0; k < 16; ++k) sum += s_sum[k];
    return sum;
  };
  const int64_t blocks = total([&](const Seq& s) { return few(s) ? (s.keys + 127) >> 7 : 0; });
  const int len = chunk_length(blocks, Hkv, slots, chunk_min, [&](int len) {
    return Hkv * total([&](const Seq& s) { return chunks(s, len); });
  });
  int2 base = make_int2(0, 0);  // units of a head, tiles
  for (int b0 = 0; b0 < a.B; b0 += 1024) {
    const Seq s = at(b0 + tid);
    const int nc = chunks(s, len), nt = tiles_of(s, few_rows);
    const int2 incl = make_int2(wave_scan(nc), wave_scan(nt));
    __syncthreads();
    if (lane == 63) s_scan[wave] = incl;
    __syncthreads();
    int2 before = base;
    for (int k = 0; k < 16; ++k) {
      if (k < wave) before = make_int2(before.x + s_scan[k].x, before.y + s_scan[k].y);
      base = make_int2(base.x + s_scan[k].x, base.y + s_scan[k].y);
    }
    if (b0 + tid < a.B) {
      joints[b0 + tid] = Joint{s.q0, few(s) ? s.rows : 0, nc, Hkv * (before.x + incl.x - nc)};
      starts[b0 + tid] = before.y + incl.y - nt;
    }
  }
  if (tid == 0) *plan = Plan{len, base.y, {0, 0}};
}

// The rows of a tile that the second kernel joins.
struct alignas(16) TileJoint {
  int q0, row0, rows, nsplit;
};

template <int D>
__global__ __launch_bounds__(512, 1) void kv_attention_paged_tile_kernel(
    PagedAttentionArgs a, PagedCache c, int few_rows, int tiles, int splits, const Plan* __restrict__ plan,
    const int* __restrict__ starts, TileJoint* __restrict__ joints, float* __restrict__ rec) {
  constexpr int KROW = 2 * D + 16;
  constexpr int NS = D / 16;   // k-steps of the score product
  constexpr int ND = D / 32;   // tiles of output channels
  constexpr int NV = D / 8;    // code words of a row
  __shared__ Stage<D> S;
  __shared__ float s_qm[8];
  __shared__ int2 s_qe[8];
  const int tid = (int)__builtin_amdgcn_workitem_id_x();
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ql = lane & 31, h = lane >> 5;
  const int G = a.Hq / c.Hkv;
  const int id = (int)__builtin_amdgcn_workgroup_id_x();
  // (heads first: an L2 reads one head's cache when there are eight.  Splits last: those that a
  // short tile does without end at once, and are not every n-th workgroup, which would leave
  // whole XCDs idle)
  const int hk = uniform(id % c.Hkv), t = uniform(id / c.Hkv % tiles);
  const int split = uniform(id / c.Hkv / tiles);
  const Tile w = find_tile(a, c.log2p, G, few_rows, tiles, plan, starts, t);
  if (!w.found) {
    if (joints && !split && !hk && !tid) joints[t] = TileJoint{0, 0, 0, 0};
    return;
  }
  const int row0 = w.i * ROWS;
  const int last = min(w.s.rows, row0 + ROWS) - 1;  // the tile's last row
  // the positions that its rows see, and this split's blocks of them
  const int keys = uniform(min(max(w.s.pos0 + last / G + 1, 0), w.s.keys));
  const int nblk = (keys + KB - 1) / KB;
  // (four blocks a split at least: 700 new tokens 36 us, with eight 39)
  const int ns = max(1, min(splits, nblk / 4));
  if (joints && !split && !hk && !tid) joints[w.index] = TileJoint{w.s.q0, row0, last + 1 - row0, ns};
  if (split >= ns) return;
  const int kb0 = uniform((int)((int64_t)nblk * split / ns));
  const int kb1 = uniform((int)((int64_t)nblk * (split + 1) / ns));

  // ---- this wave's rows
  const int wrow = row0 + 32 * wave;
  const int row = min(wrow + ql, last);
  const int tok = row / G, hq = hk * G + row - tok * G;
  const int pos = w.s.pos0 + tok;
  const int pmin = uniform(w.s.pos0 + wrow / G);

  // ---- staging: eight positions a wave; a block's parameters are prepared by one wave, in turn
  const int32_t* table = a.page_table + (int64_t)w.b * a.max_pages;
  const int pmask = (1 << c.log2p) - 1;
  const int kkey = 8 * wave + (lane >> 3);                     // key staging: position, part lane % 8
  const int vword = lane % NV, vpair = (lane / NV) & 3;        // value staging: word, two positions
  const int vkey = 8 * wave + 2 * vpair;
  struct Pages {  // lane i: the page of the 16 positions from id0 + 16 i on
    int id0, ids;
  } kpg, vpg;
  auto find_pages = [&](Pages& p, int from) {
    p.id0 = from;
    const int key = from + 16 * lane;
    p.ids = key < keys ? table[key >> c.log2p] : -1;
    // (waited for here, where it is rare: not after the branch, with all loads in flight)
    asm volatile("" : "+v"(p.ids));
  };
  uint32_t kcode[2], vcode[2];
  auto first_row = [&](Pages& p, int kb) {  // of the wave's eight positions
    const int k0 = kb * KB;
    if (k0 - p.id0 >= 1024) find_pages(p, k0);
    const int pg = __builtin_amdgcn_readlane(p.ids, ((k0 - p.id0) >> 4) + (wave >> 1));
    return c.row((uint32_t)pg < (uint32_t)c.pages ? pg : 0, hk, (k0 + 8 * wave) & pmask);
  };
  auto load_k = [&](int kb) {
    const uint8_t* src = c.kc + first_row(kpg, kb) * (D / 2);
    const uint32_t at = (uint32_t)((lane >> 3) * (D / 2) + (lane & 7) * (D / 16));
    if constexpr (D == 128) {
      const uint2 y = *reinterpret_cast<const uint2*>(src + at);
      kcode[0] = y.x;
      kcode[1] = y.y;
    } else {
      kcode[0] = *reinterpret_cast<const uint32_t*>(src + at);
    }
  };
  auto load_v = [&](int kb) {
    const uint8_t* src = c.vc + first_row(vpg, kb) * (D / 2);
    const uint32_t at = (uint32_t)(2 * vpair * (D / 2) + 4 * vword);
    vcode[0] = *reinterpret_cast<const uint32_t*>(src + at);
    vcode[1] = *reinterpret_cast<const uint32_t*>(src + at + D / 2);
  };
  auto store_k = [&](int kb, int slot) {
    const h2_t aa = __builtin_bit_cast(h2_t, S.par[kb & 3].a[kkey]);
    const uint32_t a1 = __builtin_bit_cast(uint32_t, h2_t{aa.x, aa.x});
    const uint32_t a16 = __builtin_bit_cast(uint32_t, h2_t{aa.y, aa.y});
    uint4* dst = reinterpret_cast<uint4*>(S.k[slot] + kkey * KROW + (lane & 7) * (D / 4));
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {  // codes as subnormals, times 2^15, then A c 2^-9
      const uint32_t y = kcode[i], y8 = y >> 8;
      dst[i] = make_uint4(pk_mul(pk_mul(y & 0x000F000Fu, 0x78007800u), a1),
                          pk_mul(pk_mul(y & 0x00F000F0u, 0x78007800u), a16),
                          pk_mul(pk_mul(y8 & 0x000F000Fu, 0x78007800u), a1),
                          pk_mul(pk_mul(y8 & 0x00F000F0u, 0x78007800u), a16));
    }
  };
  auto store_v = [&](int kb, int slot) {
    const uint2 s01 = *reinterpret_cast<const uint2*>(&S.par[kb & 3].ab[vkey]);
    const uint32_t a1 = __builtin_amdgcn_perm(s01.y, s01.x, 0x05040100u);
    const uint32_t b1 = __builtin_amdgcn_perm(s01.y, s01.x, 0x07060302u);
    const uint32_t a16 = pk_mul(a1, 0x2C002C00u);  // / 16
    const uint32_t x0 = __builtin_amdgcn_perm(vcode[1], vcode[0], 0x05040100u);
    const uint32_t x1 = __builtin_amdgcn_perm(vcode[1], vcode[0], 0x07060302u);
    const uint32_t y[4] = {x0, x0 >> 8, x1, x1 >> 8};
    // position 16 a + 8 b + 4 h + i of the block stands at 16 a + 8 h + 4 b + i
    uint8_t* dst = S.v[slot] + vword * VROW +
                   2 * (16 * (wave >> 1) + 8 * (vpair >> 1) + 4 * (wave & 1) + 2 * (vpair & 1));
    if (D == 128 || lane < 32) {
#pragma unroll
      for (int m = 0; m < 8; ++m)  // codes as subnormals, times 2^15, then A c 2^-9 - A z 2^-9
        *reinterpret_cast<uint32_t*>(dst + m * NV * VROW) =
            pk_fma(pk_mul(y[m >> 1] & (m & 1 ? 0x00F000F0u : 0x000F000Fu), 0x78007800u),
                   m & 1 ? a16 : a1, b1);
    }
  };
  // Parameters, lane = position: the page first, then (a turn later) the row's, then its place.
  auto page_of = [&](int kb) {
    return table[min(kb * KB + lane, keys - 1) >> c.log2p];
  };
  auto params = [&](int kb, int page) {
    const bool ok = (uint32_t)page < (uint32_t)c.pages;
    return *reinterpret_cast<const uint2*>(
        c.par + 4 * c.row(ok ? page : 0, hk, (kb * KB + lane) & pmask));
  };
  // E, F: the scaling of the block before
  auto prepare = [&](int kb, int page, uint2 p, int E, int F) {
    typename Stage<D>::Par& P = S.par[kb & 3];
    const bool ok = ((uint32_t)page < (uint32_t)c.pages) & (kb * KB + lane < keys);
    p = for_those_who_see(p);
    if (!ok) p = make_uint2(0, 0);
    const float sk = fp16_bits_to_f32((uint16_t)p.x), zk = (float)(int16_t)(p.x >> 16);
    const float sv = fp16_bits_to_f32((uint16_t)p.y), zv = (float)(int16_t)(p.y >> 16);
    // keys: A (8192 + |z|) stays below 2^28: A below 2^15, the pieces of A z 2^-13 as well.  (No
    // further below it than that takes: the other keys' bits go first.)
    const float kt = wave_max(sk * (8192.0f + fabsf(zk)));
    if (__builtin_amdgcn_ldexpf(kt, -E) >= 0x1p28f) E = __builtin_amdgcn_frexp_expf(kt) - 28;
    const float ka = __builtin_amdgcn_ldexpf(sk, -E);
    const float near = __builtin_amdgcn_fmed3f(ka * zk * 0.5f, -0x1p15f, 0x1p15f);
    const Pieces u = pieces(near), v = pieces((ka * zk * 0.5f - near) * 0x1p-12f);
    P.z[1][lane] = make_uint4(pk_f16(u.h1, u.h1), pk_f16(u.h2, u.h1), pk_f16(u.h2, u.h3), 0);
    P.z[0][lane] = make_uint4(pk_f16(v.h1, v.h1), pk_f16(v.h2, v.h1), pk_f16(v.h2, v.h3), 0);
    P.a[lane] = pk_f16(ka, ka * 0.0625f);
    // values: A stays below 2^15
    const float vt = wave_max(sv);
    if (vt > 0.0f) F = max(F, __builtin_amdgcn_frexp_expf(vt) - 15);
    const float va = __builtin_amdgcn_ldexpf(sv, -F), z = __builtin_amdgcn_fmed3f(zv, 0.0f, 15.0f);
    P.ab[lane] = pk_f16(va, -va * z * 0x1p-9f);
    P.rest[lane] = va * (zv - z) * 0x1p-9f;
    const uint64_t vm = __builtin_amdgcn_ballot_w64(ok), far = __builtin_amdgcn_ballot_w64(sv != 0.0f && zv != z);
    if (lane == 0) {
      P.E = E;
      P.F = 2 * F + (far != 0);
      P.valid[0] = (uint32_t)vm;
      P.valid[1] = (uint32_t)(vm >> 32);
    }
    return make_int2(E, F);
  };
  const bool any = kb0 < kb1;
  const int kbl = kb1 - 1;  // (past the last block the last is loaded and staged again: no branches)
  // each wave's own blocks of parameters: kb0 + 3 + wave and every eighth from there
  int page0 = -1, page1 = -1;
  uint2 par0 = make_uint2(0, 0);
  int fpage[3] = {-1, -1, -1};  // wave 0: the first three blocks, too
  uint2 fpar[3] = {};
  if (any) {
    page0 = page_of(kb0 + 3 + wave);
    page1 = page_of(kb0 + 11 + wave);
#pragma unroll
    for (int i = 0; i < 3; ++i) fpage[i] = page_of(kb0 + i);
    find_pages(kpg, kb0 * KB);
    vpg = kpg;
  }
  // the wave's query rows, whole rows at a time, and through LDS to the lanes that want them
  // (a lane that reads its row itself: 32 bytes of a line at a time, 0.3 us more)
  uint4 raw[NS];
  constexpr int LR = D / 8;  // lanes that read a row
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int i = 64 / LR * s + lane / LR, r = min(wrow + i, last);
    raw[s] = *reinterpret_cast<const uint4*>(a.q + w.s.q0 * a.ldq + (int64_t)hk * G * D + (int64_t)r * D +
                                             __shfl(tok, i) * (a.ldq - G * D) + 8 * (lane % LR));
  }
  if (any) {
    load_k(kb0);
    load_v(kb0);
    par0 = params(kb0 + 3 + wave, page0);
#pragma unroll
    for (int i = 0; i < 3; ++i) fpar[i] = params(kb0 + i, fpage[i]);
  }

  // ---- queries, rotated, times sm_scale log2(e) 2^(E + 9).  32 channels at a time are rotated by
  // a matrix product with H (its entries and the queries are exact, the sums fp32), whose rows
  // stand in such an order that half h of the lanes gets channels 16 h .. 16 h + 15 of the 32, two
  // code words; without a rotation the product is with 1.
  uint32_t qb[NS][4], zb[4] = {0, 0, 0, 0};
  auto zero_terms = [&] {  // -16 sum q for this half of the zero-points' products
    float sum = 0.0f;
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        sum = __builtin_amdgcn_fdot2(__builtin_bit_cast(h2_t, qb[s][k]),
                                     h2_t{(_Float16)1.0f, (_Float16)1.0f}, sum, false);
    sum += __shfl_xor(sum, 32);
    const Pieces v = pieces(h ? sum * -0x1p-8f : __builtin_amdgcn_fmed3f(-16.0f * sum, -65504.0f, 65504.0f));
    zb[0] = pk_f16(v.h1, v.h2);
    zb[1] = pk_f16(v.h1, v.h3);
    zb[2] = pk_f16(v.h2, v.h1);
  };
  int E;
  bool bad;  // the row is not finite: held at the end of fp16's range, it would give numbers
  {
    const int ch = 16 * ((ql >> 2) & 1) + 4 * (ql >> 3) + (ql & 3);
    auto entry = [&](int k) {
      return a.k_had ? 0x3F80u | ((uint32_t)__builtin_popcount(ch & k) << 15 & 0x8000u)
                     : (ch == k ? 0x3F80u : 0u);
    };
    uint32_t rot[2][4];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int i = 16 * (k >> 2) + 8 * h + 2 * (k & 3);
      rot[k >> 2][k & 3] = entry(i) | entry(i + 1) << 16;
    }
    static_assert(8 * 32 * KROW <= sizeof(S.k) + sizeof(S.v), "");
    uint8_t* own = &S.k[0][0] + 32 * KROW * wave;
#pragma unroll
    for (int s = 0; s < NS; ++s)
      *reinterpret_cast<uint4*>(own + (64 / LR * s + lane / LR) * KROW + 16 * (lane % LR)) = raw[s];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int s = 0; s < NS; ++s)
      raw[s] = *reinterpret_cast<const uint4*>(own + ql * KROW + 32 * s + 16 * h);
    f16_t x[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) {
#pragma unroll
      for (int r = 0; r < 16; ++r) x[d][r] = 0.0f;
#pragma unroll
      for (int k = 0; k < 2; ++k)
        x[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            __builtin_bit_cast(b8_t, make_uint4(rot[k][0], rot[k][1], rot[k][2], rot[k][3])),
            __builtin_bit_cast(b8_t, raw[2 * d + k]), x[d], 0, 0, 0);
    }
    float sm2 = a.sm_scale * LOG2E;
    if (a.k_had) {
#pragma unroll
      for (int s = 1; s < ND; s <<= 1)
#pragma unroll
        for (int d = 0; d < ND; ++d)
          if (!(d & s)) {
            const f16_t p = x[d], q = x[d + s];
            x[d] = p + q;
            x[d + s] = p - q;
          }
      sm2 *= hadamard_norm<D>();
    }
    // E: the largest query at 2^4, but the rows' mean (of their largest ones' exponents) no lower than
    // 2^-4, so that a row of garbage leaves the others their bits, and no less than the first block's
    // keys take.  A row that is too large for that, 2^19 above the mean, is made smaller as a whole:
    // its scores are over 2^16 all the same, unless the keys are tiny to the others.  Queries that
    // later keys raise beyond fp16's range, by 2^12 and more, stay at its end: a channel of theirs
    // makes over 2^21 of a score with one step of the largest key's codes.
    float qm = 0.0f;
#pragma unroll
    for (int i = 0; i < D / 2; ++i) qm = fmaxf(qm, fabsf(x[i >> 4][i & 15]));
    qm = fmaxf(qm, __shfl_xor(qm, 32));
    if (!(qm < __builtin_inff())) qm = 0.0f;
    const int qe = max(__builtin_amdgcn_frexp_expf(qm), -100);  // this row's
    const bool counts = qm > 0.0f && !h;
    const int2 qes = make_int2(wave_add(counts ? qe : 0), wave_add(counts));
    qm = wave_max(qm);
    const uint32_t kpar = for_those_who_see(fpar[0]).x;
    const float kt = wave_max(any && (uint32_t)fpage[0] < (uint32_t)c.pages &&
                                      kb0 * KB + lane < keys
                                  ? fp16_bits_to_f32((uint16_t)kpar) *
                                        (8192.0f + fabsf((float)(int16_t)(kpar >> 16)))
                                  : 0.0f);
    if (lane == 0) {
      s_qm[wave] = qm;
      s_qe[wave] = qes;
    }
    __syncthreads();
    int2 sum = make_int2(0, 0);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      qm = fmaxf(qm, s_qm[k]);
      sum = make_int2(sum.x + s_qe[k].x, sum.y + s_qe[k].y);
    }
    const int mean = (int)__builtin_floorf((float)sum.x / (float)max(sum.y, 1));
    E = uniform(max(-5 - max(__builtin_amdgcn_frexp_expf(qm), -100), sum.y ? -13 - mean : -1000) -
                __builtin_amdgcn_frexp_expf(sm2));
    if (kt > 0.0f) E = max(E, uniform(__builtin_amdgcn_frexp_expf(kt)) - 28);
    float f = __builtin_amdgcn_ldexpf(sm2, E + 9);
    f = __builtin_amdgcn_ldexpf(f, min(0, 15 - qe - __builtin_amdgcn_frexp_expf(f)));
    float check = 0.0f;
#pragma unroll
    for (int i = 0; i < D / 2; ++i) check = __builtin_fmaf(x[i >> 4][i & 15], 0.0f, check);
    check += __shfl_xor(check, 32);
    bad = check != 0.0f;
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const h2_t top = {(_Float16)65504.0f, (_Float16)65504.0f};
        h2_t p = {(_Float16)(f * x[s >> 1][8 * (s & 1) + k]),
                  (_Float16)(f * x[s >> 1][8 * (s & 1) + k + 4])};
        p = __builtin_elementwise_max(__builtin_elementwise_min(p, top), -top);
        qb[s][k] = __builtin_bit_cast(uint32_t, p);
      }
    zero_terms();
  }

  f16_t o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
  f16_t neg;  // -m in every register: what the score products start from
#pragma unroll
  for (int r = 0; r < 16; ++r) neg[r] = 0.0f;
  float l = __builtin_inff(), zsum = 0.0f;  // (l: nothing seen)
  int Eq = E, Fo = -200;  // the scaling that the queries and the outputs carry

  // QK of a tile of 32 positions in slot `slot`.  The first operands of a product are read while
  // the one before runs (two prompts of 4096 tokens: 64 channels 273 -> 263 us, 128 the same).
  constexpr int KA = 3, VA = 4;
  uint4 kz, kf[KA], vf[VA];
  auto key_at = [&](int slot, int tt, int k) {
    return *reinterpret_cast<const uint4*>(S.k[slot] + (32 * tt + ql) * KROW + 64 * (k >> 1) + 32 * h +
                                           16 * (k & 1));
  };
  auto fetch_k = [&](int kb, int slot, int tt) {
    kz = S.par[kb & 3].z[h][32 * tt + ql];
#pragma unroll
    for (int k = 0; k < KA; ++k) kf[k] = key_at(slot, tt, k);
  };
  auto scores = [&](int slot, int tt, f16_t& s) {
    uint4 rest[NS - KA];
#pragma unroll
    for (int k = KA; k < NS; ++k) rest[k - KA] = key_at(slot, tt, k);
    s = __builtin_amdgcn_mfma_f32_32x32x16_f16(
        __builtin_bit_cast(h8_t, kz),
        __builtin_bit_cast(h8_t, make_uint4(zb[0], zb[1], zb[2], zb[3])), neg, 0, 0, 0);
#pragma unroll
    for (int k = 0; k < NS; ++k)
      s = __builtin_amdgcn_mfma_f32_32x32x16_f16(
          __builtin_bit_cast(h8_t, k < KA ? kf[k < KA ? k : 0] : rest[k < KA ? 0 : k - KA]),
          __builtin_bit_cast(h8_t, make_uint4(qb[k][0], qb[k][1], qb[k][2], qb[k][3])), s, 0, 0, 0);
  };
  uint32_t wb[2][4];
  auto weights = [&](const f16_t& s, float sum) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const h2_t p = {(_Float16)__builtin_amdgcn_exp2f(s[8 * k + 2 * j]),
                        (_Float16)__builtin_amdgcn_exp2f(s[8 * k + 2 * j + 1])};
        sum = __builtin_amdgcn_fdot2(p, h2_t{(_Float16)1.0f, (_Float16)1.0f}, sum, false);
        wb[k][j] = __builtin_bit_cast(uint32_t, p);
      }
    return sum;
  };
  auto mask = [&](f16_t& s, int k0, uint32_t valid) {
    if (k0 + 31 > pmin || valid != 0xFFFFFFFFu) {
      const uint32_t vm = valid >> (4 * h);
      const int lim = pos - k0 - 4 * h;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int j = 8 * (r >> 2) + (r & 3);
        if (j > lim || !((vm >> j) & 1)) s[r] = -__builtin_inff();
      }
    }
  };
  auto row_max = [&](const f16_t& s) {
    float top = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
    return fmaxf(top, __shfl_xor(top, 32));
  };
  // After the weights of `s`, tile tt of a block: rows that had met no position before (an infinite
  // l), or now a weight beyond the range, move their reference, also under the scores `t` that were
  // formed meanwhile; then the values' zero-points beyond their codes, where the block has any.
  auto settle = [&](f16_t& s, f16_t& t, float sum, int kb, int tt, int far) {
    const uint64_t moving = __builtin_amdgcn_ballot_w64(!(sum < HUGE_SUM));
    if (!(moving | (uint64_t)far)) {
      l = sum;
      return;
    }
    if (moving) {
      const float top = row_max(s);
      const bool first = l == __builtin_inff();
      const bool move = top > -__builtin_inff() && (first || top > MID + 8.0f);
      const float by = move ? top - MID : 0.0f;
      const float f = __builtin_amdgcn_exp2f(first ? 0.0f : -by);  // (of a first one, o and zsum are 0)
      l = first && move ? 0.0f : l * f;
      zsum *= f;
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] *= f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[r] -= by;
        t[r] -= by;
        neg[r] -= by;
      }
      sum = weights(s, l);
    }
    l = sum;
    if (far) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {  // registers 4 k .. 4 k + 3: positions 8 k + 4 h and on
        const float4 z = *reinterpret_cast<const float4*>(&S.par[kb & 3].rest[32 * tt + 8 * k + 4 * h]);
        const h2_t p = __builtin_bit_cast(h2_t, wb[k >> 1][2 * (k & 1)]);
        const h2_t q = __builtin_bit_cast(h2_t, wb[k >> 1][2 * (k & 1) + 1]);
        zsum = __builtin_fmaf((float)p.x, z.x, __builtin_fmaf((float)p.y, z.y, zsum));
        zsum = __builtin_fmaf((float)q.x, z.z, __builtin_fmaf((float)q.y, z.w, zsum));
      }
    }
  };
  auto value_at = [&](int slot, int tt, int i) {
    return *reinterpret_cast<const uint4*>(S.v[slot] + (32 * (i % ND) + ql) * VROW +
                                           2 * (16 * (2 * tt + i / ND) + 8 * h));
  };
  auto fetch_v = [&](int slot, int tt) {
#pragma unroll
    for (int i = 0; i < VA; ++i) vf[i] = value_at(slot, tt, i);
  };
  auto values = [&](int slot, int tt) {
#pragma unroll
    for (int i = 0; i < 2 * ND; ++i) {
      const uint4 vv = i < VA ? vf[i < VA ? i : 0] : value_at(slot, tt, i);
      const uint32_t (&w)[4] = wb[i / ND];
      o[i % ND] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
          __builtin_bit_cast(h8_t, vv), __builtin_bit_cast(h8_t, make_uint4(w[0], w[1], w[2], w[3])),
          o[i % ND], 0, 0, 0);
    }
  };
  auto rescale_q = [&](int to) {
    if (Eq >= to) return;
    for (; Eq < to; Eq = min(Eq + 15, to)) {
      const _Float16 f = (_Float16)__builtin_amdgcn_ldexpf(1.0f, min(to - Eq, 15));
      auto grow = [&](uint32_t& x) {
        const h2_t p = __builtin_bit_cast(h2_t, x) * h2_t{f, f};
        const h2_t top = {(_Float16)65504.0f, (_Float16)65504.0f};
        x = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_elementwise_min(p, top), -top));
      };
#pragma unroll
      for (int k = 0; k < NS; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) grow(qb[k][j]);
    }
    zero_terms();
  };

  // Pipeline: while a tile's weights are formed, the next tile's scores are on the matrix cores;
  // while its values are, the codes of later blocks go to LDS: keys two blocks ahead (their first
  // tile's scores run in the block before), values one; parameters three ahead.
  if (any) {
    if (wave == 0) {
      int2 ef = make_int2(E, -200);
#pragma unroll
      for (int i = 0; i < 3; ++i) ef = prepare(kb0 + i, fpage[i], fpar[i], ef.x, ef.y);
    }
    lds_barrier();
    store_k(kb0, 0);
    load_k(min(kb0 + 1, kbl));
    store_v(kb0, 0);
    store_k(kb0 + 1, 1);
    // (keys, then values, as in the loop: the waits count the loads issued later)
    load_k(min(kb0 + 2, kbl));
    load_v(min(kb0 + 1, kbl));
    auto meta = [&](int kb) {  // E, F and its flag, valid
      const int4 x = *reinterpret_cast<const int4*>(&S.par[kb & 3].E);
      return make_int4(uniform(x.x), uniform(x.y), uniform(x.z), uniform(x.w));
    };
    auto stage_keys = [&](int kb, int slot) {
      store_k(kb + 2, slot);
      load_k(min(kb + 3, kbl));
    };
    auto stage_values = [&](int kb, int slot) {
      store_v(kb + 1, slot);
      load_v(min(kb + 2, kbl));
      if (((kb - kb0) & 7) == wave) {
        const int4 before = meta(kb + 2);
        prepare(kb + 3, page0, par0, before.x, before.y >> 1);
        page0 = page1;
        par0 = params(kb + 11, page0);
        page1 = page_of(kb + 19);
      }
    };
    int4 now = meta(kb0);
    rescale_q(now.x);
    lds_barrier();
    if (wrow > last) {  // no rows: only the staging, in step with the others
      for (int kb = kb0, s2 = 2, v1 = 1; kb < kb1; ++kb, s2 = s2 == 2 ? 0 : s2 + 1, v1 ^= 1) {
        stage_keys(kb, s2);
        stage_values(kb, v1);
        lds_barrier();
      }
      return;
    }
    f16_t s0, s1;
    fetch_k(kb0, 0, 0);
    scores(0, 0, s0);
    fetch_k(kb0, 0, 1);
    mask(s0, kb0 * KB, (uint32_t)now.z);
    if (const float top = row_max(s0); top > -__builtin_inff()) {
      l = 0.0f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        neg[r] = MID - top;
        s0[r] += MID - top;
      }
    }
    int sl = 0, vs = 0;  // slots of this block's keys and values
    for (int kb = kb0; kb < kb1; ++kb) {
      const int sl1 = sl == 2 ? 0 : sl + 1, sl2 = sl1 == 2 ? 0 : sl1 + 1;
      const int4 next = meta(kb + 1);
      const int F = now.y >> 1, far = now.y & 1;
      if (F != Fo) {
        const float f = __builtin_amdgcn_ldexpf(1.0f, max(Fo - F, -150));
        zsum *= f;
#pragma unroll
        for (int d = 0; d < ND; ++d) o[d] *= f;
        Fo = F;
      }
      mask(s0, kb * KB, (uint32_t)now.z);
      scores(sl, 1, s1);
      fetch_v(vs, 0);
      float sum = weights(s0, l);
      settle(s0, s1, sum, kb, 0, far);
      fetch_k(kb + 1, sl1, 0);
      values(vs, 0);
      stage_keys(kb, sl2);
      mask(s1, kb * KB + 32, (uint32_t)now.w);
      rescale_q(next.x);
      scores(sl1, 0, s0);
      fetch_v(vs, 1);
      sum = weights(s1, l);
      settle(s1, s0, sum, kb, 1, far);
      fetch_k(kb + 1, sl1, 1);
      values(vs, 1);
      stage_values(kb, vs ^ 1);
      lds_barrier();
      now = next;
      sl = sl1;
      vs ^= 1;
    }
  }
  if (wrow > last) return;
  if (l == __builtin_inff()) l = 0.0f;
  l += __shfl_xor(l, 32);
  zsum += __shfl_xor(zsum, 32);
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] -= zsum;
  if (bad && l > 0.0f) l = __builtin_nanf("");

  // ---- channels: o[d][r] is channel 8 word + nibble of V^T's row 32 d + 8 (r / 4) + 4 h + r % 4
  // = nibble * D / 8 + word
  const bool mine = wrow + ql <= last;
  const float back = __builtin_amdgcn_ldexpf(1.0f, Fo + 9);  // (0 where nothing was met)
  auto word = [&](int j, float* y) {  // this lane's j-th code word, j < D / 16
#pragma unroll
    for (int n = 0; n < 8; ++n)
      y[n] = D == 128 ? o[n >> 1][8 * (n & 1) + 4 * (j >> 2) + (j & 3)] : o[n >> 2][4 * (n & 3) + j];
  };
  if (ns > 1) {
    if (!mine) return;
    float* dst = rec + (int64_t)((w.index * c.Hkv + hk) * splits + split) * ROWS * (D + 2);
    const int i = 32 * wave + ql;
    if (!h) *reinterpret_cast<float2*>(dst + 2 * i) = make_float2(l == 0.0f ? LOWEST : -neg[0], l);
    dst += 2 * ROWS + i * D;
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
      float y[8];
      word(j, y);
      float4* p = reinterpret_cast<float4*>(dst + 8 * (D == 128 ? 8 * (j >> 2) + 4 * h + (j & 3) : 4 * h + j));
      p[0] = make_float4(y[0] * back, y[1] * back, y[2] * back, y[3] * back);
      p[1] = make_float4(y[4] * back, y[5] * back, y[6] * back, y[7] * back);
    }
    return;
  }
  const float f = l == 0.0f ? 0.0f : back / l;
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] *= f;
  if (a.v_had) {  // every channel bit is a bit of d, r or h
#pragma unroll
    for (int s = 1; s < D / 2; s <<= 1)
#pragma unroll
      for (int i = 0; i < D / 2; ++i)
        if (!(i & s)) {
          const float p = o[i >> 4][i & 15], q = o[(i + s) >> 4][(i + s) & 15];
          o[i >> 4][i & 15] = p + q;
          o[(i + s) >> 4][(i + s) & 15] = p - q;
        }
#pragma unroll
    for (int i = 0; i < D / 2; ++i)
      o[i >> 4][i & 15] = hadamard_norm<D>() * lane_butterfly<32>(o[i >> 4][i & 15], lane);
  }
  if (!mine) return;
  uint16_t* dst = a.out + (int64_t)(w.s.q0 + tok) * a.ldo + (int64_t)hq * D;
#pragma unroll
  for (int j = 0; j < D / 16; ++j) {
    float y[8];
    word(j, y);
    *reinterpret_cast<uint4*>(dst + 8 * (D == 128 ? 8 * (j >> 2) + 4 * h + (j & 3) : 4 * h + j)) =
        make_uint4(bf16x2_rne(y[0], y[1]), bf16x2_rne(y[2], y[3]), bf16x2_rne(y[4], y[5]),
                   bf16x2_rne(y[6], y[7]));
  }
}

// What a call's chunks or splits left: who they belong to, and their rows.
struct FewJoin {
  const Joint* joints;
  const float* rec;
  int rows, blocks;  // the most rows of a sequence and head; workgroups
};
struct TileJoin {
  const TileJoint* joints;
  const float* rec;
  int splits, blocks;
};

// Joins the chunks of a row: one workgroup per (sequence, key/value head, row), a chunk to each of
// four waves in turn.  A chain of loads, each behind the one before; the lengths and the joint go
// together.
template <int D>
__device__ __forceinline__ void join_chunks(const PagedAttentionArgs& a, int Hkv, int log2p,
                                            const FewJoin& w, int id) {
  __shared__ float s_o[4][D];
  const int lane = (int)__builtin_amdgcn_workitem_id_x() & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)__builtin_amdgcn_workitem_id_x() >> 6);
  const int G = a.Hq / Hkv;
  const int hk = id % Hkv, row = id / Hkv % w.rows, b = id / Hkv / w.rows;
  const Joint j = w.joints[b];  // (not written where the sequence has no chunks)
  const Seq s = sequence(a, log2p, G, b);
  if ((row >= s.rows) | (s.rows > w.rows) | (j.nchunk <= 1)) return;
  const int64_t size = (int64_t)w.rows * (D + 2);
  const float* first = w.rec + (int64_t)(j.unit0 + hk * j.nchunk) * size;
  auto max_sum = [&](int i) {
    return i < j.nchunk ? *reinterpret_cast<const float2*>(first + i * size + 2 * row) : make_float2(LOWEST, 0.0f);
  };
  float2 ml = max_sum(lane);
  float top = ml.x;
  for (int i = 64 + lane; i < j.nchunk; i += 64) top = fmaxf(top, max_sum(i).x);
  top = wave_max(top);
  float l = 0.0f, o[D / 64] = {};
  for (int i0 = 0; i0 < j.nchunk; i0 += 64) {
    if (i0) ml = max_sum(i0 + lane);
    const float f = __builtin_amdgcn_exp2f(ml.x - top);
    l = __builtin_fmaf(f, ml.y, l);
    const int n = min(64, j.nchunk - i0);
    const float* src = first + i0 * size + 2 * w.rows + row * D + lane * (D / 64);
    for (int k = wave; k < n; k += 32) {  // (factors past the last chunk are 0)
      float v[8][D / 64];
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < D / 64; ++e) v[i][e] = src[min(k + 4 * i, n - 1) * size + e];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float fk = __shfl(f, k + 4 * i);
#pragma unroll
        for (int e = 0; e < D / 64; ++e) o[e] = __builtin_fmaf(k + 4 * i < n ? fk : 0.0f, v[i][e], o[e]);
      }
    }
  }
  l = wave_sum(l);
#pragma unroll
  for (int e = 0; e < D / 64; ++e) s_o[wave][lane * (D / 64) + e] = o[e];
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int e = 0; e < D / 64; ++e) {
    const int d = lane * (D / 64) + e;
    o[e] = (s_o[0][d] + s_o[1][d]) + (s_o[2][d] + s_o[3][d]);
  }
  store_row<D>(a, j.q0 + row / G, hk * G + row % G, o, l, lane);
}

// Joins the splits of a tile's rows, a wave per row.
template <int D>
__device__ __forceinline__ void join_splits(const PagedAttentionArgs& a, int Hkv, const TileJoin& w, int id) {
  const int lane = (int)__builtin_amdgcn_workitem_id_x() & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)__builtin_amdgcn_workitem_id_x() >> 6);
  const int i = 4 * (id % (ROWS / 4)) + wave, hk = id / (ROWS / 4) % Hkv, t = id / (ROWS / 4) / Hkv;
  const TileJoint j = w.joints[t];
  if (i >= j.rows || j.nsplit <= 1) return;
  const int64_t size = ROWS * (D + 2);
  const float* src = w.rec + (int64_t)(t * Hkv + hk) * w.splits * size;
  float2 ml = make_float2(LOWEST, 0.0f);  // splits <= 64
  if (lane < j.nsplit) ml = *reinterpret_cast<const float2*>(src + lane * size + 2 * i);
  const float top = wave_max(ml.x);
  const float f = __builtin_amdgcn_exp2f(ml.x - top);
  const float l = wave_sum(f * ml.y);
  float o[D / 64] = {};
  src += 2 * ROWS + i * D + lane * (D / 64);
  for (int k = 0; k < j.nsplit; k += 4) {
    float v[4][D / 64];
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int e = 0; e < D / 64; ++e) v[q][e] = src[min(k + q, j.nsplit - 1) * size + e];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float fk = __shfl(f, k + q);
#pragma unroll
      for (int e = 0; e < D / 64; ++e) o[e] = __builtin_fmaf(k + q < j.nsplit ? fk : 0.0f, v[q][e], o[e]);
    }
  }
  const int G = a.Hq / Hkv, row = j.row0 + i;
  store_row<D>(a, j.q0 + row / G, hk * G + row % G, o, l, lane);
}

// (one launch for both: 1.5 us less where a call has both)
template <int D>
__global__ __launch_bounds__(256) void kv_attention_paged_join_kernel(PagedAttentionArgs a, int Hkv,
                                                                      int log2p, FewJoin few, TileJoin tile) {
  const int id = (int)__builtin_amdgcn_workgroup_id_x();
  if (id < few.blocks) join_chunks<D>(a, Hkv, log2p, few, id);
  else join_splits<D>(a, Hkv, tile, id - few.blocks);
}

}  // namespace

namespace {

// How a call is launched: the rows that the few-row kernel takes, its row tiles and units; the
// tiles of the other kernel and over how many workgroups the keys of each are split.
struct Shape {
  bool few, many, few_join, plan;
  int few_rows, row_tiles, slots, units;
  int64_t tiles;
  int splits;
};
Shape attention_shape(int64_t M, int64_t B, int64_t Hq, int64_t Hkv, int D, int64_t max_new,
                    int64_t cap) {
  const int64_t G = Hq / Hkv, most = max_new * G;
  Shape f = {};
  // The few-row kernel takes codes straight into its operands, which costs the least per position,
  // but its time grows with the row tiles, and at 64 rows of 128 channels it runs out of
  // registers: 8 new tokens of 8 heads, 4 x 5000 positions: 92 us there, 36 us as a tile that is
  // three quarters empty; 5 tokens 36 us there, 38 as a tile, with 64 x 5000 241 and 334.  64 rows
  // of 64 channels: 32 us there, 51 us as a tile.  Beside sequences of many rows it takes 16, and
  // those between go to tiles: with three row tiles every one of its workgroups would have their
  // registers (128 channels, beside a prompt of 1000: 32 single tokens of 4 heads after 5000 90 us,
  // with 48 rows 169; 32 x 5 tokens of 8 heads 166 and 187; 4 x 5 tokens 104 and 99).
  f.many = most > (D == 128 ? 48 : 64);
  f.few = !f.many || B > 1;  // a single sequence of many rows: one launch
  f.row_tiles = f.many || most <= 16 ? 1 : most <= 32 ? 2 : most <= 48 ? 3 : 4;
  f.few_rows = f.few ? (int)(f.many ? 16 : most) : 0;
  // Chunks for two workgroups a CU, or for three where they are the lightest (32 x 8000 positions of
  // 64 channels 41 us, for two 46; 8 x 32768 with 32 heads of 128 channels 211, for two 206).
  f.slots = f.row_tiles == 1 && D == 64 ? 768 : 512;
  f.few_join = f.few && cap > CHUNK_ONE;
  f.plan = B > 64;
  // (what the chunk length allows, and what the page table has room for)
  const int64_t units = (f.few_join ? 2 * f.slots : 0) + B * Hkv;
  const int64_t room = B * Hkv * (cap <= CHUNK_ONE ? 1 : (cap + CHUNK_MIN - 1) / CHUNK_MIN);
  f.units = (int)(units < room ? units : room);
  f.splits = 1;
  if (f.many) {
    // (a sequence of r rows has ceil(r / ROWS) tiles)
    f.tiles = (M * G + (ROWS - 1) * (B < M ? B : M)) / ROWS;
    const int64_t wgs = f.tiles * Hkv;
    // one workgroup per CU: the fewest splits that keep nine in ten of 256 CUs busy
    const int64_t most_splits = cap / (4 * KB);  // (that the kernel makes)
    for (int s = 1; s <= 64 && wgs * s <= 768 && (s == 1 || s <= most_splits); ++s) {
      f.splits = s;
      const int64_t rounds = (wgs * s + 255) / 256;
      if (10 * wgs * s >= 9 * 256 * rounds) break;
    }
  }
  return f;
}
// The workspace: the plan and the sequences' first tiles where there is one, the sequences' joints,
// the chunks' rows; then the tiles' joints and rows.
int64_t plan_floats(const Shape& f, int64_t B) { return f.plan ? 4 + (B + 3) / 4 * 4 : 0; }
int64_t few_floats(const Shape& f, int64_t B, int D) {
  const int64_t joints = f.plan || f.few_join ? 4 * B : 0;
  return joints + (f.few_join ? ((int64_t)f.units * f.few_rows * (D + 2) + 3) / 4 * 4 : 0);
}
int64_t tile_floats(const Shape& f, int64_t Hkv, int D) {
  return f.splits > 1 ? 4 * f.tiles + f.tiles * Hkv * f.splits * ROWS * (D + 2) : 0;
}

}  // namespace

int64_t kv_attention_paged_workspace_floats(int64_t M, int64_t B, int64_t Hq, int64_t Hkv,
                                            int head_dim, int64_t max_new) {
  const Shape f = attention_shape(M, B, Hq, Hkv, head_dim, max_new, int64_t(1) << 30);
  return plan_floats(f, B) + few_floats(f, B, head_dim) + tile_floats(f, Hkv, head_dim);
}

hipError_t launch_kv_attention_paged(const PagedAttentionArgs& a, const PagedCache& c, int head_dim,
                                     float* workspace, hipStream_t stream) {
  const Shape f = attention_shape(a.M, a.B, a.Hq, c.Hkv, head_dim, a.max_new, (int64_t)a.max_pages << c.log2p);
  Plan* plan = f.plan ? reinterpret_cast<Plan*>(workspace) : nullptr;
  int* starts = reinterpret_cast<int*>(workspace) + 4;
  float* few_at = workspace + plan_floats(f, a.B);
  Joint* joints = f.plan || f.few_join ? reinterpret_cast<Joint*>(few_at) : nullptr;
  const int chunk_min = f.few_join ? CHUNK_MIN : CHUNK_ONE;
  if (plan)
    hipLaunchKernelGGL(kv_attention_paged_plan_kernel, dim3(1), dim3(1024), 0, stream, a, c.log2p, c.Hkv,
                       f.few_rows, f.slots, chunk_min, plan, joints, starts);
  FewJoin few = {};
  TileJoin tile = {};
  if (f.few) {
    float* rec = few_at + 4 * (int64_t)a.B;
#define OFFQ_FEW(D_, RT_)                                                                        \
  hipLaunchKernelGGL((kv_attention_paged_few_kernel<D_, RT_>), dim3((unsigned)f.units), dim3(256), \
                     0, stream, a, c, f.few_rows, f.slots, chunk_min, plan, joints, rec)
    if (head_dim == 128) {
      if (f.row_tiles == 1) OFFQ_FEW(128, 1);
      else if (f.row_tiles == 2) OFFQ_FEW(128, 2);
      else OFFQ_FEW(128, 3);
    } else {
      if (f.row_tiles == 1) OFFQ_FEW(64, 1);
      else if (f.row_tiles == 2) OFFQ_FEW(64, 2);
      else if (f.row_tiles == 3) OFFQ_FEW(64, 3);
      else OFFQ_FEW(64, 4);
    }
#undef OFFQ_FEW
    if (f.few_join) few = FewJoin{joints, rec, f.few_rows, f.few_rows * c.Hkv * a.B};
  }
  if (f.many) {
    float* base = few_at + few_floats(f, a.B, head_dim);
    TileJoint* joints = f.splits > 1 ? reinterpret_cast<TileJoint*>(base) : nullptr;
    float* rec = base + 4 * f.tiles;
    const dim3 grid((unsigned)(f.tiles * c.Hkv * f.splits));
    hipLaunchKernelGGL(head_dim == 128 ? kv_attention_paged_tile_kernel<128>
                                       : kv_attention_paged_tile_kernel<64>,
                       grid, dim3(512), 0, stream, a, c, f.few_rows, (int)f.tiles, f.splits, plan, starts, joints, rec);
    if (f.splits > 1) tile = TileJoin{joints, rec, f.splits, (int)(f.tiles * c.Hkv * (ROWS / 4))};
  }
  if (few.blocks + tile.blocks)
    hipLaunchKernelGGL(head_dim == 128 ? kv_attention_paged_join_kernel<128> : kv_attention_paged_join_kernel<64>,
                       dim3((unsigned)(few.blocks + tile.blocks)), dim3(256), 0, stream, a, c.Hkv, c.log2p,
                       few, tile);
  return hipGetLastError();
}

}  // namespace offq
