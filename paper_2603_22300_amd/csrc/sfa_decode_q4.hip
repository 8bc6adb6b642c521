// SFA decode over the 4-bit cache (sfa_attn_decode_q4): int4 code values with
// uint8 indices and one float32 scale per key, int4 value rows with a bfloat16
// scale per 32 coordinates.
//
// Grid and chunks as the other decodes (decode_plan): a workgroup streams one
// chunk of one KV head for all its query heads, four wavefronts with a quarter
// of it each, 64 keys at a time:
//   scores   lane = key.  s_h = scale * ks * sum_t q4_t * qd[u_t][h], qd the dense
//            query rows in LDS; float32.
//   softmax  base 2, online, the running maximum kept uniform over the wavefront.
//   P.V      on the matrix cores, v_mfma_i32_16x16x64_i8, in whole numbers.  The
//            weights of a group of 32 coordinates, p * vs, are rounded to whole numbers
//            of 32 bits and written as four digits of a signed byte: four query heads'
//            digits are the sixteen rows of one operand, a lane of the result holds the
//            four digits' sums of one head.  The other operand is the cached nibbles as
//            they are, at the high end of a byte: 16 q.  Products and sums are exact
//            (1024 keys at most to a wavefront, 2^24); what is lost is the weights'
//            rounding alone, 2^-28 of the largest p times the group's largest value scale.
// Both operands have 16 keys of one row in a lane, and both are held key by key: the
// transposing LDS reads turn them, ds_read_b64_tr_b4 the cached nibbles and
// ds_read_b64_tr_b8 the weights.  Value rows are loaded a block of
// keys ahead and written to LDS with the 16-byte pieces of a row exchanged, so that the
// transposing reads find each key on banks of its own.  (Through registers: with
// loads sent to LDS directly, the compiler waits for them at every later LDS read.)
//
// Range: each group's weights are scaled by a power of two that follows the largest
// value scale seen in the group, as the running maximum does for p (`vexp` below).  Both
// follow lazily, p up to 2^1.9 and only upwards for the scales, so that most blocks of
// keys touch neither the maxima nor the sums.
//
// Bound by reads beside the vector unit: 64 sequences x 8 heads x 65,536 keys (d = 128, k =
// 16, 3.36 GB) 595 us, 5.6 TB/s, the vector unit 53% and the LDS 40% busy, the matrix cores
// 5%; one sequence of 3000 keys 10 us with its merge.
#include <algorithm>

#include "sfa_decode_kernel.h"

namespace sfa {
namespace {

typedef int v2i __attribute__((ext_vector_type(2)));
typedef int v4i __attribute__((ext_vector_type(4)));

__device__ __forceinline__ v2i read_tr4(const void* p) {
  return __builtin_amdgcn_ds_read_tr4_b64_v2i32((__attribute__((address_space(3))) v2i*)p);
}
__device__ __forceinline__ v2i read_tr8(const void* p) {
  return __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) v2i*)p);
}

// Sixteen nibbles q (two's complement) as bytes 16 q, in the order 0 2 4 6, 1 3 5 7 of
// each eight.
__device__ __forceinline__ v4i nibbles_i8(v2i x) {
  return v4i{(int)((uint32_t)x.x << 4 & 0xf0f0f0f0u), (int)(x.x & 0xf0f0f0f0u),
             (int)((uint32_t)x.y << 4 & 0xf0f0f0f0u), (int)(x.y & 0xf0f0f0f0u)};
}

// A whole number w as digits to the base 256, -128 to 127 each (|w| < 2^30.99).
__device__ __forceinline__ uint32_t digits(int w) { return ((uint32_t)w + 0x80808080u) ^ 0x80808080u; }
// ... and the number that four sums of digits stand for (each |sum| < 2^25).
__device__ __forceinline__ float from_digits(v4i a) {
  return fmaf((float)a[3], 0x1p24f, fmaf((float)a[2], 0x1p16f, fmaf((float)a[1], 0x1p8f, (float)a[0])));
}

__device__ __forceinline__ float pow2_field(int field) { return __uint_as_float((uint32_t)field << 23); }

// Sum over the wavefront in every lane, by DPP steps and four readlanes.
template <int CTRL>
__device__ __forceinline__ float dpp_add_step(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float wave_sum_dpp(float x) {
  x = dpp_add_step<0xb1>(x);   // quad_perm 1,0,3,2
  x = dpp_add_step<0x4e>(x);   // quad_perm 2,3,0,1
  x = dpp_add_step<0x141>(x);  // row_half_mirror
  x = dpp_add_step<0x140>(x);  // row_mirror
  auto row = [&](int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), l)); };
  return (row(0) + row(16)) + (row(32) + row(48));
}

// D: head dimension, or with ANY at least that (dd then counts).  GP: query heads
// per KV head rounded up to 4 or 8.  KC8: k / 8, or 0 to take it from p.k.
// PG: 0 contiguous, 1 pages of 64 positions or more (a block of keys has one), 2
// pages of 16 or 32.
// Wavefronts per SIMD: 8 query heads at d = 128 take two registers more than three allow;
// held to three, 64 x 4000 keys 65.6 -> 61.9 us.
template <int D, bool ANY, int GP, int KC8, int PG>
__global__ __launch_bounds__(kDecThreads, GP == 4 && D <= 128 ? 4 : D <= 128 ? 3 : 2)
void sfa_decode_q4_kernel(DecParams p, int dd, const uint16_t* vscale) {
  constexpr int NG = D / 32;  // value scale groups, two 16-coordinate tiles each
  constexpr int NP = NG < 4 || GP == 4 && D <= 128 ? NG : D / 64;  // groups whose weights are in LDS at once
  const int d = ANY ? dd : D, ng = d / 32;
  const int k = KC8 > 0 ? 8 * KC8 : p.k;
  __shared__ float qd[256][GP];  // (an index past d reads zeros)
  __shared__ __attribute__((aligned(16))) unsigned char vt[kDecWaves][64 * D / 2];
  __shared__ __attribute__((aligned(16))) uint32_t pb[kDecWaves][NP][64][GP];  // digits of the weights
  __shared__ float red_m[kDecWaves][GP], red_l[kDecWaves][GP];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool by_slot = p.by_slot;
  const int bh = by_slot ? blockIdx.x : blockIdx.y;
  unsigned slot_u = by_slot ? blockIdx.y : blockIdx.x;
  if (!by_slot && gridDim.x % 2 == 0) slot_u = (slot_u + (unsigned)bh + ((unsigned)bh >> 2)) % gridDim.x;
  const int slot = (int)slot_u;
  const int b = bh / p.Hkv, hkv = bh - b * p.Hkv;
  // The query rows this wavefront will code are read beside the length, and the first
  // block of keys before they are coded: a step of few keys is this chain of loads.
  constexpr int E = (D + 63) / 64, QH = GP / kDecWaves;
  uint32_t qbits[QH][E];
  if (p.q_dense) {
#pragma unroll
    for (int j = 0; j < QH; ++j) {
      const float* qr = p.q_dense + ((int64_t)b * p.Hq + hkv * p.G + min(wave + kDecWaves * j, p.G - 1)) * d;
#pragma unroll
      for (int e = 0; e < E; ++e) qbits[j][e] = __float_as_uint(qr[min(lane + 64 * e, d - 1)]);
    }
  }
  const int L = seq_len_of(p.seq_len, b, p.Lmax);
  const DecPlan plan = decode_plan(L, p.window, p.n_global, p.aim);
  if (slot >= plan.count) return;
  const bool winq = plan.winq;
  const int wlo = plan.wlo, wg = plan.wg;
  int chunk = slot;
  if (winq && chunk >= plan.ngc) chunk += plan.wc0 - plan.ngc;
  const int c0 = chunk * plan.c;
  const int c1 = min(L, c0 + plan.c);

  float m_run[GP], m_use[GP], l_lane[GP];  // m_use: m_run, or 0 before the first key
#pragma unroll
  for (int h = 0; h < GP; ++h) { m_run[h] = -INFINITY; m_use[h] = 0.f; l_lane[h] = 0.f; }
  constexpr int NS = GP / 4;  // operands of four heads
  v4i acc[NS][2 * NG];
#pragma unroll
  for (int t = 0; t < NS * 2 * NG; ++t) acc[t / (2 * NG)][t % (2 * NG)] = v4i{0, 0, 0, 0};
  // Per group, an exponent field that no value scale seen so far passes (255: an
  // infinity or NaN); raised to one more than the scale that passes it, so that a second
  // raise is rare.  Weights carry 2^(155 - vexp): p = 1 with a scale of that field
  // becomes 2^28 to 2^29, and the largest weight is less than 2^30.9.
  int vexp[NG];
#pragma unroll
  for (int g = 0; g < NG; ++g) vexp[g] = 0;
  float pass = -INFINITY;  // exponents past it raise the maxima: 2^1.9 once there are any

  const int64_t kv_row0 = ((int64_t)b * p.Hkv + hkv) * p.Lmax;
  const int per_wave = plan.c / kDecWaves;
  int w0 = c0 + wave * per_wave;  // a multiple of 64
  int w1 = min(c1, w0 + per_wave);
  if (winq && w0 >= wg) {
    if (w1 <= wlo) w1 = w0;
    else w0 = max(w0, wlo & ~63);
  }
  // paged: lane l holds the page of the wave's l-th page-sized run (at most 1024
  // positions and pages of 16 or more: at most 64 runs)
  int tblv = 0;
  const int pg0 = PG ? (w0 >> p.log2P) : 0;
  if constexpr (PG > 0) {
    if (w0 < w1) {
      const int npg = ((w1 - 1) >> p.log2P) - pg0 + 1;
      if (lane < npg) {
        const int pg = p.table[(int64_t)b * p.max_pages + pg0 + lane];
        tblv = min(max(pg, 0), p.num_pages - 1);
      }
    }
  }
  const int pmask = (1 << (PG ? p.log2P : 0)) - 1;
  // the cache row of position j on page pg
  auto paged_row = [&](int pg, int j) -> int64_t { return (((int64_t)pg * p.Hkv + hkv) << p.log2P) + (j & pmask); };
  // the row of a block's first key, where the others follow it (PG < 2)
  auto block_row = [&](int sb) -> int64_t {
    if constexpr (PG == 1) return paged_row(__builtin_amdgcn_readlane(tblv, (sb >> p.log2P) - pg0), sb);
    else return kv_row0 + sb;
  };

  // Value rows: 16-byte piece x of the block's 64 ng, x = lane + 64 i,
  // belongs to key x / ng and holds its piece (x % ng) ^ ((key / (16 / ng)) % ng) (ng a
  // power of two; the others keep their order).
  unsigned char* vw = vt[wave];
  const int sw_mask = (ng & (ng - 1)) == 0 ? ng - 1 : 0;
  const int sw_shift = ng >= 8 ? 1 : ng >= 4 ? 2 : ng >= 2 ? 3 : 4;
  const uint8_t* vc = (const uint8_t*)p.v;
  const uint32_t run_off = (lane / NG) * (D / 2) + (((lane % NG) ^ ((lane / NG >> sw_shift) & sw_mask)) * 16);
  u32x4 vreg[NG];
  auto load_values = [&](int sb, int page) {  // page: of this lane's key (PG 2)
    const int last = w1 - 1 - sb;
    const uint8_t* base = PG < 2 ? vc + block_row(sb) * (d / 2) : nullptr;
    if constexpr (PG < 2 && !ANY) {
      if (last >= 63) {  // a whole block: its rows are one run
#pragma unroll
        for (int i = 0; i < NG; ++i)  // (the exchange repeats after 16 keys: 8 pieces, two loads)
          vreg[i] = *(const u32x4*)(base + (NG == 8 && i % 2 ? run_off ^ 64 : run_off) + i * 1024);
        return;
      }
    }
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      if (i >= ng) break;
      const int x = lane + 64 * i, key = x / ng, kc = min(key, last);
      const int piece = (x - key * ng) ^ ((key >> sw_shift) & sw_mask);
      if constexpr (PG < 2)
        vreg[i] = *(const u32x4*)(base + (uint32_t)(kc * (d / 2) + piece * 16));
      else
        vreg[i] = *(const u32x4*)(vc + paged_row(__shfl(page, kc, 64), sb + kc) * (d / 2) + piece * 16);
    }
  };
  // A key's codes and scales (lane = key), loaded a block ahead.
  constexpr int NKC = KC8 > 0 ? KC8 : 1;
  uint2 ki[NKC];
  constexpr int NVS = !ANY && NG % 2 == 0 ? NG / 2 : NG;  // value scales, two to a word where a row is whole words
  uint32_t kq[NKC], vraw[NVS];
  float ks = 0.f;
  auto lane_row = [&](int sb, int page) -> int64_t {
    const int kc = min(lane, w1 - 1 - sb);
    return PG < 2 ? block_row(sb) + kc : paged_row(page, sb + kc);
  };
  auto load_codes = [&](int sb, int page) {
    const int64_t row = PG < 2 ? block_row(sb) : lane_row(sb, page);
    const uint32_t o = PG < 2 ? (uint32_t)min(lane, w1 - 1 - sb) : 0u;
    if constexpr (KC8 > 0) {
      const uint8_t* pi = (const uint8_t*)p.kc_idx + row * k + o * k;
      const uint8_t* pq = (const uint8_t*)p.kc_val + row * (k / 2) + o * (k / 2);
#pragma unroll
      for (int c = 0; c < KC8; ++c) {
        ki[c] = ((const uint2*)pi)[c];
        kq[c] = ((const uint32_t*)pq)[c];
      }
    }
    ks = (p.kc_scale + row)[o];
    const uint16_t* pv = vscale + row * ng + o * ng;
    if constexpr (!ANY && D == 256) {
      const u32x4 w = *(const u32x4*)pv;
#pragma unroll
      for (int g = 0; g < 4; ++g) vraw[g] = w[g];
    } else if constexpr (!ANY && D == 128) {
      const uint2 w = *(const uint2*)pv;
      vraw[0] = w.x; vraw[1] = w.y;
    } else if constexpr (!ANY && D == 64) {
      vraw[0] = *(const uint32_t*)pv;
    } else {
#pragma unroll
      for (int g = 0; g < NG; ++g) vraw[g] = g < ng ? pv[g] : 0;
    }
  };
  auto page_of = [&](int sb) -> int {
    if constexpr (PG == 2) return __shfl(tblv, (min(sb + lane, w1 - 1) >> p.log2P) - pg0, 64);
    else return 0;
  };
  // operand addresses in LDS
  const int r16 = lane & 15, key0 = lane & 48;
  // weights: a key's place in its group's block (each odd sixteen keys have their halves
  // exchanged, so that the reads of a half of each sixteen fall on all banks)
  auto place = [](int key) { return key ^ (key >> 1 & 8); };
  const int ak = r16 >> 1;  // key ak of eight in the nibbles' order
  const uint32_t* a_src[2];
#pragma unroll
  for (int m = 0; m < 2; ++m) a_src[m] = &pb[wave][0][place(key0 + 8 * m + (2 * ak & 6) + (ak >> 2))][2 * (r16 & 1)];
  const unsigned char* b_src[NG];
#pragma unroll
  for (int g = 0; g < NG; ++g)
    b_src[g] = vw + (key0 + r16) * (d / 2) + (g ^ ((r16 >> sw_shift) & sw_mask)) * 16;

  int page = 0;
  if (w0 < w1) {
    page = page_of(w0);
    load_codes(w0, page);
    load_values(w0, page);
  }

  // dense query rows
  for (int x = tid; x < 256 * GP; x += kDecThreads) (&qd[0][0])[x] = 0.f;
  __syncthreads();
  if (p.q_dense) {
#pragma unroll
    for (int j = 0; j < QH; ++j) {
      const int h = wave + kDecWaves * j;
      uint32_t key[E];
      bool sel[E];
#pragma unroll
      for (int e = 0; e < E; ++e) key[e] = topk_key(qbits[j][e], lane + 64 * e < d);
      topk_select<E>(key, k, sel);
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (h < p.G && sel[e] && lane + 64 * e < d) qd[lane + 64 * e][h] = __uint_as_float(qbits[j][e]);
    }
  } else {
    for (int x = tid; x < p.G * k; x += kDecThreads) {
      const int h = x / k, t = x - h * k;
      const int64_t qi = ((int64_t)b * p.Hq + hkv * p.G + h) * k + t;
      const int u = min(load_idx(p.q_idx, qi, p.qifmt, 255), d - 1);
      qd[u][h] = load_val(p.q_val, qi, p.qvfmt);
    }
  }
  __syncthreads();
  for (int sb = w0; sb < w1; sb += 64) {
    const int last = w1 - 1 - sb;
    const int sb_next = last >= 64 ? sb + 64 : sb;  // (the last block loads itself again, unused)
    const int page_next = page_of(sb_next);
#pragma unroll
    for (int i = 0; i < NG; ++i)
      if (i < ng) *(u32x4*)(vw + (lane + 64 * i) * 16) = vreg[i];
    load_values(sb_next, page_next);
    // scores: the code values count in sixteenths (v_cvt_off_f32_i4)
    float s[GP];
#pragma unroll
    for (int h = 0; h < GP; ++h) s[h] = 0.f;
    auto score8 = [&](uint2 iw, uint32_t qw) {
      const uint32_t qh = qw >> 4;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int u = (int)(((e < 4 ? iw.x : iw.y) >> (8 * (e & 3))) & 255u);
        const float kv = __builtin_amdgcn_cvt_off_f32_i4((int)((((e & 1) ? qh : qw) >> (8 * (e >> 1))) & 255u));
#pragma unroll
        for (int h = 0; h < GP; ++h) s[h] = fmaf(kv, qd[u][h], s[h]);
      }
    };
    if constexpr (KC8 > 0) {
#pragma unroll
      for (int c = 0; c < KC8; ++c) {
        score8(ki[c], kq[c]);
        // eight gathers in flight, not all of them: registers
#pragma unroll
        for (int h = 0; h < GP; ++h) asm volatile("" : "+v"(s[h]));
      }
    } else {
      const int64_t row = lane_row(sb, page);
      for (int c = 0; c < k / 8; ++c)
        score8(((const uint2*)((const uint8_t*)p.kc_idx + row * k))[c],
               ((const uint32_t*)((const uint8_t*)p.kc_val + row * (k / 2)))[c]);
    }
    const float kfac = p.scale_log2 * ks * 16.f;
    uint32_t vs[NG];  // the value scales, as float32 bits
#pragma unroll
    for (int g = 0; g < NG; ++g)
      vs[g] = NVS == NG ? vraw[g % NVS] << 16 : (g & 1) ? vraw[g / 2] & 0xffff0000u : vraw[g / 2] << 16;
    load_codes(sb_next, page_next);
    float t[GP];
#pragma unroll
    for (int h = 0; h < GP; ++h) t[h] = fmaf(s[h], kfac, -m_use[h]);
    const bool full = last >= 63 && (sb >= wlo || sb + 63 < wg);  // uniform: the query sees every key
    const bool ok = lane <= last && (sb + lane >= wlo || sb + lane < wg);
    if (!full) {
#pragma unroll
      for (int h = 0; h < GP; ++h) t[h] = ok ? t[h] : -INFINITY;
#pragma unroll
      for (int g = 0; g < NG; ++g) vs[g] = ok ? vs[g] : 0u;
    }
    // a key that passes a running maximum by 2^1.9, or a group's exponent
    float tmax = t[0];
#pragma unroll
    for (int h = 1; h < GP; ++h) tmax = fmaxf(tmax, t[h]);
    uint64_t up = wave_ballot(tmax > pass);
#pragma unroll
    for (int g = 0; g < NG; ++g) up |= wave_ballot(vs[g] > (uint32_t)(vexp[g] << 23 | 0x7fffff));
    if (up) {  // uniform; the first block always
      float fa[NS];
      {
        float alpha[GP];
#pragma unroll
        for (int h = 0; h < GP; ++h) {
          const float x = full || ok ? s[h] * kfac : -INFINITY;
          const float m_new = fmaxf(m_run[h], wave_max_dpp(x));
          alpha[h] = m_run[h] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run[h] - m_new);
          l_lane[h] *= alpha[h];
          m_run[h] = m_new;
          m_use[h] = m_new == -INFINITY ? 0.f : m_new;
          t[h] = x - m_use[h];
        }
        pass = m_run[0] == -INFINITY ? -INFINITY : 1.9f;
#pragma unroll
        for (int n = 0; n < NS; ++n) {  // this lane's head of the four
          fa[n] = alpha[4 * n];
#pragma unroll
          for (int h = 1; h < 4; ++h) fa[n] = lane >> 4 == h ? alpha[4 * n + h] : fa[n];
        }
      }
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const int vmax = (int)(wave_umax(vs[g] & 0x7fffffffu) >> 23);
        const int vnew = vmax <= vexp[g] ? vexp[g] : vmax == 255 ? 255 : min(vmax + 1, 254);
        const float f = vnew - vexp[g] > 126 ? 0.f : pow2_field(127 + vexp[g] - vnew);
        vexp[g] = vnew;
        if (sb == w0) continue;  // the sums are still zero
#pragma unroll
        for (int t = 0; t < NS * 2; ++t) {  // rounded to 24 bits, kept as two digits
          v4i& a = acc[t / 2][2 * g + t % 2];
          const float v = from_digits(a) * (f * fa[t / 2]);
          const float top = rintf(v * 0x1p-24f);
          a = v4i{(int)rintf(fmaf(top, -0x1p24f, v)), 0, 0, (int)top};
        }
      }
    }
    float pj[GP];
#pragma unroll
    for (int h = 0; h < GP; ++h) {
      pj[h] = __builtin_amdgcn_exp2f(t[h]);
      l_lane[h] += pj[h];
    }
#pragma unroll
    for (int g0 = 0; g0 < NG; g0 += NP) {
      if (g0 >= ng) break;
      // weights, rounded to the nearest whole number
#pragma unroll
      for (int g = g0; g < g0 + NP && g < NG; ++g) {
        if (g >= ng) break;
        const float f = __builtin_ldexpf(__uint_as_float(vs[g]), 155 - vexp[g]);
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          u32x4 w;
#pragma unroll
          for (int h = 0; h < 4; ++h) w[h] = digits((int)fmaf(pj[4 * n + h], f, 0.5f));
          *(u32x4*)&pb[wave][g - g0][place(lane)][4 * n] = w;
        }
      }
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_sched_barrier(0);
      // P.V.
      // Lane l: operand row l % 16 (digit row % 4 of head row / 4), keys 16 (l / 16) + 0..15
      // in the nibbles' order.
#pragma unroll
      for (int g = g0; g < g0 + NP && g < NG; ++g) {
        if (g >= ng) break;
        const v4i B[2] = {nibbles_i8(read_tr4(b_src[g])), nibbles_i8(read_tr4(b_src[g] + 8))};
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          const v2i lo = read_tr8(a_src[0] + (g - g0) * 64 * GP + 4 * n), hi = read_tr8(a_src[1] + (g - g0) * 64 * GP + 4 * n);
          const v4i A = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
          for (int tt = 0; tt < 2; ++tt)
            acc[n][2 * g + tt] = __builtin_amdgcn_mfma_i32_16x16x64_i8(A, B[tt], acc[n][2 * g + tt], 0, 0, 0);
        }
      }
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    page = page_next;
  }

  // The sums to LDS, with the powers of two of weights and numbers taken out (2^(155 -
  // vexp) and 16).  Lane l, register i: digit i of head l / 16, coordinate l % 16.
#pragma unroll
  for (int h = 0; h < GP; ++h) l_lane[h] = wave_sum_dpp(l_lane[h]);
  __syncthreads();  // every wavefront is done with pb
  float* red_o = (float*)&pb[0][0][0][0];  // [wave][GP][D]
  static_assert(sizeof(pb) >= sizeof(float) * kDecWaves * GP * D, "the partials fit the weights' place");
#pragma unroll
  for (int n = 0; n < NS; ++n)
#pragma unroll
    for (int t = 0; t < 2 * NG; ++t)
      red_o[(wave * GP + 4 * n + (lane >> 4)) * D + (lane & 15) + 16 * t] =
          vexp[t / 2] == 255 ? NAN : ldexpf(from_digits(acc[n][t]), vexp[t / 2] - 159);
  if (lane == 0) {
#pragma unroll
    for (int h = 0; h < GP; ++h) { red_m[wave][h] = m_run[h]; red_l[wave][h] = l_lane[h]; }
  }
  __syncthreads();
  for (int x = tid; x < p.G * d; x += kDecThreads) {
    const int h = x / d, c = x - h * d;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kDecWaves; ++w) M = fmaxf(M, red_m[w][h]);
    const float Mu = (M == -INFINITY) ? 0.f : M;
    float lsum = 0.f, osum = 0.f;
#pragma unroll
    for (int w = 0; w < kDecWaves; ++w) {
      const float sc = __builtin_amdgcn_exp2f(red_m[w][h] - Mu);
      lsum += sc * red_l[w][h];
      osum += sc * red_o[(w * GP + h) * D + c];
    }
    const int64_t part = ((int64_t)b * p.Hq + hkv * p.G + h) * p.nch + slot;
    p.ws_o[part * d + c] = osum;
    if (c == 0) { p.ws_m[part] = M; p.ws_l[part] = lsum; }
  }
}

// Merge of the chunks' partials by their LSE.  A wavefront holds a query head's row,
// lane l coordinates l + 64 i.  The output is kMergeQ4 sums, each over the chunks of
// one residue in order, added in order: by as many wavefronts (WIDE), or in turn by
// one.  Which of the two runs follows the cache's capacity; the sums, and so the bits,
// do not.  A chain of dependent loads is what this kernel's time is made of: the first
// maxima, sums and rows are read beside the length, before it is known how many of
// them count (slots past them exist, unwritten).
constexpr int kMergeQ4 = 8;
template <int NV, bool WIDE>
__global__ __launch_bounds__(WIDE ? 64 * kMergeQ4 : 256) void sfa_decode_q4_combine_kernel(DecParams p, int rows, int d,
                                                                                        void* o, int obf16, float* lse) {
  constexpr int NS = WIDE ? 1 : kMergeQ4;  // sums in this wavefront
  __shared__ float part[WIDE ? kMergeQ4 : 1][64 * NV];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int bh = WIDE ? (int)blockIdx.x : (int)blockIdx.x * 4 + wave;
  if (bh >= rows) return;  // uniform per wave; no workgroup barrier in this form
  const int64_t s0 = (int64_t)bh * p.nch;
  const int at = min(lane, p.nch - 1);
  const float m0 = p.ws_m[s0 + at], l0 = p.ws_l[s0 + at];
  float x[NS][NV];
  auto load_rows = [&](int c0) {
#pragma unroll
    for (int g = 0; g < NS; ++g) {
      const float* src = p.ws_o + (s0 + min(c0 + (WIDE ? wave : g), p.nch - 1)) * d;
#pragma unroll
      for (int i = 0; i < NV; ++i) x[g][i] = src[min(lane + 64 * i, d - 1)];
    }
  };
  load_rows(0);
  const int L = seq_len_of(p.seq_len, bh / p.Hq, p.Lmax);
  const int nc = decode_plan(L, p.window, p.n_global, p.aim).count;
  float M = lane < nc ? m0 : -INFINITY;
  for (int c = lane + 64; c < nc; c += 64) M = fmaxf(M, p.ws_m[s0 + c]);
  M = wave_max_dpp(M);
  const float Mu = (M == -INFINITY) ? 0.f : M;
  float os[NS][NV];
#pragma unroll
  for (int g = 0; g < NS; ++g)
#pragma unroll
    for (int i = 0; i < NV; ++i) os[g][i] = 0.f;
  float lsum = 0.f;
  for (int cb = 0; cb < nc; cb += 64) {  // 64 chunks' weights, one a lane
    const bool in = cb + lane < nc;
    const float w = in ? __builtin_amdgcn_exp2f((cb == 0 ? m0 : p.ws_m[s0 + cb + lane]) - Mu) : 0.f;
    lsum = in ? fmaf(w, cb == 0 ? l0 : p.ws_l[s0 + cb + lane], lsum) : lsum;
    for (int c0 = cb; c0 < min(nc, cb + 64); c0 += kMergeQ4) {
      float y[NS][NV];
#pragma unroll
      for (int g = 0; g < NS; ++g)
#pragma unroll
        for (int i = 0; i < NV; ++i) y[g][i] = x[g][i];
      if (c0 + kMergeQ4 < nc) load_rows(c0 + kMergeQ4);
#pragma unroll
      for (int g = 0; g < NS; ++g) {
        const int c = c0 + (WIDE ? wave : g);
        const float wc = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), c - cb));
#pragma unroll
        for (int i = 0; i < NV; ++i) os[g][i] = c < nc ? fmaf(wc, y[g][i], os[g][i]) : os[g][i];
      }
    }
  }
  lsum = wave_sum_dpp(lsum);
  if constexpr (WIDE) {
#pragma unroll
    for (int i = 0; i < NV; ++i) part[wave][lane + 64 * i] = os[0][i];
    __syncthreads();
    if (wave != 0) return;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float sum = os[0][i];
#pragma unroll
    for (int g = 1; g < kMergeQ4; ++g) sum += WIDE ? part[g][lane + 64 * i] : os[WIDE ? 0 : g][i];
    const float out = lsum == 0.f ? 0.f : sum / lsum;
    const int c = lane + 64 * i;
    if (c < d) {
      if (obf16) ((uint16_t*)o)[(int64_t)bh * d + c] = (uint16_t)f32_to_bf16_rne(out);
      else ((float*)o)[(int64_t)bh * d + c] = out;
    }
  }
  if (lse && lane == 0) lse[bh] = lsum == 0.f ? -INFINITY : (M + __log2f(lsum)) * kLn2;
}

template <int NV>
void launch_q4_combine(const DecParams& p, const DecodeArgs& a, hipStream_t stream) {
  const int rows = a.B * a.Hq;
  // one wavefront a row where a row's chunks are few or the rows fill the chip
  if (p.nch <= 2 * kMergeQ4 || rows >= 8192)
    hipLaunchKernelGGL((sfa_decode_q4_combine_kernel<NV, false>), dim3((rows + 3) / 4), dim3(256), 0, stream, p, rows, a.d,
                       a.o, a.obf16, a.lse);
  else
    hipLaunchKernelGGL((sfa_decode_q4_combine_kernel<NV, true>), dim3(rows), dim3(64 * kMergeQ4), 0, stream, p, rows, a.d,
                       a.o, a.obf16, a.lse);
}

template <int D, bool ANY, int GP, int KC8>
void launch_q4_t(const DecParams& p, const DecodeArgs& a, hipStream_t stream) {
  const dim3 grid = p.by_slot ? dim3(a.B * p.Hkv, p.nch) : dim3(p.nch, a.B * p.Hkv), block(kDecThreads);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, p, a.d, a.v_scale16); };
  // A block of 64 keys is one run of rows in pages of 64 and more, whose base is scalar (d =
  // 128, 64 x 4000 keys, 8 query heads a group: 61.5 us, with an address a lane 64.5).
  if (!p.table) go(sfa_decode_q4_kernel<D, ANY, GP, KC8, 0>);
  else if (p.log2P >= 6) go(sfa_decode_q4_kernel<D, ANY, GP, KC8, 1>);
  else go(sfa_decode_q4_kernel<D, ANY, GP, KC8, 2>);
}

template <int D, bool ANY, int GP>
void launch_q4_k(const DecParams& p, const DecodeArgs& a, hipStream_t stream) {
  // k known: the codes of the next block are loaded while this one is multiplied (64 x 4000
  // keys, k = 16, against codes read in their turn: d = 64 29.1 and 32.4 us, d = 128 with 8
  // query heads a group 61.5 and 72.2, d = 256 101 and 120).
  if constexpr (!ANY) {
    if (a.k == 8) return launch_q4_t<D, ANY, GP, 1>(p, a, stream);
    if (a.k == 16) return launch_q4_t<D, ANY, GP, 2>(p, a, stream);
    if (a.k == 32) return launch_q4_t<D, ANY, GP, 4>(p, a, stream);
  }
  launch_q4_t<D, ANY, GP, 0>(p, a, stream);
}

template <int D, bool ANY = false>
void launch_q4_g(const DecParams& p, const DecodeArgs& a, hipStream_t stream) {
  if (p.G <= 4) launch_q4_k<D, ANY, 4>(p, a, stream);
  else launch_q4_k<D, ANY, 8>(p, a, stream);
}

}  // namespace

// For any group and window, as decode_workspace_bytes, at any head dimension: a sequence has
// at most aim + 2 chunks below kDecodeChunk keys, or its whole chunks of kDecodeChunk.
size_t decode_q4_workspace_bytes(int B, int Hq, int Lmax, int d) {
  const int aim = decode_chunks_aim(B, (Hq + kDecMaxG - 1) / kDecMaxG, true, 1);
  const int fine = Lmax / kDecodeMinChunk + (Lmax % kDecodeMinChunk != 0), whole = decode_slots(Lmax, 0);
  const int slots = aim == 0 ? whole : std::min(fine, std::max(whole, aim + 2));
  return (size_t)B * Hq * (size_t)slots * (size_t)(d + 2) * sizeof(float);
}

hipError_t launch_attn_decode_q4(const DecodeArgs& a, hipStream_t stream) {
  const DecParams p = make_dec_params(a);
  // d known: no divisions and no absent groups in the loop (64 x 4000 keys, k = 16, against the
  // kernel of any d: d = 96 35.7 and 63.3 us, d = 256 with 8 query heads a group 101 and 202).
  if (a.d == 64) launch_q4_g<64>(p, a, stream);
  else if (a.d == 128) launch_q4_g<128>(p, a, stream);
  else if (a.d == 96) launch_q4_g<96>(p, a, stream);
  else if (a.d == 256) launch_q4_g<256>(p, a, stream);
  else launch_q4_g<256, true>(p, a, stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.d <= 64) launch_q4_combine<1>(p, a, stream);
  else if (a.d <= 128) launch_q4_combine<2>(p, a, stream);
  else launch_q4_combine<4>(p, a, stream);
  return hipGetLastError();
}

}  // namespace sfa
