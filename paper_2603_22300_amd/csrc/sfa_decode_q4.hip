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
//   P.V      on the matrix cores, v_mfma_f32_16x16x32_f16.  The weights of a group
//            of 32 coordinates are p * vs, split into two float16 pieces, p0 =
//            f16(p vs) and p1 = f16(p vs - p0): the pieces of the group's query
//            heads fill the sixteen rows of one operand, so the second piece (and
//            with it float32 accuracy, 2^-22) costs no matrix instruction.  The
//            other operand is the cached integers, exact in float16.
// Both operands have 16 or 8 keys of one row in a lane, and both are held key by
// key: the transposing LDS reads turn them, ds_read_b64_tr_b4 the cached nibbles
// as they are and ds_read_b64_tr_b16 the weights.
//
// float16 range: each group's weights are scaled by a power of two that follows
// the largest value scale seen in the group, as the running maximum does for p
// (`vexp` below): value scales of any magnitude keep their accuracy.  Both follow
// lazily, p up to 2^8 and only upwards for the scales, so that most blocks of keys
// touch neither the maxima nor the accumulators.
#include "sfa_decode_kernel.h"

namespace sfa {
namespace {

typedef int v2i __attribute__((ext_vector_type(2)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ v2i read_tr4(const void* p) {
  return __builtin_amdgcn_ds_read_tr4_b64_v2i32((__attribute__((address_space(3))) v2i*)p);
}
__device__ __forceinline__ v4s read_tr16(const void* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)p);
}

// Eight nibbles (two's complement) as float16, in the order n0 n4 n1 n5 n2 n6 n3
// n7.  A nibble with its sign bit flipped is q + 8; at the low end of a float16
// mantissa under exponent 2^10 it adds itself to 1024, at bit 4 under 2^6 to 64.
__device__ __forceinline__ f16x8 nibbles_f16(uint32_t x) {
  const uint32_t y = x >> 8;
  const h2 lo = {(_Float16)1032.f, (_Float16)1032.f}, hi = {(_Float16)72.f, (_Float16)72.f};
  const h2 a = __builtin_bit_cast(h2, (x & 0x000f000fu) ^ 0x64086408u) - lo;
  const h2 b = __builtin_bit_cast(h2, (x & 0x00f000f0u) ^ 0x54805480u) - hi;
  const h2 c = __builtin_bit_cast(h2, (y & 0x000f000fu) ^ 0x64086408u) - lo;
  const h2 d = __builtin_bit_cast(h2, (y & 0x00f000f0u) ^ 0x54805480u) - hi;
  return f16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// D: head dimension, or 256 for any d <= 256 (p.d then counts).  GP: query heads
// per KV head rounded up to 4 or 8.  KC8: k / 8, or 0 to take it from p.k.
template <int D, int GP, int KC8, bool PAGED>
__global__ __launch_bounds__(kDecThreads, GP == 4 && D <= 128 ? 3 : GP == 8 && D <= 128 ? 2 : 1) void sfa_decode_q4_kernel(DecParams p, int dd, const uint16_t* vscale) {
  constexpr int NG = D / 32;              // value scale groups, two 16-coordinate tiles each
  constexpr int PITCH = D / 2 + 8;        // bytes of a value row in LDS: rows on different banks
  const int d = D == 256 ? dd : D, ng = d / 32;
  const int k = KC8 > 0 ? 8 * KC8 : p.k;
  __shared__ float qd[D][GP];
  __shared__ __attribute__((aligned(16))) unsigned char vt[kDecWaves][64 * PITCH];
  __shared__ __attribute__((aligned(16))) _Float16 pb[kDecWaves][NG][64][2 * GP];
  __shared__ float red_m[kDecWaves][GP], red_l[kDecWaves][GP];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool by_slot = p.by_slot;
  const int bh = by_slot ? blockIdx.x : blockIdx.y;
  unsigned slot_u = by_slot ? blockIdx.y : blockIdx.x;
  if (!by_slot && gridDim.x % 2 == 0) slot_u = (slot_u + (unsigned)bh + ((unsigned)bh >> 2)) % gridDim.x;
  const int slot = (int)slot_u;
  const int b = bh / p.Hkv, hkv = bh - b * p.Hkv;
  const int L = seq_len_of(p.seq_len, b, p.Lmax);
  const DecPlan plan = decode_plan(L, p.window, p.n_global, p.aim);
  if (slot >= plan.count) return;
  const bool winq = plan.winq;
  const int wlo = plan.wlo, wg = plan.wg;
  int chunk = slot;
  if (winq && chunk >= plan.ngc) chunk += plan.wc0 - plan.ngc;
  const int c0 = chunk * plan.c;
  const int c1 = min(L, c0 + plan.c);

  // dense query rows
  if (p.q_dense) {
    constexpr int E = (D + 63) / 64;
    for (int h = wave; h < GP; h += kDecWaves) {
      const float* qr = p.q_dense + ((int64_t)b * p.Hq + hkv * p.G + min(h, p.G - 1)) * d;
      uint32_t bits[E], key[E];
      bool sel[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int c = lane + 64 * e;
        bits[e] = __float_as_uint(qr[min(c, d - 1)]);
        key[e] = topk_key(bits[e], c < d);
      }
      topk_select<E>(key, k, sel);
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (lane + 64 * e < D) qd[lane + 64 * e][h] = sel[e] && h < p.G ? __uint_as_float(bits[e]) : 0.f;
    }
  } else {
    for (int x = tid; x < D * GP; x += kDecThreads) (&qd[0][0])[x] = 0.f;
    __syncthreads();
    for (int x = tid; x < p.G * k; x += kDecThreads) {
      const int h = x / k, t = x - h * k;
      const int64_t qi = ((int64_t)b * p.Hq + hkv * p.G + h) * k + t;
      const int u = min(load_idx(p.q_idx, qi, p.qifmt, 255), d - 1);
      qd[u][h] = load_val(p.q_val, qi, p.qvfmt);
    }
  }
  __syncthreads();

  float m_run[GP], l_lane[GP];
#pragma unroll
  for (int h = 0; h < GP; ++h) { m_run[h] = -INFINITY; l_lane[h] = 0.f; }
  floatx4 acc[2 * NG];
#pragma unroll
  for (int t = 0; t < 2 * NG; ++t) acc[t] = floatx4{0.f, 0.f, 0.f, 0.f};
  // Per group, the exponent field of the largest value scale seen, at least 6; the
  // weights carry 2^(132 - vexp) (a scale of that exponent field becomes 2^5 to 2^6,
  // a weight at most 2^14).
  int vexp[NG];
#pragma unroll
  for (int g = 0; g < NG; ++g) vexp[g] = 6;

  const int64_t kv_row0 = ((int64_t)b * p.Hkv + hkv) * p.Lmax;
  const int per_wave = plan.c / kDecWaves;
  int w0 = c0 + wave * per_wave;
  int w1 = min(c1, w0 + per_wave);
  if (winq && w0 >= wg) {
    if (w1 <= wlo) w1 = w0;
    else w0 = max(w0, wlo & ~63);
  }
  auto key_ok = [&](int j) { return j >= wlo || j < wg; };
  // paged: lane l holds the page of the wave's l-th page-sized run (at most 1024
  // positions and pages of 16 or more: at most 64 runs)
  int tblv = 0;
  const int pg0 = PAGED ? (w0 >> p.log2P) : 0;
  if constexpr (PAGED) {
    if (w0 < w1) {
      const int npg = ((w1 - 1) >> p.log2P) - pg0 + 1;
      if (lane < npg) {
        const int pg = p.table[(int64_t)b * p.max_pages + pg0 + lane];
        tblv = min(max(pg, 0), p.num_pages - 1);
      }
    }
  }
  const int pmask = (1 << (PAGED ? p.log2P : 0)) - 1;
  auto row_of = [&](int j) -> int64_t {  // w0 <= j < w1, any j per lane
    if constexpr (PAGED)
      return (((int64_t)__shfl(tblv, (j >> p.log2P) - pg0, 64) * p.Hkv + hkv) << p.log2P) + (j & pmask);
    else return kv_row0 + j;
  };

  unsigned char* vw = vt[wave];
  const uint8_t* vc = (const uint8_t*)p.v;
  // A block of 64 keys in registers, loaded one block ahead: value rows (16 bytes a
  // lane and load, piece x of the rows' 64 d / 32 pieces), and lane = key: codes
  // (KC8 > 0), scales.
  constexpr int NKC = KC8 > 0 ? KC8 : 1;
  uint4 vraw[NG];
  uint2 ki[NKC];
  uint32_t kq[NKC], vs_next[NG];
  float ks_next = 0.f;
  int64_t row = 0;
  auto load_values = [&](int sb) {
    row = row_of(min(sb + lane, w1 - 1));
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      if (i >= ng) break;
      const int x = lane + 64 * i, jj = x / ng, piece = x - jj * ng;
      const int64_t vr = PAGED ? (int64_t)__shfl(row, jj, 64) : kv_row0 + min(sb + jj, w1 - 1);
      vraw[i] = *(const uint4*)(vc + vr * (d / 2) + piece * 16);
    }
  };
  auto load_codes = [&]() {  // of the rows that load_values went to
    if constexpr (KC8 > 0) {
#pragma unroll
      for (int c = 0; c < KC8; ++c) {
        ki[c] = ((const uint2*)((const uint8_t*)p.kc_idx + row * k))[c];
        kq[c] = ((const uint32_t*)((const uint8_t*)p.kc_val + row * (k / 2)))[c];
      }
    }
    ks_next = p.kc_scale[row];
#pragma unroll
    for (int g = 0; g < NG; ++g) vs_next[g] = g < ng ? vscale[row * ng + g] : 0;
  };
  if (w0 < w1) { load_values(w0); load_codes(); }
  for (int sb = w0; sb < w1; sb += 64) {
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      if (i >= ng) break;
      const int x = lane + 64 * i, jj = x / ng, piece = x - jj * ng;
      uint2* dst = (uint2*)(vw + jj * PITCH + piece * 16);
      dst[0] = make_uint2(vraw[i].x, vraw[i].y);
      dst[1] = make_uint2(vraw[i].z, vraw[i].w);
    }
    const int64_t row_here = row;
    const bool more = sb + 64 < w1;
    if (more) load_values(sb + 64);
    // scores
    float s[GP];
#pragma unroll
    for (int h = 0; h < GP; ++h) s[h] = 0.f;
    auto score8 = [&](uint2 iw, uint32_t qw) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int u = min((int)(((e < 4 ? iw.x : iw.y) >> (8 * (e & 3))) & 255u), d - 1);
        const float kv = (float)((int)(qw << (28 - 4 * e)) >> 28);
#pragma unroll
        for (int h = 0; h < GP; ++h) s[h] = fmaf(kv, qd[u][h], s[h]);
      }
    };
    if constexpr (KC8 > 0) {
#pragma unroll
      for (int c = 0; c < KC8; ++c) score8(ki[c], kq[c]);
    } else {
      for (int c = 0; c < k / 8; ++c)
        score8(((const uint2*)((const uint8_t*)p.kc_idx + row_here * k))[c],
               ((const uint32_t*)((const uint8_t*)p.kc_val + row_here * (k / 2)))[c]);
    }
    const float ks = ks_next;
    uint32_t vsb[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) vsb[g] = vs_next[g];
    if (more) load_codes();
    const float kfac = p.scale_log2 * ks;
    const bool ok = sb + lane < w1 && key_ok(sb + lane);
    float t[GP];
    bool up = false;  // this lane's key passes a running maximum by 2^8, or a group's exponent
#pragma unroll
    for (int h = 0; h < GP; ++h) {
      t[h] = ok ? s[h] * kfac : -INFINITY;
      up |= t[h] > m_run[h] + 8.f;
    }
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      vsb[g] = ok ? vsb[g] & 0x7fffu : 0u;
      up |= (int)(vsb[g] >> 7) > vexp[g];
    }
    if (wave_ballot(up)) {  // uniform; the first block always
      float fa[4];
      {
        float alpha[GP];
#pragma unroll
        for (int h = 0; h < GP; ++h) {
          const float m_new = fmaxf(m_run[h], wave_max_dpp(t[h]));
          alpha[h] = m_run[h] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run[h] - m_new);
          l_lane[h] *= alpha[h];
          m_run[h] = m_new;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) fa[i] = GP == 4 || !(lane & 16) ? alpha[i] : alpha[GP - 4 + i];
      }
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const int vnew = max(vexp[g], min((int)(wave_umax(vsb[g]) >> 7), 254));
        const float f = vnew - vexp[g] > 126 ? 0.f : __uint_as_float((uint32_t)(127 + vexp[g] - vnew) << 23);
        vexp[g] = vnew;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          acc[2 * g][i] *= f * fa[i];
          acc[2 * g + 1][i] *= f * fa[i];
        }
      }
    }
    float pj[GP];
#pragma unroll
    for (int h = 0; h < GP; ++h) {
      pj[h] = __builtin_amdgcn_exp2f(t[h] - (m_run[h] == -INFINITY ? 0.f : m_run[h]));
      l_lane[h] += pj[h];
    }
    // weights: [group][key][pieces 0 of the heads, pieces 1]
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      if (g >= ng) break;
      const float f = bf16_bits_to_f32(vsb[g]) * __uint_as_float((uint32_t)(259 - vexp[g]) << 23);
      _Float16 w[2 * GP];
#pragma unroll
      for (int h = 0; h < GP; ++h) {
        const float x = pj[h] * f;
        w[h] = (_Float16)x;
        w[GP + h] = (_Float16)(x - (float)w[h]);
      }
#pragma unroll
      for (int i = 0; i < GP / 4; ++i) ((f16x8*)&pb[wave][g][lane][0])[i] = *(f16x8*)&w[8 * i];
    }
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    // P.V.  Lane l: operand row l % 16, keys 16 (l / 16) + 8 m + 0..7, in the
    // nibbles' order 0 4 1 5 2 6 3 7.
    const int r16 = lane & 15, key0 = lane & 48;
    const int quarter = (r16 & 3) & (GP / 2 - 1);  // of the 2 GP rows (GP = 4: rows 8 to 15 repeat 0 to 7)
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      if (g >= ng) break;
      f16x8 A[2];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const int j = r16 >> 2;  // keys (j >> 1) + 4 (j & 1) for elements 0..3, and 2 more for 4..7
        const _Float16* src = &pb[wave][g][key0 + 8 * m + (j >> 1) + 4 * (j & 1)][4 * quarter];
        const v4s lo = read_tr16(src), hi = read_tr16(src + 2 * 2 * GP);
        A[m] = __builtin_bit_cast(f16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      }
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const v2i n = read_tr4(vw + (key0 + r16) * PITCH + g * 16 + tt * 8);
        acc[2 * g + tt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(A[0], nibbles_f16(n.x), acc[2 * g + tt], 0, 0, 0);
        acc[2 * g + tt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(A[1], nibbles_f16(n.y), acc[2 * g + tt], 0, 0, 0);
      }
    }
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }

  // The two pieces' sums, and the power of two of the weights.  Lane l, register i:
  // row 4 (l / 16) + i, coordinate l % 16 of the tile.
#pragma unroll
  for (int h = 0; h < GP; ++h) l_lane[h] = wave_sum(l_lane[h]);
  __syncthreads();  // every wavefront is done with pb
  float* red_o = (float*)&pb[0][0][0][0];  // [wave][GP][D]
  static_assert(sizeof(pb) >= sizeof(float) * kDecWaves * GP * D, "the partials fit the weights' place");
#pragma unroll
  for (int t = 0; t < 2 * NG; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      acc[t][i] = (acc[t][i] + __shfl_xor(acc[t][i], 4 * GP, 64)) * __uint_as_float((uint32_t)(vexp[t / 2] - 5) << 23);
  if (lane < 4 * GP) {
    const int h0 = GP == 4 ? 0 : 4 * (lane >> 4);
#pragma unroll
    for (int t = 0; t < 2 * NG; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) red_o[(wave * GP + h0 + i) * D + 16 * t + (lane & 15)] = acc[t][i];
  }
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
      const float sc = exp2f(red_m[w][h] - Mu);
      lsum += sc * red_l[w][h];
      osum += sc * red_o[(w * GP + h) * D + c];
    }
    const int64_t part = ((int64_t)b * p.Hq + hkv * p.G + h) * p.nch + slot;
    p.ws_o[part * d + c] = osum;
    if (c == 0) { p.ws_m[part] = M; p.ws_l[part] = lsum; }
  }
}

// Merge of the chunks' partials, one workgroup per query head: thread groups of d
// over the chunks, in a fixed order (as sfa_decode_combine_kernel, for any d).
constexpr int kMergeQ4 = 512;
__global__ __launch_bounds__(kMergeQ4) void sfa_decode_q4_combine_kernel(DecParams p, int d, int groups, void* o,
                                                                         int obf16, float* lse) {
  __shared__ float part[kMergeQ4];
  const int bh = blockIdx.x, b = bh / p.Hq;
  const int grp = threadIdx.x / d, dd = threadIdx.x - grp * d, lane = threadIdx.x & 63;
  const int L = seq_len_of(p.seq_len, b, p.Lmax);
  const int nc = decode_plan(L, p.window, p.n_global, p.aim).count;
  const int64_t s0 = (int64_t)bh * p.nch;
  float M = -INFINITY;
  for (int c = lane; c < nc; c += 64) M = fmaxf(M, p.ws_m[s0 + c]);
  M = wave_max(M);
  const float Mu = (M == -INFINITY) ? 0.f : M;
  float lsum = 0.f;
  for (int c = lane; c < nc; c += 64) lsum = fmaf(exp2f(p.ws_m[s0 + c] - Mu), p.ws_l[s0 + c], lsum);
  lsum = wave_sum(lsum);
  float osum = 0.f;
  if (grp < groups)
    for (int c = grp; c < nc; c += groups) osum = fmaf(exp2f(p.ws_m[s0 + c] - Mu), p.ws_o[(s0 + c) * d + dd], osum);
  part[threadIdx.x] = osum;
  __syncthreads();
  if (grp != 0) return;
  for (int g = 1; g < groups; ++g) osum += part[g * d + dd];
  const float out = lsum > 0.f ? osum / lsum : 0.f;
  if (obf16) ((uint16_t*)o)[(int64_t)bh * d + dd] = (uint16_t)f32_to_bf16_rne(out);
  else ((float*)o)[(int64_t)bh * d + dd] = out;
  if (lse && dd == 0) lse[bh] = lsum > 0.f ? (M + __log2f(lsum)) * kLn2 : -INFINITY;
}

template <int D, int GP, int KC8>
void launch_q4_t(const DecParams& p, const DecodeArgs& a, hipStream_t stream) {
  const dim3 grid = p.by_slot ? dim3(a.B * p.Hkv, p.nch) : dim3(p.nch, a.B * p.Hkv), block(kDecThreads);
  if (p.table)
    hipLaunchKernelGGL((sfa_decode_q4_kernel<D, GP, KC8, true>), grid, block, 0, stream, p, a.d, a.v_scale16);
  else
    hipLaunchKernelGGL((sfa_decode_q4_kernel<D, GP, KC8, false>), grid, block, 0, stream, p, a.d, a.v_scale16);
}

template <int D, int GP>
void launch_q4_k(const DecParams& p, const DecodeArgs& a, hipStream_t stream) {
  if (D < 256 && a.k == 16) launch_q4_t<D, GP, 2>(p, a, stream);
  else launch_q4_t<D, GP, 0>(p, a, stream);
}

template <int D>
void launch_q4_g(const DecParams& p, const DecodeArgs& a, hipStream_t stream) {
  if (p.G <= 4) launch_q4_k<D, 4>(p, a, stream);
  else launch_q4_k<D, 8>(p, a, stream);
}

}  // namespace

// For any group and window, as decode_workspace_bytes, at any head dimension.
size_t decode_q4_workspace_bytes(int B, int Hq, int Lmax, int d) {
  const int aim = decode_chunks_aim(B, (Hq + kDecMaxG - 1) / kDecMaxG, true, 1);
  return (size_t)B * Hq * (size_t)decode_most_slots(Lmax, aim) * (size_t)(d + 2) * sizeof(float);
}

hipError_t launch_attn_decode_q4(const DecodeArgs& a, hipStream_t stream) {
  const DecParams p = make_dec_params(a);
  if (a.d == 64) launch_q4_g<64>(p, a, stream);
  else if (a.d == 128) launch_q4_g<128>(p, a, stream);
  else launch_q4_g<256>(p, a, stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(sfa_decode_q4_combine_kernel, dim3(a.B * a.Hq), dim3(kMergeQ4), 0, stream, p, a.d,
                     kMergeQ4 / a.d, a.o, a.obf16, a.lse);
  return hipGetLastError();
}

}  // namespace sfa
