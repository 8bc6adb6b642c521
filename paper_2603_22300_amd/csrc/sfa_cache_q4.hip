// Append to the 4-bit cache (sfa_kv_append_q4): Top-k coding of the new keys
// (Sec. 3.1, Eqs. (3)-(4)), quantisation of code values and value rows to signed
// 4-bit numbers, q = round-half-even(x / s) in [-7, 7], and the cache write.
//
// One wavefront per (token, KV head) row, heads of a token side by side (packed
// buffers are read in order), the next row's words and slot in flight while the
// current one is coded.  Lane l holds key coordinates l + 64 e for the selection
// (sfa_topk.h) and value coordinates 2 l + 128 i, 2 l + 1 + 128 i: the 32
// coordinates of one scale are then one 16-lane row, whose maximum is four DPP
// steps, and a lane's two numbers are a byte.  Bound by the selection, as the other
// appends, so the row walk has no division and a number costs a product with the
// scale's reciprocal: only where that lands next to a half is the correctly rounded
// quotient, which decides, computed.  2 x 8192 tokens x 8 heads at d = 128, k = 16, bf16 in,
// with the codes and values for a forward beside the cache: 63 us (127 MB; 27 at a copy's
// rate), the vector and the scalar unit 73% busy.
#include "sfa_device.h"
#include "sfa_launch.h"
#include "sfa_topk.h"

namespace sfa {
namespace {

// Maximum over each 16-lane row, in every lane of it.
__device__ __forceinline__ uint32_t row16_umax(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xb1, 0xf, 0xf, false));   // quad_perm 1,0,3,2
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4e, 0xf, 0xf, false));   // quad_perm 2,3,0,1
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x141, 0xf, 0xf, false));  // row_half_mirror
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x140, 0xf, 0xf, false));  // row_mirror
}

// N numbers of a row with scale s (uniform or not): round-half-even of the float32
// quotient.  x * rcp(s) is off by less than 4 ulp, 2^-18 for the quotients here (at most
// 7.1), so it rounds as the quotient does unless it lies within 2^-16 of a half h.
// There x - h s, one fma, tells an exact tie (frequent where values and scales are
// both bfloat16), which goes to the even number; only if some quotient is near a half
// and not on it, or the reciprocal leaves the normal range, does the wavefront divide.
template <int N>
__device__ __forceinline__ void quant4(const float (&x)[N], float s, float (&q)[N]) {
  const float r = __builtin_amdgcn_rcpf(s);
  const bool tiny = s < 0x1p-100f;
  float off[N];
  bool near = tiny;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float y = x[i] * r;
    q[i] = rintf(y);
    off[i] = y - q[i];
    near |= fabsf(off[i]) > 0.5f - 0x1p-16f;
  }
  if (wave_ballot(near)) {
    bool unsure = tiny;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float h = q[i] + copysignf(0.5f, off[i]), e = fmaf(-h, s, x[i]);
      const bool at = fabsf(off[i]) > 0.5f - 0x1p-16f;
      q[i] = at ? rintf(h) : q[i];
      unsure |= at && e != 0.f;
    }
    if (wave_ballot(unsure)) {
#pragma unroll
      for (int i = 0; i < N; ++i) q[i] = s > 0.f ? rintf(x[i] / s) : 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) q[i] = fminf(fmaxf(q[i], -7.f), 7.f);
}

// x / 7, correctly rounded: the product with the rounded reciprocal and one fma
// correction of its remainder (Markstein's theorem; checked over all significands),
// the division itself where the remainder could leave the normal range.
__device__ __forceinline__ float seventh(float x) {
  const float r = 1.f / 7.f, q = x * r;
  float y = fmaf(fmaf(-7.f, q, x), r, q);
  constexpr uint32_t lo = (127u - 90) << 23, hi = (127u + 126) << 23;
  if (wave_ballot(__float_as_uint(x) - lo >= hi - lo)) {
    asm volatile("" : "+v"(x));  // (or the division is made of every row, and then not used)
    y = x / 7.f;
  }
  return y;
}

__device__ __forceinline__ int64_t clamp_len(int64_t L, int64_t cap) { return L < 0 ? 0 : (L > cap ? cap : L); }

// E: key coordinates per lane (d <= 64 E); KB, VB: bfloat16 keys / values in; V2: a
// lane's two values start on a boundary of two, and are one load.
template <int E, bool KB, bool VB, bool V2>
__global__ __launch_bounds__(256) void sfa_kv_append_q4_kernel(AppendQ4Args a) {
  constexpr int NV = E <= 2 ? 1 : 2;  // value pairs per lane
  __shared__ uint16_t ent_lds[4][256];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint16_t* ent = ent_lds[wave];
  const int64_t cap = a.table ? (int64_t)a.max_pages * a.page_size : a.page_size;

  // (b, t, h) of the wave's row, stepped by the grid's wavefronts
  const int64_t w = (int64_t)blockIdx.x * 4 + wave;
  if (w >= (int64_t)a.B * a.T * a.Hkv) return;  // uniform per wave
  int h = (int)(w % a.Hkv);
  int t = (int)(w / a.Hkv % a.T);
  int b = (int)(w / a.Hkv / a.T);

  uint32_t nk[E], nv[NV][2];  // as loaded: what would widen them here would wait for them
  // The row's place: its slot, or its position and page, as they are loaded (nothing
  // waits for them before the row's turn).
  int nplace = 0;
  int64_t npos = 0, norow, len = 0;
  int count = a.T, len_of = -1;  // of sequence len_of
  int64_t ko = b * a.st[0] + h * a.st[1] + t * a.st[2], vo = b * a.st[3] + h * a.st[4] + t * a.st[5];
  int64_t tok = (int64_t)b * a.T + t, out_row = ((int64_t)b * a.Hkv + h) * a.T + t;
  auto load_row = [&]() {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = min(lane + 64 * e, a.d - 1);
      nk[e] = KB ? (uint32_t)((const uint16_t*)a.k_new + ko)[c] : ((const uint32_t*)a.k_new + ko)[c];
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = min(2 * lane + 128 * i, a.d - 2);
      if constexpr (VB && V2) {
        nv[i][0] = *(const uint32_t*)((const uint16_t*)a.v_new + vo + c);
      } else if constexpr (VB) {
        nv[i][0] = ((const uint16_t*)a.v_new + vo)[c];
        nv[i][1] = ((const uint16_t*)a.v_new + vo)[c + 1];
      } else if constexpr (V2) {
        const uint2 two = *(const uint2*)((const uint32_t*)a.v_new + vo + c);
        nv[i][0] = two.x;
        nv[i][1] = two.y;
      } else {
        nv[i][0] = ((const uint32_t*)a.v_new + vo)[c];
        nv[i][1] = ((const uint32_t*)a.v_new + vo)[c + 1];
      }
    }
    if (a.slots) {
      nplace = a.slots[tok];
    } else {
      if (b != len_of) {
        len_of = b;
        len = clamp_len(a.seq_len[b], cap);
        if (a.n_new) count = a.n_new[b];
      }
      npos = t < count ? len + t : cap;
      nplace = a.table ? (npos < cap ? a.table[(int64_t)b * a.max_pages + (npos >> a.log2P)] : -1) : b;
    }
    norow = out_row;
  };
  load_row();
  while (true) {
    int page, slot;
    const int place = __builtin_amdgcn_readfirstlane(nplace);
    bool kept;
    if (a.slots) {
      kept = place >= 0 && place < a.num_pages * a.page_size;  // (below 2^31)
      page = a.log2P >= 0 ? place >> a.log2P : (uint32_t)place / (uint32_t)a.page_size;
      slot = place - page * a.page_size;
    } else {
      kept = npos < cap && place >= 0 && place < a.num_pages;
      page = place;
      slot = (int)(a.table ? npos & (a.page_size - 1) : npos);
    }
    // (num_pages * Hkv < 2^31)
    const int64_t crow = (int64_t)(page * a.Hkv + h) * a.page_size + slot, orow = norow;
    // (the other arrays' offsets are shifts of these two)
    const int64_t ck = crow * a.k, cv = crow * (a.d / 2);
    uint32_t bits[E], key[E], km = 0;
    float x[NV][2];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      bits[e] = KB ? nk[e] << 16 : nk[e];
      key[e] = topk_key(bits[e], lane + 64 * e < a.d);
      km = max(km, key[e]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const bool in = 2 * lane + 128 * i < a.d;
      const uint32_t v0 = VB ? nv[i][0] << 16 : nv[i][0];
      const uint32_t v1 = VB && V2 ? nv[i][0] & 0xffff0000u : VB ? nv[i][1] << 16 : nv[i][1];
      x[i][0] = in ? __uint_as_float(v0) : 0.f;
      x[i][1] = in ? __uint_as_float(v1) : 0.f;
    }
    h += a.step_h;
    t += a.step_t;
    b += a.step_b;
    ko += a.step_k;
    vo += a.step_v;
    tok += a.step_tok;
    out_row += a.step_out;
    if (h >= a.Hkv) {  // on to the next token
      h -= a.Hkv;
      ++t;
      ko += a.carry_k;
      vo += a.carry_v;
      ++tok;
      out_row += 1 - (int64_t)a.Hkv * a.T;
    }
    if (t >= a.T) {  // on to the next sequence
      t -= a.T;
      ++b;
      ko += a.wrap_k;
      vo += a.wrap_v;
      out_row += (int64_t)(a.Hkv - 1) * a.T;
    }
    const bool more = b < a.B;
    if (more) load_row();
    if (kept) {  // uniform per wave
      const uint32_t cut = topk_cut<E>(key, a.k);
      bool sel[E];
#pragma unroll
      for (int e = 0; e < E; ++e) sel[e] = key[e] >= cut;
      int sl[E];
      topk_slots<E>(sel, sl);
      // (the next row's words and place are waited for before the stores, as in
      // sfa_rope_encode_kernel)
#pragma unroll
      for (int e = 0; e < E; ++e) asm volatile("" : "+v"(nk[e]));
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        asm volatile("" : "+v"(nv[i][0]));
        if constexpr (!(VB && V2)) asm volatile("" : "+v"(nv[i][1]));
      }
      asm volatile("" : "+v"(nplace));
      // the kept values' largest magnitude is the row's: the largest key, |bits| + 1
      const float ks = seventh(__uint_as_float(wave_umax(km) - 1u));
      float kx[E], q[E];
#pragma unroll
      for (int e = 0; e < E; ++e) kx[e] = sel[e] ? __uint_as_float(bits[e]) : 0.f;
      quant4<E>(kx, ks, q);
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (sel[e] && sl[e] < a.k) ent[sl[e]] = (uint16_t)((lane + 64 * e) | ((int)q[e] & 15) << 8);
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int j = 0; j < NV; ++j) {  // (k <= d: at most 64 NV pairs)
        const int i = lane + 64 * j;
        if (i >= a.k / 2) break;
        const uint32_t two = ((const uint32_t*)ent)[i];
        ((uint16_t*)(a.kc_idx + ck))[i] = (uint16_t)((two & 255u) | ((two >> 8) & 0xff00u));
        (a.kc_val + (ck >> 1))[i] = (uint8_t)(((two >> 8) & 15u) | ((two >> 20) & 0xf0u));
      }
      if (lane == 0) a.kc_scale[crow] = ks;
      if (a.k_idx)
#pragma unroll
        for (int j = 0; j < E; ++j) {
          const int i = lane + 64 * j;
          if (i >= a.k) break;
          const int v = ent[i];
          a.k_idx[orow * a.k + i] = (int16_t)(v & 255);
          a.k_val[orow * a.k + i] = (float)((int)((uint32_t)v << 20) >> 28) * ks;
        }
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = 2 * lane + 128 * i;
        const uint32_t m = row16_umax(max(__float_as_uint(x[i][0]) & 0x7fffffffu, __float_as_uint(x[i][1]) & 0x7fffffffu));
        const uint32_t sb = f32_to_bf16_rne(seventh(__uint_as_float(m)));
        const float s = bf16_bits_to_f32(sb);
        float vq[2];
        quant4<2>(x[i], s, vq);
        if (c < a.d) {
          (a.v_cache + cv)[c / 2] = (uint8_t)(((int)vq[0] & 15) | ((int)vq[1] & 15) << 4);
          if ((lane & 15) == 0) a.v_scale[(cv >> 4) + c / 32] = (uint16_t)sb;
          if (a.v_out)
            *(uint32_t*)(a.v_out + orow * a.d + c) = f32_to_bf16_rne(vq[0] * s) | f32_to_bf16_rne(vq[1] * s) << 16;
        }
      }
    }
    if (!more) break;
  }
}

template <int E, bool KB, bool VB>
void launch_q4_v(const AppendQ4Args& a, bool v2, dim3 grid, hipStream_t stream) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a); };
  if (v2) go(sfa_kv_append_q4_kernel<E, KB, VB, true>);
  else go(sfa_kv_append_q4_kernel<E, KB, VB, false>);
}

template <bool KB, bool VB>
void launch_q4_t(const AppendQ4Args& a, bool v2, dim3 grid, hipStream_t stream) {
  if (a.d <= 64) launch_q4_v<1, KB, VB>(a, v2, grid, stream);
  else if (a.d <= 128) launch_q4_v<2, KB, VB>(a, v2, grid, stream);
  else launch_q4_v<4, KB, VB>(a, v2, grid, stream);
}

}  // namespace

hipError_t launch_kv_append_q4(AppendQ4Args a, hipStream_t stream) {
  const int64_t rows = (int64_t)a.B * a.T * a.Hkv, need = (rows + 3) / 4;
  if (need > 0) {
    // eight rows a wavefront where they fill the chip eight times over, the rest left to
    // the dispatcher (see launch_rope_encode)
    const int64_t filled = need < 2048 ? need : 2048, most = (need + 7) / 8 > filled ? (need + 7) / 8 : filled;
    const int64_t blocks = most < 1 << 22 ? most : 1 << 22;  // (a grid dimension: less than 2^32 threads)
    const dim3 grid((unsigned)blocks);
    a.log2P = -1;
    if ((a.page_size & (a.page_size - 1)) == 0)
      for (a.log2P = 0; (1 << a.log2P) < a.page_size;) ++a.log2P;
    // the step of a wavefront's walk, in heads, tokens and sequences
    int64_t step = 4 * blocks;
    a.step_h = (int)(step % a.Hkv);
    step /= a.Hkv;
    a.step_t = (int)(step % a.T);
    a.step_b = (int)(step / a.T);
    // offsets of that step, and what a carry from heads to tokens, tokens to sequences adds
    a.step_k = a.step_b * a.st[0] + a.step_h * a.st[1] + a.step_t * a.st[2];
    a.step_v = a.step_b * a.st[3] + a.step_h * a.st[4] + a.step_t * a.st[5];
    a.carry_k = a.st[2] - a.Hkv * a.st[1];
    a.carry_v = a.st[5] - a.Hkv * a.st[4];
    a.wrap_k = a.st[0] - a.T * a.st[2];
    a.wrap_v = a.st[3] - a.T * a.st[5];
    a.step_tok = (int64_t)a.step_b * a.T + a.step_t;
    a.step_out = ((int64_t)a.step_b * a.Hkv + a.step_h) * a.T + a.step_t;
    const bool v2 = ((a.st[3] | a.st[4] | a.st[5]) & 1) == 0 && (uintptr_t)a.v_new % (a.vbf16 ? 4 : 8) == 0;
    if (a.kbf16) a.vbf16 ? launch_q4_t<true, true>(a, v2, grid, stream) : launch_q4_t<true, false>(a, v2, grid, stream);
    else a.vbf16 ? launch_q4_t<false, true>(a, v2, grid, stream) : launch_q4_t<false, false>(a, v2, grid, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.slots) return hipSuccess;
  return launch_kv_advance(a.seq_len, a.n_new, a.B, a.T,
                           a.table ? (int64_t)a.max_pages * a.page_size : a.page_size, stream);
}

}  // namespace sfa
