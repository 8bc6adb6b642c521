// Append to the 4-bit cache (sfa_kv_append_q4): Top-k coding of the new keys
// (Sec. 3.1, Eqs. (3)-(4)), quantisation of code values and value rows to signed
// 4-bit numbers, q = round-half-even(x / s) in [-7, 7], and the cache write.
//
// One wavefront per (token, KV head) row.  Lane l holds key coordinates l + 64 e
// for the selection (sfa_topk.h) and value coordinates 2 l + 128 i, 2 l + 1 + 128 i:
// the 32 coordinates of one scale are then one 16-lane row, whose maximum is four
// DPP steps, and a lane's two numbers are a byte.
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

__device__ __forceinline__ float quant4(float x, float s) {
  return s > 0.f ? fminf(fmaxf(rintf(x / s), -7.f), 7.f) : 0.f;
}

__device__ __forceinline__ int64_t clamp_len(int64_t L, int64_t cap) { return L < 0 ? 0 : (L > cap ? cap : L); }

// E: key coordinates per lane (d <= 64 E); KB, VB: bfloat16 keys / values in.
template <int E, bool KB, bool VB>
__global__ __launch_bounds__(256) void sfa_kv_append_q4_kernel(AppendQ4Args a) {
  constexpr int NV = E <= 2 ? 1 : 2;  // value pairs per lane
  __shared__ uint16_t ent_lds[4][256];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint16_t* ent = ent_lds[wave];
  const int64_t cap = a.table ? (int64_t)a.max_pages * a.page_size : a.page_size;
  const int64_t rows = (int64_t)a.B * a.T * a.Hkv;
  const int groups = a.d / 32;
  for (int64_t w = (int64_t)blockIdx.x * 4 + wave; w < rows; w += (int64_t)gridDim.x * 4) {
    const int64_t tok = w / a.Hkv;  // heads of a token side by side: packed buffers are read in order
    const int h = (int)(w - tok * a.Hkv);
    const int64_t b = tok / a.T, t = tok - b * a.T;
    // the cache row (uniform per wave)
    int64_t page, slot;
    if (a.slots) {
      const int64_t s = a.slots[b * a.T + t];
      if (s < 0 || s >= (int64_t)a.num_pages * a.page_size) continue;
      page = s / a.page_size;
      slot = s - page * a.page_size;
    } else {
      const int c = a.n_new ? a.n_new[b] : a.T;
      const int64_t pos = clamp_len(a.seq_len[b], cap) + t;
      if (t >= c || pos >= cap) continue;
      page = b;
      slot = pos;
      if (a.table) {
        page = a.table[b * a.max_pages + pos / a.page_size];
        slot = pos % a.page_size;
        if (page < 0 || page >= a.num_pages) continue;
      }
    }
    const int64_t crow = (page * a.Hkv + h) * a.page_size + slot;
    const int64_t ko = b * a.st[0] + h * a.st[1] + t * a.st[2], vo = b * a.st[3] + h * a.st[4] + t * a.st[5];

    // codes
    uint32_t bits[E], key[E], km = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = lane + 64 * e, cc = min(c, a.d - 1);
      bits[e] = KB ? (uint32_t)((const uint16_t*)a.k_new + ko)[cc] << 16 : ((const uint32_t*)a.k_new + ko)[cc];
      key[e] = topk_key(bits[e], c < a.d);
      km = max(km, key[e]);
    }
    bool sel[E];
    topk_select<E>(key, a.k, sel);
    int sl[E];
    topk_slots<E>(sel, sl);
    // the kept values' largest magnitude is the row's: the largest key, |bits| + 1
    const float ks = __uint_as_float(wave_umax(km) - 1u) / 7.f;
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (sel[e] && sl[e] < a.k)
        ent[sl[e]] = (uint16_t)((lane + 64 * e) | ((int)quant4(__uint_as_float(bits[e]), ks) & 15) << 8);
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int i = lane; i < a.k / 2; i += 64) {
      const uint32_t two = ((const uint32_t*)ent)[i];
      ((uint16_t*)(a.kc_idx + crow * a.k))[i] = (uint16_t)((two & 255u) | ((two >> 8) & 0xff00u));
      (a.kc_val + crow * (a.k / 2))[i] = (uint8_t)(((two >> 8) & 15u) | ((two >> 20) & 0xf0u));
    }
    if (lane == 0) a.kc_scale[crow] = ks;
    const int64_t orow = (b * a.Hkv + h) * a.T + t;
    if (a.k_idx)
      for (int i = lane; i < a.k; i += 64) {
        const int v = ent[i];
        a.k_idx[orow * a.k + i] = (int16_t)(v & 255);
        a.k_val[orow * a.k + i] = (float)((int)((uint32_t)v << 20) >> 28) * ks;
      }
    __builtin_amdgcn_wave_barrier();

    // values
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = 2 * lane + 128 * i;
      const bool in = c < a.d;
      float x0 = 0.f, x1 = 0.f;
      if (in) {
        x0 = VB ? bf16_bits_to_f32(((const uint16_t*)a.v_new + vo)[c]) : ((const float*)a.v_new + vo)[c];
        x1 = VB ? bf16_bits_to_f32(((const uint16_t*)a.v_new + vo)[c + 1]) : ((const float*)a.v_new + vo)[c + 1];
      }
      const uint32_t m = row16_umax(max(__float_as_uint(x0) & 0x7fffffffu, __float_as_uint(x1) & 0x7fffffffu));
      const uint32_t sb = f32_to_bf16_rne(__uint_as_float(m) / 7.f);
      const float s = bf16_bits_to_f32(sb);
      const float q0 = quant4(x0, s), q1 = quant4(x1, s);
      if (in) {
        (a.v_cache + crow * (a.d / 2))[c / 2] = (uint8_t)(((int)q0 & 15) | ((int)q1 & 15) << 4);
        if ((lane & 15) == 0) a.v_scale[crow * groups + c / 32] = (uint16_t)sb;
        if (a.v_out)
          *(uint32_t*)(a.v_out + orow * a.d + c) = f32_to_bf16_rne(q0 * s) | f32_to_bf16_rne(q1 * s) << 16;
      }
    }
  }
}

template <bool KB, bool VB>
void launch_q4_t(const AppendQ4Args& a, dim3 grid, hipStream_t stream) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a); };
  if (a.d <= 64) go(sfa_kv_append_q4_kernel<1, KB, VB>);
  else if (a.d <= 128) go(sfa_kv_append_q4_kernel<2, KB, VB>);
  else go(sfa_kv_append_q4_kernel<4, KB, VB>);
}

}  // namespace

hipError_t launch_kv_append_q4(const AppendQ4Args& a, hipStream_t stream) {
  const int64_t need = ((int64_t)a.B * a.T * a.Hkv + 3) / 4;
  if (need > 0) {
    const dim3 grid((unsigned)(need < 2048 ? need : 2048));
    if (a.kbf16) a.vbf16 ? launch_q4_t<true, true>(a, grid, stream) : launch_q4_t<true, false>(a, grid, stream);
    else a.vbf16 ? launch_q4_t<false, true>(a, grid, stream) : launch_q4_t<false, false>(a, grid, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.slots) return hipSuccess;
  return launch_kv_advance(a.seq_len, a.n_new, a.B, a.T,
                           a.table ? (int64_t)a.max_pages * a.page_size : a.page_size, stream);
}

}  // namespace sfa
