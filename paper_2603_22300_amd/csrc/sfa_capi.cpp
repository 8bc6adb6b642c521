// C ABI of libsfa: argument validation, dtype dispatch, launch, error codes.
// Every check runs on the host before anything is enqueued.
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/sfa.h"
#include "sfa_device.h"
#include "sfa_launch.h"

namespace {

constexpr int kAbiVersion = 4;
constexpr int kMaxLds = 160 * 1024;  // LDS per workgroup on gfx950

// index arrays of codes; values of codes; V and O
bool is_idx(int t) { return t == SFA_I32 || t == SFA_I16 || t == SFA_U8; }
bool is_cval(int t) { return t == SFA_F32 || t == SFA_BF16 || t == SFA_F16; }
bool is_val(int t) { return t == SFA_F32 || t == SFA_BF16; }
// kernel-side format codes (sfa_device.h)
int ifmt_of(int t) { return t == SFA_I16 ? sfa::kIdxI16 : (t == SFA_U8 ? sfa::kIdxU8 : sfa::kIdxI32); }
int vfmt_of(int t) { return t == SFA_BF16 ? sfa::kValBF16 : (t == SFA_F16 ? sfa::kValF16 : sfa::kValF32); }
bool pow2_le(int g, int maxg) { return g >= 1 && g <= maxg && (g & (g - 1)) == 0; }

// Strides of [B, H, n, d] rows, coordinates contiguous: the caller's, or those of a
// contiguous array.
void row_strides(const int64_t* given, int64_t H, int64_t n, int64_t d, int64_t (&st)[3]) {
  st[0] = given ? given[0] : H * n * d;
  st[1] = given ? given[1] : n * d;
  st[2] = given ? given[2] : d;
}
bool strides_readable(const int64_t (&st)[3]) { return st[0] >= 0 && st[1] >= 0 && st[2] >= 0; }
// rows of a written array do not share elements (a dimension of one entry has no step)
bool strides_writable(const int64_t (&st)[3], int B, int H, int n, int d) {
  return strides_readable(st) && (B == 1 || st[0] >= d) && (H == 1 || st[1] >= d) && (n <= 1 || st[2] >= d);
}

// Checks and copies shared by the rotary entry points (n > 0).
bool rope_common(const sfa_rope_plan* plan, const int32_t* pos, int64_t pos_axis, int64_t pos_batch,
                 int B, int H, int n, int inverse, sfa::RopePlan& pl, sfa::RopeArgs& a) {
  if (!plan || B < 1 || H < 1 || n < 0 || pos_axis < 0 || pos_batch < 0) return false;
  if (plan->d < 2 || plan->d > 256 || plan->rot < 2 || plan->rot > plan->d || plan->rot % 2 != 0 ||
      plan->naxes < 1 || plan->naxes > SFA_ROPE_MAX_AXES || plan->pairing < 0 || plan->pairing > 1)
    return false;
  if ((long long)B * n > 0x7fffffffLL) return false;
  if (n > 0 && !pos) return false;
  pl.d = plan->d; pl.rot = plan->rot; pl.neighbours = plan->pairing; pl.inverse = inverse != 0;
  for (int i = 0; i < SFA_ROPE_MAX_PAIRS; ++i) {
    const bool used = i < plan->rot / 2;
    if (used && plan->axis[i] >= plan->naxes) return false;
    pl.freq[i] = used ? plan->freq[i] : 0.0;
    pl.axis[i] = used ? plan->axis[i] : 0;
  }
  a.pos = pos; a.pos_axis = pos_axis; a.pos_batch = pos_batch;
  a.B = B; a.H = H; a.n = n; a.d = plan->d;
  return true;
}

sfa_status from_hip(hipError_t e) { return e == hipSuccess ? SFA_OK : SFA_EHIP; }

}  // namespace

extern "C" {

int sfa_abi_version(void) { return kAbiVersion; }

const char* sfa_strerror(int status) {
  switch (status) {
    case SFA_OK: return "ok";
    case SFA_EINVAL: return "invalid argument";
    case SFA_ENOTSUP: return "unsupported shape or dtype";
    case SFA_EHIP: return "HIP runtime error";
    case SFA_ENOSPC: return "workspace too small";
    default: return "unknown status";
  }
}

sfa_status sfa_topk_encode(const float* x, int64_t rows, int d, int k, void* idx, int idx_t,
                           void* val, int val_t, void* stream) {
  if (rows < 0 || d < 1 || k < 1 || k > d) return SFA_EINVAL;
  if (!is_idx(idx_t) || !is_cval(val_t)) return SFA_EINVAL;
  if (d > 256) return SFA_ENOTSUP;
  if (rows == 0) return SFA_OK;
  if (!x || !idx || !val) return SFA_EINVAL;
  if ((rows + 3) / 4 > 0x7fffffffLL) return SFA_ENOTSUP;
  return from_hip(sfa::launch_topk_encode(x, rows, d, k, idx, ifmt_of(idx_t), val,
                                          vfmt_of(val_t), (hipStream_t)stream));
}

namespace {

sfa_status check_fwd(const void* q_idx, const void* q_val, const void* k_idx, const void* k_val,
                     const void* v, int B, int Hq, int Hkv, int n, int d, int k, float scale,
                     int idx_t, int qk_val_t, int v_t, int o_t, const void* o) {
  if (!q_idx || !q_val || !k_idx || !k_val || !v || !o) return SFA_EINVAL;
  if (B < 1 || Hq < 1 || Hkv < 1 || n < 1 || d < 1 || k < 1 || k > d) return SFA_EINVAL;
  if (Hq % Hkv != 0) return SFA_EINVAL;
  if (!is_idx(idx_t) || !is_cval(qk_val_t) || !is_val(v_t) || !is_val(o_t)) return SFA_EINVAL;
  if (!isfinite(scale)) return SFA_EINVAL;
  if (d > 256) return SFA_ENOTSUP;  // callers with matrix-core kernels only also require 64 or 128
  if ((long long)B * Hkv > 65535) return SFA_ENOTSUP;
  // per-head code and value offsets are 32-bit byte offsets in the kernels
  if ((long long)n * d > (1LL << 29) || (long long)n * k > (1LL << 29)) return SFA_ENOTSUP;
  return SFA_OK;
}

}  // namespace

size_t sfa_attn_fwd_workspace(int B, int Hkv, int n, int d, int v_t) {
  if (B < 1 || Hkv < 1 || n < 1 || (d != 64 && d != 128) || !is_val(v_t)) return 0;
  return sfa::fwd_workspace_bytes(B, Hkv, n, d, v_t == SFA_BF16);
}

sfa_status sfa_attn_fwd(const void* q_idx, const void* q_val, const void* k_idx,
                        const void* k_val, const void* v, int B, int Hq, int Hkv, int n, int d,
                        int k, int causal, int window, int n_global, float scale, int idx_t,
                        int qk_val_t, int v_t, int o_t, void* o, float* lse, void* ws,
                        size_t ws_bytes, void* stream) {
  sfa_status st = check_fwd(q_idx, q_val, k_idx, k_val, v, B, Hq, Hkv, n, d, k, scale, idx_t,
                            qk_val_t, v_t, o_t, o);
  if (st != SFA_OK) return st;
  if (window < 0 || n_global < 0) return SFA_EINVAL;
  if ((d != 64 && d != 128) || !pow2_le(Hq / Hkv, sfa::fwd_max_group())) {
    // head dimensions or group sizes without the tuned kernel: the forward of
    // float32 accuracy (any group size, no workspace)
    if (!sfa::fwd_generic_supported(d, k) || (long long)B * Hq > 65535) return SFA_ENOTSUP;
    return from_hip(sfa::launch_attn_fwd_generic(q_idx, q_val, k_idx, k_val, v, B, Hq, Hkv, n, d,
                                                 k, causal != 0, window,
                                                 window > 0 ? n_global : 0, scale,
                                                 ifmt_of(idx_t), vfmt_of(qk_val_t),
                                                 v_t == SFA_BF16, o_t == SFA_BF16, o, lse,
                                                 (hipStream_t)stream));
  }
  const size_t need = sfa::fwd_workspace_bytes(B, Hkv, n, d, v_t == SFA_BF16);
  if (need > 0 && (ws == nullptr || ws_bytes < need)) return SFA_ENOSPC;
  return from_hip(sfa::launch_attn_fwd(q_idx, q_val, k_idx, k_val, v, B, Hq, Hkv, n, d, k,
                                       causal != 0, window, window > 0 ? n_global : 0, scale,
                                       ifmt_of(idx_t),
                                       vfmt_of(qk_val_t), v_t == SFA_BF16, o_t == SFA_BF16,
                                       o, lse, ws, (hipStream_t)stream));
}

size_t sfa_attn_bwd_workspace(int B, int Hq, int Hkv, int n, int d) {
  if (B < 1 || Hq < 1 || Hkv < 1 || n < 1 || (d != 64 && d != 128)) return 0;
  return sfa::bwd_workspace_bytes(B, Hq, Hkv, n, d);
}

sfa_status sfa_attn_bwd(const void* q_idx, const void* q_val, const void* k_idx,
                        const void* k_val, const void* v, const void* o, const float* lse,
                        const void* dout, int B, int Hq, int Hkv, int n, int d, int k, int causal,
                        int window, int n_global, float scale, int idx_t, int qk_val_t, int v_t,
                        int o_t, float* dq_val,
                        float* dk_val, float* dv, void* ws, size_t ws_bytes, void* stream) {
  sfa_status st = check_fwd(q_idx, q_val, k_idx, k_val, v, B, Hq, Hkv, n, d, k, scale, idx_t,
                            qk_val_t, v_t, o_t, o);
  if (st != SFA_OK) return st;
  if (!lse || !dout || !dq_val || !dk_val || !dv) return SFA_EINVAL;
  if (window < 0 || n_global < 0) return SFA_EINVAL;
  if ((d != 64 && d != 128) || !pow2_le(Hq / Hkv, sfa::bwd_max_group())) {
    // head dimensions or group sizes without the matrix-core kernels: the
    // float32 backward (any group size, no workspace)
    if (!sfa::bwd_generic_supported(d, k) || (long long)B * Hq > 65535) return SFA_ENOTSUP;
    return from_hip(sfa::launch_attn_bwd_generic(
        q_idx, q_val, k_idx, k_val, v, o, lse, dout, B, Hq, Hkv, n, d, k, causal != 0, window,
        window > 0 ? n_global : 0, scale, ifmt_of(idx_t), vfmt_of(qk_val_t), v_t == SFA_BF16,
        o_t == SFA_BF16, dq_val, dk_val, dv, (hipStream_t)stream));
  }
  if (ws == nullptr || ws_bytes < sfa::bwd_workspace_bytes(B, Hq, Hkv, n, d)) return SFA_ENOSPC;
  return from_hip(sfa::launch_attn_bwd(q_idx, q_val, k_idx, k_val, v, o, lse, dout, B, Hq, Hkv, n,
                                       d, k, causal != 0, window, window > 0 ? n_global : 0,
                                       scale, ifmt_of(idx_t),
                                       vfmt_of(qk_val_t), v_t == SFA_BF16, o_t == SFA_BF16,
                                       dq_val, dk_val, dv, ws, (hipStream_t)stream));
}

sfa_status sfa_attn_fwd_index(const void* q_idx, const void* q_val, const void* k_idx,
                              const void* k_val, const void* v, int B, int Hq, int Hkv, int n,
                              int d, int k, int causal, float scale, int idx_t, int qk_val_t,
                              int v_t, int o_t, void* o, float* lse, void* stream) {
  sfa_status st = check_fwd(q_idx, q_val, k_idx, k_val, v, B, Hq, Hkv, n, d, k, scale, idx_t,
                            qk_val_t, v_t, o_t, o);
  if (st != SFA_OK) return st;
  if (d != 64 && d != 128) return SFA_ENOTSUP;
  if (!pow2_le(Hq / Hkv, sfa::fwd_index_rows_per_block())) return SFA_ENOTSUP;
  if (k > sfa::fwd_index_max_k()) return SFA_ENOTSUP;
  if (sfa::fwd_index_lds_bytes(d, k, v_t == SFA_BF16) > kMaxLds) return SFA_ENOTSUP;
  return from_hip(sfa::launch_attn_fwd_index(q_idx, q_val, k_idx, k_val, v, B, Hq, Hkv, n, d, k,
                                             causal != 0, scale, ifmt_of(idx_t),
                                             vfmt_of(qk_val_t), v_t == SFA_BF16,
                                             o_t == SFA_BF16, o, lse, (hipStream_t)stream));
}

size_t sfa_attn_decode_workspace(int B, int Hq, int Lmax, int d) {
  if (B < 1 || Hq < 1 || Lmax < 1 || d < 1) return 0;
  return sfa::decode_workspace_bytes(B, Hq, Lmax, d);
}

}  // extern "C"

namespace {

// Steps of the float32 decode: head dims without the tuned kernel, and caches
// that are not 16-byte aligned under a group that is not a power of two (other
// groups ask for the alignment).  Such an aligned group runs the tuned kernel
// of the next power of two, its spare heads idle: the same float32 arithmetic,
// with lanes over keys and 16-byte loads (16 sequences of 8000 keys, 12 query
// over 2 KV heads, d = 128: 2420 -> 27 us).
bool decode_generic(int d, int G, const void* v_cache, const void* kc_idx, const void* kc_val) {
  const bool aligned = ((uintptr_t)v_cache | (uintptr_t)kc_idx | (uintptr_t)kc_val) % 16 == 0;
  return (d != 64 && d != 128) || (!pow2_le(G, sfa::decode_max_group()) && !aligned);
}

// Contiguous-cache decode behind sfa_attn_decode and sfa_attn_decode_noalloc.
// ws == nullptr selects the library's static device scratch (after every
// argument check, and only if the partials fit it).
sfa_status decode_contiguous(const void* q_idx, const void* q_val, const void* kc_idx,
                             const void* kc_val, const void* v_cache, const int32_t* seq_len,
                             int B, int Hq, int Hkv, int Lmax, int d, int k, float scale,
                             int window, int n_global, int q_idx_t, int q_val_t, int kc_idx_t,
                             int kc_val_t, int v_t, int o_t, void* o, float* lse, void* ws,
                             size_t ws_bytes, bool use_scratch, void* stream) {
  if (!q_idx || !q_val || !kc_idx || !kc_val || !v_cache || !o) return SFA_EINVAL;
  if (!use_scratch && !ws) return SFA_EINVAL;
  if (B < 1 || Hq < 1 || Hkv < 1 || Lmax < 1 || d < 1 || k < 1 || k > d) return SFA_EINVAL;
  if (window < 0 || n_global < 0) return SFA_EINVAL;
  if (Lmax > (1 << 30)) return SFA_ENOTSUP;
  if (Hq % Hkv != 0) return SFA_EINVAL;
  if (!is_idx(q_idx_t) || !is_cval(q_val_t) || !is_idx(kc_idx_t) || !is_cval(kc_val_t) ||
      !is_val(v_t) || !is_val(o_t))
    return SFA_EINVAL;
  if (!isfinite(scale)) return SFA_EINVAL;
  if ((long long)B * Hkv > 65535) return SFA_ENOTSUP;
  if (d > 256 || Hq / Hkv > sfa::decode_max_group()) return SFA_ENOTSUP;
  const bool generic = decode_generic(d, Hq / Hkv, v_cache, kc_idx, kc_val);
  if (!generic && ((uintptr_t)v_cache | (uintptr_t)kc_idx | (uintptr_t)kc_val) % 16 != 0)
    return SFA_EINVAL;
  if (use_scratch) ws_bytes = sfa::noalloc_scratch_bytes();
  // (a workspace below sfa_attn_decode_workspace that holds chunks of
  // kDecodeChunk keys is taken, with those)
  if (ws_bytes < sfa::decode_workspace_bytes_min(B, Hq, Lmax, d)) return SFA_ENOSPC;
  if (use_scratch && sfa::noalloc_scratch(&ws) != hipSuccess) return SFA_EHIP;
  sfa::DecodeArgs a = {};
  a.q_idx = q_idx; a.q_val = q_val; a.kc_idx = kc_idx; a.kc_val = kc_val; a.v = v_cache;
  a.seq_len = seq_len;
  a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.Lmax = Lmax; a.d = d; a.k = k; a.scale = scale;
  a.window = window; a.n_global = window > 0 ? n_global : 0;
  a.qifmt = ifmt_of(q_idx_t); a.qvfmt = vfmt_of(q_val_t);
  a.kifmt = ifmt_of(kc_idx_t); a.kvfmt = vfmt_of(kc_val_t);
  a.vbf16 = v_t == SFA_BF16; a.obf16 = o_t == SFA_BF16;
  a.o = o; a.lse = lse; a.ws = ws;
  a.aim = sfa::decode_aim(B, Hq, Hkv, Lmax, d, window, ws_bytes, false);
  return from_hip(generic ? sfa::launch_attn_decode_generic(a, (hipStream_t)stream)
                          : sfa::launch_attn_decode(a, (hipStream_t)stream));
}

}  // namespace

extern "C" {

sfa_status sfa_attn_decode(const void* q_idx, const void* q_val, const void* kc_idx,
                           const void* kc_val, const void* v_cache, const int32_t* seq_len,
                           int B, int Hq, int Hkv, int Lmax, int d, int k, float scale,
                           int window, int n_global,
                           int q_idx_t, int q_val_t, int kc_idx_t, int kc_val_t, int v_t,
                           int o_t, void* o, float* lse, void* ws, size_t ws_bytes,
                           void* stream) {
  return decode_contiguous(q_idx, q_val, kc_idx, kc_val, v_cache, seq_len, B, Hq, Hkv, Lmax, d,
                           k, scale, window, n_global, q_idx_t, q_val_t, kc_idx_t, kc_val_t, v_t,
                           o_t, o, lse, ws, ws_bytes, false, stream);
}

sfa_status sfa_attn_decode_noalloc(const void* q_idx, const void* q_val, const void* kc_idx,
                                   const void* kc_val, const void* v_cache,
                                   const int32_t* seq_len, int B, int Hq, int Hkv, int Lmax,
                                   int d, int k, float scale, int window, int n_global,
                                   int q_idx_t, int q_val_t, int kc_idx_t, int kc_val_t, int v_t,
                                   int o_t, void* o, float* lse, void* stream) {
  return decode_contiguous(q_idx, q_val, kc_idx, kc_val, v_cache, seq_len, B, Hq, Hkv, Lmax, d,
                           k, scale, window, n_global, q_idx_t, q_val_t, kc_idx_t, kc_val_t, v_t,
                           o_t, o, lse, nullptr, 0, true, stream);
}

sfa_status sfa_attn_decode_paged(const float* q, const void* q_idx, const void* q_val,
                                 const void* kc_idx, const void* kc_val, const void* v_cache,
                                 const int32_t* block_table, int max_pages, int page_size,
                                 int num_pages, const int32_t* seq_len, int B, int Hq, int Hkv,
                                 int d, int k, float scale, int window, int n_global,
                                 int q_idx_t, int q_val_t,
                                 int kc_idx_t, int kc_val_t, int v_t, int o_t, void* o,
                                 float* lse, void* ws, size_t ws_bytes, void* stream) {
  const bool dense_q = q != nullptr;
  if (dense_q ? (q_idx || q_val) : (!q_idx || !q_val)) return SFA_EINVAL;
  if (!kc_idx || !kc_val || !v_cache || !block_table || !o || !ws) return SFA_EINVAL;
  if (B < 1 || Hq < 1 || Hkv < 1 || d < 1 || k < 1 || k > d) return SFA_EINVAL;
  if (max_pages < 1 || num_pages < 1) return SFA_EINVAL;
  if (window < 0 || n_global < 0) return SFA_EINVAL;
  if (page_size < 16 || (page_size & (page_size - 1)) != 0) return SFA_EINVAL;
  if ((long long)max_pages * page_size > (1LL << 30)) return SFA_EINVAL;
  if (Hq % Hkv != 0) return SFA_EINVAL;
  if ((!dense_q && (!is_idx(q_idx_t) || !is_cval(q_val_t))) || !is_idx(kc_idx_t) ||
      !is_cval(kc_val_t) || !is_val(v_t) || !is_val(o_t))
    return SFA_EINVAL;
  if (!isfinite(scale)) return SFA_EINVAL;
  if ((long long)B * Hkv > 65535) return SFA_ENOTSUP;
  if (d > 256 || Hq / Hkv > sfa::decode_max_group()) return SFA_ENOTSUP;
  const bool generic = decode_generic(d, Hq / Hkv, v_cache, kc_idx, kc_val);
  const int Lmax = max_pages * page_size;
  if (!generic && ((uintptr_t)v_cache | (uintptr_t)kc_idx | (uintptr_t)kc_val) % 16 != 0)
    return SFA_EINVAL;
  if (ws_bytes < sfa::decode_workspace_bytes_min(B, Hq, Lmax, d)) return SFA_ENOSPC;
  int log2P = 0;
  while ((1 << log2P) < page_size) ++log2P;
  sfa::DecodeArgs a = {};
  a.q_dense = q; a.q_idx = q_idx; a.q_val = q_val;
  a.kc_idx = kc_idx; a.kc_val = kc_val; a.v = v_cache;
  a.seq_len = seq_len; a.table = block_table;
  a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.Lmax = Lmax; a.d = d; a.k = k; a.scale = scale;
  a.max_pages = max_pages; a.log2P = log2P; a.num_pages = num_pages;
  a.window = window; a.n_global = window > 0 ? n_global : 0;
  a.qifmt = dense_q ? 0 : ifmt_of(q_idx_t); a.qvfmt = dense_q ? 0 : vfmt_of(q_val_t);
  a.kifmt = ifmt_of(kc_idx_t); a.kvfmt = vfmt_of(kc_val_t);
  a.vbf16 = v_t == SFA_BF16; a.obf16 = o_t == SFA_BF16;
  a.o = o; a.lse = lse; a.ws = ws;
  a.aim = sfa::decode_aim(B, Hq, Hkv, Lmax, d, window, ws_bytes, false);
  return from_hip(generic ? sfa::launch_attn_decode_generic(a, (hipStream_t)stream)
                          : sfa::launch_attn_decode(a, (hipStream_t)stream));
}

sfa_status sfa_kv_append(const float* k_new, const void* v_new, const int32_t* n_new,
                         int32_t* seq_len, int B, int Hkv, int T, int d, int k,
                         const int32_t* block_table, int max_pages, int page_size,
                         int num_pages, void* kc_idx, void* kc_val, void* v_cache,
                         int kc_idx_t, int kc_val_t, int v_new_t, int v_t, void* stream) {
  if (!seq_len || !kc_idx || !kc_val || !v_cache) return SFA_EINVAL;
  if (B < 1 || Hkv < 1 || T < 0 || d < 1 || k < 1 || k > d || page_size < 1) return SFA_EINVAL;
  if (T > 0 && (!k_new || !v_new)) return SFA_EINVAL;
  if (block_table && (max_pages < 1 || num_pages < 1)) return SFA_EINVAL;
  if (block_table && (long long)max_pages * page_size > (1LL << 30)) return SFA_EINVAL;
  if (block_table && (page_size & (page_size - 1)) != 0) return SFA_EINVAL;
  if (!is_idx(kc_idx_t) || !is_cval(kc_val_t) || !is_val(v_new_t) || !is_val(v_t))
    return SFA_EINVAL;
  if (kc_idx_t == SFA_I16 && d > 32767) return SFA_EINVAL;
  if (d > 256) return SFA_ENOTSUP;
  if ((long long)B * Hkv * T > (1LL << 31)) return SFA_ENOTSUP;
  sfa::AppendArgs a = {};
  a.k_new = k_new; a.v_new = v_new; a.n_new = n_new; a.seq_len = seq_len;
  a.table = block_table; a.kc_idx = kc_idx; a.kc_val = kc_val; a.v_cache = v_cache;
  a.B = B; a.Hkv = Hkv; a.T = T; a.d = d; a.k = k;
  a.page_size = page_size; a.max_pages = max_pages; a.num_pages = num_pages;
  while ((1 << a.log2P) < page_size) ++a.log2P;
  a.ifmt = ifmt_of(kc_idx_t); a.vfmt = vfmt_of(kc_val_t);
  a.vin_bf16 = v_new_t == SFA_BF16; a.vc_bf16 = v_t == SFA_BF16;
  return from_hip(sfa::launch_kv_append(a, (hipStream_t)stream));
}

sfa_status sfa_csr_to_codes(const int32_t* indptr, const void* indices, int indices_t,
                            const void* values, int values_t, int64_t rows, int d, int kmax,
                            void* idx, int idx_t, void* val, void* stream) {
  if (rows < 0 || d < 1 || kmax < 1 || kmax > d) return SFA_EINVAL;
  if (!is_idx(indices_t) || !is_idx(idx_t) || !is_cval(values_t)) return SFA_EINVAL;
  if (d > 256) return SFA_ENOTSUP;
  if (rows == 0) return SFA_OK;
  if (!indptr || !indices || !values || !idx || !val) return SFA_EINVAL;
  if ((rows + 3) / 4 > 0x7fffffffLL) return SFA_ENOTSUP;
  sfa::CsrArgs a = {};
  a.indptr = indptr; a.indices = indices; a.values = values; a.rows = rows; a.d = d;
  a.kmax = kmax; a.ifmt_in = ifmt_of(indices_t); a.vbytes = values_t == SFA_F32 ? 4 : 2;
  a.idx_out = idx; a.ifmt_out = ifmt_of(idx_t); a.val_out = val;
  return from_hip(sfa::launch_csr_to_codes(a, (hipStream_t)stream));
}

sfa_status sfa_kv_append_q8(const float* k_new, const void* v_new, const int32_t* n_new,
                            int32_t* seq_len, int B, int Hkv, int T, int d, int k,
                            const int32_t* block_table, int max_pages, int page_size,
                            int num_pages, void* kc_idx, int8_t* kc_val, float* kc_scale,
                            int8_t* v_cache, float* v_scale, int kc_idx_t, int v_new_t,
                            void* stream) {
  if (!seq_len || !kc_idx || !kc_val || !kc_scale || !v_cache || !v_scale) return SFA_EINVAL;
  if (B < 1 || Hkv < 1 || T < 0 || d < 1 || k < 1 || k > d || page_size < 1) return SFA_EINVAL;
  if (T > 0 && (!k_new || !v_new)) return SFA_EINVAL;
  if (block_table && (max_pages < 1 || num_pages < 1)) return SFA_EINVAL;
  if (block_table && (long long)max_pages * page_size > (1LL << 30)) return SFA_EINVAL;
  if (block_table && (page_size & (page_size - 1)) != 0) return SFA_EINVAL;
  if (!is_idx(kc_idx_t) || !is_val(v_new_t)) return SFA_EINVAL;
  if (d > 256) return SFA_ENOTSUP;
  if ((long long)B * Hkv * T > (1LL << 31)) return SFA_ENOTSUP;
  sfa::AppendArgs a = {};
  a.k_new = k_new; a.v_new = v_new; a.n_new = n_new; a.seq_len = seq_len;
  a.table = block_table; a.kc_idx = kc_idx; a.kc_val = kc_val; a.v_cache = v_cache;
  a.B = B; a.Hkv = Hkv; a.T = T; a.d = d; a.k = k;
  a.page_size = page_size; a.max_pages = max_pages; a.num_pages = num_pages;
  while ((1 << a.log2P) < page_size) ++a.log2P;
  a.ifmt = ifmt_of(kc_idx_t); a.vfmt = sfa::kValF32;
  a.vin_bf16 = v_new_t == SFA_BF16; a.vc_bf16 = 0;
  a.q8 = 1; a.kc_scale = kc_scale; a.v_scale = v_scale;
  return from_hip(sfa::launch_kv_append(a, (hipStream_t)stream));
}

sfa_status sfa_attn_decode_q8(const float* q, const void* q_idx, const void* q_val,
                              const void* kc_idx, const int8_t* kc_val, const float* kc_scale,
                              const int8_t* v_cache, const float* v_scale,
                              const int32_t* block_table, int max_pages, int page_size,
                              int num_pages, const int32_t* seq_len, int B, int Hq, int Hkv,
                              int d, int k, float scale, int window, int n_global, int q_idx_t,
                              int q_val_t, int kc_idx_t, int o_t, void* o, float* lse, void* ws,
                              size_t ws_bytes, void* stream) {
  const bool dense_q = q != nullptr;
  if (dense_q ? (q_idx || q_val) : (!q_idx || !q_val)) return SFA_EINVAL;
  if (!kc_idx || !kc_val || !kc_scale || !v_cache || !v_scale || !o || !ws) return SFA_EINVAL;
  if (B < 1 || Hq < 1 || Hkv < 1 || d < 1 || k < 1 || k > d || page_size < 1) return SFA_EINVAL;
  if (block_table && (max_pages < 1 || num_pages < 1)) return SFA_EINVAL;
  if (block_table && (page_size < 16 || (page_size & (page_size - 1)) != 0)) return SFA_EINVAL;
  if (window < 0 || n_global < 0) return SFA_EINVAL;
  if (Hq % Hkv != 0) return SFA_EINVAL;
  if ((!dense_q && (!is_idx(q_idx_t) || !is_cval(q_val_t))) || !is_idx(kc_idx_t) || !is_val(o_t))
    return SFA_EINVAL;
  if (!isfinite(scale)) return SFA_EINVAL;
  const long long cap = block_table ? (long long)max_pages * page_size : page_size;
  if (cap > (1LL << 30)) return SFA_ENOTSUP;
  if ((long long)B * Hkv > 65535) return SFA_ENOTSUP;
  // the 8-bit cache runs the vector decode: int16 indices, k in {8, 16, 32},
  // d in {64, 128}, a power-of-two group <= 8
  if (kc_idx_t != SFA_I16 || !sfa::decode_q8_supported(d, k, Hq / Hkv)) return SFA_ENOTSUP;
  if (((uintptr_t)v_cache | (uintptr_t)kc_idx | (uintptr_t)kc_val) % 16 != 0) return SFA_EINVAL;
  const int Lmax = (int)cap;
  if (ws_bytes < sfa::decode_workspace_bytes_min(B, Hq, Lmax, d)) return SFA_ENOSPC;
  int log2P = 0;
  if (block_table)
    while ((1 << log2P) < page_size) ++log2P;
  sfa::DecodeArgs a = {};
  a.q_dense = q; a.q_idx = q_idx; a.q_val = q_val;
  a.kc_idx = kc_idx; a.kc_val = kc_val; a.v = v_cache;
  a.kc_scale = kc_scale; a.v_scale = v_scale;
  a.seq_len = seq_len; a.table = block_table;
  a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.Lmax = Lmax; a.d = d; a.k = k; a.scale = scale;
  a.max_pages = max_pages; a.log2P = log2P; a.num_pages = num_pages;
  a.window = window; a.n_global = window > 0 ? n_global : 0;
  a.qifmt = dense_q ? 0 : ifmt_of(q_idx_t); a.qvfmt = dense_q ? 0 : vfmt_of(q_val_t);
  a.kifmt = sfa::kIdxI16; a.kvfmt = sfa::kValF32;
  a.vbf16 = 0; a.obf16 = o_t == SFA_BF16;
  a.o = o; a.lse = lse; a.ws = ws;
  a.aim = sfa::decode_aim(B, Hq, Hkv, Lmax, d, window, ws_bytes, true);
  return from_hip(sfa::launch_attn_decode_q8(a, (hipStream_t)stream));
}

sfa_status sfa_rope_plan_init(sfa_rope_plan* plan, int d, const int32_t* sections, int naxes,
                              double theta, int pairing, int order) {
  if (!plan || !sections || naxes < 1 || naxes > SFA_ROPE_MAX_AXES || d < 2) return SFA_EINVAL;
  if (!isfinite(theta) || theta < 1.0) return SFA_EINVAL;
  if (pairing != SFA_ROPE_HALVES && pairing != SFA_ROPE_NEIGHBOURS) return SFA_EINVAL;
  if (order != SFA_ROPE_SECTIONS && order != SFA_ROPE_INTERLEAVED && order != SFA_ROPE_OWN) return SFA_EINVAL;
  if (d > 256) return SFA_ENOTSUP;
  int half = 0;
  for (int a = 0; a < naxes; ++a) {
    if (sections[a] < 1 || sections[a] > d) return SFA_EINVAL;
    half += sections[a];
  }
  if (2 * half > d) return SFA_EINVAL;
  sfa_rope_plan p = {};
  p.d = d; p.rot = 2 * half; p.naxes = naxes; p.pairing = pairing;
  int i = 0;
  if (order == SFA_ROPE_INTERLEAVED) {
    for (int j = 0; i < half; ++j)
      for (int a = 0; a < naxes; ++a)
        if (j < sections[a]) p.axis[i++] = (uint8_t)a;
  } else {
    for (int a = 0; a < naxes; ++a)
      for (int j = 0; j < sections[a]; ++j) p.axis[i++] = (uint8_t)a;
  }
  i = 0;
  if (order == SFA_ROPE_OWN) {
    for (int a = 0; a < naxes; ++a)
      for (int j = 0; j < sections[a]; ++j) p.freq[i++] = pow(theta, -(double)j / sections[a]);
  } else {
    for (; i < half; ++i) p.freq[i] = pow(theta, -2.0 * i / p.rot);
  }
  *plan = p;
  return SFA_OK;
}

sfa_status sfa_rope(const void* x, const int64_t* x_strides, const int32_t* pos,
                    int64_t pos_axis_stride, int64_t pos_batch_stride, const sfa_rope_plan* plan,
                    int B, int H, int n, int inverse, int x_t, int y_t, void* y,
                    const int64_t* y_strides, void* stream) {
  sfa::RopePlan pl;
  sfa::RopeArgs a = {};
  if (!is_val(x_t) || !is_val(y_t)) return SFA_EINVAL;
  if (!rope_common(plan, pos, pos_axis_stride, pos_batch_stride, B, H, n, inverse, pl, a)) return SFA_EINVAL;
  row_strides(x_strides, H, n, a.d, a.xs);
  row_strides(y_strides, H, n, a.d, a.ys);
  if (n == 0) return SFA_OK;
  if (!strides_readable(a.xs) || !strides_writable(a.ys, B, H, n, a.d)) return SFA_EINVAL;
  if (!x || !y) return SFA_EINVAL;
  if ((uintptr_t)x % (x_t == SFA_BF16 ? 2 : 4) || (uintptr_t)y % (y_t == SFA_BF16 ? 2 : 4)) return SFA_EINVAL;
  a.x = x; a.y = y;
  a.xbf16 = x_t == SFA_BF16; a.ybf16 = y_t == SFA_BF16;
  return from_hip(sfa::launch_rope(pl, a, (hipStream_t)stream));
}

sfa_status sfa_rope_encode(const void* x, const int64_t* x_strides, const int32_t* pos,
                           int64_t pos_axis_stride, int64_t pos_batch_stride,
                           const sfa_rope_plan* plan, int B, int H, int n, int k, int x_t,
                           void* idx, int idx_t, void* val, int val_t, void* stream) {
  sfa::RopePlan pl;
  sfa::RopeArgs a = {};
  if (!is_val(x_t) || !is_idx(idx_t) || !is_cval(val_t)) return SFA_EINVAL;
  if (!rope_common(plan, pos, pos_axis_stride, pos_batch_stride, B, H, n, 0, pl, a)) return SFA_EINVAL;
  if (k < 1 || k > a.d) return SFA_EINVAL;
  row_strides(x_strides, H, n, a.d, a.xs);
  if (n == 0) return SFA_OK;
  if (!strides_readable(a.xs)) return SFA_EINVAL;
  if (!x || !idx || !val || (uintptr_t)x % (x_t == SFA_BF16 ? 2 : 4)) return SFA_EINVAL;
  a.x = x; a.idx = idx; a.val = val; a.k = k;
  a.xbf16 = x_t == SFA_BF16;
  a.ifmt = ifmt_of(idx_t); a.vfmt = vfmt_of(val_t);
  return from_hip(sfa::launch_rope_encode(pl, a, (hipStream_t)stream));
}

sfa_status sfa_rope_encode_bwd(const void* idx, int idx_t, const float* dval, const int32_t* pos,
                               int64_t pos_axis_stride, int64_t pos_batch_stride,
                               const sfa_rope_plan* plan, int B, int H, int n, int k, int dx_t,
                               void* dx, const int64_t* dx_strides, void* stream) {
  sfa::RopePlan pl;
  sfa::RopeArgs a = {};
  if (!is_val(dx_t) || !is_idx(idx_t)) return SFA_EINVAL;
  if (!rope_common(plan, pos, pos_axis_stride, pos_batch_stride, B, H, n, 1, pl, a)) return SFA_EINVAL;
  if (k < 1 || k > a.d) return SFA_EINVAL;
  row_strides(dx_strides, H, n, a.d, a.ys);
  if (n == 0) return SFA_OK;
  if (!strides_writable(a.ys, B, H, n, a.d)) return SFA_EINVAL;
  if (!idx || !dval || !dx || (uintptr_t)dx % (dx_t == SFA_BF16 ? 2 : 4)) return SFA_EINVAL;
  a.idx = const_cast<void*>(idx); a.dval = dval; a.y = dx; a.k = k;
  a.ybf16 = dx_t == SFA_BF16;
  a.ifmt = ifmt_of(idx_t);
  return from_hip(sfa::launch_rope_encode_bwd(pl, a, (hipStream_t)stream));
}

size_t sfa_page_tables_workspace(int B) {
  return B < 1 || B > (1 << 20) ? 0 : sfa::page_tables_workspace_bytes(B);
}

sfa_status sfa_page_tables(const int32_t* old_len, const int32_t* new_len, int B,
                           int32_t* block_table, int max_pages, int page_size,
                           int32_t* free_pages, int num_pages, const int32_t* free_in,
                           int32_t* free_out, int32_t* got_len, int32_t* starts, int32_t* slots,
                           int32_t* positions, int n_rows, void* ws, size_t ws_bytes,
                           void* stream) {
  if (!new_len || !block_table || !free_pages || !free_in || !free_out || !got_len || !ws) return SFA_EINVAL;
  if (B < 1 || B > (1 << 20) || max_pages < 1 || page_size < 1 || num_pages < 1 || n_rows < 0) return SFA_EINVAL;
  if ((page_size & (page_size - 1)) != 0) return SFA_EINVAL;
  if ((long long)max_pages * page_size > (1LL << 30) || (long long)num_pages * page_size > 0x7fffffffLL ||
      (long long)B * max_pages > 0x7fffffffLL)
    return SFA_EINVAL;
  if (got_len == old_len || got_len == new_len) return SFA_EINVAL;
  if ((uintptr_t)ws % 4 != 0) return SFA_EINVAL;
  if (ws_bytes < sfa::page_tables_workspace_bytes(B)) return SFA_ENOSPC;
  sfa::PageArgs a = {};
  a.old_len = old_len; a.new_len = new_len; a.free_in = free_in;
  a.table = block_table; a.free_pages = free_pages; a.free_out = free_out; a.got = got_len;
  a.starts = starts; a.slots = slots; a.pos = positions;
  a.B = B; a.max_pages = max_pages; a.num_pages = num_pages;
  a.n_rows = slots || positions ? n_rows : 0;
  while ((1 << a.log2P) < page_size) ++a.log2P;
  a.ws = (int32_t*)ws;
  return from_hip(sfa::launch_page_tables(a, (hipStream_t)stream));
}

sfa_status sfa_kv_append_q4(const void* k_new, const void* v_new, const int64_t* kv_strides,
                            const int32_t* slots, const int32_t* n_new, int32_t* seq_len, int B,
                            int Hkv, int T, int d, int k, const int32_t* block_table,
                            int max_pages, int page_size, int num_pages, uint8_t* kc_idx,
                            uint8_t* kc_val, float* kc_scale, uint8_t* v_cache, uint16_t* v_scale,
                            int16_t* k_idx, float* k_val, uint16_t* v_out, int k_new_t,
                            int v_new_t, void* stream) {
  if (!kc_idx || !kc_val || !kc_scale || !v_cache || !v_scale) return SFA_EINVAL;
  if (B < 1 || Hkv < 1 || T < 0 || d < 1 || k < 1 || k > d || page_size < 1 || num_pages < 1) return SFA_EINVAL;
  if (T > 0 && (!k_new || !v_new)) return SFA_EINVAL;
  if (slots ? (seq_len || n_new || block_table) : !seq_len) return SFA_EINVAL;
  if (!k_idx != !k_val) return SFA_EINVAL;
  if (block_table && (max_pages < 1 || (page_size & (page_size - 1)) != 0 ||
                      (long long)max_pages * page_size > (1LL << 30)))
    return SFA_EINVAL;
  if ((long long)num_pages * page_size > 0x7fffffffLL) return SFA_EINVAL;
  if (!slots && !block_table && num_pages != B) return SFA_EINVAL;
  if (!is_val(k_new_t) || !is_val(v_new_t)) return SFA_EINVAL;
  if (d > 256 || d % 32 != 0 || k % 8 != 0) return SFA_ENOTSUP;
  if ((long long)B * Hkv * T > (1LL << 31) || (long long)num_pages * Hkv > 0x7fffffffLL) return SFA_ENOTSUP;
  if (((uintptr_t)kc_idx | (uintptr_t)kc_val | (uintptr_t)v_cache | (uintptr_t)kc_scale) % 4 != 0 ||
      ((uintptr_t)v_scale | (uintptr_t)k_idx) % 2 != 0 || ((uintptr_t)k_val | (uintptr_t)v_out) % 4 != 0 ||
      (uintptr_t)k_new % (k_new_t == SFA_BF16 ? 2 : 4) != 0 || (uintptr_t)v_new % (v_new_t == SFA_BF16 ? 2 : 4) != 0)
    return SFA_EINVAL;
  sfa::AppendQ4Args a = {};
  int64_t ks[3], vs[3];
  row_strides(kv_strides, Hkv, T, d, ks);
  row_strides(kv_strides ? kv_strides + 3 : nullptr, Hkv, T, d, vs);
  if (!strides_readable(ks) || !strides_readable(vs)) return SFA_EINVAL;
  for (int i = 0; i < 3; ++i) { a.st[i] = ks[i]; a.st[3 + i] = vs[i]; }
  a.k_new = k_new; a.v_new = v_new; a.slots = slots; a.n_new = n_new; a.table = block_table; a.seq_len = seq_len;
  a.B = B; a.Hkv = Hkv; a.T = T; a.d = d; a.k = k;
  a.max_pages = max_pages; a.page_size = page_size; a.num_pages = num_pages;
  a.kbf16 = k_new_t == SFA_BF16; a.vbf16 = v_new_t == SFA_BF16;
  a.kc_idx = kc_idx; a.kc_val = kc_val; a.v_cache = v_cache; a.kc_scale = kc_scale; a.v_scale = v_scale;
  a.k_idx = k_idx; a.k_val = k_val; a.v_out = v_out;
  return from_hip(sfa::launch_kv_append_q4(a, (hipStream_t)stream));
}

size_t sfa_attn_decode_q4_workspace(int B, int Hq, int Lmax, int d) {
  if (B < 1 || Hq < 1 || Lmax < 1 || Lmax > (1 << 30) || d < 1 || d > 256) return 0;
  return sfa::decode_q4_workspace_bytes(B, Hq, Lmax, d);
}

sfa_status sfa_attn_decode_q4(const float* q, const void* q_idx, const void* q_val,
                              const uint8_t* kc_idx, const uint8_t* kc_val,
                              const float* kc_scale, const uint8_t* v_cache,
                              const uint16_t* v_scale, const int32_t* block_table, int max_pages,
                              int page_size, int num_pages, const int32_t* seq_len, int B, int Hq,
                              int Hkv, int d, int k, float scale, int window, int n_global,
                              int q_idx_t, int q_val_t, int o_t, void* o, float* lse, void* ws,
                              size_t ws_bytes, void* stream) {
  const bool dense_q = q != nullptr;
  if (dense_q ? (q_idx || q_val) : (!q_idx || !q_val)) return SFA_EINVAL;
  if (!kc_idx || !kc_val || !kc_scale || !v_cache || !v_scale || !o || !ws) return SFA_EINVAL;
  if (B < 1 || Hq < 1 || Hkv < 1 || d < 1 || k < 1 || k > d || page_size < 1) return SFA_EINVAL;
  if (block_table && (max_pages < 1 || num_pages < 1)) return SFA_EINVAL;
  if (block_table && (page_size < 16 || (page_size & (page_size - 1)) != 0)) return SFA_EINVAL;
  if (window < 0 || n_global < 0) return SFA_EINVAL;
  if (Hq % Hkv != 0) return SFA_EINVAL;
  if ((!dense_q && (!is_idx(q_idx_t) || !is_cval(q_val_t))) || !is_val(o_t)) return SFA_EINVAL;
  if (!isfinite(scale)) return SFA_EINVAL;
  const long long cap = block_table ? (long long)max_pages * page_size : page_size;
  if (cap > (1LL << 30)) return SFA_ENOTSUP;
  if ((long long)B * Hkv > 65535) return SFA_ENOTSUP;
  if (d > 256 || d % 32 != 0 || k % 8 != 0 || Hq / Hkv > sfa::decode_max_group()) return SFA_ENOTSUP;
  if (((uintptr_t)v_cache | (uintptr_t)kc_idx | (uintptr_t)kc_val | (uintptr_t)kc_scale | (uintptr_t)v_scale) % 16 != 0 ||
      (uintptr_t)ws % 4 != 0)
    return SFA_EINVAL;
  const int Lmax = (int)cap;
  if (ws_bytes < sfa::decode_q4_workspace_bytes(B, Hq, Lmax, d)) return SFA_ENOSPC;
  sfa::DecodeArgs a = {};
  if (block_table)
    while ((1 << a.log2P) < page_size) ++a.log2P;
  a.q_dense = q; a.q_idx = q_idx; a.q_val = q_val;
  a.kc_idx = kc_idx; a.kc_val = kc_val; a.v = v_cache;
  a.kc_scale = kc_scale; a.v_scale16 = v_scale;
  a.seq_len = seq_len; a.table = block_table;
  a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.Lmax = Lmax; a.d = d; a.k = k; a.scale = scale;
  a.max_pages = max_pages; a.num_pages = num_pages;
  a.window = window; a.n_global = window > 0 ? n_global : 0;
  a.qifmt = dense_q ? 0 : ifmt_of(q_idx_t); a.qvfmt = dense_q ? 0 : vfmt_of(q_val_t);
  a.obf16 = o_t == SFA_BF16;
  a.o = o; a.lse = lse; a.ws = ws;
  a.aim = sfa::decode_chunks_aim(B, Hkv, true, window);
  return from_hip(sfa::launch_attn_decode_q4(a, (hipStream_t)stream));
}

}  // extern "C"
