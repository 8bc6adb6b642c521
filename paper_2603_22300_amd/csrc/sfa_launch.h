// Internal launchers behind the C ABI (host side).  Arguments are validated
// by the ABI layer before any of these is called.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace sfa {

hipError_t launch_topk_encode(const float* x, int64_t rows, int d, int k, void* idx, int ifmt,
                              void* val, int vfmt, hipStream_t stream);

hipError_t launch_attn_fwd(const void* q_idx, const void* q_val, const void* k_idx,
                           const void* k_val, const void* v, int B, int Hq, int Hkv, int n, int d,
                           int k, int causal, int window, int n_global, float scale, int ifmt,
                           int vfmt, int vbf16, int obf16, void* o, float* lse, void* ws,
                           hipStream_t stream);
int fwd_max_group();
size_t fwd_workspace_bytes(int B, int Hkv, int n, int d, int vbf16);

// forward at float32 accuracy for head dimensions (d <= 256) and group sizes
// without the tuned kernel; no workspace
hipError_t launch_attn_fwd_generic(const void* q_idx, const void* q_val, const void* k_idx,
                                   const void* k_val, const void* v, int B, int Hq, int Hkv,
                                   int n, int d, int k, int causal, int window, int n_global,
                                   float scale, int ifmt, int vfmt, int vbf16, int obf16, void* o,
                                   float* lse, hipStream_t stream);
bool fwd_generic_supported(int d, int k);

hipError_t launch_attn_bwd(const void* q_idx, const void* q_val, const void* k_idx,
                           const void* k_val, const void* v, const void* o, const float* lse,
                           const void* dout, int B, int Hq, int Hkv, int n, int d, int k,
                           int causal, int window, int n_global, float scale, int ifmt,
                           int vfmt, int vbf16, int obf16, float* dq, float* dk, float* dv,
                           void* ws, hipStream_t stream);
size_t bwd_workspace_bytes(int B, int Hq, int Hkv, int n, int d);
int bwd_max_group();

// float32 backward for head dimensions without the matrix-core kernels
// (d <= 256); no workspace, any group size
hipError_t launch_attn_bwd_generic(const void* q_idx, const void* q_val, const void* k_idx,
                                   const void* k_val, const void* v, const void* o,
                                   const float* lse, const void* dout, int B, int Hq, int Hkv,
                                   int n, int d, int k, int causal, int window, int n_global,
                                   float scale, int ifmt, int vfmt, int vbf16, int obf16,
                                   float* dq, float* dk, float* dv, hipStream_t stream);
bool bwd_generic_supported(int d, int k);

hipError_t launch_attn_fwd_index(const void* q_idx, const void* q_val, const void* k_idx,
                                 const void* k_val, const void* v, int B, int Hq, int Hkv, int n,
                                 int d, int k, int causal, float scale, int ifmt, int vfmt,
                                 int vbf16, int obf16, void* o, float* lse, hipStream_t stream);
int fwd_index_lds_bytes(int d, int k, int vbf16);
int fwd_index_max_k();
int fwd_index_rows_per_block();

// Decode over a contiguous (table == nullptr: [B, Hkv, Lmax, ...]) or paged
// (pages [num_pages, Hkv, 1 << log2P, ...], table [B, max_pages],
// Lmax = max_pages << log2P) cache; query codes, or q_dense coded in-kernel.
struct DecodeArgs {
  const float* q_dense;
  const void *q_idx, *q_val, *kc_idx, *kc_val, *v;
  const int32_t* seq_len;
  const int32_t* table;
  int B, Hq, Hkv, Lmax, d, k;
  int max_pages, log2P, num_pages;
  int window, n_global;  // token pattern (window 0: none)
  float scale;
  int qifmt, qvfmt, kifmt, kvfmt, vbf16, obf16;
  void* o;
  float* lse;
  void* ws;
  int aim;  // tuned decode: decode_chunks_aim, or 0 where ws holds kDecodeChunk chunks only
  // 8-bit cache (launch_attn_decode_q8): float32 scale per key row / value row
  const float* kc_scale;
  const float* v_scale;
  const uint16_t* v_scale16;  // 4-bit cache (launch_attn_decode_q4): bfloat16 scale per 32 values
};
// Most keys of a decode workgroup (one context chunk), and of the float32
// decode's; the workspace holds one partial (m, l, o) per chunk, query head
// and sequence.
constexpr int kDecodeChunk = 4096;
// Fewest keys of a chunk (64 per wavefront), and the workgroups that the
// tuned decode aims at by cutting sequences into smaller chunks (decode_plan):
// one per compute unit; more for the 8-bit cache, whose waves do more
// arithmetic per byte, and under a token window, which fills its first and
// last chunk only partly.
constexpr int kDecodeMinChunk = 256;
constexpr int kDecodeTarget = 256, kDecodeTargetQ8 = 1024, kDecodeTargetWindow = 2048;
// Chunks per (sequence, KV head) that a step over B * Hkv of them aims at.
// 0: every chunk has kDecodeChunk keys (B * Hkv alone passes the target); 1: the same,
// but a sequence that fits one smaller chunk has that.
inline int decode_chunks_aim(int B, int Hkv, bool q8, int window) {
  const int target = window > 0 ? kDecodeTargetWindow : q8 ? kDecodeTargetQ8 : kDecodeTarget;
  return (int)(target / ((int64_t)B * Hkv));
}
// Partial slots per (sequence, query head) of a step that reads at most
// `span` keys of each sequence with that aim (decode_plan).
inline int decode_slots(int span, int aim) {
  auto up = [](int a, int b) { return a / b + (a % b != 0); };
  const int big = up(span, kDecodeChunk), fine = up(span, kDecodeMinChunk);
  const int most = aim > big ? aim : big;
  return fine < most ? fine : most;
}
hipError_t launch_attn_decode(const DecodeArgs& a, hipStream_t stream);
// Workspace of any step of these sizes, and of one in chunks of kDecodeChunk
// keys (never more than the former).
size_t decode_workspace_bytes(int B, int Hq, int Lmax, int d);
size_t decode_workspace_bytes_min(int B, int Hq, int Lmax, int d);
// The aim of a step with a workspace of ws_bytes (at least the minimum).
int decode_aim(int B, int Hq, int Hkv, int Lmax, int d, int window, size_t ws_bytes, bool q8);
int decode_max_group();
// float32 decode for head dimensions without the tuned kernel (d <= 256);
// same partial layout, in chunks of kDecodeChunk keys; Hq / Hkv <= decode_max_group()
hipError_t launch_attn_decode_generic(const DecodeArgs& a, hipStream_t stream);

// Static device scratch of the allocation-free decode (one copy per GPU):
// its size, and its device address on the current device (looked up once per
// device).
size_t noalloc_scratch_bytes();
hipError_t noalloc_scratch(void** out);

// Decode over the 8-bit cache: int8 code values (int16 indices, k in
// {8, 16, 32}) and int8 value rows with their scales; d in {64, 128}, Hq /
// Hkv a power of two <= 8.
hipError_t launch_attn_decode_q8(const DecodeArgs& a, hipStream_t stream);
bool decode_q8_supported(int d, int k, int G);

// KV-cache append: Top-k coding of new keys and copy of their values into a
// contiguous (table == nullptr: [B, Hkv, P, ...]) or paged cache, then
// seq_len[b] += the appended count (clamped to the capacity).
struct AppendArgs {
  const float* k_new;
  const void* v_new;
  const int32_t* n_new;
  int32_t* seq_len;
  const int32_t* table;
  void *kc_idx, *kc_val, *v_cache;
  int B, Hkv, T, d, k;
  int page_size, max_pages, num_pages;
  int log2P;  // paged: page_size == 1 << log2P
  int ifmt, vfmt, vin_bf16, vc_bf16;
  // 8-bit cache: kc_val and v_cache hold int8, with one float32 scale per
  // key row (kc_scale) and value row (v_scale)
  int q8;
  float* kc_scale;
  float* v_scale;
};
hipError_t launch_kv_append(const AppendArgs& a, hipStream_t stream);

// CSR codes (row r: entries indptr[r] .. indptr[r+1]-1) to fixed rows of kmax
// entries, padded with zero values at the lowest free coordinates.
struct CsrArgs {
  const int32_t* indptr;
  const void* indices;
  const void* values;
  int64_t rows;
  int d, kmax;
  int ifmt_in, vbytes;  // index format; value storage bytes (copied bitwise)
  void* idx_out;
  int ifmt_out;
  void* val_out;
};
hipError_t launch_csr_to_codes(const CsrArgs& a, hipStream_t stream);

// Rotary positions (the device's part of an sfa_rope_plan).
struct RopePlan {
  int d, rot;
  int neighbours;  // pairs (2i, 2i + 1) rather than (i, i + rot/2)
  int inverse;     // turn back
  double freq[128];
  uint8_t axis[128];
};
struct RopeArgs {
  const void* x;
  int64_t xs[3], ys[3];  // element strides of batch, head, token
  const int32_t* pos;
  int64_t pos_axis, pos_batch;
  int B, H, n, d, k;
  int xbf16, ybf16;
  void* y;  // rotated rows, or the backward's dx
  void *idx, *val;
  const float* dval;
  int ifmt, vfmt;
  int units, heads, tokens;  // set by the launchers
};
hipError_t launch_rope(const RopePlan& pl, RopeArgs a, hipStream_t stream);
hipError_t launch_rope_encode(const RopePlan& pl, RopeArgs a, hipStream_t stream);
hipError_t launch_rope_encode_bwd(const RopePlan& pl, RopeArgs a, hipStream_t stream);

// Block tables, free list and slot map from old and new lengths.
struct PageArgs {
  const int32_t *old_len, *new_len, *free_in;
  int32_t *table, *free_pages, *free_out, *got, *starts, *slots, *pos;
  int B, max_pages, log2P, num_pages, n_rows;
  int32_t* ws;
};
size_t page_tables_workspace_bytes(int B);
hipError_t launch_page_tables(const PageArgs& a, hipStream_t stream);

// Append to the 4-bit cache.
struct AppendQ4Args {
  const void *k_new, *v_new;
  int64_t st[6];  // element strides: k batch, head, token, v batch, head, token
  const int32_t *slots, *n_new, *table;
  int32_t* seq_len;
  int B, Hkv, T, d, k;
  int max_pages, page_size, num_pages;
  int kbf16, vbf16;
  uint8_t *kc_idx, *kc_val, *v_cache;
  float* kc_scale;
  uint16_t* v_scale;
  int16_t* k_idx;
  float* k_val;
  uint16_t* v_out;
  // set by the launcher
  int log2P, step_h, step_t, step_b;
  int64_t step_k, step_v, step_tok, step_out, carry_k, carry_v, wrap_k, wrap_v;
};
hipError_t launch_kv_append_q4(AppendQ4Args a, hipStream_t stream);
// seq_len[b] += the appended count, clamped to the capacity (sfa_cache.hip)
hipError_t launch_kv_advance(int32_t* seq_len, const int32_t* n_new, int B, int T, int64_t cap,
                             hipStream_t stream);

// Decode over the 4-bit cache (DecodeArgs: kc_val, v, kc_scale and v_scale16 its
// arrays, aim from decode_chunks_aim).
size_t decode_q4_workspace_bytes(int B, int Hq, int Lmax, int d);
hipError_t launch_attn_decode_q4(const DecodeArgs& a, hipStream_t stream);

}  // namespace sfa
