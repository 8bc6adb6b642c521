// Block tables, free list and slot map on the device, from old and new request
// lengths (sfa_page_tables).
//
// With have / want the pages of a sequence's old / new length, F the free count
// and exclusive prefix sums over the sequences of what each gives back (rel0) and
// takes (need0), every page's place is known without any order of execution:
//   the j-th page given back by b stands at F + rel0[b] + j of the free list,
//   the j-th page taken by b stood at S - 1 - (need0[b] + j), S = F + sum rel,
// and a place at or past F is a page given back in this call, found by a binary
// search of rel0.  One workgroup makes the sums (`plan`); then every sequence's
// table entries and token rows are independent (`fill`): entries that are read
// (a shrinking row's, the free list below F) are not the ones that are written
// (a growing row's, the free list from F on).
// A generation step is bound by launches: one workgroup then does both parts.
#include "sfa_device.h"
#include "sfa_launch.h"

namespace sfa {
namespace {

constexpr int kPlanThreads = 1024;

// The scratch: header, then the prefix sums.  A step of few sequences has it in LDS, and
// their lengths behind it: its time is a chain of reads of these (22 sequences, pages
// given back and taken: 13.6 -> 11.6 us).
constexpr int kLocal = 1024;
struct PageWs {
  int32_t* head;   // F, S, new count, tokens in all
  int32_t* rel0;   // [B]
  int32_t* need0;  // [B]
  int32_t* row0;   // [B]
  const int32_t *old_len, *new_len;
  __device__ __forceinline__ explicit PageWs(const PageArgs& a)
      : head(a.ws), rel0(a.ws + 4), need0(a.ws + 4 + a.B), row0(a.ws + 4 + 2 * a.B), old_len(a.old_len), new_len(a.new_len) {}
  __device__ __forceinline__ explicit PageWs(int32_t (&lds)[4 + 5 * kLocal])
      : head(lds), rel0(lds + 4), need0(lds + 4 + kLocal), row0(lds + 4 + 2 * kLocal), old_len(lds + 4 + 3 * kLocal),
        new_len(lds + 4 + 4 * kLocal) {}
};

// A sequence's lengths and pages.
struct SeqPages {
  int old_len, new_len, have, want, rel, need, count;
  __device__ __forceinline__ SeqPages(const PageArgs& a, const PageWs& ws, int b) {
    const int cap = a.max_pages << a.log2P, up = (1 << a.log2P) - 1;
    old_len = ws.old_len ? min(max(ws.old_len[b], 0), cap) : 0;
    new_len = min(max(ws.new_len[b], 0), cap);
    have = (old_len + up) >> a.log2P;
    want = (new_len + up) >> a.log2P;
    rel = max(have - want, 0);
    need = max(want - have, 0);
    count = max(new_len - old_len, 0);
  }
};

// Sum of two counts, at most 2^31 - 1 (the tokens of a call may pass it: rows
// that far on lie behind any token buffer).
__device__ __forceinline__ int add_sat(int x, int y) { return (int)min((uint32_t)x + (uint32_t)y, 0x7fffffffu); }

__device__ __forceinline__ int wave_scan(int x, int lane) {  // inclusive
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x = add_sat(x, y);
  }
  return x;
}

__device__ __forceinline__ void plan(const PageArgs& a, const PageWs& ws) {
  __shared__ int part[3][kPlanThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int base[3] = {0, 0, 0};  // sums over the sequences before these
  for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
    const int b = b0 + tid;
    int v[3] = {0, 0, 0}, in[3];
    if (b < a.B) {
      const SeqPages s(a, ws, b);
      v[0] = s.rel; v[1] = s.need; v[2] = s.count;
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      const int upto = wave_scan(v[q], lane);
      if (lane == 63) part[q][wave] = upto;
      const int below = __shfl_up(upto, 1, 64);
      in[q] = lane > 0 ? below : 0;
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      int before = 0, all = 0;
#pragma unroll
      for (int w = 0; w < kPlanThreads / 64; ++w) {
        if (w < wave) before = add_sat(before, part[q][w]);
        all = add_sat(all, part[q][w]);
      }
      in[q] = add_sat(in[q], add_sat(base[q], before));
      base[q] = add_sat(base[q], all);
    }
    if (b < a.B) {
      ws.rel0[b] = in[0]; ws.need0[b] = in[1]; ws.row0[b] = in[2];
      if (a.starts) a.starts[b] = in[2];
    }
    __syncthreads();
  }
  const int F = min(max(a.free_in[0], 0), a.num_pages);
  const int S = (int)min((int64_t)F + base[0], (int64_t)a.num_pages);
  const int left = S - min(S, base[1]);
  for (int b = tid; b < a.B; b += kPlanThreads) {  // each thread its own sequences
    const SeqPages s(a, ws, b);
    const int grant = min(max(S - ws.need0[b], 0), s.need);
    a.got[b] = s.new_len <= s.old_len ? s.new_len
                                      : (int)min((int64_t)s.new_len, (int64_t)(s.have + grant) << a.log2P);
  }
  if (tid == 0) {
    ws.head[0] = F; ws.head[1] = S; ws.head[2] = left; ws.head[3] = base[2];
    if (a.starts) a.starts[a.B] = base[2];
  }
  __syncthreads();  // free_out may be free_in: every thread has read it
  if (tid == 0) a.free_out[0] = left;
}

// The page at place p < S of the free list with this call's pages pushed; rel0 as in
// the scratch, or a copy of it.
__device__ __forceinline__ int stack_page(const PageArgs& a, const PageWs& ws, const int32_t* rel0, int F, int p) {
  if (p < F) return a.free_pages[p];
  const int q = p - F;
  int lo = 0, hi = a.B;  // the last sequence with rel0 <= q
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (rel0[mid] <= q) lo = mid; else hi = mid;
  }
  const SeqPages s(a, ws, lo);
  return a.table[(int64_t)lo * a.max_pages + s.want + (q - rel0[lo])];
}

// Sequence b's table entries, pushed pages and token rows, by `lanes` threads.
__device__ __forceinline__ void fill(const PageArgs& a, const PageWs& ws, int b, int me, int lanes,
                                     const int32_t* all_rel0) {
  const int F = ws.head[0], S = ws.head[1], left = ws.head[2];
  const SeqPages s(a, ws, b);
  const int rel0 = ws.rel0[b], need0 = ws.need0[b], row0 = ws.row0[b];
  int32_t* row = a.table + (int64_t)b * a.max_pages;
  for (int j = me; j < s.rel; j += lanes) {
    const uint32_t p = (uint32_t)F + (uint32_t)(rel0 + j);  // (may pass 2^31 where lengths and list disagree)
    if (p < (uint32_t)left) a.free_pages[p] = row[s.want + j];
  }
  const int grant = min(max(S - need0, 0), s.need);
  for (int j = me; j < grant; j += lanes) row[s.have + j] = stack_page(a, ws, all_rel0, F, S - 1 - need0 - j);
  const int rows = min(s.count, a.n_rows - row0);  // (may be negative)
  for (int t = me; t < rows; t += lanes) {
    const int pos = s.old_len + t, j = pos >> a.log2P;
    if (a.slots) {
      // a new page's id from where the entry above takes it: the entry may not be written yet
      int page = -1;
      if (j < s.have) page = row[j];
      else if (j - s.have < grant) page = stack_page(a, ws, all_rel0, F, S - 1 - need0 - (j - s.have));
      a.slots[row0 + t] = page >= 0 && page < a.num_pages ? (page << a.log2P) + (pos & ((1 << a.log2P) - 1)) : -1;
    }
    if (a.pos) a.pos[row0 + t] = pos;
  }
}

__device__ __forceinline__ void fill_behind(const PageArgs& a, const PageWs& ws, int64_t me, int64_t threads) {
  for (int64_t i = ws.head[3] + me; i < a.n_rows; i += threads) {
    if (a.slots) a.slots[i] = -1;
    if (a.pos) a.pos[i] = -1;
  }
}

// group: threads per sequence (a power of two).  LOCAL: B <= kLocal.
template <bool LOCAL>
__global__ __launch_bounds__(kPlanThreads) void sfa_page_step_kernel(PageArgs a, int group) {
  auto both = [&](const PageWs& ws) {
    plan(a, ws);
    __syncthreads();
    for (int b = threadIdx.x / group; b < a.B; b += kPlanThreads / group)
      fill(a, ws, b, threadIdx.x & (group - 1), group, ws.rel0);
    fill_behind(a, ws, threadIdx.x, kPlanThreads);
  };
  if constexpr (LOCAL) {
    __shared__ int32_t lds[4 + 5 * kLocal];
    if ((int)threadIdx.x < a.B) {  // (kLocal threads)
      lds[4 + 3 * kLocal + threadIdx.x] = a.old_len ? a.old_len[threadIdx.x] : 0;
      lds[4 + 4 * kLocal + threadIdx.x] = a.new_len[threadIdx.x];
    }
    __syncthreads();
    both(PageWs(lds));
  } else {
    both(PageWs(a));
  }
}

__global__ __launch_bounds__(kPlanThreads) void sfa_page_plan_kernel(PageArgs a) { plan(a, PageWs(a)); }

// LOCAL (B <= kLocal): the prefix sums that the searches walk, in LDS: a search is a
// chain of dependent reads, and most pages that are taken beside others given back are
// found by one (256 sequences, a million rows: 21 -> 9.5 us).
template <bool LOCAL>
__global__ __launch_bounds__(256) void sfa_page_fill_kernel(PageArgs a) {
  __shared__ int32_t rel0[LOCAL ? kLocal : 1];
  const PageWs ws(a);
  const int32_t* src = ws.rel0;
  if constexpr (LOCAL) {
    for (int i = threadIdx.x; i < a.B; i += 256) rel0[i] = src[i];
    __syncthreads();
  }
  fill(a, ws, blockIdx.x, blockIdx.y * 256 + threadIdx.x, gridDim.y * 256, LOCAL ? rel0 : src);
  const int64_t blocks = (int64_t)gridDim.x * gridDim.y, me = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  fill_behind(a, ws, me * 256 + threadIdx.x, blocks * 256);
}

}  // namespace

size_t page_tables_workspace_bytes(int B) { return ((size_t)3 * B + 4) * sizeof(int32_t); }

hipError_t launch_page_tables(const PageArgs& a, hipStream_t stream) {
  // One workgroup for a step's tokens, or a few prompts' (its 16 wavefronts keep
  // up with the second launch to about four rows a thread).
  if (a.n_rows <= 4 * kPlanThreads && a.B <= 4 * kPlanThreads) {
    int group = 64;
    while (group > 1 && (int64_t)group * a.B > kPlanThreads) group >>= 1;
    if (a.B <= kLocal) hipLaunchKernelGGL(sfa_page_step_kernel<true>, dim3(1), dim3(kPlanThreads), 0, stream, a, group);
    else hipLaunchKernelGGL(sfa_page_step_kernel<false>, dim3(1), dim3(kPlanThreads), 0, stream, a, group);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(sfa_page_plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // a row a thread where the sequences share the rows evenly, in at most 4096 workgroups
  int64_t slices = (a.n_rows / a.B + 255) / 256;
  if (slices * a.B > 4096) slices = 4096 / a.B;
  if (slices < 1) slices = 1;
  const dim3 grid(a.B, (unsigned)slices);
  if (a.B <= kLocal) hipLaunchKernelGGL(sfa_page_fill_kernel<true>, grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(sfa_page_fill_kernel<false>, grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace sfa
