// Rotary positions with several axes on gfx950: the rotation of dense heads
// (sfa_rope), the same fused with Top-k coding (sfa_rope_encode; Sec. 3.1,
// Eqs. (3)-(4)) and its straight-through backward (sfa_rope_encode_bwd; Eq. (6)).
//
// Pair i turns by the angle pos[axis(i)] * f_i.  Angle, cosine and sine are
// float64 (a position of a million times f_0 = 1 leaves 2^-33 of a radian there
// and a sixteenth of one in float32); both are rounded to float32.  A product of
// two float32 numbers is exact in float64, so x1 c - x2 s rounds once there and
// once to float32: the row that the Top-k selection sees does not depend on the
// order of operations, and neither does the selection.  The float64 unit runs
// at the rate of the float32 one here, and an angle serves every head of its token.
#include "sfa_device.h"
#include "sfa_launch.h"
#include "sfa_topk.h"

namespace sfa {
namespace {

// cos and sin of an angle |a| <= 2^31, rounded to float32.  Reduction by
// n * pi/2 with pi/2 in two float64 pieces (the products inside the fma are
// exact: the error is 2^-53 of the remainder plus n 2^-107), then the Taylor
// polynomials on [-pi/4, pi/4]: their first terms left out are below
// (pi/4)^19/19! = 8e-20 and (pi/4)^18/18! = 2e-18.
__device__ __forceinline__ void turn(double a, float& c, float& s) {
  const double n = rint(a * 0.63661977236758134308);
  double r = fma(-n, 1.5707963267948965580, a);
  r = fma(-n, 6.1232339957367658860e-17, r);
  const double z = r * r;
  double p = 1.0 / 355687428096000.0;  // 1/17!
  p = fma(p, z, -1.0 / 1307674368000.0);
  p = fma(p, z, 1.0 / 6227020800.0);
  p = fma(p, z, -1.0 / 39916800.0);
  p = fma(p, z, 1.0 / 362880.0);
  p = fma(p, z, -1.0 / 5040.0);
  p = fma(p, z, 1.0 / 120.0);
  p = fma(p, z, -1.0 / 6.0);
  const double sn = fma(p * z, r, r);
  double q = 1.0 / 20922789888000.0;  // 1/16!
  q = fma(q, z, -1.0 / 87178291200.0);
  q = fma(q, z, 1.0 / 479001600.0);
  q = fma(q, z, -1.0 / 3628800.0);
  q = fma(q, z, 1.0 / 40320.0);
  q = fma(q, z, -1.0 / 720.0);
  q = fma(q, z, 1.0 / 24.0);
  q = fma(q, z, -1.0 / 2.0);
  const double cs = fma(q, z, 1.0);
  const int k = (int)(long long)n & 3;
  const double c0 = (k & 1) ? sn : cs, s0 = (k & 1) ? cs : sn;
  c = (float)((k == 1 || k == 2) ? -c0 : c0);
  s = (float)((k & 2) ? -s0 : s0);
}

// y1 = x1 c - x2 s, y2 = x2 c + x1 s, each rounded to float32 once.
__device__ __forceinline__ void rotate(float x1, float x2, float c, float s, float& y1, float& y2) {
  const double a = x1, b = x2, cd = c, sd = s;
  y1 = (float)fma(a, cd, -(b * sd));
  y2 = (float)fma(b, cd, a * sd);
}

// VP consecutive elements, VP * size bytes aligned.
template <int VP, typename T>
__device__ __forceinline__ void load_vec(const T* p, float (&v)[VP]) {
  if constexpr (VP == 4 && sizeof(T) == 4) {
    const float4 w = *(const float4*)p;
    v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
  } else if constexpr (VP == 4) {
    const uint2 w = *(const uint2*)p;
    v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xffff0000u);
    v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xffff0000u);
  } else {
#pragma unroll
    for (int i = 0; i < VP; ++i) v[i] = sizeof(T) == 4 ? (float)p[i] : bf16_bits_to_f32((uint32_t)p[i]);
  }
}

// float32 -> bfloat16 bits, nearest even, NaN kept.
__device__ __forceinline__ uint32_t to_bf16(float x) {
  return x != x ? 0x7fc0u : f32_to_bf16_rne(x);
}

template <int VP, typename T>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[VP]) {
  if constexpr (VP == 4 && sizeof(T) == 4) {
    *(float4*)p = make_float4(v[0], v[1], v[2], v[3]);
  } else if constexpr (VP == 4) {
    *(uint2*)p = make_uint2(to_bf16(v[0]) | (to_bf16(v[1]) << 16), to_bf16(v[2]) | (to_bf16(v[3]) << 16));
  } else {
#pragma unroll
    for (int i = 0; i < VP; ++i) {
      if constexpr (sizeof(T) == 4) p[i] = v[i];
      else p[i] = (T)to_bf16(v[i]);
    }
  }
}

// A lane's piece of a row: VP pairs, or the 2 VP coordinates past rot that are
// copied.  off0 / off1: the two runs of VP coordinates it reads and writes
// (pairing halves: the first and the second of each pair; neighbours: 2 VP
// consecutive ones, pair by pair).
template <int VP>
struct Unit {
  bool turned;
  int pair, off0, off1, n1;  // n1: coordinates of the second run inside the row
  __device__ __forceinline__ Unit(const RopePlan& pl, int u) {
    const int half = pl.rot / 2, nr = half / VP;
    turned = u < nr;
    pair = turned ? u * VP : 0;
    if (turned) {
      off0 = pl.neighbours ? 2 * pair : pair;
      off1 = pl.neighbours ? off0 + VP : pair + half;
    } else {
      off0 = pl.rot + (u - nr) * 2 * VP;
      off1 = off0 + VP;
    }
    n1 = min(VP, max(0, pl.d - off1));
  }
};

template <int VP>
__device__ __forceinline__ void unit_turns(const RopePlan& pl, const int32_t* pos, int64_t pos_axis, bool turned,
                                           int pair, float (&c)[VP], float (&s)[VP]) {
#pragma unroll
  for (int i = 0; i < VP; ++i) {
    c[i] = 1.f; s[i] = 0.f;
    if (turned) {
      turn((double)pos[pl.axis[pair + i] * pos_axis] * pl.freq[pair + i], c[i], s[i]);
      if (pl.inverse) s[i] = -s[i];
    }
  }
}

// The two runs of a unit, rotated in place (F32: in float32; else rounded once).
template <int VP, bool F32 = false>
__device__ __forceinline__ void unit_rotate(bool neighbours, const float (&c)[VP], const float (&s)[VP],
                                            float (&a)[VP], float (&b)[VP]) {
  float r[2 * VP];
#pragma unroll
  for (int i = 0; i < VP; ++i) { r[i] = a[i]; r[VP + i] = b[i]; }
#pragma unroll
  for (int i = 0; i < VP; ++i) {
    const float x1 = neighbours ? r[2 * i] : a[i], x2 = neighbours ? r[2 * i + 1] : b[i];
    float y1, y2;
    if constexpr (F32) {
      y1 = fmaf(x1, c[i], -(x2 * s[i]));
      y2 = fmaf(x2, c[i], x1 * s[i]);
    } else {
      rotate(x1, x2, c[i], s[i], y1, y2);
    }
    if (neighbours) { r[2 * i] = y1; r[2 * i + 1] = y2; }
    else { r[i] = y1; r[VP + i] = y2; }
  }
#pragma unroll
  for (int i = 0; i < VP; ++i) { a[i] = r[i]; b[i] = r[VP + i]; }
}

// The workgroup's place in a grid of token blocks (block_grid).
__device__ __forceinline__ uint32_t block_of() { return blockIdx.z * gridDim.x + blockIdx.x; }

// A workgroup takes a run of tokens, one lane per unit of a token's row, and all
// heads of its slice (grid y) with the lane's cosines and sines in registers.
// Bound by memory: 16-byte accesses (VP = 4) where rot, d, strides and addresses
// allow them, single elements (VP = 1) otherwise.  8 heads x 32,768 tokens of a packed bf16
// projection to float32 (d = 128, three axes): 44 us, 4.5 TB/s.
template <int VP, typename XT, typename YT>
__global__ __launch_bounds__(256) void sfa_rope_kernel(RopePlan pl, RopeArgs a) {
  const int U = a.units, r = threadIdx.x / U, u = threadIdx.x - r * U;
  const uint32_t tok = block_of() * (uint32_t)(256 / U) + r;  // (B * n < 2^31, and the last block near it)
  if (r >= 256 / U || tok >= (uint32_t)(a.B * a.n)) return;
  const uint32_t b = a.B == 1 ? 0 : tok / (uint32_t)a.n, t = tok - b * a.n;
  const Unit<VP> un(pl, u);
  float c[VP], s[VP];
  unit_turns<VP>(pl, a.pos + b * a.pos_batch + t, a.pos_axis, un.turned, un.pair, c, s);
  const int h0 = blockIdx.y * a.heads, h1 = min(a.H, h0 + a.heads);
  const XT* x = (const XT*)a.x + b * a.xs[0] + h0 * a.xs[1] + t * a.xs[2];
  YT* y = (YT*)a.y + b * a.ys[0] + h0 * a.ys[1] + t * a.ys[2];
  for (int h = h0; h < h1; ++h, x += a.xs[1], y += a.ys[1]) {
    float p[VP], q[VP];
    load_vec<VP>(x + un.off0, p);
    if (un.n1 == VP) {
      load_vec<VP>(x + un.off1, q);
    } else {
#pragma unroll
      for (int i = 0; i < VP; ++i) q[i] = 0.f;
    }
    if (un.turned) unit_rotate<VP>(pl.neighbours, c, s, p, q);
    store_vec<VP>(y + un.off0, p);
    if (un.n1 == VP) store_vec<VP>(y + un.off1, q);
  }
}

// One wavefront codes one row at a time (as topk_encode_kernel), a token's heads
// in turn with the lane's cosines and sines in registers; the next row's loads
// are in flight while the current one is selected.  A coordinate's partner is
// loaded beside it, unless both lie in the lane already (SAME: pairing halves,
// rot = d = 128 or 256: coordinates l + 64 e and l + 64 (e + E/2)).
// IF, VF: output formats, or -1 to read them from the arguments.
// Bound by the scalar unit, 82% busy with the selection: 32 heads x 32,768 rows of 128
// float32, k = 16: 192 us, 3.5 TB/s.
template <int E, int IF, int VF, bool XB, bool SAME>
__global__ __launch_bounds__(256) void sfa_rope_encode_kernel(RopePlan pl, RopeArgs a) {
  __shared__ uint2 ent_lds[4][E <= 1 ? 64 : 64 * E];  // kept entries of R rows: bits, coordinate
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint2* ent = ent_lds[wave];
  const int ifmt = IF >= 0 ? IF : a.ifmt, vfmt = VF >= 0 ? VF : a.vfmt;
  const uint32_t ntok = (uint32_t)(a.B * a.n);  // (< 2^31)
  const int half = pl.rot / 2;
  constexpr int EP = SAME ? E / 2 : E;
  int axis[EP], part[EP];
  float sign[EP];
  double freq[EP];
  bool turned[EP];
#pragma unroll
  for (int e = 0; e < EP; ++e) {
    const int c = min(lane + 64 * e, a.d - 1);
    turned[e] = SAME || c < pl.rot;
    const bool second = pl.neighbours ? (c & 1) : c >= half;
    const int pair = turned[e] ? (pl.neighbours ? c >> 1 : (second ? c - half : c)) : 0;
    axis[e] = pl.axis[pair];
    freq[e] = pl.freq[pair];
    part[e] = !turned[e] ? c : pl.neighbours ? c ^ 1 : (second ? c - half : c + half);
    sign[e] = second ? 1.f : -1.f;
  }
  const uint32_t stride = gridDim.x * 4;
  uint32_t tok = blockIdx.x * 4 + wave;
  if (tok >= ntok) return;  // uniform per wave
  const int h0 = blockIdx.y * a.heads, h1 = min(a.H, h0 + a.heads);
  // Stores: as many rows (heads of one token) as have 64 entries, and at least one.  An
  // entry's lane is then its place in a row of its own, and a store instruction is whole
  // runs of k (stored from where they are selected, a row took two partial ones a format).
  const int R = a.k <= 64 ? 64 / a.k : 1;
  const int my_row = a.k <= 64 ? lane / a.k : 0;
  const int64_t row_step = (int64_t)a.n * a.k, my_off = my_row * row_step + (lane - my_row * a.k);
  // A row's words, and a token's positions, are loaded one row ahead, past the end
  // of a token's heads too.
  uint32_t nx[E], np[SAME ? 1 : E];
  auto load_row = [&](int64_t o) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = min(lane + 64 * e, a.d - 1);
      nx[e] = XB ? (uint32_t)((const uint16_t*)a.x + o)[c] : ((const uint32_t*)a.x + o)[c];
      if constexpr (!SAME)
        np[e] = XB ? (uint32_t)((const uint16_t*)a.x + o)[part[e]] : ((const uint32_t*)a.x + o)[part[e]];
    }
  };
  int npos[EP];
  uint32_t b, t;
  auto open_token = [&]() {
    b = a.B == 1 ? 0 : tok / (uint32_t)a.n;
    t = tok - b * a.n;
    const int32_t* pos = a.pos + b * a.pos_batch + t;
#pragma unroll
    for (int e = 0; e < EP; ++e) npos[e] = pos[axis[e] * a.pos_axis];
    load_row(b * a.xs[0] + t * a.xs[2] + h0 * a.xs[1]);
  };
  auto value = [](uint32_t v) { return XB ? bf16_bits_to_f32(v) : __uint_as_float(v); };
  open_token();
  while (true) {
    const int64_t x0 = b * a.xs[0] + t * a.xs[2], o_base = ((int64_t)b * a.H * a.n + t) * a.k;
    float co[EP], si[EP];
#pragma unroll
    for (int e = 0; e < EP; ++e) {
      turn((double)npos[e] * freq[e], co[e], si[e]);
      if (!SAME) si[e] *= sign[e];
    }
    tok += stride;  // (no wrap: ntok and the grid's wavefronts are below 2^31)
    const bool more = tok < ntok;
    int held = 0;
    for (int h = h0; h < h1; ++h) {
      uint32_t bits[E], key[E];
      if constexpr (SAME) {
#pragma unroll
        for (int e = 0; e < EP; ++e) {
          float y1, y2;
          rotate(value(nx[e]), value(nx[e + EP]), co[e], si[e], y1, y2);
          bits[e] = __float_as_uint(y1);
          bits[e + EP] = __float_as_uint(y2);
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float x = value(nx[e]);
          const float y = (float)fma((double)x, (double)co[e], (double)value(np[e]) * (double)si[e]);
          bits[e] = __float_as_uint(turned[e] ? y : x);
        }
      }
#pragma unroll
      for (int e = 0; e < E; ++e) key[e] = topk_key(bits[e], lane + 64 * e < a.d);
      if (h + 1 < h1) load_row(x0 + (h + 1) * a.xs[1]);
      else if (more) open_token();
      const uint32_t cut = topk_cut<E>(key, a.k);
      bool sel[E];
#pragma unroll
      for (int e = 0; e < E; ++e) sel[e] = key[e] >= cut;
      int slot[E];
      topk_slots<E>(sel, slot);
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (sel[e] && slot[e] < a.k) ent[held * a.k + slot[e]] = make_uint2(bits[e], lane + 64 * e);
      if (++held < R && h + 1 < h1) continue;
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      const int64_t o0 = o_base + (h + 1 - held) * row_step + my_off;
#pragma unroll
      for (int e = 0; e < E; ++e) {  // (more than one only where k > 64)
        const int i = lane + 64 * e;
        if (64 * e >= held * a.k) break;
        if (i < held * a.k) {
          const uint2 w = ent[i];
          store_code(a.idx, a.val, o0 + 64 * e, (int)w.y, w.x, ifmt, vfmt);
        }
      }
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      held = 0;
    }
    if (!more) break;
  }
}

// dx = R^T scatter(idx, dval).  A wavefront takes R = 64 / U tokens (U: units of a
// row), a lane one unit of one of them, and the heads of its slice in turn: the
// code entries, NE a lane and loaded a head ahead, are scattered into float32 rows
// of LDS, each lane reads its unit back, turns and stores it, and the entries'
// places are cleared again.  The rotation is float32 here (a product and an fma, off
// by 2^-24 of each term: no selection hangs on it).  Bound by memory: it writes d
// values for the k entries it reads (32 heads x 32,768 rows of 128 to bf16, k = 16: 89 us, 4.5
// TB/s).
constexpr int kBwdLds = 4 * 512;  // floats; a wavefront's R d are at most 512 (U >= d / 8), or d where U >= 64
template <int VP, int NE, typename YT>
__global__ __launch_bounds__(256) void sfa_rope_bwd_kernel(RopePlan pl, RopeArgs a) {
  __shared__ float rows_lds[kBwdLds];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float* rows = rows_lds + wave * (kBwdLds / 4);
  const int U = a.units, R = a.tokens, d = a.d;
  constexpr int NIT = VP == 1 ? 2 : 1;  // up to 128 units where VP = 1
  const uint32_t ntok = (uint32_t)(a.B * a.n), tok0 = (block_of() * 4 + wave) * (uint32_t)R;  // (as above)
  if (tok0 >= ntok) return;  // uniform per wave; no workgroup barrier below
  const int here = (int)min((uint32_t)R, ntok - tok0);
  const int h0 = blockIdx.y * a.heads, h1 = min(a.H, h0 + a.heads);

  // Entry e of the wave's tokens: token e / k (exact: e < 2^11, so (e + 1/2) / k is
  // 1/(2k) or more from an integer).  Lanes past the last entry repeat it.
  const float inv_k = 1.f / (float)a.k;
  int64_t at[NE];
  int place[NE], ci[NE];
  float cg[NE];
#pragma unroll
  for (int j = 0; j < NE; ++j) {
    const int e = min(lane + 64 * j, here * a.k - 1), r = (int)(((float)e + 0.5f) * inv_k);
    const uint32_t tok = tok0 + r, b = a.B == 1 ? 0 : tok / (uint32_t)a.n;
    at[j] = (((int64_t)b * a.H + h0) * a.n + (tok - b * a.n)) * a.k + (e - r * a.k);
    place[j] = r * d;
  }
  auto load_entries = [&]() {
#pragma unroll
    for (int j = 0; j < NE; ++j) {
      ci[j] = min(load_idx(a.idx, at[j], a.ifmt, 255), d - 1);
      cg[j] = a.dval[at[j]];
      at[j] += (int64_t)a.n * a.k;
    }
  };
  load_entries();
  for (int i = lane; i < R * d; i += 64) rows[i] = 0.f;

  float c[NIT][VP], s[NIT][VP];
  int row[NIT], off0[NIT], off1[NIT];
  bool two[NIT], turned[NIT];
  int64_t yo[NIT];
#pragma unroll
  for (int it = 0; it < NIT; ++it) {
    const int v = min(lane + 64 * it, here * U - 1);  // lanes past the last unit repeat it: no branch around the
    row[it] = v / U;                                   // stores, so a wait for the entries is not one for them too
    const Unit<VP> un(pl, v - row[it] * U);
    const uint32_t tok = tok0 + row[it];
    const uint32_t b = a.B == 1 ? 0 : tok / (uint32_t)a.n, t = tok - b * a.n;
    off0[it] = un.off0; off1[it] = un.off1; two[it] = VP == 4 || un.n1 == VP; turned[it] = un.turned;
    unit_turns<VP>(pl, a.pos + b * a.pos_batch + t, a.pos_axis, un.turned, un.pair, c[it], s[it]);
    yo[it] = b * a.ys[0] + t * a.ys[2] + h0 * a.ys[1];
  }
  for (int h = h0; h < h1; ++h) {
    int here_at[NE];
#pragma unroll
    for (int j = 0; j < NE; ++j) {
      here_at[j] = place[j] + ci[j];
      rows[here_at[j]] = cg[j];
    }
    if (h + 1 < h1) load_entries();
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int it = 0; it < NIT; ++it) {
      if (it > 0 && here * U <= 64 * it) break;  // uniform
      float p[VP], q[VP];
      const float* src = rows + row[it] * d;
      load_vec<VP>(src + off0[it], p);
      if (two[it]) load_vec<VP>(src + off1[it], q);
      else {
#pragma unroll
        for (int i = 0; i < VP; ++i) q[i] = 0.f;
      }
      if (turned[it]) unit_rotate<VP, true>(pl.neighbours, c[it], s[it], p, q);
      YT* y = (YT*)a.y + yo[it];
      store_vec<VP>(y + off0[it], p);
      if (two[it]) store_vec<VP>(y + off1[it], q);
      yo[it] += a.ys[1];
    }
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int j = 0; j < NE; ++j) rows[here_at[j]] = 0.f;
  }
}

// Whether rows can be read and written four elements at a time: units of four
// pairs (or eight copied coordinates) tile the row, and every row starts on a
// four-element boundary (32 heads x 32,768 tokens, d = 128, bf16 rows 136 apart, from the
// first coordinate and from the second: rotation 165 and 175 us, backward 130 and 217).
bool vec_rows(const RopePlan& pl, const void* p, const int64_t* st, int bytes) {
  return ((uintptr_t)p % (4 * bytes)) == 0 && (st[0] | st[1] | st[2]) % 4 == 0 && pl.rot % 8 == 0 &&
         (pl.d - pl.rot) % 8 == 0;
}

int units_of(const RopePlan& pl, int vp) { return pl.rot / 2 / vp + (pl.d - pl.rot + 2 * vp - 1) / (2 * vp); }

// Heads per slice: all of a token's where the tokens alone fill the chip with
// `want` workgroups, else as few as make that many.
int heads_per_slice(int64_t blocks, int H, int64_t want) {
  int64_t slices = (want + blocks - 1) / blocks;
  if (slices > H) slices = H;
  if (slices > 65535) slices = 65535;
  return (int)((H + slices - 1) / slices);
}

// Token blocks by slices of the heads.  A grid dimension holds less than 2^32 threads:
// blocks past 2^20 go to the third, in equal parts.
dim3 block_grid(int64_t blocks, int slices) {
  const int64_t z = (blocks + (1 << 20) - 1) >> 20;
  return dim3((unsigned)((blocks + z - 1) / z), (unsigned)slices, (unsigned)z);
}

template <int VP>
void launch_rope_t(const RopePlan& pl, const RopeArgs& a, dim3 grid, hipStream_t stream) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, pl, a); };
  if (a.xbf16) a.ybf16 ? go(sfa_rope_kernel<VP, uint16_t, uint16_t>) : go(sfa_rope_kernel<VP, uint16_t, float>);
  else a.ybf16 ? go(sfa_rope_kernel<VP, float, uint16_t>) : go(sfa_rope_kernel<VP, float, float>);
}

template <int E, bool XB, bool SAME>
void launch_encode_f(const RopePlan& pl, const RopeArgs& a, dim3 grid, hipStream_t stream) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, pl, a); };
  if (a.ifmt == kIdxI32 && a.vfmt == kValF32) go(sfa_rope_encode_kernel<E, kIdxI32, kValF32, XB, SAME>);
  else if (a.ifmt == kIdxI16 && a.vfmt == kValBF16) go(sfa_rope_encode_kernel<E, kIdxI16, kValBF16, XB, SAME>);
  else if (a.ifmt == kIdxU8 && a.vfmt == kValF16) go(sfa_rope_encode_kernel<E, kIdxU8, kValF16, XB, SAME>);
  else go(sfa_rope_encode_kernel<E, -1, -1, XB, SAME>);
}

template <int E, bool XB>
void launch_encode_s(const RopePlan& pl, const RopeArgs& a, dim3 grid, hipStream_t stream) {
  if constexpr (E > 1) {
    if (!pl.neighbours && pl.rot == pl.d && pl.d == 64 * E) return launch_encode_f<E, XB, true>(pl, a, grid, stream);
  }
  launch_encode_f<E, XB, false>(pl, a, grid, stream);
}

template <bool XB>
void launch_encode_e(const RopePlan& pl, const RopeArgs& a, dim3 grid, hipStream_t stream) {
  if (a.d <= 64) launch_encode_s<1, XB>(pl, a, grid, stream);
  else if (a.d <= 128) launch_encode_s<2, XB>(pl, a, grid, stream);
  else launch_encode_s<4, XB>(pl, a, grid, stream);
}

template <int VP, int NE>
void launch_bwd_t(const RopePlan& pl, const RopeArgs& a, dim3 grid, hipStream_t stream) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, pl, a); };
  if (a.ybf16) go(sfa_rope_bwd_kernel<VP, NE, uint16_t>);
  else go(sfa_rope_bwd_kernel<VP, NE, float>);
}

}  // namespace

hipError_t launch_rope(const RopePlan& pl, RopeArgs a, hipStream_t stream) {
  const bool vec = vec_rows(pl, a.x, a.xs, a.xbf16 ? 2 : 4) && vec_rows(pl, a.y, a.ys, a.ybf16 ? 2 : 4);
  a.units = units_of(pl, vec ? 4 : 1);
  const int per = 256 / a.units;
  const int64_t blocks = ((int64_t)a.B * a.n + per - 1) / per;
  a.heads = heads_per_slice(blocks, a.H, 2048);
  const dim3 grid = block_grid(blocks, (a.H + a.heads - 1) / a.heads);
  if (vec) launch_rope_t<4>(pl, a, grid, stream);
  else launch_rope_t<1>(pl, a, grid, stream);
  return hipGetLastError();
}

hipError_t launch_rope_encode(const RopePlan& pl, RopeArgs a, hipStream_t stream) {
  // A wavefront takes the heads of one token, about 32 rows (several tokens where
  // the heads are fewer), and leaves the rest to the dispatcher: in a grid that just
  // fills the chip, wavefronts of equal shares end far apart (32 heads x 32,768
  // tokens: 275 us with 8192 wavefronts of four tokens, 221 with 32,768 of one).
  const int64_t ntok = (int64_t)a.B * a.n;
  a.heads = heads_per_slice(ntok, a.H, 4 * 2048);
  const int64_t slices = (a.H + a.heads - 1) / a.heads, need = (ntok + 3) / 4;
  const int64_t per = a.heads >= 32 ? 1 : 32 / a.heads, full = (2047 + slices) / slices;
  const int64_t filled = need < full ? need : full, blocks = (need + per - 1) / per;
  const int64_t most = blocks > filled ? blocks : filled;
  const dim3 grid((unsigned)(most < 1 << 22 ? most : 1 << 22), (unsigned)slices);  // (as block_grid: 2^32 threads)
  if (a.xbf16) launch_encode_e<true>(pl, a, grid, stream);
  else launch_encode_e<false>(pl, a, grid, stream);
  return hipGetLastError();
}

hipError_t launch_rope_encode_bwd(const RopePlan& pl, RopeArgs a, hipStream_t stream) {
  const bool vec = vec_rows(pl, a.y, a.ys, a.ybf16 ? 2 : 4) && a.d % 4 == 0;
  a.units = units_of(pl, vec ? 4 : 1);
  a.tokens = a.units >= 64 ? 1 : 64 / a.units;
  const int64_t blocks = ((int64_t)a.B * a.n + 4 * a.tokens - 1) / (4 * a.tokens);
  // (32 heads, 32,768 tokens: 89 us in one slice, 98 in four, 126 in sixteen, each with its
  // sines again; 12 heads, 8 x 1024 tokens at d = 64: 11.0 with three heads a slice,
  // 14.5 with one, 15.8 with all)
  a.heads = heads_per_slice(blocks, a.H, 2048);
  if (a.heads < 3) a.heads = a.H < 3 ? a.H : 3;
  const dim3 grid = block_grid(blocks, (a.H + a.heads - 1) / a.heads);
  // code entries a lane holds: at most 64 k / U, k <= 8 U (VP = 4) or 2 U
  const int ne = (a.tokens * a.k + 63) / 64;
  if (vec) {
    if (ne <= 1) launch_bwd_t<4, 1>(pl, a, grid, stream);
    else if (ne <= 2) launch_bwd_t<4, 2>(pl, a, grid, stream);
    else if (ne <= 4) launch_bwd_t<4, 4>(pl, a, grid, stream);
    else launch_bwd_t<4, 8>(pl, a, grid, stream);
  } else {
    if (ne <= 1) launch_bwd_t<1, 1>(pl, a, grid, stream);
    else launch_bwd_t<1, 4>(pl, a, grid, stream);
  }
  return hipGetLastError();
}

}  // namespace sfa
