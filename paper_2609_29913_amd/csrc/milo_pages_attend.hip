// Attention over the paged 8-bit cache (include/milo.h: milo_attend_pages):
//   out = sum_r 2^(x_r) v_r / sum_r 2^(x_r),  x_r = scale log2(e) s_page (q . code_r)
// in one pass over the rows, with the exponent m that the sums are relative to
// (Running).  The codes go from memory straight into registers in the order the
// matrix instructions take them, are converted there and used by all columns (query
// x head of one KV head) of a tile; the scores' registers are, as they stand, the
// weights' operand of the value product, so nothing goes through LDS but the sums of
// waves that share a tile.
// Bounds, with measured times between calls:
//  - few columns a tile: the cache is read once.  14B heads, 64 requests of 8192 rows,
//    E4M3: 1.08 GB in 182 .. 186 us, 5.8 TB/s, where a copy moves 5.1 (half of it
//    writes); 7B heads, 32 requests of 257 .. 16384 rows, INT8: 0.28 GB in 63 us, 4.4
//    TB/s, of which 5 are the join and about 5 the start.  One request of 131001 rows:
//    0.13 GB in 39 us, 28 of them reading (4.8 TB/s), 6 the join of 64 parts a tile.
//  - many columns: the vector units and the matrix units together, which hardly
//    overlap here (2048 queries, the last of 8192 rows, 7B heads, E4M3: 232 us, 905
//    TFLOP/s, where a matrix product of 16384^3 reaches 1328; the matrix units are busy
//    39% of the cycles, the vector units issue in 69% of them).  Half of the vector
//    instructions are the codes' conversions, which INT8 needs more of (about 300 us).
//  - in between (32 columns): the longest tile (8 requests of 100 .. 3000 rows, 1 .. 37
//    queries that see all of them, 14B heads: 27 us; the first tiles end after 9).
//  - one short request: the launch (9 us between calls, 7 on the GPU).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "milo_attend.h"
#include "milo_pages.h"

namespace milo {
namespace {

constexpr int kPagesThreads = 256;   // four waves
constexpr int kPagesWaves = kPagesThreads / 64;
constexpr int kLeastShare = 4;       // positions (64 rows each) of a share, as a rule
constexpr int kLongShare = 24;       // and before every CU gets a second one

struct PagesArgs {
  milo_pages p;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* starts;   // NULL: request i's only query is row i
  const uint16_t* q;
  void* out;
  const float* ctx_o;      // [n_tok * H_q][d] attention over the compressed context (NULL: none)
  const float2* ctx_ml;    // its maximum in log2 units and its sum
  int64_t q_stride;
  float* part_o;           // [2 grid][columns of a tile][d] parts of tiles that workgroups share
  float2* part_ml;         // their maxima (log2 units) and sums
  int4* meta;              // [grid] the tile that begins in a workgroup and ends in a later one
  float qscale;            // scale * log2(e)
  int32_t least_tiles;     // what the host knows of the number of tiles
  uint32_t G_inv, tt_inv;  // ceil(2^16 / G), ceil(2^32 / tt) (tiles_of)
  int32_t whole_tiles;     // 1: a workgroup takes one whole tile, no shares
  int32_t n_req, n_tok, H_q, G, width, lg_page, causal, out_bf16;
};

__device__ inline int start_of(const PagesArgs& a, int i) {
  return a.starts ? min(max(a.starts[i], 0), a.n_tok) : i;
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// eight codes as bf16, exactly
template <int FMT>
__device__ __forceinline__ bf16x8 codes_bf16(uint32_t lo, uint32_t hi) {
  bf16x8 v;
  if constexpr (FMT == MILO_KV_INT8) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = (__bf16)(float)(int8_t)(lo >> (8 * e));
      v[4 + e] = (__bf16)(float)(int8_t)(hi >> (8 * e));
    }
  } else {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1];
    v[4] = c[0]; v[5] = c[1]; v[6] = d[0]; v[7] = d[1];
  }
  return v;
}

// eight codes as fp16, exactly.  INT8: with the sign bit turned, byte u = code + 128
// under the high byte 0x64 is the fp16 value 1024 + u.
template <int FMT>
__device__ __forceinline__ f16x8 codes_f16(uint32_t lo, uint32_t hi) {
  f16x2 x[4];
  if constexpr (FMT == MILO_KV_INT8) {
    const f16x2 off = {(_Float16)1152.f, (_Float16)1152.f};
    lo ^= 0x80808080u;
    hi ^= 0x80808080u;
    x[0] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u)) - off;
    x[1] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u)) - off;
    x[2] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u)) - off;
    x[3] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u)) - off;
  } else {
    x[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false);
    x[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
    x[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false);
    x[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
  }
  return f16x8{x[0][0], x[0][1], x[1][0], x[1][1], x[2][0], x[2][1], x[3][0], x[3][1]};
}

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int lane_of(int v, int l) { return __builtin_amdgcn_readlane(v, l); }
__device__ __forceinline__ float lane_of(float v, int l) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l));
}

__device__ inline Request request_of(const PagesArgs& a, int r) {
  Request q;
  q.start = start_of(a, r);
  q.m = a.starts ? max(0, start_of(a, r + 1) - q.start) : 1;
  q.n = (int)min((int64_t)max(a.lens[r], 0), (int64_t)a.width << a.lg_page);
  return q;
}

// column c < 256 of a tile: its query and head (c < 256 and G <= 16: exact)
__device__ inline int col_token(const PagesArgs& a, int c) { return (int)(c * a.G_inv >> 16); }
__device__ inline int64_t col_offset(const PagesArgs& a, int c) {
  const int tok = col_token(a, c);
  return (int64_t)tok * a.H_q + c - tok * a.G;
}

// merges a column's result with the compressed context's and stores 4 dims of it
__device__ inline void finish(const PagesArgs& a, int64_t col, int d, int D, float m, float l, float4 o) {
  if (a.ctx_ml) {
    const float2 cm = a.ctx_ml[col];
    const float4 co = *reinterpret_cast<const float4*>(a.ctx_o + col * D + d);
    const float mx = fmaxf(m, cm.x);
    const float fp = m == -INFINITY ? (l == 0.f ? 0.f : l) : exp2_hw(m - mx), fc = exp2_hw(cm.x - mx) * cm.y;
    l = l * fp + fc;
    o.x = o.x * fp + co.x * fc;
    o.y = o.y * fp + co.y * fc;
    o.z = o.z * fp + co.z * fc;
    o.w = o.w * fp + co.w * fc;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  o.x *= inv;
  o.y *= inv;
  o.z *= inv;
  o.w *= inv;
  if (a.out_bf16) {
    uint2 w;
    w.x = bf16_bits(o.x) | bf16_bits(o.y) << 16;
    w.y = bf16_bits(o.z) | bf16_bits(o.w) << 16;
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + col * D + d) = w;
  } else {
    *reinterpret_cast<float4*>(static_cast<float*>(a.out) + col * D + d) = o;
  }
}

// Pages of one request as a wave reads them: lane i holds where the head's codes of page
// base + i begin and its scales, so a step takes them without waiting for memory.  The values' scale stands
// as its logarithm, which joins the score (see add_step), and as its reciprocal; a
// page of less than 2^-96 (none at all, as a rule) adds no values: it counts with the least
// of the other scales, and its reciprocal is negative.
struct Window {
  int base, id;
  uint32_t lo, hi;  // first byte of the page and head
  float ks;        // scale of the keys, times the call's, in log2 units
  float lv, rv;    // log2 of the values' scale, 1 / scale
};
constexpr float kMinValueScale = 1.262177448e-29f;  // 2^-96
__device__ __forceinline__ bool no_values(float rv) { return __float_as_int(rv) < 0; }

// Ids first, so that the codes' loads need not wait for the scales.
__device__ inline void window_ids(const PagesArgs& a, int req, int base, int last_page, Window& w) {
  w.base = base;
  w.id = a.table[(int64_t)req * a.width + min(base + (int)(threadIdx.x & 63), last_page)];
}

template <int D>
__device__ inline void window_loads(const PagesArgs& a, int head, Window& w) {
  const bool in = (uint32_t)w.id < (uint32_t)a.p.n_pages;
  if (!in) w.id = 0;
  const int64_t at = (int64_t)w.id * a.p.n_kv_heads + head, byte = (at << a.lg_page) * D;
  w.lo = (uint32_t)byte;
  w.hi = (uint32_t)(byte >> 32);
  w.ks = a.p.k_scale[at];
  w.lv = a.p.v_scale[at];
  w.rv = in ? 1.f : __uint_as_float(0x7FC00000u);
}

__device__ inline void window_scales(const PagesArgs& a, Window& w) {
  const float vs = w.lv, bad = w.rv;  // bad: 1, or NaN where the page is none
  w.ks *= a.qscale * bad;
  w.lv = __builtin_amdgcn_logf(vs);
  w.rv = vs == vs ? exp2_hw(-w.lv) : 1.f;
  const bool none = vs < kMinValueScale;
  if (__any(none)) {
    float least = none || vs != vs ? INFINITY : w.lv;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) least = fminf(least, __shfl_xor(least, o));
    if (least == INFINITY) least = 0.f;
    if (none) {
      w.lv = least;
      w.rv = -exp2_hw(-least);
    }
  }
}

// One step's codes (GS groups of 16 rows) and scales.
template <int D, int GS>
struct Step {
  uint4 k[GS][D / 64], v[GS][D / 64];
  float ks[GS], lv[GS], rv[GS];
  bool plain;  // every page adds values
};

template <int D, int GS>
__device__ __forceinline__ void load_codes(const PagesArgs& a, int head, const Window& w, int row, int last_page,
                                           Step<D, GS>& st) {
  const uint32_t lane16 = 16 * (threadIdx.x & 63);
#pragma unroll
  for (int g = 0; g < GS; ++g) {
    const int r = row + 16 * g, li = min(r >> a.lg_page, last_page) - w.base;
    const int64_t at = ((int64_t)lane_of((int)w.hi, li) << 32 | (uint32_t)lane_of((int)w.lo, li)) +
                       (r & ((1 << a.lg_page) - 1)) * D;
    const uint8_t* kp = static_cast<const uint8_t*>(a.p.k_codes) + at;
    const uint8_t* vp = static_cast<const uint8_t*>(a.p.v_codes) + at;
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
      st.k[g][j] = *reinterpret_cast<const uint4*>(kp + 1024 * j + lane16);
      st.v[g][j] = *reinterpret_cast<const uint4*>(vp + 1024 * j + lane16);
    }
  }
}

template <int D, int GS>
__device__ __forceinline__ void take_scales(const PagesArgs& a, const Window& w, int row, int last_page, Step<D, GS>& st) {
  st.plain = true;
#pragma unroll
  for (int g = 0; g < GS; ++g) {
    const int li = min((row + 16 * g) >> a.lg_page, last_page) - w.base;
    st.ks[g] = lane_of(w.ks, li);
    st.lv[g] = lane_of(w.lv, li);
    st.rv[g] = lane_of(w.rv, li);
    st.plain &= !no_values(st.rv[g]);
  }
}

template <int D, int GS>
__device__ __forceinline__ void load_step(const PagesArgs& a, int req, int head, Window& w, int row, int last_page,
                                          Step<D, GS>& st) {
  if ((row >> a.lg_page) - w.base >= 64) {
    window_ids(a, req, row >> a.lg_page, last_page, w);
    window_loads<D>(a, head, w);
    window_scales(a, w);
  }
  load_codes(a, head, w, row, last_page, st);
  take_scales(a, w, row, last_page, st);
}

// A wave's running softmax over NT tiles of 16 columns: lane (n = l % 16, q = l / 16)
// holds of column n the exponent m that sums are relative to (all four q alike, -inf
// before any row), its own part of the sum, and dims
// 16 t + 4 q .. + 3 of the outputs.
template <int D, int NT>
struct Running {
  f32x4 o[NT][D / 16];
  float m[NT], l[NT];
};

// Adds a step's rows.  Scores: 16x16x32 products keys x queries, so lane (n, q) holds
// rows 4 q .. 4 q + 3 of each group for column n; two groups' weights are, as they
// stand, the right operand of the product with the values' 32 rows in the order the
// codes are stored in.  A row's weight is taken with its values' scale, 2^(s + log2 v),
// to 2^m, m at first 7 below the largest such exponent: fp16 then holds it with 2^-11
// (2^-22 in two parts) of itself or, if it is less than 2^-21 of the largest, with 2^-32 of
// that, whatever the pages' scales; the sum takes the scale out again.  m moves only when
// a weight passes 2^15, which fp16 still holds.
template <bool MASKED, int D, int FMT, int PARTS, int NT, int GS>
__device__ __forceinline__ void add_step(const Step<D, GS>& st, const bf16x8 (&qf)[NT][D / 32], int row,
                                         int n, const int (&vis)[NT], Running<D, NT>& run) {
  const int lane = threadIdx.x & 63, q4 = (lane >> 4) * 4;
  // products first where two waves compete: the other's arithmetic fills the gaps (5%)
  __builtin_amdgcn_s_setprio(1);
  // two groups at a time: as many independent sums as hide a product's latency
  f32x4 s[GS][NT];
#pragma unroll
  for (int g0 = 0; g0 < GS; g0 += 2) {
#pragma unroll
    for (int g = g0; g < g0 + 2; ++g)
#pragma unroll
      for (int t = 0; t < NT; ++t) s[g][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < D / 64; ++j)
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int g = g0; g < g0 + 2; ++g) {
          const uint4& raw = st.k[g][j];
          const bf16x8 kf = half == 0 ? codes_bf16<FMT>(raw.x, raw.y) : codes_bf16<FMT>(raw.z, raw.w);
#pragma unroll
          for (int t = 0; t < NT; ++t) s[g][t] = mfma16(kf, qf[t][2 * j + half], s[g][t]);
        }
    __builtin_amdgcn_sched_barrier(0);
  }
  __builtin_amdgcn_s_setprio(0);
  // the conversions of the phases stay in them: moved up, they cost registers (spills)
  __builtin_amdgcn_sched_barrier(0);
  // exponents of the weights, relative to m (0 before any row)
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const float m0 = run.m[t] == -INFINITY ? 0.f : run.m[t];
    float mx = -INFINITY;
#pragma unroll
    for (int g = 0; g < GS; ++g) {
      const float base = st.lv[g] - m0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x = fmaf(s[g][t][i], st.ks[g], base);
        if (MASKED && row + 16 * g + q4 + i >= vis[t]) x = -INFINITY;
        s[g][t][i] = x;
        mx = fmaxf(mx, x);
      }
    }
    if (__any(mx > (run.m[t] == -INFINITY ? -INFINITY : 15.f))) {
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      // up by what the largest passes 2^7 (from none: there, up or down)
      const float up = mx == -INFINITY ? 0.f : run.m[t] == -INFINITY ? mx - 7.f : fmaxf(mx - 7.f, 0.f);
      const float f = run.m[t] == -INFINITY ? 0.f : exp2_hw(-up);
      if (mx != -INFINITY) run.m[t] = m0 + up;
      run.l[t] *= f;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) run.o[t][c] *= f;
#pragma unroll
      for (int g = 0; g < GS; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[g][t][i] -= up;
    }
  }
  f16x8 w[GS / 2][NT][PARTS];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
#pragma unroll
    for (int g = 0; g < GS; ++g) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x = exp2_hw(s[g][t][i]);
        const int e = (g & 1) * 4 + i;
        sum += x;
        if (MASKED && no_values(st.rv[g])) x = 0.f;
        w[g / 2][t][0][e] = (_Float16)x;
        if constexpr (PARTS == 2) w[g / 2][t][1][e] = (_Float16)(x - (float)w[g / 2][t][0][e]);
      }
      run.l[t] = fmaf(sum, MASKED ? fabsf(st.rv[g]) : st.rv[g], run.l[t]);
    }
  }
  __builtin_amdgcn_s_setprio(1);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int g = 0; g < GS; g += 2) {
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
      __builtin_amdgcn_sched_barrier(0);
      uint32_t va[4] = {st.v[g][j].x, st.v[g][j].y, st.v[g][j].z, st.v[g][j].w};
      uint32_t vb[4] = {st.v[g + 1][j].x, st.v[g + 1][j].y, st.v[g + 1][j].z, st.v[g + 1][j].w};
      if constexpr (FMT == MILO_KV_E4M3 && MASKED) {  // rows behind the request's last hold anything, NaN among it
        const int na = min(max(n - row - 16 * g - q4, 0), 4), nb = min(max(n - row - 16 * g - 16 - q4, 0), 4);
        const uint32_t ka = na == 4 ? ~0u : (1u << 8 * na) - 1u, kb = nb == 4 ? ~0u : (1u << 8 * nb) - 1u;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          va[c] &= ka;
          vb[c] &= kb;
        }
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const f16x8 vf = codes_f16<FMT>(va[c], vb[c]);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int p = 0; p < PARTS; ++p) run.o[t][4 * j + c] = mfma16(vf, w[g / 2][t][p], run.o[t][4 * j + c]);
      }
    }
  }
  __builtin_amdgcn_s_setprio(0);
}

// One workgroup's share of the call: the tiles, or parts of tiles, between two positions
// (milo_pages.h).  SHARE: its waves split a tile's rows (16 NT columns) and join their
// sums through LDS, else its columns (64 NT columns, every wave reads all rows, three of
// four times from L1).  Two waves to a SIMD, 256 registers each: with one of 64 columns
// the 2048-query chunk takes 367 us against 266 at the time, since nothing then fills a
// wave's waits.  Rows are read a step ahead, 64 of them at 16 columns, else 32.
template <int D, int FMT, int PARTS, int NT, bool SHARE>
__global__ __launch_bounds__(kPagesThreads, 2) void pages_kernel(PagesArgs a) {
  constexpr int GS = NT == 1 ? 4 : 2, ROWS = 16 * GS;
  constexpr int COLS = SHARE ? 16 * NT : 16 * NT * kPagesWaves;
  constexpr int OS = D + 4;  // row stride of a column's partial in LDS
  __shared__ uint32_t wave_cost[kPagesWaves];
  __shared__ Place begin;
  __shared__ Request reqs[kPagesThreads];  // all of them where there are no more than threads
  // two sets in turn: a wave writes a tile's while others still read the last one's
  __shared__ float joined[2][2][kPagesWaves][16 * NT];
  // waves' sums on their way together: all four waves', or, of 32 columns, two at a time
  constexpr int PW = NT == 1 ? kPagesWaves : kPagesWaves / 2;
  __shared__ __align__(16) float part[SHARE ? PW * 16 * NT * OS : 4];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int tt = COLS / a.G, H = a.p.n_kv_heads;

  // the call's work and this workgroup's share of it
  const int chunk = (a.n_req + kPagesThreads - 1) / kPagesThreads;
  const auto get = [&](int r) {
    const Request q = chunk == 1 ? reqs[r] : request_of(a, r);
    return Request{q.start, q.m, q.n};
  };
  // (sums that stop at 2^32 - 1: only q_starts that are no running sums get there)
  uint32_t own = 0;  // of this thread's requests
  for (int r = tid * chunk; r < min((tid + 1) * chunk, a.n_req); ++r) {
    const Request q = request_of(a, r);
    if (chunk == 1) reqs[tid] = q;
    const int all = tiles_of(q.m, tt, a.tt_inv);
    own = sat_add(own, a.whole_tiles ? all : tiles_cost(q, all, all, tt, a.causal));
  }
  if ((uint64_t)own * H >> 32) own = ~0u;
  else own *= H;
  uint32_t upto = wave_scan(own);
  if (lane == 63) wave_cost[wave] = upto;
  __syncthreads();
  uint32_t sum = 0;
#pragma unroll
  for (int k = 0; k < kPagesWaves; ++k) {
    const uint32_t c = wave_cost[k];
    if (k < wave) upto = sat_add(upto, c);
    sum = sat_add(sum, c);
  }
  const int X = uniform(sum > INT32_MAX / 2 ? 0 : (int)sum);
  if (a.whole_tiles && (int)blockIdx.x >= X) return;
  // As many shares as keep kLeastShare each, up to one a CU, or two of kLongShare (8 requests
  // of 9000 rows, 14B heads: 37.5 us in 256 shares of 37 positions, 42.9 in 512 of 18; 32
  // requests of 8320 on average, 7B heads, 71.7 in 256, 65.1 in 512 of 33), not in between,
  // where some CUs have twice the others' work; one for a tile where that is about as many, so
  // that tiles of like length are not cut.
  int W = X / kLeastShare;
  if (W < 2 * a.least_tiles) W = a.least_tiles;
  else if (W > (int)gridDim.x / 2) W = X < kLongShare * (int)gridDim.x ? gridDim.x / 2 : gridDim.x;
  W = min(min((int)gridDim.x, W), X / kTileCost);
  if (W >= kXcds) W -= W % kXcds;
  W = max(W, 1);
  const int L = uniform((int)((uint32_t)(X + W - 1) / (uint32_t)W));
  // A sixth more for the first workgroup of a CU and less for the second where tiles are cut
  // anyway (2048-query chunk 254 -> 243 us, 32 requests of 8320 rows on average, 14B heads,
  // 122 -> 111; as many uniform tiles as shares, which this would cut: 186 -> 193).
  const int La = W == 2 * kCus && a.least_tiles < W ? L + L / 6 : L;
  int4* meta = a.meta + blockIdx.x;
  // consecutive shares on one XCD, whose L2 then holds the rows that tiles share
  const int w = W >= kXcds ? (int)(blockIdx.x % kXcds) * (W / kXcds) + blockIdx.x / kXcds : blockIdx.x;
  int b0 = blockIdx.x, b1 = 0;
  if (!a.whole_tiles) {
    if (tid == 0) *meta = make_int4(-1, 0, 0, 0);
    if ((int)blockIdx.x >= W) return;
    b0 = (int)min((int64_t)X, share_at(w, L, La));
    b1 = (int)min((int64_t)X, share_at(w + 1, L, La));
    if (b0 >= b1) return;
  }

  // The thread one of whose requests holds position b0 finds the tile.
  if ((uint32_t)b0 < upto && (uint32_t)b0 >= upto - own) {
    Place at;
    if (!a.whole_tiles) {
      at = place_of(get, tid * chunk, (int)(upto - own), b0, H, tt, a.tt_inv, a.causal);
    } else {  // a request's last tiles, which see most, first; its heads side by side
      int x = b0 - (int)(upto - own);
      for (at.r = tid * chunk;; ++at.r) {
        at.rq = get(at.r);
        at.all = tiles_of(at.rq.m, tt, a.tt_inv);
        if (x < H * at.all) break;
        x -= H * at.all;
      }
      at.head = x % H;
      at.tile = at.all - 1 - x / H;
      at.head0 = at.cost = at.p0 = 0;
      at.p1 = 1;  // the whole of what the workgroup does
    }
    begin = at;
  }
  __syncthreads();
  Place at{uniform(begin.r), uniform(begin.head), uniform(begin.tile), uniform(begin.all), uniform(begin.p0),
           uniform(begin.p1), uniform(begin.head0), uniform(begin.cost),
           Request{uniform(begin.rq.start), uniform(begin.rq.m), uniform(begin.rq.n)}};
  if (a.whole_tiles) b0 = 0, b1 = 1;
  bool first = true;
  int parity = 0;
  for (int pos = b0; pos < b1;) {
    const int j0 = uniform(at.tile * tt), ntok = uniform(min(tt, at.rq.m - at.tile * tt)), n = uniform(at.rq.n);
    const int req = uniform(at.r), g = uniform(at.head), start = uniform(at.rq.start), m = uniform(at.rq.m);
    const int vis_hi = uniform(seen_upto(at.rq, j0 + ntok, a.causal));
    const int p0 = uniform(at.p0), p1 = uniform(at.p1);
    const int ra = uniform(row_at(b0, p0, p1, vis_hi)), rb = uniform(row_at(b1, p0, p1, vis_hi));
    const bool whole = b0 <= p0 && b1 >= p1;
    const int slot = 2 * w + (first ? 0 : 1);

    // this wave's rows and columns
    const int col0 = SHARE ? 0 : wave * 16 * NT, ncol = ntok * a.G;
    const int64_t q0 = (int64_t)(start + j0) * a.H_q + g * a.G;  // the tile's first column in out
    int wa = ra, wb = rb;
    if (SHARE) {
      const int steps = (rb - ra + ROWS - 1) / ROWS;
      wa = ra + steps * wave / kPagesWaves * ROWS;
      wb = min(rb, ra + steps * (wave + 1) / kPagesWaves * ROWS);
    }
    const bool works = wa < wb && col0 < ncol;
    const int last_page = (n - 1) >> a.lg_page;
    Window win;
    if (works) window_ids(a, req, wa >> a.lg_page, last_page, win);
    Running<D, NT> run;
    int vis[NT], vis_lo = n;
    bf16x8 qf[NT][D / 32];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int c = col0 + 16 * t + (lane & 15), tok = col_token(a, c);
      vis[t] = 0;
#pragma unroll
      for (int k = 0; k < D / 32; ++k) qf[t][k] = bf16x8{};
      if (c < ncol) {
        const Request me{start, m, n};
        vis[t] = seen_upto(me, j0 + tok + 1, a.causal);
        const uint16_t* src = a.q + (int64_t)(start + j0 + tok) * a.q_stride + (int64_t)(g * a.G + c - tok * a.G) * D;
#pragma unroll
        for (int k = 0; k < D / 32; ++k)
          qf[t][k] = *reinterpret_cast<const bf16x8*>(src + 64 * (k / 2) + 16 * (lane >> 4) + 8 * (k % 2));
      }
      run.m[t] = -INFINITY;
      run.l[t] = 0.f;
#pragma unroll
      for (int c2 = 0; c2 < D / 16; ++c2) run.o[t][c2] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // steps below vis_lo need no mask: the fewest rows a column of this wave sees
    if (col0 < ncol) {
      const Request me{start, m, n};
      vis_lo = seen_upto(me, j0 + col_token(a, col0) + 1, a.causal);
    }
    vis_lo = uniform(vis_lo);
    wa = uniform(wa);
    wb = uniform(wb);
    if (works) {
      Step<D, GS> s0, s1;
      window_loads<D>(a, g, win);
      load_codes(a, g, win, wa, last_page, s0);
      window_scales(a, win);
      take_scales(a, win, wa, last_page, s0);
      int row = wa;
      for (; row + 2 * ROWS <= min(vis_lo, wb) && s0.plain; row += 2 * ROWS) {
        load_step(a, req, g, win, row + ROWS, last_page, s1);
        add_step<false, D, FMT, PARTS, NT, GS>(s0, qf, row, n, vis, run);
        if (!s1.plain) {
          s0 = s1;
          row += ROWS;
          break;
        }
        // (the same rows again behind the last: a load that may not be there makes the compiler
        // wait for the newest one in its stead)
        load_step(a, req, g, win, row + 2 * ROWS < wb ? row + 2 * ROWS : row + ROWS, last_page, s0);
        add_step<false, D, FMT, PARTS, NT, GS>(s1, qf, row + ROWS, n, vis, run);
      }
      for (; row < wb; row += ROWS) {  // the last ones, whose rows not every column sees
        if (row + ROWS < wb) load_step(a, req, g, win, row + ROWS, last_page, s1);
        add_step<true, D, FMT, PARTS, NT, GS>(s0, qf, row, n, vis, run);
        if (row + ROWS < wb) s0 = s1;
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      run.l[t] += __shfl_xor(run.l[t], 16);
      run.l[t] += __shfl_xor(run.l[t], 32);
    }
    if (SHARE) {
      auto& wave_m = joined[parity][0];
      auto& wave_l = joined[parity][1];
      parity ^= 1;
      // join the waves: factors relative to the largest maximum, sums in wave order
#pragma unroll
      for (int t = 0; t < NT; ++t)
        if (lane < 16) {
          wave_m[wave][16 * t + lane] = run.m[t];
          wave_l[wave][16 * t + lane] = run.l[t];
        }
      __syncthreads();
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int c = 16 * t + (lane & 15);
        float mx = wave_m[0][c];
#pragma unroll
        for (int k = 1; k < kPagesWaves; ++k) mx = fmaxf(mx, wave_m[k][c]);
        const float f = run.m[t] == -INFINITY ? 1.f : exp2_hw(run.m[t] - mx);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) run.o[t][k] *= f;
      }
      float* mine = &part[((wave & (PW - 1)) * 16 * NT + (lane & 15)) * OS + 4 * (lane >> 4)];
      const auto put = [&] {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int k = 0; k < D / 16; ++k) *reinterpret_cast<f32x4*>(mine + 16 * t * OS + 16 * k) = run.o[t][k];
      };
      if constexpr (PW < kPagesWaves) {
        if (wave >= PW) put();
        __syncthreads();
        if (wave < PW) {
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int k = 0; k < D / 16; ++k) run.o[t][k] += *reinterpret_cast<const f32x4*>(mine + 16 * t * OS + 16 * k);
          put();  // where it has read
        }
      } else {
        put();
      }
      __syncthreads();
      for (int x = tid; x < ncol * (D / 4); x += kPagesThreads) {
        const int c = x / (D / 4), d = x % (D / 4) * 4;
        float mx = wave_m[0][c], l = 0.f;
#pragma unroll
        for (int k = 1; k < kPagesWaves; ++k) mx = fmaxf(mx, wave_m[k][c]);
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < kPagesWaves; ++k) {
          const float wm = wave_m[k][c];
          l += wave_l[k][c] * (wm == -INFINITY ? 1.f : exp2_hw(wm - mx));
        }
#pragma unroll
        for (int k = 0; k < PW; ++k) {
          const float4 y = *reinterpret_cast<const float4*>(&part[(k * 16 * NT + c) * OS + d]);
          o.x += y.x;
          o.y += y.y;
          o.z += y.z;
          o.w += y.w;
        }
        if (whole) {
          finish(a, q0 + col_offset(a, c), d, D, mx, l, o);
        } else {
          *reinterpret_cast<float4*>(a.part_o + ((int64_t)slot * COLS + c) * D + d) = o;
          if (d == 0) a.part_ml[(int64_t)slot * COLS + c] = make_float2(mx, l);
        }
      }
    } else {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int c = col0 + 16 * t + (lane & 15);
        if (c < ncol) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const int d = 16 * k + 4 * (lane >> 4);
            const float4 o = make_float4(run.o[t][k][0], run.o[t][k][1], run.o[t][k][2], run.o[t][k][3]);
            if (whole) finish(a, q0 + col_offset(a, c), d, D, run.m[t], run.l[t], o);
            else *reinterpret_cast<float4*>(a.part_o + ((int64_t)slot * COLS + c) * D + d) = o;
          }
          if (!whole && lane < 16) a.part_ml[(int64_t)slot * COLS + c] = make_float2(run.m[t], run.l[t]);
        }
      }
    }
    // a tile that begins here and goes on in the next workgroups: joined afterwards
    if (tid == 0 && b0 <= p0 && b1 < p1) {
      const int we = share_of(p1 - 1, L, La);
      *meta = make_int4((int)q0, ncol, slot, we);
    }
    first = false;
    pos = p1;
    if (pos < b1) next_tile(get, at, H, tt, a.tt_inv, a.causal);
  }
}

// A column's sums as parts are added to them, each relative to 2^m.
struct Joined {
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  __device__ void add(float2 ml, const float4& y) {
    if (ml.x == -INFINITY && ml.y == 0.f) return;  // a part without rows
    const float mx = fmaxf(m, ml.x);
    const float f = m == -INFINITY ? 1.f : exp2_hw(m - mx), fy = ml.x == -INFINITY ? 1.f : exp2_hw(ml.x - mx);
    l = l * f + ml.y * fy;
    o.x = o.x * f + y.x * fy;
    o.y = o.y * f + y.y * fy;
    o.z = o.z * f + y.z * fy;
    o.w = o.w * f + y.w * fy;
    m = mx;
  }
};

constexpr int kJoinBlocks = 16;  // workgroups for a tile's columns

// Joins the parts of the tile that begins in share w and ends in share we: its own
// slot and the first slot of the shares after it.  Of few parts, each lane of D / 4
// threads takes a column; of many, a workgroup's PL lanes share CB columns at a time, each
// every PL-th part in turn, U at once, and are joined in order.  Bound by the reading of
// the parts where tiles are wide (456 tiles of 128 columns in two parts each, 60 MB: 18
// us), else by its start and the chain of a lane's parts (4 tiles of 64 parts: 6 us).
template <int D, int COLS>
__global__ __launch_bounds__(kPagesThreads) void pages_join_kernel(PagesArgs a) {
  constexpr int CB = COLS / kJoinBlocks < 4 ? COLS / kJoinBlocks : 4;
  constexpr int TPC = D / 4, PL = kPagesThreads / TPC, U = 4;
  static_assert(CB <= PL, "a lane finishes a column");
  __shared__ float2 lane_ml[PL][CB];
  __shared__ float4 lane_o[PL][CB][TPC];
  const int4 mt = a.meta[blockIdx.x];
  if (mt.x < 0) return;
  const int s0 = mt.z, we = mt.w, w = s0 >> 1, dq = threadIdx.x % TPC, pl = threadIdx.x / TPC;
  const auto part_at = [&](int k, int c) { return (int64_t)(k == w ? s0 : 2 * k) * COLS + c; };
  const auto few = [&](auto n) {  // at most n parts
    constexpr int N = decltype(n)::value;
    const int c = blockIdx.y * PL + pl;
    if (c >= mt.y) return;
    float2 ml[N];
    float4 y[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int64_t at = part_at(min(w + u, we), c);
      ml[u] = a.part_ml[at];
      y[u] = *reinterpret_cast<const float4*>(a.part_o + at * D + 4 * dq);
    }
    Joined s;
#pragma unroll
    for (int u = 0; u < N; ++u)
      if (w + u <= we) s.add(ml[u], y[u]);
    finish(a, mt.x + col_offset(a, c), 4 * dq, D, s.m, s.l, s.o);
  };
  static_assert(PL * kJoinBlocks >= COLS, "a lane for each column");
  if (we - w == 1) return few(std::integral_constant<int, 2>());
  if (we - w < 8) return few(std::integral_constant<int, 8>());
  for (int c0 = blockIdx.y * CB; c0 < mt.y; c0 += kJoinBlocks * CB) {
    Joined s[CB];
    for (int k0 = w + pl; k0 <= we; k0 += PL * U) {
      float2 ml[CB][U];
      float4 y[CB][U];
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int64_t at = part_at(min(k0 + u * PL, we), min(c0 + c, mt.y - 1));
          ml[c][u] = a.part_ml[at];
          y[c][u] = *reinterpret_cast<const float4*>(a.part_o + at * D + 4 * dq);
        }
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (k0 + u * PL <= we) s[c].add(ml[c][u], y[c][u]);
    }
#pragma unroll
    for (int c = 0; c < CB; ++c) {
      if (dq == 0) lane_ml[pl][c] = make_float2(s[c].m, s[c].l);
      lane_o[pl][c][dq] = s[c].o;
    }
    __syncthreads();
    if (pl < CB && c0 + pl < mt.y) {
      Joined all;
#pragma unroll
      for (int k = 0; k < PL; ++k) all.add(lane_ml[k][pl], lane_o[k][pl][dq]);
      finish(a, mt.x + col_offset(a, c0 + pl), 4 * dq, D, all.m, all.l, all.o);
    }
    __syncthreads();
  }
}

int64_t round256(int64_t x) { return (x + 255) / 256 * 256; }

constexpr int kGrid = 512;  // workgroups that share the work: two on every CU
constexpr int64_t kMaxColumns = 1 << 23;  // 256 threads for each of 17 / 16 as many tiles fit a launch's 2^32

// How a call's columns are tiled: 16 or 32 to a workgroup whose waves split the rows where
// requests bring few queries each, else 128 whose waves split the columns.  By the average
// request's columns, so that one kernel serves the call: up to 16 the cache's reading
// bounds, and 16 columns waste least; up to 112 the tiles of 128 would be few and
// partly empty (8 requests of 1 .. 37 queries, 14B heads: 36 us in tiles of 32 against 57 in
// tiles of 64 by columns, when these were measured); beyond, tiles of 32 would
// read the rows four times.
enum Tiling { kFew, kSome, kMany };
Tiling tiling_of(int32_t n_req, int32_t n_tok, int G) {
  const int64_t cols = (int64_t)n_tok * G;
  return cols <= 16 * (int64_t)n_req ? kFew : cols <= 112 * (int64_t)n_req ? kSome : kMany;
}
int tile_columns(Tiling t) { return t == kFew ? 16 : t == kSome ? 32 : 128; }

template <int D, int FMT, int PARTS>
void launch_pages(const PagesArgs& a, Tiling t, int grid, hipStream_t s) {
  if (t == kFew) hipLaunchKernelGGL((pages_kernel<D, FMT, PARTS, 1, true>), dim3(grid), dim3(kPagesThreads), 0, s, a);
  else if (t == kSome) hipLaunchKernelGGL((pages_kernel<D, FMT, PARTS, 2, true>), dim3(grid), dim3(kPagesThreads), 0, s, a);
  else hipLaunchKernelGGL((pages_kernel<D, FMT, PARTS, 2, false>), dim3(grid), dim3(kPagesThreads), 0, s, a);
}

template <int D>
void launch_pages(const PagesArgs& a, Tiling t, int grid, hipStream_t s) {
  const bool e4m3 = a.p.format == MILO_KV_E4M3;
  if (a.out_bf16) {
    if (e4m3) launch_pages<D, MILO_KV_E4M3, 1>(a, t, grid, s);
    else launch_pages<D, MILO_KV_INT8, 1>(a, t, grid, s);
  } else {
    if (e4m3) launch_pages<D, MILO_KV_E4M3, 2>(a, t, grid, s);
    else launch_pages<D, MILO_KV_INT8, 2>(a, t, grid, s);
  }
  if (a.whole_tiles) return;
  // most workgroups find no tile and leave
  const dim3 grid_of_parts(kGrid, kJoinBlocks);
  if (t == kFew) hipLaunchKernelGGL((pages_join_kernel<D, 16>), grid_of_parts, dim3(kPagesThreads), 0, s, a);
  else if (t == kSome) hipLaunchKernelGGL((pages_join_kernel<D, 32>), grid_of_parts, dim3(kPagesThreads), 0, s, a);
  else hipLaunchKernelGGL((pages_join_kernel<D, 128>), grid_of_parts, dim3(kPagesThreads), 0, s, a);
}

}  // namespace
}  // namespace milo

using namespace milo;

extern "C" {

int64_t milo_attend_pages_work(int32_t n_req, int32_t n_tok, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                               int with_cache) {
  if (n_req < 0 || n_tok < 0 || n_kv_heads < 1 || n_q_heads < n_kv_heads || head_dim < 1) return 0;
  const int64_t cols = (int64_t)n_tok * n_q_heads, slot_cols = 2 * kGrid * tile_columns(tiling_of(n_req, n_tok, n_q_heads / n_kv_heads));
  int64_t bytes = round256(kGrid * (int64_t)sizeof(int4)) + round256(slot_cols * 8) + round256(slot_cols * head_dim * 4);
  if (with_cache) bytes += round256(cols * 8) + round256(cols * head_dim * 4);
  return bytes;
}

int milo_attend_pages(milo_cache* cache, const int32_t* block_table, int32_t n_sel, const milo_pages* pages,
                      const int32_t* page_table, int32_t table_width, const int32_t* lens, const int32_t* q_starts,
                      int32_t n_req, const uint16_t* q, int64_t q_stride, int32_t n_tok, int32_t n_q_heads,
                      int32_t causal, float scale, void* out, int32_t out_format, void* work, void* hip_stream) {
  clear_error();
  if (const int e = check_pages(pages); e != MILO_OK) return e;
  const int H = pages->n_kv_heads, d = pages->head_dim;
  if (n_req < 0 || n_tok < 0) return pages_fail(MILO_ERR_INVALID_ARG, "n_req and n_tok must be >= 0");
  if (n_req > kMaxPagesReq) return pages_fail(MILO_ERR_UNSUPPORTED, "n_req must be at most 2^24");
  if (!q_starts && n_tok != n_req)
    return pages_fail(MILO_ERR_INVALID_ARG, "without q_starts n_tok (%d) must equal n_req (%d)", n_tok, n_req);
  if (n_q_heads < 1 || n_q_heads % H != 0)
    return pages_fail(MILO_ERR_INVALID_ARG, "n_q_heads (%d) must be a positive multiple of n_kv_heads (%d)", n_q_heads, H);
  const int G = n_q_heads / H;
  if (G > kMaxGroup) return pages_fail(MILO_ERR_UNSUPPORTED, "more than %d query heads per KV head", kMaxGroup);
  if (table_width < 1) return pages_fail(MILO_ERR_INVALID_ARG, "table_width must be >= 1");
  if ((int64_t)table_width * pages->page_tokens > INT32_MAX)
    return pages_fail(MILO_ERR_UNSUPPORTED, "table_width times page_tokens must be below 2^31");
  if ((int64_t)n_tok * n_q_heads > kMaxColumns)
    return pages_fail(MILO_ERR_UNSUPPORTED, "n_tok times n_q_heads must be at most 2^23");
  if (causal != 0 && causal != 1) return pages_fail(MILO_ERR_INVALID_ARG, "causal must be 0 or 1 (got %d)", causal);
  if (!std::isfinite(scale)) return pages_fail(MILO_ERR_INVALID_ARG, "scale must be finite");
  if (out_format != MILO_OUT_F32 && out_format != MILO_OUT_BF16)
    return pages_fail(MILO_ERR_INVALID_ARG, "out_format must be MILO_OUT_F32 or MILO_OUT_BF16 (got %d)", out_format);
  if (!cache && n_sel != 0) return pages_fail(MILO_ERR_INVALID_ARG, "blocks are selected (n_sel = %d) without a cache", n_sel);
  if (cache) {
    int ch = 0, cd = 0;
    cache_heads(cache, &ch, &cd);
    if (ch != H || cd != d)
      return pages_fail(MILO_ERR_INVALID_ARG, "the cache has %d KV heads of %d dims, the pages %d of %d", ch, cd, H, d);
    if (n_sel < 0) return pages_fail(MILO_ERR_INVALID_ARG, "n_sel must be >= 0");
  }
  if (n_req == 0 || n_tok == 0) return MILO_OK;
  if (!page_table || !lens) return pages_fail(MILO_ERR_INVALID_ARG, "page_table / lens must be non-NULL");
  if (const int e = check_rows("q", q, q_stride, (int64_t)n_q_heads * d); e != MILO_OK) return e;
  if (!out || !aligned_to(out, 16)) return pages_fail(MILO_ERR_INVALID_ARG, "out must be non-NULL and 16-byte aligned");
  if (!work || !aligned_to(work, 256)) return pages_fail(MILO_ERR_INVALID_ARG, "work must be non-NULL and 256-byte aligned");
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  PagesArgs a{};
  const Tiling tiling = tiling_of(n_req, n_tok, G);
  // about as many tiles as there are at least (one a request, if each has queries), and at most
  const int tt = tile_columns(tiling) / G;
  const int64_t least = (int64_t)H * std::max((n_tok + tt - 1) / tt, std::min(n_req, n_tok));
  const int64_t most = (int64_t)H * (n_tok / tt + std::min(n_req, n_tok));
  // Whole tiles, without parts to join, where no request can be long: up to 1024 rows
  // (measured, one request, 7B heads: 1024 rows 10.3 us against 13.3 in shares, 2048 rows
  // 15.7 against 13.4), up to 4096 of many tiles (64 requests, 7B heads, 4096 rows each: 55.9
  // against 61.9; 0.5B heads 22.3 against 22.0); and where many columns make tiles enough to
  // even out (with about as many as workgroups run at once, 2048 queries after 6144 rows take
  // 258 us whole and 263 in shares, 0.5B heads 177 and 165, 1024 14B queries, the last of 4096
  // rows, 123 and 114).  Not where there are many requests, since every workgroup reads them
  // all (requests of up to 64 rows: 1024 of 0.5B heads 27 us whole and 36 in shares, 2048 101
  // and 62, 512 of 14B heads 59 and 68, 1024 138 and 74).  Where positions might not fit 31
  // bits (a table far wider than any request), whole tiles or nothing.
  const int64_t rows = (int64_t)table_width * pages->page_tokens;
  const bool fit = most * (kTileCost + rows / kRowAlign + 1) <= INT32_MAX / 2;
  if (!fit && most * n_req > (int64_t)1 << 26)
    return pages_fail(MILO_ERR_UNSUPPORTED, "%d requests of up to %lld rows are too many for one call", n_req, (long long)rows);
  a.whole_tiles = !fit || (most * n_req <= (int64_t)1 << 22 &&
                           (rows <= 1024 || (rows <= 4096 && least >= kGrid / 4) ||
                            (tiling != kFew && least >= 2 * kGrid)));
  const int64_t slot_cols = 2 * kGrid * tile_columns(tiling);
  char* w = static_cast<char*>(work);
  a.meta = reinterpret_cast<int4*>(w);
  w += round256(kGrid * (int64_t)sizeof(int4));
  a.part_ml = reinterpret_cast<float2*>(w);
  w += round256(slot_cols * 8);
  a.part_o = reinterpret_cast<float*>(w);
  w += round256(slot_cols * d * 4);
  if (cache && n_sel > 0) {
    if (q_stride != (int64_t)n_q_heads * d)
      return pages_fail(MILO_ERR_UNSUPPORTED, "with a cache the rows of q must follow one another (stride %lld)",
                        (long long)q_stride);
    const int64_t cols = (int64_t)n_tok * n_q_heads;
    float2* ml = reinterpret_cast<float2*>(w);
    float* o = reinterpret_cast<float*>(w + round256(cols * 8));
    int e = MILO_ERR_OUT_OF_MEMORY;
    try {
      e = attend_context(cache, block_table, n_sel, n_tok, n_q_heads, q, scale, o, ml, hip_stream);
    } catch (...) {  // its plan lives in host containers
      e = pages_fail(MILO_ERR_OUT_OF_MEMORY, "no host memory for the work plan");
    }
    if (e != MILO_OK) return e;
    a.ctx_o = o;
    a.ctx_ml = ml;
  }
  a.p = *pages;
  a.table = page_table;
  a.lens = lens;
  a.starts = q_starts;
  a.q = q;
  a.out = out;
  a.q_stride = q_stride;
  a.qscale = scale * 1.4426950408889634f;
  a.n_req = n_req;
  a.n_tok = n_tok;
  a.H_q = n_q_heads;
  a.G = G;
  a.width = table_width;
  a.lg_page = log2_page(pages->page_tokens);
  a.causal = causal;
  a.out_bf16 = out_format == MILO_OUT_BF16;
  a.least_tiles = (int)std::min<int64_t>(kGrid, least);
  a.G_inv = (65536 + G - 1) / G;
  a.tt_inv = reciprocal(tt);
  const int grid = a.whole_tiles ? (int)most : kGrid;
  if (d == 64) launch_pages<64>(a, tiling, grid, s);
  else launch_pages<128>(a, tiling, grid, s);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? MILO_OK : pages_fail(MILO_ERR_HIP, "attention kernel: %s", hipGetErrorString(e));
}

}  // extern "C"
