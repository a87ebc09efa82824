// Internal definitions of the paged 8-bit cache (include/milo.h): the order of
// the codes in a page, the conversions of both formats and the host checks that
// its entry points share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cstdio>

#include "milo.h"
#include "milo_internal.h"

namespace milo {

// Byte of (token t, dim c) in a page's codes of one head.  16 rows of a head are
// one run of 16 d bytes: as keys 16-byte pieces of 16 dims of one token, so that
// lane l of a wave loading bytes 16 l .. holds dims 16 (l / 16) .. of token l % 16,
// the A operand (tokens x dims) of two 16x16x32 products; as values pieces of four
// tokens of one dim, four dim tiles to a lane, the A operand (dims x tokens) of four.
__host__ __device__ inline int key_byte(int t, int c, int d) {
  return ((t >> 4) * (d >> 4) + (c >> 4)) * 256 + (t & 15) * 16 + (c & 15);
}
__host__ __device__ inline int value_byte(int t, int c, int d) {
  return ((t >> 4) * (d >> 6) + (c >> 6)) * 1024 + ((t & 15) >> 2) * 256 + (c & 15) * 16 + ((c & 63) >> 4) * 4 + (t & 3);
}

constexpr int kMaxPagesReq = 1 << 24;   // requests of a call
constexpr int kMaxPagesRows = 1 << 27;  // rows stored or loaded by a call: a launch has 2^32 threads at most
constexpr int kMaxPagesHeads = 32767;   // KV heads: a launch has 65536 workgroups at most in y

// log2 of the page size, or -1 where it is none of 16, 32, 64, 128
inline int log2_page(int page_tokens) {
  for (int k = 4; k <= 7; ++k)
    if (page_tokens == 1 << k) return k;
  return -1;
}

template <typename... A>
int pages_fail(int code, const char* fmt, A... a) {
  char buf[256];
  std::snprintf(buf, sizeof buf, fmt, a...);
  return report_error(code, buf);
}
inline int pages_fail(int code, const char* msg) { return report_error(code, msg); }

inline bool aligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// MILO_OK, or the code of the first thing wrong with a pool's description
inline int check_pages(const milo_pages* p) {
  if (!p) return pages_fail(MILO_ERR_INVALID_ARG, "pages is NULL");
  if (p->n_pages < 1) return pages_fail(MILO_ERR_INVALID_ARG, "n_pages must be >= 1 (got %d)", p->n_pages);
  if (p->n_kv_heads < 1) return pages_fail(MILO_ERR_INVALID_ARG, "n_kv_heads must be >= 1 (got %d)", p->n_kv_heads);
  if (log2_page(p->page_tokens) < 0)
    return pages_fail(MILO_ERR_UNSUPPORTED, "page_tokens %d not supported (16, 32, 64 or 128)", p->page_tokens);
  if (p->head_dim != 64 && p->head_dim != 128)
    return pages_fail(MILO_ERR_UNSUPPORTED, "head_dim %d not supported (64 or 128)", p->head_dim);
  if (p->n_kv_heads > kMaxPagesHeads)
    return pages_fail(MILO_ERR_UNSUPPORTED, "n_kv_heads %d not supported (at most %d)", p->n_kv_heads, kMaxPagesHeads);
  if ((int64_t)p->n_pages * p->page_tokens > INT32_MAX)
    return pages_fail(MILO_ERR_UNSUPPORTED, "%d pages of %d tokens exceed 2^31 - 1 slots", p->n_pages, p->page_tokens);
  if (p->format != MILO_KV_INT8 && p->format != MILO_KV_E4M3)
    return pages_fail(MILO_ERR_INVALID_ARG, "format must be MILO_KV_INT8 or MILO_KV_E4M3 (got %d)", p->format);
  if (!p->k_codes || !p->v_codes || !p->k_scale || !p->v_scale)
    return pages_fail(MILO_ERR_INVALID_ARG, "k_codes / v_codes / k_scale / v_scale must be non-NULL");
  if (!aligned_to(p->k_codes, 16) || !aligned_to(p->v_codes, 16))
    return pages_fail(MILO_ERR_INVALID_ARG, "k_codes / v_codes must be 16-byte aligned");
  return MILO_OK;
}

// a row stride in elements for rows of `width` bf16 values read 16 bytes at a time
inline int check_rows(const char* name, const void* p, int64_t stride, int64_t width) {
  if (!p) return pages_fail(MILO_ERR_INVALID_ARG, "%s is NULL", name);
  if (!aligned_to(p, 16)) return pages_fail(MILO_ERR_INVALID_ARG, "%s must be 16-byte aligned", name);
  if (stride < width || stride % 8 != 0)
    return pages_fail(MILO_ERR_INVALID_ARG, "%s: row stride %lld must be a multiple of 8, at least %lld", name,
                      (long long)stride, (long long)width);
  return MILO_OK;
}

// ---- the work of an attention call -------------------------------------------------
// Request r's m queries are cut into column tiles of tt tokens; tile k sees vis(k) of
// its n rows.  Positions number the work, kRowAlign rows each: request by request, KV
// head by KV head, tile by tile, the first k tiles of a head kTileCost k + (vis(0) + ..
// + vis(k - 1)) / kRowAlign long, rounded down (requests without queries take none).
// Share w of W has the positions [w L, (w + 1) L) of X, L = ceil(X / W), in whatever tiles
// they fall (or a sixth more or less, share_at), so lengths may differ as they like (the
// last shares may be short or empty); a tile's rows are cut at multiples of kRowAlign.  All of it follows from the lengths, on the
// device; the host sees to it that X fits 31 bits.
constexpr int kRowAlign = 64;
constexpr int kTileCost = 2;  // what a tile costs besides its rows

constexpr int kCus = 256;
constexpr int kXcdCus = kCus / kXcds;

// Where share k begins.  Of two shares to a CU, the workgroup that came first is served first
// (with equal shares of a 2048-query chunk it ends after 211 us, the other after 254): the
// first kXcdCus of an XCD's shares have La positions, the others 2 L - La.  La = L: all alike.
__host__ __device__ inline int64_t share_at(int k, int L, int La) {
  if (La == L) return (int64_t)k * L;
  const int j = k % (2 * kXcdCus);
  return (int64_t)(k - j) * L + (j < kXcdCus ? j * La : kXcdCus * La + (j - kXcdCus) * (2 * L - La));
}
// the share that holds a position
__host__ __device__ inline int share_of(int pos, int L, int La) {
  if (La == L) return (int)((uint32_t)pos / (uint32_t)L);
  const int xcd = pos / (2 * kXcdCus * L), rest = pos - xcd * 2 * kXcdCus * L;
  return 2 * kXcdCus * xcd + (rest < kXcdCus * La ? rest / La : kXcdCus + (rest - kXcdCus * La) / (2 * L - La));
}

struct Request {
  int start, m, n;  // first query, queries, rows held
};

// ceil(x / tt) for x <= 2^24 and tt <= 128 by the reciprocal ceil(2^32 / tt) (0 for tt = 1)
__host__ __device__ inline int tiles_of(int m, int tt, uint32_t tt_inv) {
  const uint32_t x = (uint32_t)(m + tt - 1);
  return tt == 1 ? (int)x : (int)(((uint64_t)x * tt_inv) >> 32);
}
inline uint32_t reciprocal(int tt) { return (uint32_t)((((uint64_t)1 << 32) + tt - 1) / tt); }

// rows that query number j - 1 of the request sees (at most its last one's)
__host__ __device__ inline int seen_upto(const Request& q, int j, int causal) {
  if (!causal) return q.n;
  const int v = q.n - q.m + (j < q.m ? j : q.m);
  return v > 0 ? v : 0;
}

// positions of the first k of a request's `all` tiles
__host__ __device__ inline int tiles_cost(const Request& q, int k, int all, int tt, int causal) {
  if (k <= 0) return 0;
  int64_t sum;
  if (!causal) {
    sum = (int64_t)k * q.n;
  } else {
    // tile i sees max(0, base + (i + 1) tt) rows, the request's last tile n
    const int whole = k < all ? k : all - 1, base = q.n - q.m;
    int skip = base < 0 ? -base / tt : 0;  // tiles that see nothing
    if (skip > whole) skip = whole;
    sum = (int64_t)(whole - skip) * base + (int64_t)tt * (((int64_t)whole * (whole + 1) - (int64_t)skip * (skip + 1)) / 2);
    if (k >= all) sum += q.n;
  }
  return (int)(sum / kRowAlign) + k * kTileCost;
}

// the row at which boundary b cuts the tile at positions [p0, p1) that sees vis rows
__host__ __device__ inline int row_at(int b, int p0, int p1, int vis) {
  if (b >= p1) return vis;
  if (b <= p0 + kTileCost) return 0;
  return (b - p0 - kTileCost) * kRowAlign;
}

struct Place {
  int r, head, tile, all;  // all: tiles of the request
  int p0, p1;              // positions of the tile
  int head0, cost;         // first position of the head's tiles, and how many
  Request rq;
};

// sets the positions of the tile that `at` names
__host__ __device__ inline void set_tile(Place& at, int tt, int causal) {
  at.p0 = at.head0 + tiles_cost(at.rq, at.tile, at.all, tt, causal);
  at.p1 = at.tile + 1 < at.all ? at.head0 + tiles_cost(at.rq, at.tile + 1, at.all, tt, causal) : at.head0 + at.cost;
}

// the tile that holds position b, where request r0's work begins at p <= b
template <typename Get>
__host__ __device__ inline Place place_of(const Get& get, int r0, int p, int b, int H, int tt, uint32_t tt_inv, int causal) {
  Place at;
  for (at.r = r0;; ++at.r) {
    at.rq = get(at.r);
    at.all = tiles_of(at.rq.m, tt, tt_inv);
    at.cost = tiles_cost(at.rq, at.all, at.all, tt, causal);
    if (b - p < H * at.cost) break;
    p += H * at.cost;
  }
  at.head = (int)((uint32_t)(b - p) / (uint32_t)at.cost);
  at.head0 = p + at.head * at.cost;
  int t0 = 0, t1 = at.all;
  while (t1 - t0 > 1) {
    const int mid = (t0 + t1) >> 1;
    if (at.head0 + tiles_cost(at.rq, mid, at.all, tt, causal) <= b) t0 = mid;
    else t1 = mid;
  }
  at.tile = t0;
  set_tile(at, tt, causal);
  return at;
}

// the tile after (there is one)
template <typename Get>
__host__ __device__ inline void next_tile(const Get& get, Place& at, int H, int tt, uint32_t tt_inv, int causal) {
  if (++at.tile >= at.all) {
    at.tile = 0;
    at.head0 += at.cost;
    if (++at.head >= H) {
      at.head = 0;
      do at.rq = get(++at.r);
      while (at.rq.m == 0);
      at.all = tiles_of(at.rq.m, tt, tt_inv);
      at.cost = tiles_cost(at.rq, at.all, at.all, tt, causal);
    }
  }
  set_tile(at, tt, causal);
}

#ifdef __HIPCC__

__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }
// sums over the lanes up to this one, which stop at 2^32 - 1
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
#define MILO_FROM(ctrl, rows) x = sat_add(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, rows, 0xF, false))
  MILO_FROM(0x111, 0xF);  // 1, 2, 4, 8 lanes before, in rows of 16
  MILO_FROM(0x112, 0xF);
  MILO_FROM(0x114, 0xF);
  MILO_FROM(0x118, 0xF);
  MILO_FROM(0x142, 0xA);  // rows 0 and 2 to rows 1 and 3
  MILO_FROM(0x143, 0xC);  // row 1 to rows 2 and 3
#undef MILO_FROM
  return x;
}

__device__ __forceinline__ float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }
__device__ __forceinline__ uint32_t bf16_bits(float x) {  // round half to even
  const __bf16 h = (__bf16)x;
  return __builtin_bit_cast(uint16_t, h);
}

// the four codes of a dword as fp32 values, exactly
template <int FMT>
__device__ __forceinline__ float4 code_values(uint32_t w) {
  if constexpr (FMT == MILO_KV_INT8) {
    return make_float4((float)(int8_t)w, (float)(int8_t)(w >> 8), (float)(int8_t)(w >> 16), (float)(int8_t)(w >> 24));
  } else {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    return make_float4(lo[0], lo[1], hi[0], hi[1]);
  }
}

// four values already divided by their scale as codes, rounded half to even
template <int FMT>
__device__ __forceinline__ uint32_t codes_of(float4 x) {
  if constexpr (FMT == MILO_KV_INT8) {
    auto one = [](float v) { return (uint32_t)(int)fminf(fmaxf(rintf(v), -127.f), 127.f) & 255u; };
    return one(x.x) | one(x.y) << 8 | one(x.z) << 16 | one(x.w) << 24;
  } else {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x.x, x.y, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x.z, x.w, w, true);
  }
}

// scale of rows whose largest magnitude has the bf16 bits `amax` (sign cleared);
// NaN where a value is not finite
template <int FMT>
__device__ __forceinline__ float scale_of(uint32_t amax) {
  if (amax >= 0x7F80u) return __uint_as_float(0x7FC00000u);
  const float a = bf16_value(amax);
  if constexpr (FMT == MILO_KV_INT8) {
    return __fdiv_rn(a, 127.f);
  } else {
    if (amax == 0) return 0.f;
    // a = 1.f x 2^k <= 448 x 2^e = 1.75 x 2^(e+8); subnormal a: e at its bound
    const int k = (int)(amax >> 7) - 127;
    const int e = k - 8 + ((amax & 127u) > 96u ? 1 : 0);
    return __uint_as_float((uint32_t)(max(e, -126) + 127) << 23);
  }
}

// x under scale s; a page and head without any magnitude (s = 0) or that holds
// NaN has codes 0
template <int FMT>
__device__ __forceinline__ float4 over(float4 x, float s) {
  if (!(s > 0.f)) return make_float4(0.f, 0.f, 0.f, 0.f);
  return make_float4(__fdiv_rn(x.x, s), __fdiv_rn(x.y, s), __fdiv_rn(x.z, s), __fdiv_rn(x.w, s));
}

#endif  // __HIPCC__

}  // namespace milo
