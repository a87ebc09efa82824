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
  if (p->n_kv_heads > 65535)
    return pages_fail(MILO_ERR_UNSUPPORTED, "n_kv_heads %d not supported (at most 65535)", p->n_kv_heads);
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

#ifdef __HIPCC__

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
