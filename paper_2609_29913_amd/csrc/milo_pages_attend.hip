// Attention over the paged 8-bit cache (include/milo.h: milo_attend_pages).
#include <hip/hip_runtime.h>

#include <cmath>

#include "milo_attend.h"
#include "milo_pages.h"

namespace milo {
namespace {

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
  float qscale;            // scale * log2(e)
  int32_t n_req, n_tok, H_q, G, width, lg_page, causal, out_bf16;
};

__device__ inline int start_of(const PagesArgs& a, int i) {
  return a.starts ? min(max(a.starts[i], 0), a.n_tok) : i;
}

// Rows a query sees: all n of its request, or, as query j of m, its own and those before.
__device__ inline int seen_by(const PagesArgs& a, int n, int j, int m) { return a.causal ? max(0, n - m + j + 1) : n; }

template <int D, int FMT>
__global__ __launch_bounds__(64) void pages_simple_kernel(PagesArgs a) {
  __shared__ float qs[D], ps[64];
  const int lane = threadIdx.x, h = blockIdx.y, g = h / a.G, P = 1 << a.lg_page;
  const int t = blockIdx.x;
  // the request: the last with start <= t
  int lo = 0, hi = a.n_req;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start_of(a, mid) <= t) lo = mid;
    else hi = mid;
  }
  const int s0 = start_of(a, lo), s1 = a.starts ? start_of(a, lo + 1) : lo + 1;
  if (t < s0 || t >= s1) return;
  const int64_t cap = (int64_t)a.width << a.lg_page;
  const int n = (int)min((int64_t)max(a.lens[lo], 0), cap);
  const int seen = seen_by(a, n, t - s0, s1 - s0);
  for (int c = lane; c < D; c += 64) qs[c] = bf16_value(a.q[(int64_t)t * a.q_stride + (int64_t)h * D + c]);
  __syncthreads();
  float m = -INFINITY, l = 0.f, o[D / 64] = {};
  for (int r0 = 0; r0 < seen; r0 += 64) {
    const int r = r0 + lane;
    float s = -INFINITY;
    if (r < seen) {
      const int id = a.table[(int64_t)lo * a.width + (r >> a.lg_page)];
      if ((uint32_t)id < (uint32_t)a.p.n_pages) {
        const int64_t ph = (int64_t)id * a.p.n_kv_heads + g;
        const uint8_t* kc = (const uint8_t*)a.p.k_codes + ph * P * D;
        float dot = 0.f;
        for (int c = 0; c < D; c += 4) {
          const float4 x = code_values<FMT>(*(const uint32_t*)(kc + key_byte(r & (P - 1), c, D)));
          dot += x.x * qs[c] + x.y * qs[c + 1] + x.z * qs[c + 2] + x.w * qs[c + 3];
        }
        s = dot * (a.p.k_scale[ph] * a.qscale);
      } else {
        s = __uint_as_float(0x7FC00000u);
      }
    }
    float mx = s;
    for (int k = 32; k > 0; k >>= 1) mx = fmaxf(mx, __shfl_xor(mx, k));
    mx = fmaxf(mx, m);
    const float ref = mx == -INFINITY ? 0.f : mx;
    const float p = exp2f(s - ref), f = exp2f(m - ref);
    float sum = p;
    for (int k = 32; k > 0; k >>= 1) sum += __shfl_xor(sum, k);
    l = l * f + sum;
    m = mx;
    __syncthreads();
    ps[lane] = p;
    __syncthreads();
    for (int k = 0; k < D / 64; ++k) o[k] *= f;
    for (int u = 0; u < 64 && r0 + u < seen; ++u) {
      const int rr = r0 + u, id = a.table[(int64_t)lo * a.width + (rr >> a.lg_page)];
      if ((uint32_t)id >= (uint32_t)a.p.n_pages) continue;
      const int64_t ph = (int64_t)id * a.p.n_kv_heads + g;
      const uint8_t* vc = (const uint8_t*)a.p.v_codes + ph * P * D;
      const float w = ps[u] * a.p.v_scale[ph];
      for (int k = 0; k < D / 64; ++k) o[k] += w * code_values<FMT>(vc[value_byte(rr & (P - 1), lane + 64 * k, D)]).x;
    }
  }
  const int64_t col = (int64_t)t * a.H_q + h;
  if (a.ctx_ml) {
    const float2 cm = a.ctx_ml[col];
    const float mx = fmaxf(m, cm.x), fp = m == -INFINITY && l == 0.f ? 0.f : exp2f(m - mx), fc = exp2f(cm.x - mx) * cm.y;
    l = l * fp + fc;
    for (int k = 0; k < D / 64; ++k) o[k] = o[k] * fp + fc * a.ctx_o[col * D + lane + 64 * k];
  }
  for (int k = 0; k < D / 64; ++k) {
    const float x = l == 0.f ? 0.f : o[k] / l;
    if (a.out_bf16) ((uint16_t*)a.out)[col * D + lane + 64 * k] = (uint16_t)bf16_bits(x);
    else ((float*)a.out)[col * D + lane + 64 * k] = x;
  }
}

int64_t round256(int64_t x) { return (x + 255) / 256 * 256; }

}  // namespace
}  // namespace milo

using namespace milo;

extern "C" {

int64_t milo_attend_pages_work(int32_t n_tok, int32_t n_q_heads, int32_t head_dim, int with_cache) {
  if (n_tok < 0 || n_q_heads < 1 || head_dim < 1) return 0;
  const int64_t cols = (int64_t)n_tok * n_q_heads;
  return with_cache ? round256(cols * 8) + round256(cols * head_dim * 4) + 256 : 256;
}

int milo_attend_pages(milo_cache* cache, const int32_t* block_table, int32_t n_sel, const milo_pages* pages,
                      const int32_t* page_table, int32_t table_width, const int32_t* lens, const int32_t* q_starts,
                      int32_t n_req, const uint16_t* q, int64_t q_stride, int32_t n_tok, int32_t n_q_heads,
                      int32_t causal, float scale, void* out, int32_t out_format, void* work, void* hip_stream) {
  clear_error();
  if (const int e = check_pages(pages); e != MILO_OK) return e;
  const int H = pages->n_kv_heads, d = pages->head_dim;
  if (n_req < 0 || n_tok < 0) return pages_fail(MILO_ERR_INVALID_ARG, "n_req and n_tok must be >= 0");
  if (!q_starts && n_tok != n_req)
    return pages_fail(MILO_ERR_INVALID_ARG, "without q_starts n_tok (%d) must equal n_req (%d)", n_tok, n_req);
  if (n_q_heads < 1 || n_q_heads % H != 0)
    return pages_fail(MILO_ERR_INVALID_ARG, "n_q_heads (%d) must be a positive multiple of n_kv_heads (%d)", n_q_heads, H);
  const int G = n_q_heads / H;
  if (G > kMaxGroup) return pages_fail(MILO_ERR_UNSUPPORTED, "more than %d query heads per KV head", kMaxGroup);
  if (table_width < 1) return pages_fail(MILO_ERR_INVALID_ARG, "table_width must be >= 1");
  if ((int64_t)table_width * pages->page_tokens > INT32_MAX)
    return pages_fail(MILO_ERR_UNSUPPORTED, "table_width times page_tokens must be below 2^31");
  if ((int64_t)n_tok * n_q_heads > (int64_t)1 << 24) return pages_fail(MILO_ERR_UNSUPPORTED, "too many query columns");
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
  if (cache && n_sel > 0) {
    if (q_stride != (int64_t)n_q_heads * d)
      return pages_fail(MILO_ERR_UNSUPPORTED, "with a cache the rows of q must follow one another (stride %lld)",
                        (long long)q_stride);
    const int64_t cols = (int64_t)n_tok * n_q_heads;
    float2* ml = static_cast<float2*>(work);
    float* o = reinterpret_cast<float*>(static_cast<char*>(work) + round256(cols * 8));
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
  const dim3 grid(n_tok, n_q_heads);
  const bool e4m3 = pages->format == MILO_KV_E4M3;
  if (d == 64) {
    if (e4m3) hipLaunchKernelGGL((pages_simple_kernel<64, MILO_KV_E4M3>), grid, dim3(64), 0, s, a);
    else hipLaunchKernelGGL((pages_simple_kernel<64, MILO_KV_INT8>), grid, dim3(64), 0, s, a);
  } else {
    if (e4m3) hipLaunchKernelGGL((pages_simple_kernel<128, MILO_KV_E4M3>), grid, dim3(64), 0, s, a);
    else hipLaunchKernelGGL((pages_simple_kernel<128, MILO_KV_INT8>), grid, dim3(64), 0, s, a);
  }
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? MILO_OK : pages_fail(MILO_ERR_HIP, "attention kernel: %s", hipGetErrorString(e));
}

}  // extern "C"
