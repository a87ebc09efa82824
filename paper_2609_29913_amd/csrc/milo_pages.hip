// Paged 8-bit cache (include/milo.h): the step's bookkeeping (milo_pages_plan),
// the quantising append (milo_pages_store) and the read back to bf16
// (milo_pages_load).  Attention over the pages is in milo_pages_attend.hip.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "milo_pages.h"

namespace milo {
namespace {

// ---------------------------------------------------------------------------
// Plan.  pages(n) = ceil(n / P); request i takes max(pages(n') - pages(n), 0)
// pages from the ring's head on and gives back max(pages(n) - pages(n'), 0), both
// at places given by running sums over the requests, so nothing depends on the
// order of execution.  One workgroup forms the three sums (new rows, pages taken,
// pages given back) and what stops the step; a grid then writes slots and pages.
// ---------------------------------------------------------------------------
constexpr int kPlanThreads = 1024;
constexpr int kFillThreads = 256;
constexpr int kMaxPlanReq = 1 << 24;

enum PlanStatus : int { kPoolShort = 1, kRowNarrow = 2, kBadLength = 4, kSlotsShort = 8, kBadRing = 16 };

struct PlanArgs {
  const int32_t* lens;
  const int32_t* delta;
  int32_t* table;
  int32_t* ring;
  const int32_t* ring_state;
  int32_t* ring_state_out;
  int32_t* lens_out;
  int32_t* starts;
  int32_t* slots;
  int32_t* status;
  int32_t* taken;   // [n_req] pages taken by the requests before
  int32_t* given;   // [n_req] pages given back by the requests before
  int32_t* total;   // [6] pages taken, given back, status, head, count, new rows
  int32_t n_req, lg_page, width, n_pages, n_slots;
};

struct Sums {
  int64_t rows, taken, given;
};

__device__ inline Sums add(Sums a, Sums b) { return {a.rows + b.rows, a.taken + b.taken, a.given + b.given}; }

// what request i adds to the sums; *flags: what is wrong with it
__device__ inline Sums plan_one(const PlanArgs& a, int i, int* flags) {
  const int64_t n = a.lens[i], m = n + a.delta[i], cap = (int64_t)a.width << a.lg_page;
  if (n < 0 || m < 0) {
    *flags |= kBadLength;
    return {0, 0, 0};
  }
  if (n > cap || m > cap) {
    *flags |= kRowNarrow;
    return {0, 0, 0};
  }
  const int64_t r = (1 << a.lg_page) - 1, p0 = (n + r) >> a.lg_page, p1 = (m + r) >> a.lg_page;
  return {m > n ? m - n : 0, p1 > p0 ? p1 - p0 : 0, p0 > p1 ? p0 - p1 : 0};
}

__global__ __launch_bounds__(kPlanThreads) void plan_scan_kernel(PlanArgs a) {
  __shared__ Sums wave_sum[kPlanThreads / 64];
  __shared__ int all_flags;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) all_flags = 0;
  Sums carry{0, 0, 0};
  int flags = 0;
  for (int base = 0; base < a.n_req; base += kPlanThreads) {
    const int i = base + tid;
    const Sums own = i < a.n_req ? plan_one(a, i, &flags) : Sums{0, 0, 0};
    Sums inc = own;
    for (int o = 1; o < 64; o <<= 1) {
      const Sums up{__shfl_up(inc.rows, o), __shfl_up(inc.taken, o), __shfl_up(inc.given, o)};
      if (lane >= o) inc = add(inc, up);
    }
    __syncthreads();  // the last round's sums have been read
    if (lane == 63) wave_sum[wave] = inc;
    __syncthreads();
    Sums before = carry;
    for (int w = 0; w < wave; ++w) before = add(before, wave_sum[w]);
    for (int w = 0; w < kPlanThreads / 64; ++w) carry = add(carry, wave_sum[w]);
    if (i < a.n_req) {
      // sums past 2^31 are cut: such a step is stopped below and they are not used
      a.starts[i] = (int32_t)(before.rows + inc.rows - own.rows);
      a.taken[i] = (int32_t)(before.taken + inc.taken - own.taken);
      a.given[i] = (int32_t)(before.given + inc.given - own.given);
    }
  }
  __syncthreads();
  if (flags) atomicOr(&all_flags, flags);
  __syncthreads();
  flags = all_flags;
  const int64_t head = a.ring_state[0], count = a.ring_state[1], n = a.n_pages;
  if (head < 0 || head >= n || count < 0 || count > n || count + carry.given > n) flags |= kBadRing;
  else if (carry.taken > count) flags |= kPoolShort;
  if (carry.rows > a.n_slots) flags |= kSlotsShort;
  for (int i = tid; i < a.n_req; i += kPlanThreads) {
    a.lens_out[i] = a.lens[i] + (flags ? 0 : a.delta[i]);
    if (flags) a.starts[i] = 0;
  }
  __syncthreads();  // ring_state is read by every thread before it may be written
  if (tid == 0) {
    a.starts[a.n_req] = flags ? 0 : (int32_t)carry.rows;
    a.ring_state_out[0] = (int32_t)(flags ? head : (head + carry.taken) % n);
    a.ring_state_out[1] = (int32_t)(flags ? count : count - carry.taken + carry.given);
    a.status[0] = flags;
    a.total[0] = flags ? 0 : (int32_t)carry.taken;
    a.total[1] = flags ? 0 : (int32_t)carry.given;
    a.total[2] = flags;
    a.total[3] = (int32_t)head;
    a.total[4] = (int32_t)count;
    a.total[5] = flags ? 0 : (int32_t)carry.rows;
  }
}

// the last i with first[i] <= x (first[0] = 0 <= x, not decreasing)
__device__ inline int owner_of(const int32_t* first, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

__global__ __launch_bounds__(kFillThreads) void plan_fill_kernel(PlanArgs a) {
  const int taken = a.total[0], given = a.total[1], rows = a.total[5], head = a.total[3], count = a.total[4];
  const int P = 1 << a.lg_page;
  const int64_t items = (int64_t)a.n_slots + taken + given;
  for (int64_t x = (int64_t)blockIdx.x * kFillThreads + threadIdx.x; x < items; x += (int64_t)gridDim.x * kFillThreads) {
    if (x < a.n_slots) {
      int slot = -1;
      if (x < rows) {
        const int i = owner_of(a.starts, a.n_req, (int)x);
        const int n = a.lens_out[i] - a.delta[i];  // length before (delta > 0 here)
        const int row = n + (int)x - a.starts[i], pg = row >> a.lg_page, held = (n + P - 1) >> a.lg_page;
        const int id = pg < held ? a.table[(int64_t)i * a.width + pg]
                                 : a.ring[((int64_t)head + a.taken[i] + pg - held) % a.n_pages];
        if ((uint32_t)id < (uint32_t)a.n_pages) slot = (id << a.lg_page) + (row & (P - 1));
      }
      a.slots[x] = slot;
    } else if (x < (int64_t)a.n_slots + taken) {
      const int y = (int)(x - a.n_slots), i = owner_of(a.taken, a.n_req, y);
      const int held = (a.lens_out[i] - a.delta[i] + P - 1) >> a.lg_page;
      a.table[(int64_t)i * a.width + held + y - a.taken[i]] = a.ring[((int64_t)head + y) % a.n_pages];
    } else {
      const int y = (int)(x - a.n_slots - taken), i = owner_of(a.given, a.n_req, y);
      const int kept = (a.lens_out[i] + P - 1) >> a.lg_page;
      a.ring[((int64_t)head + count + y) % a.n_pages] = a.table[(int64_t)i * a.width + kept + y - a.given[i]];
    }
  }
}

// ---------------------------------------------------------------------------
// Store.  One wave per (row, KV head): the row that begins a page's run of new
// rows does the whole run of that page, the others leave at once.
// ---------------------------------------------------------------------------
constexpr int kRowThreads = 256;

struct StoreArgs {
  milo_pages p;
  const uint16_t* k;
  const uint16_t* v;
  int64_t k_stride, v_stride;
  const int32_t* slots;
  int32_t n_tok, lg_page, n_slots;
};

__device__ inline uint32_t wave_max(uint32_t x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, o));
  return x;
}

// keys (VALUES false) or values of rows t0 .. t0 + run - 1 into offsets off .. of
// a page and head
template <int D, int FMT, bool VALUES>
__device__ void store_side(const uint16_t* x, int64_t stride, uint8_t* codes, float* scale_at, int off, int run) {
  const int lane = threadIdx.x & 63;
  uint32_t amax = 0;
  for (int i = lane; i < run * D; i += 64) amax = max(amax, (uint32_t)x[(int64_t)(i / D) * stride + i % D] & 0x7FFFu);
  amax = wave_max(amax);
  const float was = *scale_at;
  float s = scale_of<FMT>(amax);
  if (off > 0 && !(s >= was)) s = was >= s || was != was ? was : s;  // the larger, NaN before all
  if (off > 0 && s != was && s == s) {  // rows that are held, under the larger scale
    for (int i = lane; i < off * D; i += 64) {
      const int b = VALUES ? value_byte(i / D, i % D, D) : key_byte(i / D, i % D, D);
      const float c = code_values<FMT>(codes[b]).x;
      codes[b] = (uint8_t)codes_of<FMT>(over<FMT>(make_float4(__fmul_rn(c, was), 0.f, 0.f, 0.f), s));
    }
  }
  for (int i = lane; i < run * D; i += 64) {
    const int t = off + i / D, c = i % D;
    const float f = bf16_value(x[(int64_t)(i / D) * stride + c]);
    codes[VALUES ? value_byte(t, c, D) : key_byte(t, c, D)] = (uint8_t)codes_of<FMT>(over<FMT>(make_float4(f, 0.f, 0.f, 0.f), s));
  }
  if (lane == 0) *scale_at = s;
}

template <int D, int FMT>
__global__ __launch_bounds__(kRowThreads) void store_kernel(StoreArgs a) {
  const int H = a.p.n_kv_heads;
  const int64_t item = (int64_t)blockIdx.x * (kRowThreads / 64) + (threadIdx.x >> 6);
  const int t = (int)(item / H), h = (int)(item % H);
  if (t >= a.n_tok) return;
  const int slot = a.slots[t], P = 1 << a.lg_page;
  if ((uint32_t)slot >= (uint32_t)a.n_slots) return;
  const int off = slot & (P - 1), page = slot >> a.lg_page;
  if (off > 0 && t > 0 && a.slots[t - 1] == slot - 1) return;  // inside another row's run
  int run = 1;
  while (run < P - off && t + run < a.n_tok && a.slots[t + run] == slot + run) ++run;
  const int64_t ph = (int64_t)page * H + h;
  store_side<D, FMT, false>(a.k + (int64_t)t * a.k_stride + h * D, a.k_stride, (uint8_t*)a.p.k_codes + ph * P * D,
                            a.p.k_scale + ph, off, run);
  store_side<D, FMT, true>(a.v + (int64_t)t * a.v_stride + h * D, a.v_stride, (uint8_t*)a.p.v_codes + ph * P * D,
                           a.p.v_scale + ph, off, run);
}

// ---------------------------------------------------------------------------
// Load.  One wave per (row, KV head).
// ---------------------------------------------------------------------------
struct LoadArgs {
  milo_pages p;
  uint16_t* k;
  uint16_t* v;
  int64_t k_stride, v_stride;
  const int32_t* slots;
  int32_t n_tok, lg_page, n_slots;
};

template <int D, int FMT>
__global__ __launch_bounds__(kRowThreads) void load_kernel(LoadArgs a) {
  const int lane = threadIdx.x & 63, H = a.p.n_kv_heads;
  const int64_t item = (int64_t)blockIdx.x * (kRowThreads / 64) + (threadIdx.x >> 6);
  const int t = (int)(item / H), h = (int)(item % H);
  if (t >= a.n_tok) return;
  const int slot = a.slots[t], P = 1 << a.lg_page;
  const bool in = (uint32_t)slot < (uint32_t)a.n_slots;
  const int64_t ph = in ? (int64_t)(slot >> a.lg_page) * H + h : 0;
  const uint8_t* kc = (const uint8_t*)a.p.k_codes + ph * P * D;
  const uint8_t* vc = (const uint8_t*)a.p.v_codes + ph * P * D;
  for (int c = lane; c < D; c += 64) {
    if (a.k) {
      const float x = in ? a.p.k_scale[ph] * code_values<FMT>(kc[key_byte(slot & (P - 1), c, D)]).x : 0.f;
      a.k[(int64_t)t * a.k_stride + h * D + c] = (uint16_t)bf16_bits(x);
    }
    if (a.v) {
      const float x = in ? a.p.v_scale[ph] * code_values<FMT>(vc[value_byte(slot & (P - 1), c, D)]).x : 0.f;
      a.v[(int64_t)t * a.v_stride + h * D + c] = (uint16_t)bf16_bits(x);
    }
  }
}


#define MILO_PAGES_DISPATCH(kernel, a, grid, threads, s)                                            \
  do {                                                                                              \
    const bool e4m3 = (a).p.format == MILO_KV_E4M3;                                                 \
    if ((a).p.head_dim == 64) {                                                                     \
      if (e4m3) hipLaunchKernelGGL((kernel<64, MILO_KV_E4M3>), grid, dim3(threads), 0, s, a);       \
      else hipLaunchKernelGGL((kernel<64, MILO_KV_INT8>), grid, dim3(threads), 0, s, a);            \
    } else {                                                                                        \
      if (e4m3) hipLaunchKernelGGL((kernel<128, MILO_KV_E4M3>), grid, dim3(threads), 0, s, a);      \
      else hipLaunchKernelGGL((kernel<128, MILO_KV_INT8>), grid, dim3(threads), 0, s, a);           \
    }                                                                                               \
  } while (0)

int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? MILO_OK : pages_fail(MILO_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace
}  // namespace milo

using namespace milo;

extern "C" {

int64_t milo_pages_plan_work(int32_t n_req) { return n_req < 0 ? 0 : 8 * (int64_t)n_req + 64; }

int milo_pages_plan(const int32_t* lens, const int32_t* delta, int32_t n_req, int32_t page_tokens, int32_t* table,
                    int32_t table_width, int32_t* ring, int32_t n_pages, const int32_t* ring_state,
                    int32_t* ring_state_out, int32_t* lens_out, int32_t* starts, int32_t* slots, int32_t n_slots,
                    int32_t* status, void* work, void* hip_stream) {
  clear_error();
  if (n_req < 0 || n_slots < 0) return pages_fail(MILO_ERR_INVALID_ARG, "n_req and n_slots must be >= 0");
  if (n_req > kMaxPlanReq) return pages_fail(MILO_ERR_UNSUPPORTED, "more than %d requests", kMaxPlanReq);
  const int lg = log2_page(page_tokens);
  if (lg < 0) return pages_fail(MILO_ERR_UNSUPPORTED, "page_tokens %d not supported (16, 32, 64 or 128)", page_tokens);
  if (table_width < 1 || n_pages < 1) return pages_fail(MILO_ERR_INVALID_ARG, "table_width and n_pages must be >= 1");
  if ((int64_t)n_pages * page_tokens > INT32_MAX || (int64_t)table_width * page_tokens > INT32_MAX)
    return pages_fail(MILO_ERR_UNSUPPORTED, "n_pages and table_width times page_tokens must be below 2^31");
  if (n_req > 0 && (!lens || !delta || !table || !lens_out))
    return pages_fail(MILO_ERR_INVALID_ARG, "lens / delta / table / lens_out must be non-NULL");
  if (!ring || !ring_state || !ring_state_out || !starts || !status || (n_slots > 0 && !slots))
    return pages_fail(MILO_ERR_INVALID_ARG, "ring / ring_state / ring_state_out / starts / slots / status must be non-NULL");
  if (!work || !aligned_to(work, 16)) return pages_fail(MILO_ERR_INVALID_ARG, "work must be non-NULL and 16-byte aligned");
  PlanArgs a{};
  a.lens = lens;
  a.delta = delta;
  a.table = table;
  a.ring = ring;
  a.ring_state = ring_state;
  a.ring_state_out = ring_state_out;
  a.lens_out = lens_out;
  a.starts = starts;
  a.slots = slots;
  a.status = status;
  a.total = static_cast<int32_t*>(work);
  a.taken = a.total + 16;
  a.given = a.taken + n_req;
  a.n_req = n_req;
  a.lg_page = lg;
  a.width = table_width;
  a.n_pages = n_pages;
  a.n_slots = n_slots;
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  hipLaunchKernelGGL(plan_scan_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
  if (const int e = launched("plan kernel"); e != MILO_OK) return e;
  const int64_t items = (int64_t)n_slots + n_slots / page_tokens + n_req;
  const int grid = (int)std::min<int64_t>(2048, items / kFillThreads + 1);
  hipLaunchKernelGGL(plan_fill_kernel, dim3(grid), dim3(kFillThreads), 0, s, a);
  return launched("plan kernel");
}

int milo_pages_store(const milo_pages* pages, const uint16_t* k, int64_t k_stride, const uint16_t* v, int64_t v_stride,
                     const int32_t* slots, int32_t n_tok, void* hip_stream) {
  clear_error();
  if (const int e = check_pages(pages); e != MILO_OK) return e;
  if (n_tok < 0) return pages_fail(MILO_ERR_INVALID_ARG, "n_tok must be >= 0");
  if (n_tok == 0) return MILO_OK;
  const int64_t D = (int64_t)pages->n_kv_heads * pages->head_dim;
  if (const int e = check_rows("k", k, k_stride, D); e != MILO_OK) return e;
  if (const int e = check_rows("v", v, v_stride, D); e != MILO_OK) return e;
  if (!slots) return pages_fail(MILO_ERR_INVALID_ARG, "slots is NULL");
  StoreArgs a{};
  a.p = *pages;
  a.k = k;
  a.v = v;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.slots = slots;
  a.n_tok = n_tok;
  a.lg_page = log2_page(pages->page_tokens);
  a.n_slots = pages->n_pages * pages->page_tokens;
  const int64_t waves = (int64_t)n_tok * pages->n_kv_heads, wgs = (waves + kRowThreads / 64 - 1) / (kRowThreads / 64);
  if (wgs > INT32_MAX) return pages_fail(MILO_ERR_UNSUPPORTED, "too many rows");
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  MILO_PAGES_DISPATCH(store_kernel, a, dim3((uint32_t)wgs), kRowThreads, s);
  return launched("store kernel");
}

int milo_pages_load(const milo_pages* pages, const int32_t* slots, int32_t n_tok, uint16_t* k_out, int64_t k_stride,
                    uint16_t* v_out, int64_t v_stride, void* hip_stream) {
  clear_error();
  if (const int e = check_pages(pages); e != MILO_OK) return e;
  if (n_tok < 0) return pages_fail(MILO_ERR_INVALID_ARG, "n_tok must be >= 0");
  if (n_tok == 0) return MILO_OK;
  if (!k_out && !v_out) return pages_fail(MILO_ERR_INVALID_ARG, "k_out and v_out are both NULL");
  const int64_t D = (int64_t)pages->n_kv_heads * pages->head_dim;
  if (k_out)
    if (const int e = check_rows("k_out", k_out, k_stride, D); e != MILO_OK) return e;
  if (v_out)
    if (const int e = check_rows("v_out", v_out, v_stride, D); e != MILO_OK) return e;
  if (!slots) return pages_fail(MILO_ERR_INVALID_ARG, "slots is NULL");
  LoadArgs a{};
  a.p = *pages;
  a.k = k_out;
  a.v = v_out;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.slots = slots;
  a.n_tok = n_tok;
  a.lg_page = log2_page(pages->page_tokens);
  a.n_slots = pages->n_pages * pages->page_tokens;
  const int64_t waves = (int64_t)n_tok * pages->n_kv_heads, wgs = (waves + kRowThreads / 64 - 1) / (kRowThreads / 64);
  if (wgs > INT32_MAX) return pages_fail(MILO_ERR_UNSUPPORTED, "too many rows");
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  MILO_PAGES_DISPATCH(load_kernel, a, dim3((uint32_t)wgs), kRowThreads, s);
  return launched("load kernel");
}

}  // extern "C"
