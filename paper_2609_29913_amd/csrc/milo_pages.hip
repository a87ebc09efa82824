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
// pages given back) and what stops the step, since the sums need every request and
// there are few (256 requests, a row each: 31 KB in all); a grid then writes slots and
// pages, each finding its request by binary search.  Where one workgroup can write them
// as well, it does: latency bounds both, and a launch costs about 3 us.  A decode step of
// 256 requests takes 7.2 us on the GPU in one launch, 10.4 between calls; 32 prompts of
// up to 4096 rows (65k slots) 2.8 + 4.5 us in two, 13 between calls.
// ---------------------------------------------------------------------------
constexpr int kPlanThreads = 1024;
constexpr int kFillThreads = 256;
constexpr int kOneLaunch = 4096;  // new rows that one workgroup writes the slots of

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

// Sums that stop at 2^32 - 1, past every limit they are held against.
struct Sums {
  uint32_t rows, taken, given;
};

__device__ __forceinline__ Sums add(Sums a, Sums b) {
  return {sat_add(a.rows, b.rows), sat_add(a.taken, b.taken), sat_add(a.given, b.given)};
}

// what a request of n rows and change delta adds to the sums; *flags: what is wrong with it
__device__ inline Sums plan_one(const PlanArgs& a, int n, int delta, int* flags) {
  const int64_t m = (int64_t)n + delta, cap = (int64_t)a.width << a.lg_page;
  if (n < 0 || m < 0) {
    *flags |= kBadLength;
    return {0, 0, 0};
  }
  if (n > cap || m > cap) {
    *flags |= kRowNarrow;
    return {0, 0, 0};
  }
  const int r = (1 << a.lg_page) - 1, p0 = (int)(((int64_t)n + r) >> a.lg_page), p1 = (int)((m + r) >> a.lg_page);
  return {(uint32_t)max(delta, 0), (uint32_t)max(p1 - p0, 0), (uint32_t)max(p0 - p1, 0)};
}

// x < 2 n_pages as an index of the ring
__device__ inline int ring_at(const PlanArgs& a, int64_t x) { return (int)(x >= a.n_pages ? x - a.n_pages : x); }

// the slot of packed new row x, which is row `row` of request i, whose first `held` pages
// are in the table and whose others are the ring's from the taken-th on
__device__ inline int slot_at(const PlanArgs& a, int i, int row, int held, int taken, int head) {
  const int pg = row >> a.lg_page, P = 1 << a.lg_page;
  const int id = pg < held ? a.table[(int64_t)i * a.width + pg] : a.ring[ring_at(a, (int64_t)head + taken + pg - held)];
  return (uint32_t)id < (uint32_t)a.n_pages ? (id << a.lg_page) + (row & (P - 1)) : -1;
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

// FILL: n_req <= kPlanThreads; the workgroup also writes slots and pages, the sums in
// LDS, so that a decode step's plan is one launch.
template <bool FILL>
__global__ __launch_bounds__(kPlanThreads) void plan_scan_kernel(PlanArgs a) {
  constexpr int kPlanWaves = kPlanThreads / 64;
  __shared__ int first[FILL ? 4 : 1][FILL ? kPlanThreads : 1];  // starts, taken, given, length before
  __shared__ Sums wave_sum[kPlanWaves];
  __shared__ int all_flags;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int head = a.ring_state[0], count = a.ring_state[1];
  if (tid == 0) all_flags = 0;
  Sums carry{0, 0, 0};
  int flags = 0;
  for (int base = 0; base < a.n_req; base += kPlanThreads) {
    const int i = base + tid;
    const int n = i < a.n_req ? a.lens[i] : 0, delta = i < a.n_req ? a.delta[i] : 0;
    const Sums own = plan_one(a, n, delta, &flags);
    const Sums inc{wave_scan(own.rows), wave_scan(own.taken), wave_scan(own.given)};
    __syncthreads();  // the last round's sums have been read
    if (lane == 63) wave_sum[wave] = inc;
    __syncthreads();
    Sums before = carry;
#pragma unroll
    for (int w = 0; w < kPlanWaves; ++w) {
      const Sums s = wave_sum[w];
      if (w < wave) before = add(before, s);
      carry = add(carry, s);
    }
    if (i < a.n_req) {
      // (sums that stopped are not used: the step is refused below)
      const Sums at{before.rows + inc.rows - own.rows, before.taken + inc.taken - own.taken,
                    before.given + inc.given - own.given};
      if constexpr (FILL) {
        first[0][i] = (int32_t)at.rows;
        first[1][i] = (int32_t)at.taken;
        first[2][i] = (int32_t)at.given;
        first[3][i] = n;
      } else {
        a.starts[i] = (int32_t)at.rows;
        a.taken[i] = (int32_t)at.taken;
        a.given[i] = (int32_t)at.given;
      }
    }
  }
  if (flags) atomicOr(&all_flags, flags);
  __syncthreads();
  flags = all_flags;
  if (head < 0 || head >= a.n_pages || count < 0 || count > a.n_pages || carry.given > (uint32_t)(a.n_pages - count))
    flags |= kBadRing;
  else if (carry.taken > (uint32_t)count)
    flags |= kPoolShort;
  if (carry.rows > (uint32_t)a.n_slots) flags |= kSlotsShort;
  const int rows = flags ? 0 : (int)carry.rows, taken = flags ? 0 : (int)carry.taken, given = flags ? 0 : (int)carry.given;
  for (int i = tid; i < a.n_req; i += kPlanThreads) {
    if constexpr (FILL) {
      a.starts[i] = flags ? 0 : first[0][i];
      a.lens_out[i] = first[3][i] + (flags ? 0 : a.delta[i]);
    } else {
      if (flags) a.starts[i] = 0;
      a.lens_out[i] = a.lens[i] + (flags ? 0 : a.delta[i]);
    }
  }
  if (tid == 0) {  // every thread has read ring_state, which this may be, before the barriers above
    a.starts[a.n_req] = rows;
    a.ring_state_out[0] = flags ? head : ring_at(a, (int64_t)head + taken);
    a.ring_state_out[1] = count - taken + given;
    a.status[0] = flags;
    if constexpr (!FILL) {
      a.total[0] = taken;
      a.total[1] = given;
      a.total[3] = head;
      a.total[4] = count;
      a.total[5] = rows;
    }
  }
  if constexpr (FILL) {
    const int P = 1 << a.lg_page, items = a.n_slots + taken + given;
    for (int x = tid; x < items; x += kPlanThreads) {
      if (x < a.n_slots) {
        int slot = -1;
        if (x < rows) {
          const int i = owner_of(first[0], a.n_req, x), n = first[3][i];
          slot = slot_at(a, i, n + x - first[0][i], (n + P - 1) >> a.lg_page, first[1][i], head);
        }
        a.slots[x] = slot;
      } else if (x < a.n_slots + taken) {
        const int y = x - a.n_slots, i = owner_of(first[1], a.n_req, y), held = (first[3][i] + P - 1) >> a.lg_page;
        a.table[(int64_t)i * a.width + held + y - first[1][i]] = a.ring[ring_at(a, (int64_t)head + y)];
      } else {
        const int y = x - a.n_slots - taken, i = owner_of(first[2], a.n_req, y);
        const int kept = (first[3][i] + a.delta[i] + P - 1) >> a.lg_page;
        a.ring[ring_at(a, (int64_t)head + count + y)] = a.table[(int64_t)i * a.width + kept + y - first[2][i]];
      }
    }
  }
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
        slot = slot_at(a, i, n + (int)x - a.starts[i], (n + P - 1) >> a.lg_page, a.taken[i], head);
      }
      a.slots[x] = slot;
    } else if (x < (int64_t)a.n_slots + taken) {
      const int y = (int)(x - a.n_slots), i = owner_of(a.taken, a.n_req, y);
      const int held = (a.lens_out[i] - a.delta[i] + P - 1) >> a.lg_page;
      a.table[(int64_t)i * a.width + held + y - a.taken[i]] = a.ring[ring_at(a, (int64_t)head + y)];
    } else {
      const int y = (int)(x - a.n_slots - taken), i = owner_of(a.given, a.n_req, y);
      const int kept = (a.lens_out[i] + P - 1) >> a.lg_page;
      a.ring[ring_at(a, (int64_t)head + count + y)] = a.table[(int64_t)i * a.width + kept + y - a.given[i]];
    }
  }
}

// ---------------------------------------------------------------------------
// Store and load.  A wave takes a page's (or 16 output rows') part of one KV head and
// side at a time, in groups of 16 rows: lane (q, ch) has rows 4 q .. 4 q + 3 and dims
// 8 ch .. 8 ch + 7, four 16-byte accesses on the bf16 side; on the codes' side 8 bytes
// of keys per row, or per dim the dword of a value's four rows.  With 64 dims a wave
// holds two groups.  The new rows of 16 tokens stay in registers between the maximum and
// the codes, so they are read once; larger runs are read twice, the second time from L2.
// Measured: store, 4200 rows of 4 KV heads of 128 dims (13 MB in and out) 8.3 us, 64
// single rows of 8 heads 6.4 (slot, scale, codes and stores wait for one another); load,
// 64k rows of 8 heads (131 MB of codes to 262 MB) 84 us, a copy's 5.2 TB/s counting the 40
// MB of codes that are fetched a second time; 1k rows of 4 heads 3.9 us.
// ---------------------------------------------------------------------------
constexpr int kRowThreads = 256;

struct StoreArgs {
  milo_pages p;
  const uint16_t* k;
  const uint16_t* v;
  int64_t k_stride, v_stride;
  const int32_t* slots;
  int32_t n_tok, lg_page, n_slots;
  int32_t chunk;  // rows of the call a workgroup looks at
  int32_t share;  // waves that share a page's rows: 1 or 4 (all: they meet at a barrier)
};

__device__ inline uint32_t wave_max(uint32_t x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, o));
  return x;
}

__device__ inline uint32_t abs_max2(uint32_t m, uint32_t x) {  // both halves
  const uint32_t lo = max(m & 0xFFFFu, x & 0x7FFFu), hi = max(m >> 16, (x >> 16) & 0x7FFFu);
  return lo | hi << 16;
}

// eight bf16 values (16 bytes) under scale s as eight codes; E4M3 scales are powers
// of two, whose reciprocal is exact
template <int FMT>
__device__ __forceinline__ uint2 codes_of_row(const uint4& x, float s) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = bf16_value(w[i] & 0xFFFFu);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
  if (!(s > 0.f)) return make_uint2(0, 0);
  if constexpr (FMT == MILO_KV_E4M3) {
    const float r = 1.f / s;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] *= r;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __fdiv_rn(f[i], s);
  }
  return make_uint2(codes_of<FMT>(make_float4(f[0], f[1], f[2], f[3])), codes_of<FMT>(make_float4(f[4], f[5], f[6], f[7])));
}

// the four codes of a dword under scale `was`, under scale s
template <int FMT>
__device__ __forceinline__ uint32_t rescaled(uint32_t w, float was, float s) {
  const float4 c = code_values<FMT>(w);
  return codes_of<FMT>(over<FMT>(make_float4(__fmul_rn(c.x, was), __fmul_rn(c.y, was), __fmul_rn(c.z, was),
                                             __fmul_rn(c.w, was)), s));
}

// byte b of words a, b, c, d as one word
__device__ __forceinline__ uint32_t gather_byte(uint32_t a, uint32_t b, uint32_t c, uint32_t d, int k) {
  const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x0C0C0000u | (uint32_t)(4 + k) << 8 | (uint32_t)k);
  const uint32_t hi = __builtin_amdgcn_perm(d, c, 0x0C0C0000u | (uint32_t)(4 + k) << 8 | (uint32_t)k);
  return lo | hi << 16;
}

// rows x .. (run of them) into offsets off .. of a page and head: keys (VALUES false)
// or values.  `share` waves, this one `mine`, take its groups in turn and their largest
// magnitudes together through `seen`.
template <int D, int FMT, bool VALUES>
__device__ void store_side(const uint16_t* x, int64_t stride, uint8_t* codes, float* scale_at, int off, int run, int mine,
                           int share, uint32_t* seen, bool works) {
  constexpr int LPG = D / 2, GPW = 64 / LPG;  // lanes of a group of 16 rows, groups of a wave
  const int lane = threadIdx.x & 63, sub = mine * GPW + lane / LPG, step = share * GPW;
  const int ch = lane % (D / 8), q = lane % LPG / (D / 8);
  const float was = works && off > 0 ? *scale_at : 0.f;
  const int g0 = off >> 4, g1 = works ? (off + run + 15) >> 4 : 0;
  uint4 v[4];
  const auto load = [&](int g) {  // the group's new rows, zeros in the others
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = 16 * g + 4 * q + i - off;
      v[i] = t >= 0 && t < run ? *reinterpret_cast<const uint4*>(x + (int64_t)t * stride + 8 * ch) : make_uint4(0, 0, 0, 0);
    }
  };
  uint32_t mx = 0;
  for (int g = g0 + sub; g < g1; g += step) {
    load(g);
#pragma unroll
    for (int i = 0; i < 4; ++i) mx = abs_max2(abs_max2(abs_max2(abs_max2(mx, v[i].x), v[i].y), v[i].z), v[i].w);
  }
  mx = wave_max(max(mx & 0xFFFFu, mx >> 16));
  if (share > 1) {
    if (lane == 0) seen[threadIdx.x >> 6] = mx;
    __syncthreads();
    for (int k = 0; k < share; ++k) mx = max(mx, seen[(threadIdx.x >> 6) - mine + k]);
  }
  if (!works) return;
  float s = scale_of<FMT>(mx);
  if (off > 0 && !(s >= was)) s = was >= s || was != was ? was : s;  // the larger, NaN before all
  const bool grew = off > 0 && s != was && s == s;
  const bool loaded = g1 - g0 <= step;  // the new rows are still in registers
  for (int g = grew ? (g0 + sub) % step : g0 + sub; g < g1; g += step) {
    if (g >= g0 && !loaded) load(g);
    uint2 c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = g < g0 ? make_uint2(0, 0) : codes_of_row<FMT>(v[i], s);
    const int t0 = 16 * g + 4 * q;
    if constexpr (!VALUES) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = t0 + i;
        uint2* at = reinterpret_cast<uint2*>(codes + key_byte(t, 8 * ch, D));
        if (t >= off) {
          if (t < off + run) *at = c[i];
        } else if (grew) {
          const uint2 w = *at;
          *at = make_uint2(rescaled<FMT>(w.x, was, s), rescaled<FMT>(w.y, was, s));
        }
      }
    } else {
      // which of the quad's rows are new and which held
      uint32_t fresh = 0, held = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = t0 + i;
        if (t >= off && t < off + run) fresh |= 255u << 8 * i;
        if (t < off) held |= 255u << 8 * i;
      }
      if (fresh || (held && grew)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          uint32_t w = e < 4 ? gather_byte(c[0].x, c[1].x, c[2].x, c[3].x, e) : gather_byte(c[0].y, c[1].y, c[2].y, c[3].y, e - 4);
          uint32_t* at = reinterpret_cast<uint32_t*>(codes + value_byte(t0, 8 * ch + e, D));
          if (fresh != ~0u) {
            const uint32_t old = *at;
            w = (w & fresh) | (old & ~fresh);
            if (grew) w = (w & ~held) | (rescaled<FMT>(old, was, s) & held);
          }
          *at = w;
        }
      }
    }
  }
  if (lane == 0 && mine == 0) *scale_at = s;
}

// Workgroups: `chunk` rows of the call by 4 / share of the 2 H (head, side) pairs.  A row
// that begins a run (rows that follow one another in a page) brings the run with it; the
// others are passed over.  All four waves go through the same runs.
template <int D, int FMT>
__global__ __launch_bounds__(kRowThreads) void store_kernel(StoreArgs a) {
  __shared__ uint32_t seen[2][kRowThreads / 64];  // in turn: a wave may still read the last run's
  const int H = a.p.n_kv_heads, P = 1 << a.lg_page, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), mine = wave & (a.share - 1);
  const int pair = (blockIdx.y * (kRowThreads / 64) + wave) / a.share;
  const bool works = pair < 2 * H;
  const int h = pair >> 1;
  int turn = 0;
  // the rows that begin a run, by one look at the chunk's slots
  const int64_t t0 = (int64_t)blockIdx.x * a.chunk, tl = t0 + lane;
  const bool mine_to_see = lane < a.chunk && tl < a.n_tok;
  const int slot_l = mine_to_see ? a.slots[tl] : -1, last_l = mine_to_see && tl > 0 ? a.slots[tl - 1] : -1;
  const bool in = (uint32_t)slot_l < (uint32_t)a.n_slots;
  uint64_t begins = __ballot(in && ((slot_l & (P - 1)) == 0 || tl == 0 || last_l != slot_l - 1));
  for (; begins; begins &= begins - 1) {
    const int l = __builtin_ctzll(begins);
    const int64_t t = t0 + l;
    const int slot = __builtin_amdgcn_readlane(slot_l, l), off = slot & (P - 1);
    int run = 0;  // rows whose slots go on from this one's in the page
    for (int k = 0; k < P; k += 64) {
      const int r = k + lane;
      const bool on = r < P - off && t + r < a.n_tok && a.slots[t + r] == slot + r;
      const uint64_t m = __ballot(on);
      run += ~m == 0 ? 64 : __builtin_ctzll(~m);
      if (~m != 0) break;
    }
    const int64_t ph = (int64_t)(slot >> a.lg_page) * H + (works ? h : 0);
    if (pair & 1)
      store_side<D, FMT, true>(a.v + t * a.v_stride + h * D, a.v_stride, (uint8_t*)a.p.v_codes + ph * P * D,
                               a.p.v_scale + ph, off, run, mine, a.share, seen[turn], works);
    else
      store_side<D, FMT, false>(a.k + t * a.k_stride + h * D, a.k_stride, (uint8_t*)a.p.k_codes + ph * P * D,
                                a.p.k_scale + ph, off, run, mine, a.share, seen[turn], works);
    turn ^= 1;
  }
}

struct LoadArgs {
  milo_pages p;
  uint16_t* k;
  uint16_t* v;
  int64_t k_stride, v_stride;
  const int32_t* slots;
  int32_t n_tok, lg_page, n_slots;
};

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) { return bf16_bits(a) | bf16_bits(b) << 16; }

// Waves: 16 output rows (32 with 64 dims) by (head, side) pairs.  Rows may come from
// anywhere; where a lane's four follow one another, as a request's do, their values
// are in one or two dwords per dim.
template <int D, int FMT>
__global__ __launch_bounds__(kRowThreads) void load_kernel(LoadArgs a) {
  constexpr int LPG = D / 2, GPW = 64 / LPG;
  const int H = a.p.n_kv_heads, P = 1 << a.lg_page, lane = threadIdx.x & 63;
  const int pair = blockIdx.y * (kRowThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (pair >= 2 * H) return;
  const int h = pair >> 1;
  const bool values = pair & 1;
  uint16_t* out = values ? a.v : a.k;
  if (!out) return;
  const int64_t stride = values ? a.v_stride : a.k_stride;
  const uint8_t* codes = static_cast<const uint8_t*>(values ? a.p.v_codes : a.p.k_codes);
  const float* scales = values ? a.p.v_scale : a.p.k_scale;
  const int ch = lane % (D / 8), q = lane % LPG / (D / 8);
  const int64_t j0 = ((int64_t)blockIdx.x * GPW + lane / LPG) * 16 + 4 * q;
  int slot[4];
  float s[4];
  const uint8_t* base[4];  // the row's page and head
  bool in[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    slot[i] = j0 + i < a.n_tok ? a.slots[j0 + i] : -1;
    in[i] = (uint32_t)slot[i] < (uint32_t)a.n_slots;
    const int64_t ph = (int64_t)(in[i] ? slot[i] >> a.lg_page : 0) * H + h;
    s[i] = scales[ph];
    base[i] = codes + ph * P * D;
    slot[i] = in[i] ? slot[i] & (P - 1) : 0;
  }
  uint2 c[4];  // the rows' eight codes
  if (!values) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = *reinterpret_cast<const uint2*>(base[i] + key_byte(slot[i], 8 * ch, D));
  } else {
    const uint8_t* at[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) at[i] = base[i] + value_byte(slot[i] & ~3, 8 * ch, D);
    const bool one = at[0] == at[3] && at[1] == at[0] && at[2] == at[0];
    const bool two = (at[1] == at[0] || at[1] == at[3]) && (at[2] == at[0] || at[2] == at[3]);
    // dim 8 ch + e of the same rows lies e dwords of 16 bytes on (value_byte)
    uint32_t w[4][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[0][e] = *reinterpret_cast<const uint32_t*>(at[0] + 16 * e);
    if (one) {
#pragma unroll
      for (int e = 0; e < 8; ++e) w[1][e] = w[2][e] = w[3][e] = w[0][e];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) w[3][e] = *reinterpret_cast<const uint32_t*>(at[3] + 16 * e);
      if (two) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          w[1][e] = at[1] == at[0] ? w[0][e] : w[3][e];
          w[2][e] = at[2] == at[0] ? w[0][e] : w[3][e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          w[1][e] = *reinterpret_cast<const uint32_t*>(at[1] + 16 * e);
          w[2][e] = *reinterpret_cast<const uint32_t*>(at[2] + 16 * e);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int sh = (slot[i] & 3) * 8;
      c[i].x = (w[i][0] >> sh & 255u) | (w[i][1] >> sh & 255u) << 8 | (w[i][2] >> sh & 255u) << 16 | (w[i][3] >> sh & 255u) << 24;
      c[i].y = (w[i][4] >> sh & 255u) | (w[i][5] >> sh & 255u) << 8 | (w[i][6] >> sh & 255u) << 16 | (w[i][7] >> sh & 255u) << 24;
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (j0 + i >= a.n_tok) continue;
    const float4 x = code_values<FMT>(c[i].x), y = code_values<FMT>(c[i].y);
    uint4 r = make_uint4(bf16_pair(s[i] * x.x, s[i] * x.y), bf16_pair(s[i] * x.z, s[i] * x.w),
                         bf16_pair(s[i] * y.x, s[i] * y.y), bf16_pair(s[i] * y.z, s[i] * y.w));
    if (!in[i]) r = make_uint4(0, 0, 0, 0);
    // past the caches, which the codes then have: 64k rows of 14B heads 85 us against 91, with the
    // read of them that follows 144 either way; 32k rows 31 against 43
    typedef uint32_t Line __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(__builtin_bit_cast(Line, r), reinterpret_cast<Line*>(out + (j0 + i) * stride + h * D + 8 * ch));
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
  if (n_req > kMaxPagesReq) return pages_fail(MILO_ERR_UNSUPPORTED, "more than %d requests", kMaxPagesReq);
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
  if (n_req <= kPlanThreads && n_slots <= kOneLaunch) {
    hipLaunchKernelGGL(plan_scan_kernel<true>, dim3(1), dim3(kPlanThreads), 0, s, a);
    return launched("plan kernel");
  }
  hipLaunchKernelGGL(plan_scan_kernel<false>, dim3(1), dim3(kPlanThreads), 0, s, a);
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
  if (n_tok > kMaxPagesRows) return pages_fail(MILO_ERR_UNSUPPORTED, "n_tok must be at most 2^27");
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
  // Few rows: a workgroup for each, since each may begin a run; many: one for 16 of them,
  // most of which are inside another's run.  The four waves share a page's rows where it has
  // groups for them (4096 rows, pages of 64, 7B heads: 15.6 us with one wave each).
  a.chunk = n_tok <= 2048 ? 1 : 16;
  const int groups = pages->page_tokens / (pages->head_dim == 64 ? 32 : 16);
  a.share = groups >= 4 ? 4 : 1;
  const dim3 grid((n_tok + a.chunk - 1) / a.chunk, (2 * pages->n_kv_heads * a.share + 3) / 4);
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  MILO_PAGES_DISPATCH(store_kernel, a, grid, kRowThreads, s);
  return launched("store kernel");
}

int milo_pages_load(const milo_pages* pages, const int32_t* slots, int32_t n_tok, uint16_t* k_out, int64_t k_stride,
                    uint16_t* v_out, int64_t v_stride, void* hip_stream) {
  clear_error();
  if (const int e = check_pages(pages); e != MILO_OK) return e;
  if (n_tok < 0) return pages_fail(MILO_ERR_INVALID_ARG, "n_tok must be >= 0");
  if (n_tok > kMaxPagesRows) return pages_fail(MILO_ERR_UNSUPPORTED, "n_tok must be at most 2^27");
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
  const int rows = pages->head_dim == 64 ? 32 : 16;
  const dim3 grid((uint32_t)(((int64_t)n_tok + rows - 1) / rows), (2 * pages->n_kv_heads + 3) / 4);
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  MILO_PAGES_DISPATCH(load_kernel, a, grid, kRowThreads, s);
  return launched("load kernel");
}

}  // extern "C"
