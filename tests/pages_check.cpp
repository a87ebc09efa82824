// Checks the division of a paged attention call's work into shares (milo_pages.h) on the
// host: over random batches every tile's rows are covered once, in order, by consecutive
// shares, and the shares agree on who holds what.  Prints "ok <calls> <tiles> <split tiles>".
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "milo_pages.h"

namespace milo {
int report_error(int code, const char*) { return code; }
}
using namespace milo;

#define CHECK(c)                                                       \
  do {                                                                 \
    if (!(c)) {                                                        \
      std::printf("line %d: %s (call %d)\n", __LINE__, #c, call);      \
      return 1;                                                        \
    }                                                                  \
  } while (0)

int main() {
  std::mt19937 rng(11);
  auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
  long tiles_seen = 0, split = 0;
  int call = 0;
  for (int tt = 1; tt <= 128; ++tt)
    for (int k = 0; k < 2000; ++k) {
      const int m = k < 500 ? k : pick(0, 1 << 24);
      CHECK(tiles_of(m, tt, reciprocal(tt)) == (m + tt - 1) / tt);
    }
  for (; call < 3000; ++call) {
    const int n_req = pick(1, call % 3 ? 6 : 400), H = pick(1, 8), tt = pick(1, 128), causal = pick(0, 1);
    const uint32_t inv = reciprocal(tt);
    const int long_n = call % 5 == 0 ? 100000 : 700, many = call % 4 == 0 ? 900 : 5;
    std::vector<Request> req(n_req);
    int start = 0;
    for (auto& q : req) {
      q.m = pick(0, 3) ? pick(0, many) : pick(0, 1);
      q.n = pick(0, 3) ? pick(0, long_n) : pick(0, 2) * 64;
      q.start = start;
      start += q.m;
    }
    int calls_out = 0;
    const auto get = [&](int r) {
      if (r < 0 || r >= n_req) {
        ++calls_out;
        return Request{0, 1, 0};
      }
      return req[r];
    };
    std::vector<int> pre(n_req + 1, 0);
    for (int r = 0; r < n_req; ++r) {
      const int all = (req[r].m + tt - 1) / tt;
      int64_t rows = 0;
      for (int k = 0; k <= all; ++k) {
        CHECK(tiles_cost(req[r], k, all, tt, causal) == rows / kRowAlign + k * kTileCost);
        if (k < all) rows += seen_upto(req[r], (k + 1) * tt, causal);
      }
      const int64_t next = pre[r] + (int64_t)H * tiles_cost(req[r], all, all, tt, causal);
      CHECK(next < INT32_MAX);
      pre[r + 1] = (int)next;
    }
    const int X = pre[n_req];
    if (X == 0) continue;
    const bool two = call % 4 == 3;  // two shares a CU, of different lengths
    const int W = two ? 2 * kCus : std::min(pick(1, 512), X), L = (X + W - 1) / W, La = two ? L + L / 6 : L;
    // the tiles in order, each with the row up to which it is done
    int r = 0, head = 0, tile = 0, done = 0, parts = 0, last_end = -1;
    while (req[r].m == 0) ++r;
    for (int w = 0; w < W; ++w) {
      CHECK(share_at(w, L, La) < share_at(w + 1, L, La));
      const int b0 = (int)std::min<int64_t>(X, share_at(w, L, La)), b1 = (int)std::min<int64_t>(X, share_at(w + 1, L, La));
      if (b0 >= X) continue;
      int lo = 0;
      while (pre[lo + 1] <= b0) ++lo;
      lo = lo > 2 ? lo - pick(0, 2) : lo;  // any request before will do
      Place at = place_of(get, lo, pre[lo], b0, H, tt, inv, causal);
      bool first = true;
      for (int pos = b0; pos < b1;) {
        CHECK(calls_out == 0 && at.r == r && at.head == head && at.tile == tile);
        const Request q = at.rq;
        const int j0 = tile * tt, ntok = std::min(tt, q.m - j0), vis = seen_upto(q, j0 + ntok, causal);
        CHECK(ntok >= 1 && vis <= q.n);
        const int p0 = at.p0, p1 = at.p1;
        CHECK(p0 <= pos && pos < p1 && (first || p0 == pos));
        const int ra = row_at(b0, p0, p1, vis), rb = row_at(b1, p0, p1, vis);
        CHECK(ra == done && ra <= rb && rb <= vis && (ra % kRowAlign == 0 || ra == vis) && (rb % kRowAlign == 0 || rb == vis));
        CHECK(share_of(pos, L, La) == w && share_of(std::min(p1, b1) - 1, L, La) == w);
        const bool whole = b0 <= p0 && b1 >= p1;
        CHECK(!whole || (ra == 0 && rb == vis && parts == 0));
        if (!whole && b0 <= p0) last_end = share_of(p1 - 1, L, La);
        if (!whole) CHECK(parts == 0 ? b0 <= p0 && b1 < p1 : first);
        done = rb;
        ++parts;
        pos = p1;
        if (b1 >= p1) {  // the tile ends here
          CHECK(done == vis && (whole || last_end == w));
          ++tiles_seen;
          split += parts > 1;
          done = parts = 0;
          if (++tile >= (req[r].m + tt - 1) / tt) {
            tile = 0;
            if (++head >= H) {
              head = 0;
              do ++r;
              while (r < n_req && req[r].m == 0);
            }
          }
        }
        first = false;
        if (pos < b1) next_tile(get, at, H, tt, inv, causal);
      }
    }
    CHECK(r == n_req && calls_out == 0 && share_at(W, L, La) >= X);
  }
  std::printf("ok %d %ld %ld\n", call, tiles_seen, split);
  return 0;
}
