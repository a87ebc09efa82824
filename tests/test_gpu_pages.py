"""The paged 8-bit cache on the GPU against the fp64 oracle.

Bookkeeping, codes and scales are held to equality.  Attention is held to worst-case bounds,
element by element, from the roundings on the way (u = 2^-24 that of fp32, size = the average
of |values| under the softmax, reach = the largest sum |q_c k_c| scale of a score):
 - a score is a sum of d exact products and three roundings more: (d + 8) u reach, which a
   weight takes on as a relative error;
 - a weight enters the value product as one fp16 (2^-11) for bf16 output, as two (2^-22) for
   fp32 output, or, small, off by 2^-32 of the largest (each of n rows of codes up to 448, under
   the largest scale, for the largest weight peak); 2^-22 covers the exponential;
 - sums of up to n weights or weighted values, and their rescalings: (n / 8 + 64) u;
 - the output's own rounding, 2^-8 of it as bf16."""
import numpy as np
import pytest
import torch

import oracle
import synth
from paper_2609_29913_amd import milo

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
FMTS = {"int8": milo.MILO_KV_INT8, "e4m3": milo.MILO_KV_E4M3}


def i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def bf16(x):
    return torch.as_tensor(np.asarray(x, dtype=np.float32), device="cuda").to(torch.bfloat16)


def f64(x):
    return x.double().cpu().numpy()


def key_byte(t, c, d):
    return ((t // 16) * (d // 16) + c // 16) * 256 + (t % 16) * 16 + c % 16


def value_byte(t, c, d):
    return ((t // 16) * (d // 64) + c // 64) * 1024 + (t % 16) // 4 * 256 + c % 16 * 16 + c % 64 // 16 * 4 + t % 4


def put(pages, rows_k, rows_v, ks, vs):
    """Code values [n_pages][P][H][d] and scales into the pool's storage."""
    P, d = pages.page_tokens, pages.head_dim
    t, c = np.arange(P)[:, None], np.arange(d)[None]
    for rows, codes, at in ((rows_k, pages.k_codes, key_byte(t, c, d)), (rows_v, pages.v_codes, value_byte(t, c, d))):
        raw = np.zeros(codes.shape)
        raw[:, :, at.reshape(-1)] = rows.transpose(0, 2, 1, 3).reshape(*codes.shape[:2], -1)
        codes.view(torch.uint8).copy_(torch.from_numpy(raw).float().to(codes.dtype).view(torch.uint8))
    pages.k_scale.copy_(torch.from_numpy(ks))
    pages.v_scale.copy_(torch.from_numpy(vs))


def get(pages, side):
    """The pool's code values [n_pages][P][H][d]."""
    P, d = pages.page_tokens, pages.head_dim
    t, c = np.arange(P)[:, None], np.arange(d)[None]
    codes = pages.k_codes if side == "k" else pages.v_codes
    at = (key_byte if side == "k" else value_byte)(t, c, d)
    raw = codes.float().double().cpu().numpy()[:, :, at.reshape(-1)]
    return raw.reshape(*codes.shape[:2], P, d).transpose(0, 2, 1, 3).copy()


def random_pool(rng, n_pages, P, H, d, fmt):
    """A pool of random codes, with its rows and scales."""
    pages = milo.milo_pages_create(n_pages, P, H, d, FMTS[fmt])
    rows, scales = [], []
    for _ in range(2):
        x = rng.standard_normal((n_pages, P, H, d)) * (40 if fmt == "int8" else 100)
        rows.append(np.clip(np.rint(x), -127, 127) if fmt == "int8" else oracle.e4m3_round(np.clip(x, -448, 448)))
        scales.append((rng.random((n_pages, H)) * 0.02 + 0.01).astype(np.float32))
    put(pages, *rows, *scales)
    return pages, rows, scales


# ---- plan -----------------------------------------------------------------------------------

def run_plan(lens, delta, P, table, ring, head, count, n_slots, **kw):
    t, r = i32(table), i32(ring)
    got = milo.milo_pages_plan(i32(lens), i32(delta), P, t, r, i32([head, count]), n_slots, **kw)
    lens_out, starts, slots, state, status = [x.cpu().numpy() for x in got]
    return int(status[0]), lens_out, starts, slots, t.cpu().numpy(), r.cpu().numpy(), tuple(state)


def same_plan(got, want):
    assert got[0] == want[0]
    for g, w in zip(got[1:], want[1:]):
        assert np.array_equal(np.asarray(g), np.asarray(w))


@pytest.mark.parametrize("P", [16, 128])
@pytest.mark.parametrize("n_req", [0, 1, 63, 1024, 2500])
def test_plan_steps(P, n_req):
    rng = np.random.default_rng(n_req + P)
    width, n_pages = 6, 3 * n_req + 5
    lens, table = np.zeros(n_req, dtype=np.int64), np.full((n_req, width), -9)
    ring, head, count = rng.permutation(n_pages), n_pages - 2, n_pages
    for step in range(6):
        delta = np.where(rng.random(n_req) < 0.3, -rng.integers(0, lens + 1), rng.integers(0, 2 * P if step == 0 else 3, n_req))
        want = oracle.pages_plan(lens, delta, P, table, ring, head, count, int(np.maximum(delta, 0).sum()) + 3)
        same_plan(run_plan(lens, delta, P, table, ring, head, count, len(want[3])), want)
        _, lens, _, _, table, ring, (head, count) = want
        lens = np.asarray(lens, dtype=np.int64)


def test_plan_long_prompts():
    lens, delta = [3, 0, 40, 17], [70001, 0, 5000, -17]
    table, ring = np.full((4, 4400), -1), np.random.default_rng(2).permutation(4800)
    table[0, 0], table[2, :3], table[3, :2] = 4801, [4802, 4803, 4804], [4805, 4806]
    ring = np.concatenate([ring, [-1] * 10])
    want = oracle.pages_plan(lens, delta, 16, table, ring, 0, 4800, 75001)
    assert want[0] == 0
    same_plan(run_plan(lens, delta, 16, table, ring, 0, 4800, 75001), want)


@pytest.mark.parametrize("what,status", [
    (dict(count=2), 1), (dict(delta=[200, 1, 1]), 2), (dict(delta=[-21, 1, 1]), 4), (dict(lens=[-1, 3, 3]), 4),
    (dict(n_slots=10), 8), (dict(head=30), 16), (dict(head=-1), 16), (dict(count=31), 16), (dict(delta=[-20, 1, 1], count=29), 16),
    (dict(delta=[200, -9, 1], n_slots=0), 14), (dict(delta=[2 ** 31 - 1, 2 ** 31 - 1, 0]), 2)])
def test_plan_refuses_a_step_as_a_whole(what, status):
    f = dict(lens=[20, 3, 3], delta=[40, 1, 20], P=16, table=np.arange(15).reshape(3, 5), ring=np.arange(30), head=29, count=9,
             n_slots=64)
    f.update(what)
    want = oracle.pages_plan(**{("page_tokens" if k == "P" else k): v for k, v in f.items()})
    assert want[0] == status
    same_plan(run_plan(**f), want)


def test_plan_in_place_and_captured():
    """lens and ring_state updated in place, a decode loop replayed from a graph."""
    n, P = 37, 16
    lens, delta = i32(np.arange(n) % 20), i32([1] * n)
    state, ring, table = i32([5, 150]), i32(np.arange(200)), i32(np.arange(200, 200 + 3 * n).reshape(n, 3))
    ref = [x.cpu().numpy().copy() for x in (lens, table, ring, state)]
    outs = dict(lens_out=lens, ring_state_out=state, starts=i32([0] * (n + 1)), slots=i32([0] * n), status=i32([9]),
                work=torch.zeros(milo.lib().milo_pages_plan_work(n) // 4, dtype=torch.int32, device="cuda"))
    call = lambda: milo.milo_pages_plan(lens, delta, P, table, ring, state, **outs)  # noqa: E731
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    h = (int(ref[3][0]), int(ref[3][1]))
    for step in range(20):
        want = oracle.pages_plan(ref[0], [1] * n, P, ref[1], ref[2], *h, n)
        g.replay() if step % 3 else call()
        got = (int(outs["status"]), lens.cpu().numpy(), outs["starts"].cpu().numpy(), outs["slots"].cpu().numpy(),
               table.cpu().numpy(), ring.cpu().numpy(), tuple(state.tolist()))
        same_plan(got, want)
        ref[0], ref[1], ref[2], h = np.asarray(want[1]), want[4], want[5], want[6]


# ---- store and load ---------------------------------------------------------------------------

def check_pool(pages, rows, scales):
    for side, i in (("k", 0), ("v", 1)):
        got = (pages.k_scale if side == "k" else pages.v_scale).cpu().numpy()
        assert np.array_equal(got, scales[i], equal_nan=True), side
        assert np.array_equal(get(pages, side), rows[i]), side


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("P,H,d", [(16, 2, 64), (32, 1, 128), (64, 8, 128), (128, 3, 64)])
def test_store_appends(P, H, d, fmt):
    """Requests that start, grow by odd counts and restart pages, in rows of a wider buffer, some
    of them not stored; pages nobody writes keep every byte."""
    rng = np.random.default_rng(P + d)
    pages, rows, scales = random_pool(rng, 12, P, H, d, fmt)
    order = rng.permutation(12)
    for step, (first, n) in enumerate([(0, 1), (1, 5), (6, 2 * P + 3), (2 * P + 9, 1), (P - 1, 2), (3 * P, P), (0, 4)]):
        pos = np.arange(first, first + n)
        slots = order[pos // P] * P + pos % P
        more = np.array([-1, 12 * P, slots[0]])                    # rows that are not stored; a second page's start
        more[2] = order[8 + step % 4] * P
        slots = np.concatenate([slots, more])
        x = rng.standard_normal((2, n + 3, H, d)) * np.exp(rng.standard_normal((2, n + 3, 1, 1)))
        x[:, 0, 0] = 0 if step % 2 else x[:, 0, 0] * 9
        wide = bf16(rng.standard_normal((n + 3, 2 * H + 1, d)))
        wide[:, :H], wide[:, H:2 * H] = bf16(x[0]), bf16(x[1])
        k, v = wide[:, :H], wide[:, H:2 * H]
        for i, y in enumerate((k, v)):
            oracle.pages_store(rows[i], scales[i], P, f64(y), slots, fmt == "e4m3")
        milo.milo_pages_store(pages, k, v, i32(slots))
        check_pool(pages, rows, scales)
        milo.milo_pages_store(pages, k, v, i32(slots))             # the same rows again change nothing
        check_pool(pages, rows, scales)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_store_single_rows_of_many_requests(fmt):
    rng = np.random.default_rng(8)
    pages, rows, scales = random_pool(rng, 300, 16, 4, 128, fmt)
    for off in (0, 7, 8, 15):
        x = [bf16(rng.standard_normal((300, 4, 128)) * 2) for _ in range(2)]
        slots = rng.permutation(300) * 16 + off
        for i in range(2):
            oracle.pages_store(rows[i], scales[i], 16, f64(x[i]), slots, fmt == "e4m3")
        milo.milo_pages_store(pages, *x, i32(slots))
        check_pool(pages, rows, scales)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_store_extreme_values(fmt):
    """Zeros, the smallest and largest bf16 values, and values that are not finite: the page and
    head then holds NaN, the other heads and pages do not."""
    pages, rows, scales = random_pool(np.random.default_rng(1), 6, 16, 3, 64, fmt)
    x = np.zeros((8, 3, 64), dtype=np.float32)
    x[1] = 2.0 ** -133
    x[2], x[2, 1, 5] = 2.0 ** -126, -2.0 ** -120
    x[3], x[3, 2, 9] = 1.0, 3.3895e38
    x[4, 0, 3], x[4, 1, 60], x[4, 2] = np.inf, np.nan, 0.5
    x[5], x[6], x[7] = 0.25, 1.5, -np.inf
    slots = np.array([0, 16, 32, 48, 64, 65, 66, 5 * 16 + 3])
    k, v = bf16(x), bf16(x[::-1].copy())
    for i, y in enumerate((k, v)):
        oracle.pages_store(rows[i], scales[i], 16, f64(y), slots, fmt == "e4m3")
    milo.milo_pages_store(pages, k, v, i32(slots))
    check_pool(pages, rows, scales)
    assert np.isnan(scales[0][4, 0]) and not np.isnan(scales[0][4, 2])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("P,H,d", [(16, 2, 64), (64, 8, 128), (128, 1, 128)])
def test_load(P, H, d, fmt):
    rng = np.random.default_rng(3)
    pages, rows, scales = random_pool(rng, 9, P, H, d, fmt)
    runs = np.concatenate([np.arange(5 * P, 7 * P), np.arange(P // 2, P + 9), np.arange(3 * P)])
    for slots in (rng.integers(0, 9 * P, 77), runs, np.array([5]), np.array([-1, 9 * P, 3, 3, 2 ** 31 - 1, 9 * P - 1, -2 ** 31])):
        want = []
        for i in range(2):
            x = np.zeros((len(slots), H, d), dtype=np.float32)
            for j, s in enumerate(slots):
                if 0 <= s < 9 * P:
                    x[j] = rows[i][s // P, s % P].astype(np.float32) * scales[i][s // P][:, None]
            want.append(bf16(x))
        wide = torch.full((len(slots), 2 * H + 1, d), 7.0, dtype=torch.bfloat16, device="cuda")
        milo.milo_pages_load(pages, i32(slots), wide[:, :H], wide[:, H:2 * H])
        assert torch.equal(wide[:, :H], want[0]) and torch.equal(wide[:, H:2 * H], want[1]) and bool((wide[:, 2 * H] == 7).all())
        one = torch.empty((len(slots), H, d), dtype=torch.bfloat16, device="cuda")
        milo.milo_pages_load(pages, i32(slots), None, one)
        assert torch.equal(one, want[1])
        milo.milo_pages_load(pages, i32(slots), k_out=one)
        assert torch.equal(one, want[0])


# ---- attention ----------------------------------------------------------------------------------

class Batch:
    """Requests of given lengths and query counts over a pool, pages in random places."""

    def __init__(self, seed, lens, counts, heads, P, fmt, spread=1.0, spare=4):
        H_q, H, d = heads
        rng = np.random.default_rng(seed)
        need = [-(-n // P) for n in lens]
        self.pages, self.rows, self.scales = random_pool(rng, sum(need) + spare, P, H, d, fmt)
        ids = rng.permutation(sum(need) + spare)
        self.table = np.full((len(lens), max(need + [1]) + 1), -1)
        at = 0
        for i, m in enumerate(need):
            self.table[i, :m] = ids[at:at + m]
            at += m
        self.lens, self.counts, self.P = np.array(lens), np.array(counts), P
        self.starts = np.concatenate([[0], np.cumsum(counts)]).astype(int)
        self.scale = spread / np.sqrt(d)
        self.q = bf16(rng.standard_normal((int(self.starts[-1]), H_q, d)))

    def kv(self, i):
        t = np.arange(self.lens[i])
        pg = self.table[i, t // self.P]
        return [self.rows[s][pg, t % self.P] * self.scales[s][pg][:, :, None].astype(np.float64) for s in range(2)]

    def want(self, causal):
        parts = [oracle.attend_pages(*self.kv(i), f64(self.q[self.starts[i]:self.starts[i + 1]]), self.scale, causal)
                 for i in range(len(self.lens))]
        return [np.concatenate([p[k] for p in parts]) for k in range(4)]

    def run(self, causal=True, dtype=torch.float32, **kw):
        out = torch.full(self.q.shape, float("nan"), dtype=dtype, device="cuda")
        milo.milo_attend_pages(self.pages, i32(self.table), i32(self.lens), kw.pop("q", self.q), self.scale, out,
                               q_starts=i32(self.starts), causal=causal, **kw)
        return out

    def check(self, got, want):
        out, size, reach, peak = want
        n, d = max(int(self.lens.max()), 1), out.shape[-1]
        lost = 2.0 ** -11 if got.dtype == torch.bfloat16 else 2.0 ** -22
        small = n * 2.0 ** -32 * 448 * np.nanmax(self.scales[1]) * peak[..., None]
        rel = (d + 8) * U * reach[..., None] + 2.0 ** -22 + (n / 8 + 64) * U
        tol = (2 * rel + lost) * size + small + (2.0 ** -8 * np.abs(out) if got.dtype == torch.bfloat16 else 0) + 1e-30
        err = np.abs(f64(got) - out)
        assert np.all(np.isfinite(f64(got))) and np.all(err <= tol), float(np.max(err / tol))


HEADS = {"0.5b": (14, 2, 64), "7b": (28, 4, 128), "14b": (40, 8, 128), "one": (1, 1, 64), "sixteen": (32, 2, 128)}
SHAPES = {
    "one_row": ([1], [1], "0.5b", 16),
    "edges_16": ([15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257], [1] * 15, "7b", 16),
    "edges_128": ([127, 128, 129, 1, 255, 257, 0, 1000], [1] * 8, "14b", 128),
    "long": ([5000], [1], "one", 64),
    "ragged": ([3, 4000, 0, 1, 700, 2049], [1] * 6, "sixteen", 32),
    "none_and_one": ([0, 5, 0], [1, 1, 1], "one", 16),
    "few": ([40, 41, 300, 7, 2000], [2, 8, 5, 7, 3], "7b", 16),
    "no_queries": ([40, 41, 300], [0, 3, 0], "0.5b", 32),
    "chunk": ([333], [333], "7b", 32),
    "chunk_after": ([700, 90, 64], [130, 90, 1], "14b", 64),
    "more_queries_than_rows": ([5, 0, 60], [9, 4, 80], "0.5b", 16),
    "chunk_sixteen": ([200, 129], [70, 129], "sixteen", 128),
}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("name", sorted(SHAPES))
def test_attend(name, fmt, dtype):
    lens, counts, heads, P = SHAPES[name]
    b = Batch(sorted(SHAPES).index(name), lens, counts, HEADS[heads], P, fmt)
    for causal in (True, False):
        want = b.want(causal)
        got = b.run(causal, dtype)
        b.check(got, want)
        assert torch.equal(got, b.run(causal, dtype))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("spread", [8.0, -1.0, 0.0])
def test_attend_sharp_negative_and_flat_scales(spread, dtype):
    b = Batch(77, [900, 65, 130], [1, 6, 40], HEADS["7b"], 16, "int8", spread=spread)
    b.check(b.run(True, dtype), b.want(True))


@pytest.mark.parametrize("lens,counts", [([30000, 17, 9000], [1, 1, 1]), ([20011], [21]), ([12000, 300], [3, 150])])
def test_attend_long(lens, counts):
    """Requests whose rows are split over many workgroups and joined."""
    b = Batch(5, lens, counts, HEADS["0.5b"], 64, "e4m3")
    got = b.run()
    b.check(got, b.want(True))
    assert torch.equal(got, b.run())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attend_values_of_very_different_scales(dtype):
    """Pages whose values lie 2^40 apart, pages of zeros, requests of each kind alone: what small
    pages hold is not lost to the large ones' requests beside them."""
    b = Batch(21, [64, 100, 16, 400, 48], [1, 2, 1, 3, 1], HEADS["0.5b"], 16, "int8")
    for i, (lo, hi) in enumerate([(-70, -70), (-20, 20), (0, 0), (-4, 14), (-60, 30)]):
        for j, pg in enumerate(b.table[i, :-(-b.lens[i] // 16)]):
            b.scales[1][pg] = 0.0 if i == 2 or j == 1 else np.float32(2.0) ** (lo if j % 2 else hi)
    put(b.pages, *b.rows, *b.scales)
    b.lens = np.asarray(b.lens)
    want = b.want(True)
    got = b.run(True, dtype)
    whole = b.scales[1].copy()
    for i in range(5):  # each request against the scales of its own pages
        at = slice(b.starts[i], b.starts[i + 1])
        b.scales[1] = whole[b.table[i, :-(-b.lens[i] // 16)]]
        b.check(got[at], [w[at] for w in want])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attend_a_row_that_takes_the_weight_and_adds_nothing(dtype):
    """One row with nearly all of the weight and values of zero before thousands that share the
    rest: what is left of the output is theirs, to the usual error."""
    b = Batch(22, [9000, 500], [1, 1], HEADS["one"], 16, "int8")
    for i in range(2):
        first = b.table[i, 0]
        b.rows[0][first, 0], b.rows[1][first, 0] = 0, 0
        q = f64(b.q[i, 0])
        b.rows[0][first, 0, 0] = np.rint(127 * q / np.abs(q).max())
        b.scales[0][first] = np.float32((np.log(2e5) + 5) / (b.scale * (q @ b.rows[0][first, 0, 0])))
    put(b.pages, *b.rows, *b.scales)
    want = b.want(True)
    assert want[3].min() > 0.9
    b.check(b.run(True, dtype), want)


def test_attend_many_requests():
    rng = np.random.default_rng(6)
    lens = rng.integers(0, 90, 1500)
    b = Batch(6, list(lens), [1] * 1500, HEADS["one"], 16, "int8")
    b.check(b.run(), b.want(True))
    out = torch.full(b.q.shape, float("nan"), device="cuda")
    milo.milo_attend_pages(b.pages, i32(b.table), i32(b.lens), b.q, b.scale, out)     # without q_starts
    b.check(out, b.want(True))


@pytest.mark.parametrize("counts", [[1, 1, 1], [5, 1, 40]])
def test_attend_rows_behind_a_request_do_not_matter(counts):
    """NaN codes and NaN scales everywhere a request does not look, and queries of no request."""
    b = Batch(9, [50, 17, 129], counts, HEADS["7b"], 16, "e4m3")
    for i in range(3):
        n = b.lens[i]
        last = b.table[i, (n - 1) // 16]
        t = np.arange(16)[n % 16 or 16:]
        for codes, at in ((b.pages.k_codes, key_byte), (b.pages.v_codes, value_byte)):
            raw = codes.view(torch.uint8)
            for tt in t:
                raw[last][:, torch.from_numpy(at(tt, np.arange(128), 128)).cuda()] = 0x7F
    spare = [x for x in range(b.pages.n_pages) if x not in b.table]
    b.pages.k_scale[spare], b.pages.v_scale[spare] = float("nan"), float("nan")
    b.table[b.table < 0] = spare[0]
    n, pad = b.q.shape[0], 3
    wide = torch.full((n + pad, 30, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:n, :28] = b.q
    out = torch.full((n + pad, 28, 128), 7.0, device="cuda")
    milo.milo_attend_pages(b.pages, i32(b.table), i32(b.lens), wide[:, :28], b.scale, out, q_starts=i32(b.starts))
    b.check(out[:n], b.want(True))
    assert bool((out[n:] == 7).all())


def test_attend_causal_queries_do_not_see_a_later_page_of_nan():
    b = Batch(10, [64, 40], [40, 30], HEADS["0.5b"], 16, "int8")
    want = b.want(True)
    b.pages.k_scale[int(b.table[0, 3])], b.pages.v_scale[int(b.table[0, 3])] = float("nan"), float("nan")
    got = b.run()
    seen = np.arange(40) + 25 > 48
    assert bool(torch.isnan(got[:40][torch.from_numpy(seen).cuda()]).all())
    ok = np.concatenate([~seen, np.ones(30, bool)])
    b.check(got[torch.from_numpy(ok).cuda()], [w[ok] for w in want])


def test_attend_bad_pages_and_lengths():
    """Lengths out of range are cut, a page out of range makes its request NaN, starts are cut."""
    b = Batch(11, [50, 33, 20], [1, 1, 1], HEADS["0.5b"], 16, "int8")
    want = b.want(True)
    table = b.table.copy()
    table[1, 1] = b.pages.n_pages
    out = torch.full(b.q.shape, 7.0, device="cuda")
    milo.milo_attend_pages(b.pages, i32(table), i32([50, 33, -5]), b.q, b.scale, out)
    b.check(out[:1], [w[:1] for w in want])
    assert bool(torch.isnan(out[1]).all()) and bool((out[2] == 0).all())
    out.fill_(7.0)
    milo.milo_attend_pages(b.pages, i32(b.table), i32(b.lens), b.q, b.scale, out, q_starts=i32([-4, 1, 2, 9]))
    b.check(out, want)
    b2 = Batch(12, [64], [1], HEADS["0.5b"], 16, "int8")
    out = torch.full(b2.q.shape, 7.0, device="cuda")
    milo.milo_attend_pages(b2.pages, i32(b2.table[:, :4]), i32([1 << 30]), b2.q, b2.scale, out)
    b2.check(out, b2.want(True))


def test_attend_on_another_stream():
    b = Batch(13, [700, 90, 64], [13, 90, 1], HEADS["7b"], 64, "int8")
    want = b.want(True)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for stream in (s, s.cuda_stream):
        out = torch.full(b.q.shape, float("nan"), device="cuda")
        args = [i32(b.table), i32(b.lens), b.q, b.scale, out]
        starts = i32(b.starts)
        torch.cuda.synchronize()
        milo.milo_attend_pages(b.pages, *args, q_starts=starts, stream=stream)
        s.synchronize()
        b.check(out, want)


# ---- together -------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_with_a_compressed_context(fmt):
    """The pages take the place of the dense tails: milo_attend_decode's result on the rows the
    pages hold, at the bar of the compressed blocks' roundings (1e-2)."""
    from helpers import GpuLayer, max_rel_l2, oracle_args
    inp = synth.make_problem(31, [300, 256, 700], [64, 40, 96], n_kv_heads=4, head_dim=128, n_q=3, n_q_heads=28, tail_cap=80)
    b = Batch(31, [80, 0, 33], [1, 1, 1], HEADS["7b"], 16, fmt)
    b.q = torch.from_numpy(inp.q.view(np.int16)).cuda().view(torch.bfloat16)
    a = oracle_args(inp)
    a["table"] = [2, 0]
    a["tail_len"] = b.lens
    for side, name in ((0, "tail_k"), (1, "tail_v")):
        a[name] = np.zeros((3, 80, 4, 128))
        for i in range(3):
            a[name][i, :b.lens[i]] = b.kv(i)[side]
    ref = oracle.attend_latent(**a)
    gl = GpuLayer(inp)
    try:
        for dtype in (torch.float32, torch.bfloat16):
            b.scale = inp.scale
            got = b.run(True, dtype, cache=gl.cache, block_table=[2, 0])
            assert max_rel_l2(f64(got), ref) <= 1e-2
        pages_only = b.run(True, cache=gl.cache, block_table=[])
        assert torch.equal(pages_only, b.run(True))
        with pytest.raises(milo.MiloError):   # rows of q apart
            milo.milo_attend_pages(b.pages, i32(b.table), i32(b.lens), torch.zeros((3, 30, 128), dtype=torch.bfloat16,
                                   device="cuda")[:, :28], b.scale, torch.empty(b.q.shape, device="cuda"),
                                   cache=gl.cache, block_table=[0])
    finally:
        gl.free()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_a_serving_loop(fmt):
    """Prompts enter, requests decode from a captured graph, one ends and its pages serve another:
    plan, store and attend together, against rows quantised by the oracle."""
    rng = np.random.default_rng(40)
    H_q, H, d = HEADS["0.5b"]
    P, n_req, n_pages, width = 16, 4, 24, 8
    pages = milo.milo_pages_create(n_pages, P, H, d, FMTS[fmt])
    rows = [np.zeros((n_pages, P, H, d)) for _ in range(2)]
    scales = [np.zeros((n_pages, H), dtype=np.float32) for _ in range(2)]
    lens, table, ring, state = i32([0] * n_req), i32(np.full((n_req, width), -1)), i32(np.arange(n_pages)), i32([0, n_pages])
    host = [[0] * n_req, np.full((n_req, width), -1), np.arange(n_pages), (0, n_pages)]

    def step(delta, bufs=None, graph=None):
        n = int(np.maximum(delta, 0).sum())
        x = bf16(rng.standard_normal((n, H_q + 2 * H, d)))
        if bufs is None:
            bufs = dict(x=x, delta=i32(delta), out=torch.empty((n, H_q, d), device="cuda"), starts=i32([0] * (n_req + 1)),
                        slots=i32([0] * n), status=i32([0]),
                        work=torch.empty(milo.lib().milo_attend_pages_work(n_req, n, H_q, H, d, 0), dtype=torch.uint8, device="cuda"),
                        plan=torch.empty(milo.lib().milo_pages_plan_work(n_req) // 4, dtype=torch.int32, device="cuda"))
        else:
            bufs["x"].copy_(x)

        def call():
            milo.milo_pages_plan(lens, bufs["delta"], P, table, ring, state, lens_out=lens, ring_state_out=state,
                                 starts=bufs["starts"], slots=bufs["slots"], status=bufs["status"], work=bufs["plan"])
            y = bufs["x"]
            milo.milo_pages_store(pages, y[:, H_q:H_q + H], y[:, H_q + H:], bufs["slots"])
            milo.milo_attend_pages(pages, table, lens, y[:, :H_q], d ** -0.5, bufs["out"], q_starts=bufs["starts"],
                                   work=bufs["work"])

        if graph is None:
            call()
        elif isinstance(graph, list):
            g = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(g):
                call()
            graph.append(g)
            g.replay()
        else:
            graph.replay()
        st, host[0], starts, slots, host[1], host[2], host[3] = oracle.pages_plan(
            host[0], delta, P, host[1], host[2], *host[3], n)
        assert st == 0 and int(bufs["status"]) == 0
        for side in range(2):
            y = f64(x[:, H_q + side * H:H_q + (side + 1) * H])
            oracle.pages_store(rows[side], scales[side], P, y, slots, fmt == "e4m3")
        b = Batch.__new__(Batch)
        b.rows, b.scales, b.table, b.lens, b.P = rows, scales, host[1], np.array(host[0]), P
        b.starts, b.scale, b.q, b.counts = np.array(starts), d ** -0.5, x[:, :H_q], None
        b.check(bufs["out"], b.want(True))
        check_pool(pages, rows, scales)
        return bufs

    step([33, 5, 0, 60])
    graph = []
    bufs = step([1, 1, 1, 1], graph=graph)
    for k in range(18):
        step([1, 1, 1, 1], bufs, graph[0])
    step([-int(host[0][0]), 2, -3, 0])
    step([90, 0, 4, 1])
    for k in range(3):
        step([1, 1, 1, 1], bufs, graph[0])


def test_pages_feed_the_encoder():
    """Rows read back are the encoder's input: the singular values of a request's rows."""
    rng = np.random.default_rng(50)
    pages = milo.milo_pages_create(8, 32, 2, 64)
    x = rng.standard_normal((200, 8)) @ rng.standard_normal((8, 128))
    k = bf16(x).view(200, 2, 64)
    slots = i32(np.random.default_rng(1).permutation(8)[np.arange(200) // 32] * 32 + np.arange(200) % 32)
    milo.milo_pages_store(pages, k, k, slots)
    got = torch.empty((200, 2, 64), dtype=torch.bfloat16, device="cuda")
    milo.milo_pages_load(pages, slots, k_out=got)
    # a code is off by half a step, amax / 254 at most, and bf16 by 2^-8 of the value
    assert bool(((got - k).abs().float() <= k.abs().float().max() / 254 + k.abs().float() * 2.0 ** -7).all())
    sigma, _ = milo.milo_block_svd([got.view(200, 128)])
    want = np.linalg.svd(f64(got).reshape(200, 128), compute_uv=False)
    assert np.allclose(sigma[0].cpu().numpy()[:8], want[:8], rtol=1e-3)


def test_arguments_of_the_binding():
    b = Batch(60, [20, 30], [1, 1], HEADS["0.5b"], 16, "int8")
    out = torch.full(b.q.shape, 7.0, device="cuda")
    good = dict(pages=b.pages, page_table=i32(b.table), lens=i32(b.lens), q=b.q, scale=b.scale, out=out)
    bad = [dict(q=b.q.float()), dict(q=b.q[:, :, :32]), dict(q=b.q.transpose(0, 1)), dict(out=out.double()), dict(out=out[:1]),
           dict(lens=i32([20])), dict(lens=i32(b.lens).long()), dict(page_table=i32(b.table)[:, ::2]), dict(q_starts=i32([0, 1])),
           dict(cache=12345), dict(block_table=[0]), dict(work=torch.empty(8, dtype=torch.uint8, device="cuda")), dict(pages=None)]
    for kw in bad:
        with pytest.raises(ValueError):
            milo.milo_attend_pages(**{**good, **kw})
    k = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    for args in ((k.float(), k, i32([0, 1])), (k, k[:1], i32([0, 1])), (k, k, i32([0])), (k, k[:, :1], i32([0, 1])),
                 (k, k.transpose(0, 1), i32([0, 1]))):
        with pytest.raises(ValueError):
            milo.milo_pages_store(b.pages, *args)
    for kw in (dict(), dict(k_out=k[:1]), dict(v_out=k.float()), dict(k_out=k[:1].expand(2, 2, 64))):
        with pytest.raises(ValueError):
            milo.milo_pages_load(b.pages, i32([0, 1]), **kw)
    for kw in (dict(n_slots=None), dict(slots=i32([0, 0]), n_slots=3), dict(n_slots=2, starts=i32([0, 0])),
               dict(n_slots=2, work=i32([0]))):
        with pytest.raises(ValueError):
            milo.milo_pages_plan(i32([1, 2]), i32([1, 1]), 16, i32(b.table), i32([0, 1, 2]), i32([0, 3]), **kw)
    torch.cuda.synchronize()
    assert bool((out == 7).all())
