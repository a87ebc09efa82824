"""The paged 8-bit cache at its limits: batches that take the other ways to divide the work,
pools and outputs past 4 GiB, calls at once, graphs that share a workspace, starts that are none.
Attention is held to the bounds that tests/test_gpu_pages.py derives, or to equality."""
import numpy as np
import pytest
import torch

import synth
from paper_2609_29913_amd import milo
from test_gpu_pages import FMTS, HEADS, Batch, bf16, f64, i32

pytestmark = pytest.mark.gpu


def work_for(b, n_sel=0):
    need = milo.lib().milo_attend_pages_work(len(b.lens), b.q.shape[0], b.q.shape[1], b.pages.n_kv_heads, b.q.shape[2], n_sel)
    return torch.empty(need, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("longest,counts", [(6000, 1), (700, 1), (5000, 5)])
def test_attend_hundreds_of_requests(longest, counts):
    """More requests than a workgroup has threads, in shares (a long one among them) and whole."""
    rng = np.random.default_rng(longest)
    lens = rng.integers(0, 60, 700)
    lens[[3, 699]] = longest, longest // 2
    n = np.full(700, counts)
    n[::3] = counts - 1
    b = Batch(longest, list(lens), list(n), HEADS["one"], 16, "int8")
    got = b.run()
    b.check(got, b.want(True))
    assert torch.equal(got, b.run())


@pytest.mark.parametrize("fmt,dtype", [("int8", torch.float32), ("e4m3", torch.bfloat16)])
@pytest.mark.parametrize("req,queries,rows,heads", [(90, 1, 9000, "0.5b"), (2, 1000, 7000, "0.5b"), (24, 5, 9000, "14b")])
def test_attend_more_work_than_units(req, queries, rows, heads, fmt, dtype):
    """Two shares to a unit, of different lengths, for each tiling; pages that requests share."""
    H_q, H, d = HEADS[heads]
    rng = np.random.default_rng(req)
    b = Batch(req, [2000], [1], HEADS[heads], 16, fmt)
    b.lens, b.counts = rng.integers(rows // 2, rows, req), np.full(req, queries)
    b.table = rng.integers(0, b.pages.n_pages, (req, -(-rows // 16)))
    b.starts = np.arange(req + 1) * queries
    b.q = bf16(rng.standard_normal((req * queries, H_q, d)))
    got = b.run(True, dtype)
    b.check(got, b.want(True))
    assert torch.equal(got, b.run(True, dtype))


def test_attend_thousands_of_short_requests():
    """Too many for every workgroup of a whole tile to read them: shares of many tiles each."""
    rng = np.random.default_rng(8)
    b = Batch(8, list(rng.integers(0, 60, 3000)), list(rng.integers(0, 3, 3000)), HEADS["0.5b"], 16, "e4m3")
    got = b.run()
    b.check(got, b.want(True))
    assert torch.equal(got, b.run())


@pytest.mark.parametrize("req,counts,heads", [(4, 820, "14b"), (200, 5, "14b")])
def test_attend_whole_tiles_of_many_columns(req, counts, heads):
    rng = np.random.default_rng(req)
    lens = rng.integers(900, 1100, req)
    lens[0] = 1100
    b = Batch(req, list(lens), [counts] * req, HEADS[heads], 16, "e4m3")
    for dtype in (torch.float32, torch.bfloat16):
        b.check(b.run(True, dtype), b.want(True))


def test_attend_a_table_far_wider_than_the_rows():
    """Where 31 bits might not number the work, were the lengths what the table allows."""
    b = Batch(1, list(range(1, 65)), [1] * 64, HEADS["14b"], 128, "int8")
    wide = torch.full((64, 1 << 20), -1, dtype=torch.int32, device="cuda")
    wide[:, :b.table.shape[1]] = i32(b.table)
    out = torch.full(b.q.shape, float("nan"), device="cuda")
    milo.milo_attend_pages(b.pages, wide, i32(b.lens), b.q, np.float32(b.scale), out)
    b.check(out, b.want(True))


@pytest.mark.parametrize("n_req", [3, 65536])
def test_attend_starts_that_descend(n_req):
    """Undefined rows, but no access out of range; the next call is right."""
    b = Batch(2, [6000, 40, 70], [30, 3, 4063], HEADS["0.5b"], 16, "int8")
    starts = np.zeros(n_req + 1, dtype=np.int64)
    starts[1::2] = 4096
    table = i32(b.table[np.zeros(n_req, dtype=int)])
    out = torch.zeros(b.q.shape, device="cuda")
    milo.milo_attend_pages(b.pages, table, i32([6000] * n_req), b.q, b.scale, out, q_starts=i32(starts))
    torch.cuda.synchronize()
    lo = 33                                             # (the last request's columns are too many for the oracle)
    got = b.run()[:lo]
    want = [w[:lo] for w in Batch.want(_first(b, 2), True)]
    b.check(got, want)


def _first(b, n):
    c = Batch.__new__(Batch)
    c.__dict__.update(b.__dict__)
    c.lens, c.counts = b.lens[:n], b.counts[:n]
    return c


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_pages_past_4_gib(fmt):
    """The last pages of a pool of 5.2 GB a side work as those of a small pool."""
    H, d, P, n_pages = 8, 128, 128, 40000
    rng = np.random.default_rng(3)
    n = 1000
    x = bf16(rng.standard_normal((n, 3 * H, d)))
    got = []
    for size, first in ((8, 0), (n_pages, n_pages - 8)):
        pages = milo.milo_pages_create(size, P, H, d, FMTS[fmt])
        slots = torch.arange(n, dtype=torch.int32, device="cuda") + first * P
        milo.milo_pages_store(pages, x[:, :H], x[:, H:2 * H], slots)
        k, v = (torch.empty((n, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        milo.milo_pages_load(pages, slots, k, v)
        outs = [k, v]
        table = i32(np.arange(first, first + 8)[None])
        for queries in (1, 40):
            out = torch.empty((queries, H, d), device="cuda")
            milo.milo_attend_pages(pages, table, i32([n]), x[:queries, 2 * H:], d ** -0.5, out, q_starts=i32([0, queries]))
            outs.append(out)
        got.append(outs)
        del pages
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_load_past_4_gib():
    """An output of more than 2^31 elements, the same slots again and again."""
    H, d, n = 8, 128, 2100000
    pages = milo.milo_pages_create(4, 16, H, d)
    x = bf16(np.random.default_rng(4).standard_normal((64, H, d)))
    milo.milo_pages_store(pages, x, x, torch.arange(64, dtype=torch.int32, device="cuda"))
    slots = torch.arange(n, device="cuda").remainder(64).int()
    out = torch.empty((n, H, d), dtype=torch.bfloat16, device="cuda")
    milo.milo_pages_load(pages, slots, v_out=out)
    one = torch.empty((64, H, d), dtype=torch.bfloat16, device="cuda")
    milo.milo_pages_load(pages, slots[:64], v_out=one)
    whole = out[:n // 64 * 64].view(-1, 64, H, d)
    for part in whole.split(4096):
        assert bool((part == one).all())
    assert torch.equal(out[n // 64 * 64:], one[:n % 64])


def test_attend_two_calls_at_once():
    """Different batches on two streams, workspaces made by the calls, again and again."""
    bs = [Batch(20, [9000, 33], [1, 1], HEADS["7b"], 64, "int8"), Batch(21, [5000, 800], [40, 3], HEADS["14b"], 16, "e4m3")]
    want = [b.run() for b in bs]
    for b, w in zip(bs, want):
        b.check(w, b.want(True))
    args = [(b.pages, i32(b.table), i32(b.lens), b.q, b.scale) for b in bs]
    starts = [i32(b.starts) for b in bs]
    outs = [[torch.zeros_like(w) for _ in range(10)] for w in want]
    streams = [torch.cuda.Stream() for _ in bs]
    torch.cuda.synchronize()
    for k in range(10):
        for i in range(2):
            milo.milo_attend_pages(*args[i], outs[i][k], q_starts=starts[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        for o in outs[i]:
            assert torch.equal(o, want[i])


def test_two_graphs_share_a_workspace():
    """Graphs of different calls over one workspace, replayed in turn with eager calls between."""
    bs = [Batch(22, [9000, 33, 0], [1, 1, 1], HEADS["0.5b"], 64, "int8"), Batch(23, [5000, 800], [140, 3], HEADS["0.5b"], 16, "e4m3")]
    want = [b.run() for b in bs]
    work = max((work_for(b) for b in bs), key=lambda w: w.numel())
    args = [(b.pages, i32(b.table), i32(b.lens), b.q, b.scale) for b in bs]
    starts, outs, graphs = [i32(b.starts) for b in bs], [torch.zeros_like(w) for w in want], []
    torch.cuda.synchronize()
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            milo.milo_attend_pages(*args[i], outs[i], q_starts=starts[i], work=work)
        graphs.append(g)
    for k in range(4):
        for i in range(2):
            outs[i].zero_()
            graphs[i].replay()
        for i in range(2):
            assert torch.equal(outs[i], want[i])
        assert torch.equal(bs[k % 2].run(), want[k % 2])


def test_a_captured_call_with_a_compressed_context():
    """The call's shape once eagerly, then recorded: replays follow queries and lengths."""
    from helpers import GpuLayer
    inp = synth.make_problem(32, [300, 256, 700], [64, 40, 96], n_kv_heads=4, head_dim=128, n_q=3, n_q_heads=28, tail_cap=80)
    b = Batch(32, [80, 7, 33], [1, 1, 1], HEADS["7b"], 16, "int8")
    gl = GpuLayer(inp)
    try:
        table, lens, q, work = i32(b.table), i32(b.lens), b.q.clone(), work_for(b, 1)
        out = torch.zeros(q.shape, device="cuda")

        def call(o):
            milo.milo_attend_pages(b.pages, table, lens, q, b.scale, o, cache=gl.cache, block_table=[2, 0], work=work)
        call(out)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(out)
        for k in range(4):
            q.copy_(torch.roll(b.q, k, 0))
            lens.copy_(i32([80 - k, 7 * k, 33 + k]))
            out.zero_()
            g.replay()
            eager = torch.zeros_like(out)
            call(eager)
            nan = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
            nan[1] = 7 * k > 16                          # the request's second page is -1
            assert torch.equal(torch.isnan(out), nan) and torch.equal(torch.isnan(eager), nan)
            assert torch.equal(out[~nan], eager[~nan])
        # queries that see no rows of their own have the context's result (scaled by a sum and divided by
        # it again: less than ten roundings)
        lens.zero_()
        g.replay()
        want = torch.empty_like(out)
        milo.milo_attend_decode(gl.cache, [2, 0], q, None, None, None, b.scale, want)
        assert float((out - want).abs().max()) <= 1e-5 * float(want.abs().max())
    finally:
        gl.free()


def test_attend_with_a_context_on_another_stream():
    from helpers import GpuLayer
    inp = synth.make_problem(33, [300, 200], [64, 40], n_kv_heads=4, head_dim=128, n_q=2, n_q_heads=28, tail_cap=80)
    b = Batch(33, [500, 20], [1, 1], HEADS["7b"], 16, "e4m3")
    gl = GpuLayer(inp)
    try:
        want = b.run(cache=gl.cache, block_table=[1, 0])
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        args = (b.pages, i32(b.table), i32(b.lens), b.q, b.scale)
        out = torch.zeros_like(want)
        torch.cuda.synchronize()
        milo.milo_attend_pages(*args, out, cache=gl.cache, block_table=[1, 0], stream=s)
        s.synchronize()
        assert torch.equal(out, want)
        assert f64(out).shape == (2, 28, 128)
    finally:
        gl.free()
