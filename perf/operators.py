"""Performance cases of the paged 8-bit cache: what a serving program calls each step.

Four operators, through the public entry points of ``paper_2609_29913_amd.milo``:

- ``plan``    block tables and slot maps from request lengths (``milo_pages_plan``)
- ``store``   keys and values quantised into pages, read back (``milo_pages_store``)
- ``load``    rows of pages back to bf16 (``milo_pages_load``)
- ``attend``  attention of a ragged batch of queries over its pages (``milo_attend_pages``):
              single tokens, chunks (causal), and queries that see every row (cross attention)

A page holds ``page`` tokens of every KV head in 8 bits, INT8 or E4M3, with one fp32 scale
per page and head, for keys and values apart.  Storage (groups of 16 tokens, so that a
matrix instruction's operand is one contiguous load):

    keys    [page][head][token / 16][dim / 16][token % 16][dim % 16]
    values  [page][head][token / 16][dim / 64][token % 16 / 4][dim % 16][dim % 64 / 16][token % 4]
"""
import math
import random

import torch

own = False

# (query heads, KV heads, head dimension) of the layers the repository's workloads name
HEADS = {"0.5b": (14, 2, 64), "7b": (28, 4, 128), "14b": (40, 8, 128)}


def _case(kind, heads, fmt, page, req, lo, hi, **more):
    """req requests whose lengths lie in lo .. hi; new: tokens each adds in this step."""
    c = {"kind": kind, "heads": heads, "fmt": fmt, "page": page, "req": req, "lo": lo, "hi": hi, "new": 1,
         "ragged_new": False, "causal": True, "out": "bf16", "layout": 1}
    c.update(more)
    return c


def listed():
    return [
        # a decode step's bookkeeping: a token each, some requests ending
        _case("plan", "7b", "int8", 16, 256, 1, 4096, new=1, ends=True, name="plan_decode_256"),
        # prompts of a whole batch entering at once
        _case("plan", "7b", "int8", 64, 32, 0, 0, new=4096, ragged_new=True, ends=False, name="plan_prompts_32"),
        # a decode step's rows into half-filled pages
        _case("store", "14b", "int8", 16, 64, 1, 8192, name="store_decode_64"),
        # a prompt's rows
        _case("store", "7b", "e4m3", 64, 4, 0, 3000, new=2048, ragged_new=True, name="store_prompts_8k"),
        # a request's older rows on their way to the encoder
        _case("load", "7b", "int8", 32, 1, 1024, 1024, name="load_block_1k"),
        # a batch's whole rows
        _case("load", "14b", "e4m3", 64, 16, 3000, 5000, name="load_batch_64k"),
        # one request's first tokens on the smallest model: launches and latency
        _case("attend", "0.5b", "int8", 16, 1, 301, 301, out="fp32", name="attend_small"),
        # a serving batch of ragged lengths
        _case("attend", "7b", "int8", 16, 32, 257, 16384, name="attend_7b_b32"),
        # a large batch: the cache read at full rate
        _case("attend", "14b", "e4m3", 64, 64, 8192, 8192, name="attend_14b_b64"),
        # one long request: its rows split over the whole GPU
        _case("attend", "7b", "int8", 64, 1, 131001, 131001, out="fp32", name="attend_7b_128k"),
        # a chunk of a prompt after rows that are there
        _case("attend", "7b", "e4m3", 32, 1, 8192, 8192, new=2048, name="attend_chunk_2k"),
        # short queries over an encoder's states of other lengths, every row seen
        _case("attend", "14b", "int8", 32, 8, 100, 3000, new=37, ragged_new=True, causal=False, name="attend_cross_8"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["plan", "store", "load", "attend", "attend", "attend"])
    heads, fmt, page = rng.choice(sorted(HEADS)), rng.choice(["int8", "e4m3"]), rng.choice([16, 32, 64, 128])
    more = {"layout": rng.randrange(1 << 30), "out": rng.choice(["bf16", "fp32"])}
    if kind == "plan":
        req = log_int(1, 1000)
        if rng.random() < 0.5:
            return _case(kind, heads, fmt, page, req, 0, log_int(2, 8192), ends=rng.random() < 0.5, **more)
        return _case(kind, heads, fmt, page, req, 0, log_int(2, 500), new=log_int(2, max(2, 100000 // req)),
                     ragged_new=True, ends=False, **more)
    if kind == "store":
        req = log_int(1, 200)
        if rng.random() < 0.5:
            return _case(kind, heads, fmt, page, req, 0, log_int(2, 4096), **more)
        return _case(kind, heads, fmt, page, req, 0, log_int(2, 500), new=log_int(2, max(2, 8000 // req)),
                     ragged_new=True, **more)
    if kind == "load":
        req = log_int(1, 64)
        return _case(kind, heads, fmt, page, req, 1, log_int(2, 64000 // req), **more)
    style = rng.choice(["decode", "decode", "few", "chunk", "cross"])
    if style == "decode":
        req = log_int(1, 128)
        hi = log_int(2, min(131072, 400000 // req))
        return _case(kind, heads, fmt, page, req, rng.choice([0, hi // 2]), hi, **more)
    if style == "few":
        req = log_int(1, 64)
        return _case(kind, heads, fmt, page, req, 8, log_int(10, min(32768, 200000 // req)), new=rng.randint(2, 8), **more)
    if style == "chunk":
        req = log_int(1, 8)
        new = log_int(16, 1500 // req)
        return _case(kind, heads, fmt, page, req, 0, log_int(2, 8000 // req) + new, new=new, ragged_new=rng.random() < 0.5, **more)
    return _case(kind, heads, fmt, page, log_int(1, 16), 1, log_int(2, 4000), new=log_int(1, 64), ragged_new=True,
                 causal=False, **more)


def _shape(case):
    """What the case fixes, whatever the seed: lengths before the step, tokens each request
    adds (below 0: rows it gives up), rows after it."""
    rng = random.Random(case["layout"])
    before, delta = [], []
    for _ in range(case["req"]):
        n = rng.randint(case["lo"], case["hi"])
        a = rng.randint(0, case["new"]) if case["ragged_new"] else case["new"]
        if case["kind"] == "plan" and case["ends"] and rng.random() < 0.2:
            a = -n if rng.random() < 0.5 else -min(n, 3)
        if case["kind"] == "attend":  # hi counts the rows after the step
            a = min(a, n) if case["causal"] else a
            n = n - a if case["causal"] else n
        before.append(n)
        delta.append(a)
    if case["kind"] != "plan" and sum(delta) == 0:
        delta[0] = 1
    after = [n + (a if case["causal"] else 0) for n, a in zip(before, delta)]
    return before, delta, after


def work(case):
    h_q, n_kv, d = HEADS[case["heads"]]
    P, D = case["page"], n_kv * d
    before, delta, after = _shape(case)
    pages = [-(-n // P) for n in after]
    new = sum(max(a, 0) for a in delta)
    if case["kind"] == "plan":
        moved = sum(abs(p - -(-n // P)) for p, n in zip(pages, before))
        return {"bytes": 4 * (4 * case["req"] + 1 + new + 2 * moved), "flops": 0}
    touched = [-(-n // P) - b // P for n, b in zip(after, before)]
    if case["kind"] == "store":
        # the new rows in bf16, their codes, the touched pages' scales; their rows read back
        rows = sum(n - b // P * P for n, b in zip(after, before))
        return {"bytes": 6 * new * D + 8 * sum(touched) * n_kv + 6 * rows * D + 4 * (new + rows), "flops": 0}
    rows = sum(after)
    if case["kind"] == "load":
        return {"bytes": 6 * rows * D + 8 * sum(pages) * n_kv + 4 * rows, "flops": 0}
    if case["causal"]:
        seen = sum(a * (n - a) + a * (a + 1) // 2 for n, a in zip(after, delta))
    else:
        seen = sum(a * n for n, a in zip(after, delta))
    rows = sum(n for n, a in zip(after, delta) if a)
    size = 2 if case["out"] == "bf16" else 4
    return {"bytes": 2 * rows * D + 8 * sum(pages) * n_kv + 4 * sum(pages) + new * h_q * d * (2 + size),
            "flops": 4 * seen * h_q * d}


def _order(n, gen):
    return torch.randperm(n, generator=gen, device="cuda", dtype=torch.int64).to(torch.int32)


def prepare(case, seed):
    h_q, n_kv, d = HEADS[case["heads"]]
    P = case["page"]
    before, delta, after = _shape(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    held = [-(-n // P) for n in before]
    total = [-(-max(n, b) // P) for n, b in zip(after, before)]
    width = max(1, max(total)) + 1
    n_pages = sum(total) + 3
    ids = _order(n_pages, gen)
    st = {"case": case, "P": P, "n_kv": n_kv, "d": d, "h_q": h_q, "n_pages": n_pages,
          "lens": i32(before), "delta": i32(delta)}
    # the pages the requests hold, scattered over the pool; the others in the ring of free ones
    held_t, at = i32(held), torch.arange(width, device="cuda")
    first = torch.cumsum(held_t, 0) - held_t
    if case["kind"] == "plan":
        own_page = at[None] < held_t[:, None]
        pick = (first[:, None] + at[None]).clamp(max=n_pages - 1)
        st["table"] = torch.where(own_page, ids[pick], -1).to(torch.int32)
        n_held, head = sum(held), n_pages // 3
        ring = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
        ring[(torch.arange(n_pages - n_held, device="cuda") + head) % n_pages] = ids[n_held:]
        st["ring"], st["ring_state"] = ring, i32([head, n_pages - n_held])
        n = sum(max(a, 0) for a in delta)
        st["outs"] = {"lens_out": i32([0] * len(before)), "ring_state_out": i32([0, 0]), "starts": i32([0] * (len(before) + 1)),
                      "slots": torch.empty(n + 5, dtype=torch.int32, device="cuda"), "status": i32([0])}
        return st
    total_t = i32(total)
    first = torch.cumsum(total_t, 0) - total_t
    pick = (first[:, None] + at[None]).clamp(max=n_pages - 1)
    st["table"] = torch.where(at[None] < total_t[:, None], ids[pick], -1).to(torch.int32)
    st["after"] = i32(after)
    # codes with the spread that rows of a page have under their common scale
    shape = (n_pages, n_kv, P * d)
    for side in ("k", "v"):
        if case["fmt"] == "int8":
            c = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float16).mul_(40).round_().clamp_(-127, 127)
            st[side + "_codes"] = c.to(torch.int8)
            st[side + "_scale"] = torch.rand((n_pages, n_kv), generator=gen, device="cuda") * 0.02 + 0.015
        else:
            c = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float16).mul_(100).clamp_(-448, 448)
            st[side + "_codes"] = c.to(torch.float8_e4m3fn)
            e = torch.randint(-8, -5, (n_pages, n_kv), generator=gen, device="cuda")
            st[side + "_scale"] = torch.ldexp(torch.ones((), device="cuda"), e)
        del c
    delta_t, before_t = i32([max(a, 0) for a in delta]), i32(before)
    n_new = sum(max(a, 0) for a in delta)

    def slots_of(first_row, count, n):
        """Slots of `count` rows of each request from `first_row` on, one request after another."""
        who = torch.repeat_interleave(torch.arange(len(before), device="cuda"), count.long(), output_size=n)
        row = torch.arange(n, device="cuda") - (torch.cumsum(count, 0) - count)[who] + first_row[who]
        return (st["table"][who, row // P] * P + row % P).to(torch.int32)

    if case["kind"] == "store":
        amp = torch.exp(torch.randn((1, n_kv, d), generator=gen, device="cuda") * 0.3)
        fused = torch.randn((n_new, 2, n_kv, d), generator=gen, device="cuda") * amp[:, None]
        fused = fused.to(torch.bfloat16)  # rows as a fused projection leaves them
        st["k"], st["v"] = fused[:, 0], fused[:, 1]
        st["slots"] = slots_of(before_t, delta_t, n_new)
        start = before_t // P * P
        rows = sum(n - b // P * P for n, b in zip(after, before))
        st["read"] = slots_of(start, st["after"] - start, rows)
    elif case["kind"] == "load":
        st["read"] = slots_of(before_t * 0, st["after"], sum(after))
    else:
        st["q"] = torch.randn((n_new, h_q, d), generator=gen, device="cuda").to(torch.bfloat16)
        st["starts"] = torch.nn.functional.pad(torch.cumsum(delta_t, 0), (1, 0)).to(torch.int32)
        st["max_new"] = max(delta)
        st["scale"] = 1.0 / math.sqrt(d)
        st["out"] = torch.empty((n_new, h_q, d), dtype=torch.bfloat16 if case["out"] == "bf16" else torch.float32, device="cuda")
        return st
    n = st["read"].numel()
    st["k_out"] = torch.empty((n, n_kv, d), dtype=torch.bfloat16, device="cuda")
    st["v_out"] = torch.empty((n, n_kv, d), dtype=torch.bfloat16, device="cuda")
    return st


# ---- plain form ---------------------------------------------------------------------------

def _k_rows(codes, P, d):
    """Keys' codes [..., P * d] as rows [..., P, d] in fp32."""
    lead = codes.shape[:-1]
    c = codes.reshape(*lead, P // 16, d // 16, 16, 16).transpose(-3, -2)
    return c.reshape(*lead, P, d).float()


def _v_rows(codes, P, d):
    lead = codes.shape[:-1]
    c = codes.reshape(*lead, P // 16, d // 64, 4, 16, 4, 4)
    n = len(lead)
    c = c.permute(*range(n), n, n + 2, n + 5, n + 1, n + 4, n + 3)
    return c.reshape(*lead, P, d).float()


def _pick(codes, ids):
    if codes.dtype == torch.int8:
        return codes[ids]
    return codes.view(torch.uint8)[ids].view(torch.float8_e4m3fn)


def _token_rows(codes, side, P, d, page, tok):
    """Codes of single tokens (page, tok) [n] as rows [n][head][dim] in fp32."""
    raw = codes if codes.dtype == torch.int8 else codes.view(torch.uint8)
    lead, g, t = raw.shape[:2], tok // 16, tok % 16
    if side == "k":
        c = raw.view(*lead, P // 16, d // 16, 16, 16)[page, :, g, :, t]
    else:
        c = raw.view(*lead, P // 16, d // 64, 4, 16, 4, 4)[page, :, g, :, t // 4, :, :, t % 4].transpose(-1, -2)
    c = c.reshape(page.numel(), lead[1], d)
    return (c if codes.dtype == torch.int8 else c.view(torch.float8_e4m3fn)).float()


def _quantise(x, scale, fmt):
    """Codes, as fp32, of x under its scale."""
    x = torch.where(scale > 0, x / torch.where(scale > 0, scale, 1.0), 0.0)
    if fmt == "int8":
        return x.round().clamp(-127, 127)
    return x.to(torch.float8_e4m3fn).float()


def _scale_of(amax, fmt):
    if fmt == "int8":
        return amax / torch.full_like(amax, 127.0)
    m, e = torch.frexp(amax)  # amax = m 2^e, 0.5 <= m < 1; 448 = 0.875 2^9
    e = torch.where(m > 0.875, e - 8, e - 9).clamp(min=-126)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), 0.0)


def _plan(st):
    lens, delta, P, table, ring = st["lens"].long(), st["delta"].long(), st["P"], st["table"], st["ring"]
    n_pages, n_slots = ring.numel(), st["outs"]["slots"].numel()
    head, count = st["ring_state"].long().unbind()
    after = lens + delta
    grow = delta.clamp(min=0)
    starts = torch.nn.functional.pad(torch.cumsum(grow, 0), (1, 0))
    p0, p1 = (lens + P - 1) // P, (after + P - 1) // P
    alloc, freed = (p1 - p0).clamp(min=0), (p0 - p1).clamp(min=0)
    a_end, f_end = torch.cumsum(alloc, 0), torch.cumsum(freed, 0)
    col = torch.arange(table.shape[1], device=table.device)
    # the new entries of the table: ring ids in request order
    new = (col >= p0[:, None]) & (col < p1[:, None])
    nth = head + (a_end - alloc)[:, None] + col - p0[:, None]
    table = torch.where(new, ring[nth % n_pages], table)
    # the pages given up, behind the free ones
    out = (col >= p1[:, None]) & (col < p0[:, None])
    nth = head + count + (f_end - freed)[:, None] + col - p1[:, None]
    room = torch.cat([ring, ring[:1]])
    room[torch.where(out, nth % n_pages, n_pages).reshape(-1)] = table.reshape(-1)
    state = torch.stack([(head + a_end[-1]) % n_pages, count - a_end[-1] + f_end[-1]])
    # slots of the new rows
    j = torch.arange(n_slots, device=table.device)
    who = torch.searchsorted(starts, j, right=True).sub(1).clamp(max=lens.numel() - 1)
    row = (lens[who] + j - starts[who])
    inside = j < starts[-1]
    slot = table[who, (row // P).clamp(max=table.shape[1] - 1)] * P + row % P
    slots = torch.where(inside, slot, -1)
    i32 = lambda v: v.to(torch.int32)  # noqa: E731
    return {"table": i32(table), "lens": i32(after), "starts": i32(starts), "slots": i32(slots), "ring": i32(room[:n_pages]),
            "ring_state": i32(state), "status": torch.zeros(1, dtype=torch.int32, device=table.device)}


def _read_rows(st, side, scale, new_rows=None):
    """Rows of st["read"] under `scale`; new_rows (codes of st["slots"]) over the ones in the pages."""
    P, d, fmt, codes = st["P"], st["d"], st["case"]["fmt"], st[side + "_codes"]
    page, off = st["read"].long() // P, st["read"].long() % P
    rows = _token_rows(codes, side, P, d, page, off)
    if new_rows is not None:
        # rows that were there, under the page's scale of now
        was, now = st[side + "_scale"][page][..., None], scale[page][..., None]
        rows = torch.where(was == now, rows, _quantise(rows * was, now, fmt))
        at = torch.zeros(st["n_pages"] * P, dtype=torch.int64, device=page.device)
        at[st["read"].long()] = torch.arange(page.numel(), device=page.device)
        rows[at[st["slots"].long()]] = new_rows
    return (rows * scale[page][..., None]).to(torch.bfloat16)


def _store_side(st, side):
    P, fmt = st["P"], st["case"]["fmt"]
    x, slots, was = st[side].float(), st["slots"].long(), st[side + "_scale"]
    page = slots // P
    amax = torch.zeros_like(was).index_reduce(0, page, x.abs().amax(-1), "amax")
    first = torch.full((st["n_pages"],), P, device=x.device).index_reduce(0, page, slots % P, "amin")
    new = _scale_of(amax, fmt)
    scale = torch.where(first[:, None] == P, was, torch.where(first[:, None] == 0, new, torch.maximum(was, new)))
    return _read_rows(st, side, scale, _quantise(x, scale[page][..., None], fmt)), scale


def _attend(st):
    P, d, n_kv, h_q = st["P"], st["d"], st["n_kv"], st["h_q"]
    G, W, n = h_q // n_kv, st["max_new"], st["starts"][1:] - st["starts"][:-1]
    ids = st["table"].long().clamp(min=0)
    req, L = ids.shape[0], ids.shape[1] * P
    keys = _k_rows(_pick(st["k_codes"], ids), P, d).mul_(st["k_scale"][ids][..., None, None])
    keys = keys.transpose(1, 2).reshape(req, n_kv, L, d)
    j = torch.arange(W, device="cuda")
    row = (st["starts"][:-1, None] + j).clamp(max=st["q"].shape[0] - 1).long()
    q = st["q"][row].float().view(req, W, n_kv, G, d).transpose(1, 2).reshape(req, n_kv, W * G, d)
    s = torch.matmul(q, keys.transpose(2, 3)).mul_(st["scale"]).view(req, n_kv, W, G, L)
    del keys
    seen = st["after"][:, None].expand(req, W)
    if st["case"]["causal"]:
        seen = seen - n[:, None] + j + 1
    s.masked_fill_((torch.arange(L, device="cuda") >= seen[..., None])[:, None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    s = s.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    den = s.sum(-1, keepdim=True)
    values = _v_rows(_pick(st["v_codes"], ids), P, d).mul_(st["v_scale"][ids][..., None, None])
    values = values.transpose(1, 2).reshape(req, n_kv, L, d)
    o = torch.matmul(s.view(req, n_kv, W * G, L), values).view(req, n_kv, W, G, d)
    o = torch.where(den > 0, o / den, 0.0).transpose(1, 2).reshape(req, W, h_q, d)
    t = torch.arange(st["q"].shape[0], device="cuda")
    who = torch.searchsorted(st["starts"][1:].contiguous(), t, right=True)
    return o[who, t - st["starts"][who]].to(st["out"].dtype)


# ---- the framework's operators -----------------------------------------------------------

def _pages(st):
    from paper_2609_29913_amd import milo
    if "pages" not in st:  # the handle that a program keeps with its buffers
        st["pages"] = milo.MiloPages(st["k_codes"], st["v_codes"], st["k_scale"], st["v_scale"], st["P"])
    return milo, st["pages"]


def run(st):
    kind = st["case"]["kind"]
    if not own:
        if kind == "plan":
            return _plan(st)
        if kind == "store":
            (k, ks), (v, vs) = _store_side(st, "k"), _store_side(st, "v")
            return {"k": k, "v": v, "k_scale": ks, "v_scale": vs}
        if kind == "load":
            return {"k": _read_rows(st, "k", st["k_scale"]), "v": _read_rows(st, "v", st["v_scale"])}
        return {"out": _attend(st)}
    if kind == "plan":
        from paper_2609_29913_amd import milo
        o = st["outs"]
        milo.milo_pages_plan(st["lens"], st["delta"], st["P"], st["table"], st["ring"], st["ring_state"], **o)
        return {"table": st["table"], "lens": o["lens_out"], "starts": o["starts"], "slots": o["slots"], "ring": st["ring"],
                "ring_state": o["ring_state_out"], "status": o["status"]}
    milo, pages = _pages(st)
    if kind == "attend":
        milo.milo_attend_pages(pages, st["table"], st["after"], st["q"], st["scale"], st["out"], q_starts=st["starts"],
                               causal=st["case"]["causal"])
        return {"out": st["out"]}
    if kind == "store":
        milo.milo_pages_store(pages, st["k"], st["v"], st["slots"])
    milo.milo_pages_load(pages, st["read"], st["k_out"], st["v_out"])
    got = {"k": st["k_out"], "v": st["v_out"]}
    if kind == "store":
        got.update(k_scale=st["k_scale"], v_scale=st["v_scale"])
    return got


# ---- 64 bits, from the definitions ---------------------------------------------------------

def _value(codes):
    """8-bit codes as float64, E4M3 from its bits: sign, 4 exponent bits (bias 7), 3 fraction bits."""
    if codes.dtype == torch.int8:
        return codes.double()
    b = codes.view(torch.uint8).long()
    e, f = (b >> 3) & 15, (b & 7).double()
    v = torch.where(e == 0, f / 8 * 2.0 ** -6, (1 + f / 8) * torch.pow(2.0, (e - 7).double()))
    return torch.where(b >= 128, -v, v)


def _row64(st, side, page, tok):
    """Codes of rows (page, token) [n], as float64 [n][head][dim], by the storage formula."""
    P, d = st["P"], st["d"]
    dim = torch.arange(d, device="cuda")
    t, c = tok[:, None], dim[None]
    if side == "k":
        at = ((t // 16 * (d // 16) + c // 16) * 16 + t % 16) * 16 + c % 16
    else:
        at = ((((t // 16 * (d // 64) + c // 64) * 4 + t % 16 // 4) * 16 + c % 16) * 4 + c % 64 // 16) * 4 + t % 4
    raw = st[side + "_codes"]
    raw = raw if raw.dtype == torch.int8 else raw.view(torch.uint8)
    got = raw[page[:, None, None], torch.arange(st["n_kv"], device="cuda")[None, :, None], at[:, None, :]]
    return _value(got if st["case"]["fmt"] == "int8" else got.view(torch.float8_e4m3fn))


def _code64(x, s, fmt):
    x = torch.where(s > 0, x / torch.where(s > 0, s, 1.0), torch.zeros_like(x))
    if fmt == "int8":
        return torch.round(x).clamp(-127, 127)
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -9))).clamp(min=-6)
    step = torch.pow(2.0, e - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    if case["kind"] == "plan":
        return None
    st = prepare(case, seed)
    P, fmt = st["P"], case["fmt"]
    if case["kind"] in ("store", "load"):
        got = {}
        read = st["read"].long()
        for side in ("k", "v"):
            scale = st[side + "_scale"].double()
            rows = torch.empty((read.numel(), st["n_kv"], st["d"]), dtype=torch.float64, device="cuda")
            for i in range(0, read.numel(), 8192):
                r = read[i:i + 8192]
                rows[i:i + 8192] = _row64(st, side, r // P, r % P)
            if case["kind"] == "store":
                slots, x, old = st["slots"].long(), st[side].double(), scale.clone()
                big = x.abs().amax(-1)
                for s in torch.unique(slots // P).tolist():
                    mine = slots // P == s
                    a = big[mine].amax(0)
                    if fmt == "int8":
                        a = (a / 127).float().double()  # a scale is stored in fp32
                    else:
                        e = torch.ceil(torch.log2(a.clamp(min=1e-300) / 448)).clamp(min=-126)
                        a = torch.where(a > 0, torch.pow(2.0, e), a)
                    scale[s] = a if (slots[mine] % P).min() == 0 else torch.maximum(old[s], a)
                was, now = old[read // P][..., None], scale[read // P][..., None]
                rows = torch.where(was == now, rows, _code64(rows * was, now, fmt))
                order = torch.argsort(read)
                at = order[torch.searchsorted(read[order], slots)]
                rows[at] = _code64(x, scale[slots // P][..., None], fmt)
                got[side + "_scale"] = scale
            got[side] = rows * scale[read // P][..., None]
        return got
    G, lens, starts = st["h_q"] // st["n_kv"], st["after"].tolist(), st["starts"].tolist()
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    for i, n in enumerate(lens):
        a, b = starts[i], starts[i + 1]
        if a == b or n == 0:
            continue
        t = torch.arange(n, device="cuda")
        page = st["table"][i].long()[t // P]
        K = _row64(st, "k", page, t % P) * st["k_scale"].double()[page][..., None]
        V = _row64(st, "v", page, t % P) * st["v_scale"].double()[page][..., None]
        last = t[None] < (n - (b - a) + torch.arange(b - a, device="cuda") + 1 if case["causal"] else
                          torch.full((b - a,), n, device="cuda"))[:, None]
        for h in range(st["h_q"]):
            s = (st["q"][a:b, h].double() @ K[:, h // G].T.contiguous()) * st["scale"]
            p = torch.softmax(s.masked_fill(~last, -math.inf), -1).nan_to_num(0.0)
            out[a:b, h] = p @ V[:, h // G].contiguous()
    return {"out": out}
