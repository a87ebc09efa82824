"""The paged cache's entry points refuse what they do not take, on the host and before any
GPU work: sizes, alignment, strides, formats and NULLs in the C functions, types and shapes in
the Python ones."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2609_29913_amd import milo

A = 4096  # a plausible aligned address that is never followed: each call fails first
INV, UNS = milo.MILO_ERR_INVALID_ARG, milo.MILO_ERR_UNSUPPORTED


def pool(**kw):
    f = dict(n_pages=8, page_tokens=16, n_kv_heads=2, head_dim=64, format=0, k_codes=A, v_codes=A, k_scale=A, v_scale=A)
    f.update(kw)
    return milo.milo_pages(*[f[n] for n, _ in milo.milo_pages._fields_])


BAD_POOLS = [(dict(n_pages=0), INV), (dict(n_kv_heads=0), INV), (dict(page_tokens=24), UNS), (dict(page_tokens=8), UNS),
             (dict(page_tokens=256), UNS), (dict(head_dim=96), UNS), (dict(format=2), INV), (dict(format=-1), INV),
             (dict(k_codes=None), INV), (dict(v_codes=None), INV), (dict(k_scale=None), INV), (dict(v_scale=None), INV),
             (dict(k_codes=A + 8), INV), (dict(v_codes=A + 4), INV), (dict(n_pages=1 << 27), UNS),
             (dict(n_kv_heads=1 << 17), UNS), (dict(n_kv_heads=32768), UNS)]


def attend(p=None, **kw):
    f = dict(cache=None, block_table=None, n_sel=0, pages=ctypes.byref(pool()) if p is None else p, page_table=A,
             table_width=4, lens=A, q_starts=A, n_req=3, q=A, q_stride=256, n_tok=5, n_q_heads=4, causal=1, scale=0.125,
             out=A, out_format=0, work=A, hip_stream=None)
    f.update(kw)
    return milo.lib().milo_attend_pages(*f.values())


@pytest.mark.parametrize("kw,code", BAD_POOLS)
def test_bad_pools(kw, code):
    p = ctypes.byref(pool(**kw))
    L = milo.lib()
    assert L.milo_pages_store(p, A, 128, A, 128, A, 3, None) == code and milo.milo_last_error()
    assert L.milo_pages_load(p, A, 3, A, 128, A, 128, None) == code
    assert attend(p) == code


def test_more_rows_than_a_launch_takes():
    L, p = milo.lib(), ctypes.byref(pool())
    assert L.milo_pages_store(p, A, 128, A, 128, A, (1 << 27) + 1, None) == UNS
    assert L.milo_pages_load(p, A, (1 << 27) + 1, A, 128, A, 128, None) == UNS


def test_null_pool():
    L = milo.lib()
    assert L.milo_pages_store(None, A, 128, A, 128, A, 3, None) == INV
    assert L.milo_pages_load(None, A, 3, A, 128, A, 128, None) == INV
    assert attend(ctypes.POINTER(milo.milo_pages)()) == INV


@pytest.mark.parametrize("args", [
    (None, 128, A, 128, A, 3), (A, 128, None, 128, A, 3), (A, 128, A, 128, None, 3), (A, 120, A, 128, A, 3),
    (A, 128, A, 132, A, 3), (A + 2, 128, A, 128, A, 3), (A, 128, A + 8, 128, A, 3), (A, 128, A, 128, A, -1)])
def test_store_refuses(args):
    assert milo.lib().milo_pages_store(ctypes.byref(pool()), *args, None) == INV


@pytest.mark.parametrize("args", [
    (A, 3, None, 128, None, 128), (None, 3, A, 128, A, 128), (A, -1, A, 128, A, 128), (A, 3, A, 120, A, 128),
    (A, 3, A, 128, A, 130), (A, 3, A + 2, 128, None, 0), (A, 3, None, 0, A + 8, 128)])
def test_load_refuses(args):
    assert milo.lib().milo_pages_load(ctypes.byref(pool()), *args, None) == INV


@pytest.mark.parametrize("kw,code", [
    (dict(n_req=-1), INV), (dict(n_tok=-1), INV), (dict(q_starts=None), INV), (dict(n_q_heads=3), INV),
    (dict(n_q_heads=0), INV), (dict(n_q_heads=34, q_stride=34 * 64), UNS), (dict(table_width=0), INV),
    (dict(table_width=1 << 28), UNS), (dict(causal=2), INV), (dict(scale=float("nan")), INV),
    (dict(scale=float("inf")), INV), (dict(out_format=2), INV), (dict(page_table=None), INV), (dict(lens=None), INV),
    (dict(q=None), INV), (dict(q=A + 2), INV), (dict(q_stride=192), INV), (dict(q_stride=260), INV), (dict(out=None), INV),
    (dict(out=A + 8), INV), (dict(work=None), INV), (dict(work=A + 128), INV), (dict(n_sel=1), INV),
    (dict(n_tok=1 << 23), UNS), (dict(n_tok=(1 << 21) + 1), UNS), (dict(n_req=(1 << 24) + 1), UNS),
    (dict(n_req=1 << 14, n_tok=1 << 14, table_width=1 << 22), UNS)])
def test_attend_refuses(kw, code):
    assert attend(**kw) == code and milo.milo_last_error()


def plan(**kw):
    f = dict(lens=A, delta=A, n_req=3, page_tokens=16, table=A, table_width=4, ring=A, n_pages=8, ring_state=A,
             ring_state_out=A, lens_out=A, starts=A, slots=A, n_slots=5, status=A, work=A, hip_stream=None)
    f.update(kw)
    return milo.lib().milo_pages_plan(*f.values())


@pytest.mark.parametrize("kw,code", [
    (dict(n_req=-1), INV), (dict(n_slots=-1), INV), (dict(page_tokens=48), UNS), (dict(table_width=0), INV),
    (dict(n_pages=0), INV), (dict(n_pages=1 << 28), UNS), (dict(table_width=1 << 28), UNS), (dict(n_req=1 << 25), UNS),
    (dict(work=A + 4), INV)] + [(dict([(n, None)]), INV) for n in
                                ("lens", "delta", "table", "ring", "ring_state", "ring_state_out", "lens_out", "starts",
                                 "slots", "status", "work")])
def test_plan_refuses(kw, code):
    assert plan(**kw) == code and milo.milo_last_error()


def test_nothing_to_do_is_no_error():
    L, p = milo.lib(), ctypes.byref(pool())
    assert L.milo_pages_store(p, None, 0, None, 0, None, 0, None) == 0
    assert L.milo_pages_load(p, None, 0, None, 0, None, 0, None) == 0
    assert attend(n_req=0, n_tok=0) == 0 and attend(n_tok=0) == 0


def test_host_tensors_are_refused():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):
        milo.MiloPages(torch.zeros((2, 2, 1024), dtype=torch.int8), torch.zeros((2, 2, 1024), dtype=torch.int8),
                       torch.zeros(2, 2), torch.zeros(2, 2), 16)
    with pytest.raises(ValueError):
        milo.milo_pages_plan(i32(2), i32(2), 16, i32(2, 4), i32(8), i32(2), 4)
    for call in (lambda: milo.milo_pages_store(np.zeros(3), None, None, None), lambda: milo.milo_pages_load(None, i32(2)),
                 lambda: milo.milo_attend_pages(None, i32(2, 4), i32(2), torch.zeros(2, 4, 64), 1.0, torch.zeros(2, 4, 64))):
        with pytest.raises(ValueError):
            call()
