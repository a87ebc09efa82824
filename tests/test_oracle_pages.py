"""The paged cache's oracle against things other than itself: torch's E4M3 type, closed
forms of the scales, torch's attention, and invariants of the page bookkeeping (every page
held once or free once, slots that follow the table, nothing changed by a refused step)."""
import math

import numpy as np
import pytest
import torch

import oracle


def test_e4m3_rounding_is_that_of_the_type():
    bits = torch.arange(0, 0x7F80, dtype=torch.int32).to(torch.int16)
    x = bits.view(torch.bfloat16).float()
    x = x[x <= 448]
    want = x.to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oracle.e4m3_round(x.numpy()), want)
    assert np.array_equal(oracle.e4m3_round(-x.numpy()), -want)


@pytest.mark.parametrize("amax,scale", [(448.0, 1.0), (449.0, 2.0), (224.0, 0.5), (1.75, 2.0 ** -8), (1.76, 2.0 ** -7),
                                        (2.0 ** -140, 2.0 ** -126), (0.0, 0.0)])
def test_e4m3_scale_is_the_smallest_power_that_holds_it(amax, scale):
    assert oracle.pages_scale(amax, True) == scale


def test_int8_scale_and_codes():
    x = np.linspace(-6.35, 6.35, 255, dtype=np.float32)     # 127 steps of 0.05 each way
    s = oracle.pages_scale(np.abs(x).max(), False)
    c = oracle.pages_codes(x, s, False)
    assert c.min() == -127 and c.max() == 127 and np.all(np.abs(x - c * s) <= 0.5000001 * s)
    assert math.isnan(oracle.pages_scale(math.inf, False)) and math.isnan(oracle.pages_scale(math.nan, True))
    assert np.all(oracle.pages_codes(x, np.float32(0), False) == 0)


def test_store_grows_a_page_and_starts_it_afresh():
    rows, scales = np.zeros((2, 16, 1, 1)), np.zeros((2, 1), dtype=np.float32)
    oracle.pages_store(rows, scales, 16, np.full((3, 1, 1), 1.27), np.array([16, 17, 18]), False)
    assert np.all(rows[1, :3, 0, 0] == 127) and scales[0, 0] == 0
    oracle.pages_store(rows, scales, 16, np.full((1, 1, 1), 12.7), np.array([19]), False)
    assert list(rows[1, :4, 0, 0]) == [13, 13, 13, 127]      # 1.27 / 0.1 = 12.7
    oracle.pages_store(rows, scales, 16, np.full((1, 1, 1), 0.1), np.array([20]), False)
    assert rows[1, 4, 0, 0] == 1 and scales[1, 0] == np.float32(12.7) / np.float32(127)
    oracle.pages_store(rows, scales, 16, np.full((1, 1, 1), np.nan), np.array([21]), False)
    assert np.isnan(scales[1, 0])
    oracle.pages_store(rows, scales, 16, np.full((1, 1, 1), 1.27), np.array([16]), False)
    assert scales[1, 0] == np.float32(1.27) / np.float32(127)


@pytest.mark.parametrize("causal", [False, True])
def test_attention_is_torch_attention(causal):
    rng = np.random.default_rng(5)
    k, v, q = rng.standard_normal((23, 2, 64)), rng.standard_normal((23, 2, 64)), rng.standard_normal((7, 6, 64))
    out, size, _, _ = oracle.attend_pages(k, v, q, 0.3, causal)
    mask = torch.ones(7, 23, dtype=torch.bool).tril(16) if causal else torch.ones(7, 23, dtype=torch.bool)
    rep = lambda x: torch.from_numpy(x).transpose(0, 1).repeat_interleave(3, 0)  # noqa: E731
    want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q).transpose(0, 1), rep(k), rep(v),
                                                            attn_mask=mask, scale=0.3).transpose(0, 1).numpy()
    assert np.allclose(out, want, rtol=0, atol=1e-12) and np.all(size >= np.abs(out) - 1e-12)


def test_a_query_before_every_row_gets_zeros():
    out, _, _, _ = oracle.attend_pages(np.ones((2, 1, 64)), np.ones((2, 1, 64)), np.ones((4, 1, 64)), 1.0, True)
    assert np.all(out[:2] == 0) and np.all(out[2:] == 1)


@pytest.mark.parametrize("seed", range(20))
def test_plan_keeps_every_page_in_one_place(seed):
    rng = np.random.default_rng(seed)
    P, n_req, width, n_pages = 16, 6, 9, 40
    lens = np.zeros(n_req, dtype=np.int64)
    table = np.full((n_req, width), -7)
    ring, head, count = rng.permutation(n_pages), int(rng.integers(n_pages)), n_pages
    for _ in range(30):
        delta = np.where(rng.random(n_req) < 0.3, -rng.integers(0, lens + 1), rng.integers(0, 40, n_req))
        before = (table.copy(), ring.copy(), head, count)
        status, lens2, starts, slots, table, ring, (head, count) = oracle.pages_plan(lens, delta, P, table, ring, head, count, 200)
        if status:
            assert np.array_equal(table, before[0]) and np.array_equal(ring, before[1]) and (head, count) == before[2:]
            assert np.all(slots == -1) and not any(starts) and np.array_equal(lens2, lens)
            continue
        assert np.array_equal(lens2, lens + delta) and starts[-1] == np.maximum(delta, 0).sum()
        held = [int(x) for i in range(n_req) for x in table[i, :-(-lens2[i] // P)]]
        free = [int(ring[(head + k) % n_pages]) for k in range(count)]
        assert sorted(held + free) == list(range(n_pages))
        for i in range(n_req):
            for j, r in enumerate(range(int(lens[i]), int(lens2[i]))):
                assert slots[starts[i] + j] == table[i, r // P] * P + r % P
        lens = np.array(lens2)
