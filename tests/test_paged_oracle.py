"""Pins of the paged-cache oracle: a step worked out by hand, and attention
against the contiguous-cache oracle and closed forms."""

import numpy as np

from oracle import paged_oracle as PO
from oracle import qmatmul_oracle as O


def test_plan_by_hand():
    # Pages of 16.  Request 0 holds 15 tokens (1 page) and gets 2: positions 15, 16, one new page.
    # Request 1 has ended with 17 tokens: pages 5 and 6 go back.  Request 2 holds nothing and gets 16: one page.
    # The ring starts at its last entry: free pages 9, 3, 4 in this order.
    r = PO.plan_step([15, 17, 0], [2, -1, 16], [[7, -1, -1], [5, 6, -1], [-1, -1, -1]],
                     [3, 4, -1, -1, -1, -1, -1, -1, -1, 9], [9, 3], 16, 20)
    assert r["tables"] == [[7, 9, -1], [5, 6, -1], [3, -1, -1]]
    assert r["positions"] == [15, 16] + list(range(16)) + [-1, -1]
    assert r["slots"] == [7 * 16 + 15, 9 * 16] + [48 + j for j in range(16)] + [-1, -1]
    assert r["offsets"] == [0, 2, 2, 18] and r["lens"] == [17, 0, 16] and r["kv_lens"] == [17, 0, 16]
    assert r["ring"] == [1, 3] and r["free_ring"][:5] == [3, 4, 5, 6, -1] and r["refused"] == [0]


def test_plan_refusals_by_hand():
    # One free page: request 0 takes it, request 1 needs one and is refused, request 2 needs none and goes on,
    # request 3 would pass its table of 2 pages.
    r = PO.plan_step([16, 16, 3, 30], [1, 1, 1, 3], [[0, -1], [1, -1], [2, -1], [3, 4]], [8, -1, -1], [0, 1], 16, 8)
    assert r["kv_lens"] == [17, 0, 4, 0] and r["lens"] == [17, 16, 4, 30] and r["refused"] == [2]
    assert r["offsets"] == [0, 1, 2, 3, 6] and r["positions"] == [16, -1, 3, -1, -1, -1, -1, -1]
    assert r["tables"] == [[0, 8], [1, -1], [2, -1], [3, 4]] and r["ring"] == [1, 0]


def test_plan_with_a_prefix_by_hand():
    # Two shared pages of 16: request 0 begins behind them, request 1 ends and keeps them, request 2 is idle.
    r = PO.plan_step([0, 50, 0], [3, -1, 0], [[8, 9, -1, -1], [8, 9, 3, 4], [8, 9, -1, -1]], [5, -1, -1, -1], [0, 1], 16,
                     4, prefix_pages=2)
    assert r["tables"][0] == [8, 9, 5, -1] and r["positions"] == [32, 33, 34, -1] and r["slots"][:3] == [80, 81, 82]
    assert r["lens"] == [35, 0, 32] and r["kv_lens"] == [35, 0, 32] and r["free_ring"] == [5, 3, 4, -1]
    assert r["ring"] == [1, 2]


def test_attention_equals_the_contiguous_oracle():
    rng = np.random.default_rng(0)
    hq, hkv, d, page, n, new = 4, 2, 64, 16, 37, 5
    k, v = (rng.standard_normal((hkv, 48, d)).astype(np.float16) for _ in range(2))
    ids = [4, 0, 2]
    kp, vp = (rng.standard_normal((6, hkv, page, d)).astype(np.float16) for _ in range(2))
    for pool, rows in ((kp, k), (vp, v)):
        for at, p in enumerate(ids):
            pool[p] = rows[:, 16 * at:16 * at + 16]
    q = rng.standard_normal((new, hq, d)).astype(np.float16)
    for tables, prefix in ([[ids], None], [[[1, 1, 2]], [4, 0]]):
        o, _ = PO.paged_attention(q, kp, vp, tables, [0, new], [n], 0.125, prefix)
        ref = O.attention_prefill(q.transpose(1, 0, 2), k[:, :n], v[:, :n], 0.125, p0=n - new)
        np.testing.assert_allclose(o.transpose(1, 0, 2), ref, rtol=1e-12, atol=1e-12)


def test_attention_closed_forms():
    # Equal keys: the mean of the visible values; a request without keys: zeros.
    kp = np.zeros((2, 1, 16, 64), np.float16)
    vp = np.zeros((2, 1, 16, 64), np.float16)
    vp[1, 0, :, 0] = np.arange(16)
    q = np.ones((3, 1, 64), np.float16)
    o, size = PO.paged_attention(q, kp, vp, [[1], [0]], [0, 2, 3], [5, 0], 1.0)
    assert o[0, 0, 0] == 1.5 and o[1, 0, 0] == 2.0 and not o[2].any() and size[1, 0, 0] == 2.0
