"""qkv_plan against the oracle: pages from the ring, page tables, positions,
slots and lengths of a step, and what it refuses."""

import random

import pytest
import torch

from oracle import paged_oracle as PO
from paper_2607_00501_amd import binding as B

pytestmark = pytest.mark.gpu


def _state(rng, n, page, most_ctx, most_new, width=None, prefix_pages=0, ended=0.1, count=None, head=None):
    lens = [prefix_pages * page + rng.randrange(0, most_ctx + 1) for _ in range(n)]
    new = [-1 if rng.random() < ended else rng.randrange(0, most_new + 1) for _ in range(n)]
    held = [-(-x // page) for x in lens]
    width = width or max(-(-(x + most_new) // page) for x in lens) + 1
    need = sum(max(0, -(-(x + t) // page) - h) for x, t, h in zip(lens, new, held) if t > 0)
    count = need + rng.randrange(0, 10) if count is None else count
    n_pages = prefix_pages + sum(h - prefix_pages for h in held) + count + 1
    ids = list(range(n_pages))
    rng.shuffle(ids)
    at, tables = prefix_pages, []
    for h in held:
        tables.append((ids[:prefix_pages] + ids[at:at + h - prefix_pages] + [-1] * width)[:max(width, 1)])
        at += h - prefix_pages
    head = rng.randrange(n_pages) if head is None else head
    ring = [-1] * n_pages
    for j in range(count):
        ring[(head + j) % n_pages] = ids[at + j]
    return lens, new, tables, ring, [head, count]


def _check(lens, new, tables, free_ring, ring, page, max_tokens, prefix_pages=0):
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    t, f = dev(tables), dev(free_ring)
    p = B.qkv_plan(dev(lens), dev(new), t, f, dev(ring), page, max_tokens, prefix_pages)
    got = dict(lens=p.lens, kv_lens=p.kv_lens, offsets=p.offsets, positions=p.positions, slots=p.slots, ring=p.ring,
               refused=p.refused, tables=t, free_ring=f)
    want = PO.plan_step(lens, new, tables, free_ring, ring, page, max_tokens, prefix_pages)
    for k, v in got.items():
        assert v.tolist() == want[k], k
    return p


@pytest.mark.parametrize("n,page,most_ctx,most_new,prefix_pages", [
    (1, 16, 0, 1, 0), (1, 16, 40, 1, 0), (1, 256, 700, 3000, 2), (2, 16, 17, 17, 0), (63, 32, 100, 1, 1),
    (64, 64, 500, 2, 0), (65, 16, 300, 40, 3), (200, 16, 2000, 1, 0), (513, 128, 1000, 1, 4), (1024, 16, 90, 60, 0),
    (1023, 32, 0, 63, 0)])
def test_plan_matches_the_oracle(n, page, most_ctx, most_new, prefix_pages):
    rng = random.Random(n * 1000 + page + most_ctx)
    for pad in (0, 37):
        s = _state(rng, n, page, most_ctx, most_new, prefix_pages=prefix_pages)
        tokens = sum(max(t, 0) for t in s[1])
        _check(*s, page, tokens + pad, prefix_pages)


@pytest.mark.parametrize("n,page,most_new", [(5, 16, 30), (100, 32, 50), (1000, 16, 20)])
def test_plan_refuses_what_does_not_fit(n, page, most_new):
    rng = random.Random(n)
    lens, new, tables, free_ring, ring = _state(rng, n, page, 200, most_new, count=max(1, n // 2))
    tokens = sum(max(t, 0) for t in new)
    _check(lens, new, tables, free_ring, ring, page, tokens)                       # pages run out
    _check(lens, new, tables, free_ring, ring, page, tokens // 2)                  # tokens do not fit
    _check(lens, new, tables, free_ring, [ring[0], 0], page, tokens)               # nothing is free
    narrow = max(1, len(tables[0]) // 2)
    _check(lens, new, [t[:narrow] for t in tables], free_ring, ring, page, tokens)  # tables too short


def test_plan_with_senseless_lengths_and_rings():
    lens, new = [5, -3, 2 ** 31 - 1, 40, -(2 ** 31)], [3, 4, 1, -1, -1]
    tables = [[0, 1, -1]] * 5
    _check(lens, new, tables, [7, 6, 5, -1], [1, 2], 16, 20)
    _check([5, 9], [2 ** 31 - 1, 2 ** 31 - 1], tables[:2], [7, 6, 5, -1], [1, 2], 16, 20)
    for ring in ([4, 2], [-1, 2], [0, 5], [0, -1]):
        _check([15, 3], [3, 2], tables[:2], [7, 6, 5, -1], ring, 16, 8)
    _check([16], [1], [[0, -1]], [3], [0, 1], 16, 0)                               # no room for any token


def test_plan_gives_pages_back_around_the_ring():
    # 3 free pages at the ring's end, 4 come back around its start; none of them is used in this step.
    lens, new = [40, 20, 16], [-1, 13, -1]
    tables = [[0, 1, 2, -1], [3, 4, -1, -1], [5, -1, -1, -1]]
    p = _check(lens, new, tables, [-1] * 5 + [6, 7, 8], [5, 3], 16, 13)
    assert p.ring.tolist() == [6, 6]


def test_plan_begins_behind_the_prefix():
    """Lengths below the prefix count as the prefix, also where it fills the table."""
    tables = [[8, 9, -1, -1], [8, 9, 3, 4], [8, 9, -1, -1], [8, 9, 2, -1], [8, 9, -1, -1]]
    ring = [5, 6, 7] + [-1] * 7
    for lens in ([0, 50, 0, 33, 0], [32, 31, 17, 48, 1]):
        for new in ([3, -1, 0, 20, 33], [17, 1, -1, -1, 40], [0, 0, 0, 0, 0]):
            _check(lens, new, tables, ring, [0, 3], 16, 64, prefix_pages=2)
    _check([0, 10, 64], [0, 1, -1], tables[:3], ring, [0, 3], 16, 64, prefix_pages=4)


def test_plan_is_the_same_when_repeated_and_in_replayed_graphs():
    """A captured plan follows the lengths: each replay takes the state that the
    program wrote in between, with eager work around it."""
    rng = random.Random(3)
    page, n, cap = 16, 40, 64
    lens, new, tables, free_ring, ring = _state(rng, n, page, 100, 1, ended=0, count=300, width=30)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    l, t, tb, fr, rg = dev(lens), dev(new), dev(tables), dev(free_ring), dev(ring)
    out = B.empty_kv_plan(n, cap)
    call = lambda: B.qkv_plan(l, t, tb, fr, rg, page, cap, out=out)
    call()
    first = [x.clone() for x in (out.slots, out.lens, out.ring, tb, fr)]
    call()
    for a, b in zip(first, (out.slots, out.lens, out.ring, tb, fr)):
        assert torch.equal(a, b)
    tb.copy_(dev(tables))
    fr.copy_(dev(free_ring))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for step in range(20):
        new = [-1 if rng.random() < 0.03 else rng.randrange(0, 3) for _ in range(n)]
        t.copy_(dev(new))
        g.replay()
        want = PO.plan_step(lens, new, tables, free_ring, ring, page, cap)
        for k, v in dict(lens=out.lens, kv_lens=out.kv_lens, offsets=out.offsets, positions=out.positions,
                         slots=out.slots, ring=out.ring, tables=tb, free_ring=fr).items():
            assert v.tolist() == want[k], (step, k)
        l.copy_(out.lens)
        rg.copy_(out.ring)
        lens, tables, free_ring, ring = want["lens"], want["tables"], want["free_ring"], want["ring"]
