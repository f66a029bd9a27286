"""Buffers of the paged cache's calls that share bytes are refused before any
device work (no GPU needed)."""

import ctypes

import pytest

from paper_2607_00501_amd import binding as B

EINVAL = 1
at = ctypes.c_void_p


def _call(name, args, **changed):
    status = getattr(B.lib(), name)(*dict(args, **changed).values())
    return status, B.qm_last_error()


# 300 requests of 40 pages, 2,000 tokens (two workgroups): every buffer in a place of its own.
SIZES = dict(lens=1200, new_lens=1200, tables=48000, free_ring=4000, ring=8, lens_out=1200, kv_lens=1200, offsets=1204,
             positions=8000, slots=16000, ring_out=8, refused=4)
READ = ("lens", "new_lens", "ring")
PLACE = {k: 0x100000 * (i + 1) for i, k in enumerate(SIZES)}
PLAN = dict(lens=None, new_lens=None, n_req=300, page_size=16, tables=None, max_pages=40, prefix_pages=0, free_ring=None,
            ring=None, n_pages=1000, max_tokens=2000, lens_out=None, kv_lens=None, offsets=None, positions=None,
            slots=None, ring_out=None, refused=None, stream=None)
PLAN.update({k: at(v) for k, v in PLACE.items()})


@pytest.mark.parametrize("one,other", [(a, b) for a in SIZES for b in SIZES
                                       if a != b and not (a in READ and b in READ)])   # (what is only read may be the same)
def test_plan_buffers_share_no_bytes(one, other):
    step = 8 if one == "slots" else 4
    for place in (PLACE[other], PLACE[other] + SIZES[other] // 8 * 8 - step, PLACE[other] - (SIZES[one] // 8 * 8 - step)):
        if place + SIZES[one] <= PLACE[other] or place >= PLACE[other] + SIZES[other] or place % step:
            continue
        status, error = _call("qkv_plan", PLAN, **{one: at(place)})
        assert status == EINVAL and one in error and other in error, (place - PLACE[other], error)
