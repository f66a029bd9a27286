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


def _pairs(sizes, written):
    return [(a, b) for a in written for b in sizes if a != b]


APPEND_SIZES = dict(q=20 * 4 * 64 * 4, k=20 * 2 * 64 * 4, v=20 * 2 * 64 * 4, positions=80, slots=160, q_norm=128,
                    k_norm=128, table=50 * 64 * 4, q_out=20 * 4 * 64 * 2, k_pages=8 * 2 * 16 * 64 * 2,
                    v_pages=8 * 2 * 16 * 64 * 2)
APPEND = dict(q=0, k=0, v=0, hq=4, hkv=2, d=64, tokens=20, positions=0, slots=0, interleaved=0, q_norm=0, k_norm=0,
              eps=1e-6, table=0, table_len=50, q_out=0, k_pages=0, v_pages=0, n_pages=8, page_size=16, stream=None)
ATTEND_SIZES = dict(q=30 * 4 * 64 * 2, k_pages=10 * 2 * 16 * 64 * 2, v_pages=10 * 2 * 16 * 64 * 2, tables=3 * 4 * 4,
                    prefix=8, offsets=16, kv_lens=12, out=30 * 4 * 64 * 2)
ATTEND = dict(q=0, k_pages=0, v_pages=0, n_pages=10, page_size=16, tables=0, max_pages=4, prefix=0, prefix_pages=2,
              offsets=0, kv_lens=0, n_req=3, tokens=30, hq=4, hkv=2, d=64, scale=0.1, out=0, workspace=at(0x40000000),
              ws_bytes=1 << 40, stream=None)
for args, sizes in ((APPEND, APPEND_SIZES), (ATTEND, ATTEND_SIZES)):
    args.update({k: at(0x100000 * (i + 1)) for i, k in enumerate(sizes)})


def _check(name, args, sizes, one, other):
    """`one` over the first and the last 16 bytes of `other`, and with its own last ones over the first."""
    base = args[other].value
    for place in (base, base + max(0, sizes[other] - 16) // 16 * 16, base - max(0, sizes[one] - 16) // 16 * 16):
        if place < base + sizes[other] and base < place + sizes[one]:
            status, error = _call(name, args, **{one: at(place)})
            assert status == EINVAL and one in error and other in error, (place - base, error)


@pytest.mark.parametrize("one,other", _pairs(APPEND_SIZES, ("q_out", "k_pages", "v_pages")))
def test_append_buffers_share_no_bytes(one, other):
    _check("qkv_rope_append", APPEND, APPEND_SIZES, one, other)


@pytest.mark.parametrize("one,other", _pairs(ATTEND_SIZES, ("out",)))
def test_attention_buffers_share_no_bytes(one, other):
    _check("qattn_paged_f16", ATTEND, ATTEND_SIZES, one, other)


@pytest.mark.gpu
def test_attention_workspace_shares_no_bytes():
    import torch
    from tests.test_gpu_paged_limits import _inputs
    q, k, v, tables, offsets, kv_lens, prefix = _inputs(3, 4, 2, 64, 16, [100, 70], [1, 40], 2)
    need = B.qattn_paged_workspace_bytes(4, 2, 64, 2, 41, 2)
    big = torch.zeros(need + q.numel() * 2, dtype=torch.uint8, device="cuda")
    tail = big[need:].view(torch.float16).view(41, -1)
    for first in (0, 16):
        call = lambda: B.qattn_paged_f16(q, k, v, tables, offsets, kv_lens, 0.1, prefix=prefix, out=tail,
                                         workspace=big[first:])
        if first == 0:
            call()                                                   # (side by side)
        else:
            with pytest.raises(B.QmError) as e:
                call()
            assert e.value.status == EINVAL
