"""qkv_rope_append: the bits of the contiguous cache's RoPE and append at the
pages' rows, tokens without a place left alone, the rotation in 64 bits."""

import numpy as np
import pytest
import torch

from oracle import qmatmul_oracle as O
from paper_2607_00501_amd import binding as B

pytestmark = pytest.mark.gpu

THETA = 5e5


def _inputs(seed, t, hq, hkv, d, norm):
    g = torch.Generator(device="cuda").manual_seed(seed)
    f = lambda *s: torch.randn(s, generator=g, device="cuda")
    gains = [(1 + 0.1 * f(d)).half() for _ in range(2)] if norm else [None, None]
    return f(t, hq * d), f(t, hkv * d), f(t, hkv * d), gains


@pytest.mark.parametrize("hq,hkv,d,page,t,p0", [
    (16, 8, 128, 16, 1, 0), (16, 8, 128, 16, 1, 77), (32, 8, 64, 32, 33, 15), (24, 8, 128, 64, 100, 3),
    (1, 1, 64, 256, 5, 250), (14, 2, 128, 128, 257, 1000), (7, 7, 64, 16, 600, 0)])
@pytest.mark.parametrize("norm,interleaved", [(False, False), (True, False), (False, True)])
def test_append_equals_the_contiguous_cache(hq, hkv, d, page, t, p0, norm, interleaved):
    q, k, v, (qn, kn) = _inputs(t + d, t, hq, hkv, d, norm)
    max_len = -(-(p0 + t) // page) * page
    table = B.qdec_rope_table(max_len, d, THETA)
    kc, vc = (torch.zeros((hkv, max_len, d), dtype=torch.float16, device="cuda") for _ in range(2))
    want = B.qdec_rope_append_rows(q, k, v, p0, THETA, kc, vc, interleaved=interleaved, q_norm=qn, k_norm=kn,
                                   table=table)
    n_pages = max_len // page + 3
    ids = torch.randperm(n_pages, device="cuda")
    pos = torch.arange(p0, p0 + t, device="cuda")
    slots = ids[pos // page] * page + pos % page
    kp, vp = (torch.full((n_pages, hkv, page, d), 9.0, dtype=torch.float16, device="cuda") for _ in range(2))
    order = torch.randperm(t, device="cuda")              # tokens in any order
    got = B.qkv_rope_append(q[order], k[order], v[order], pos[order].int(), slots[order], table, kp, vp,
                            interleaved=interleaved, q_norm=qn, k_norm=kn)
    assert torch.equal(got, want.transpose(0, 1)[order])
    untouched = torch.ones((n_pages, page), dtype=torch.bool, device="cuda")
    untouched[ids[pos // page], pos % page] = False
    for pool, cache in ((kp, kc), (vp, vc)):
        assert torch.equal(pool[ids[pos // page], :, pos % page], cache[:, p0:p0 + t].transpose(0, 1))
        assert (pool.transpose(1, 2)[untouched] == 9.0).all()


def test_append_leaves_tokens_without_a_place():
    hq, hkv, d, page, n_pages, t = 4, 2, 64, 16, 3, 8
    q, k, v, _ = _inputs(1, t, hq, hkv, d, False)
    table = B.qdec_rope_table(20, d, THETA)
    kp, vp = (torch.full((n_pages, hkv, page, d), 9.0, dtype=torch.float16, device="cuda") for _ in range(2))
    q_out = torch.full((t, hq, d), 9.0, dtype=torch.float16, device="cuda")
    slots = torch.tensor([-1, 5, n_pages * page, 2 ** 40, 7, 9, 11, -(2 ** 62)], device="cuda")
    pos = torch.tensor([3, 3, 3, 3, -1, 20, 19, 3], dtype=torch.int32, device="cuda")
    B.qkv_rope_append(q, k, v, pos, slots, table, kp, vp, q_out=q_out)
    there = [i for i in range(t) if (q_out[i] != 9.0).any()]
    assert there == [1, 6]
    rows = (kp.transpose(1, 2).reshape(-1, hkv * d) != 9.0).any(1).nonzero().flatten().tolist()
    assert rows == [5, 11]
    assert torch.equal(vp[0, :, 5].reshape(-1), v[1].half()) and torch.equal(vp[0, :, 11].reshape(-1), v[6].half())


def test_append_in_64_bits():
    """One rounding to fp16 of a rotation in fp32: within half a step (2^-11), plus
    three fp32 roundings of the products' size."""
    hq, hkv, d, page, t = 3, 1, 128, 32, 50
    q, k, v, _ = _inputs(5, t, hq, hkv, d, False)
    max_len = 4096
    table = B.qdec_rope_table(max_len, d, THETA)
    pos = torch.randint(0, max_len, (t,), device="cuda", dtype=torch.int32)
    kp, vp = (torch.zeros((2, hkv, page, d), dtype=torch.float16, device="cuda") for _ in range(2))
    got = B.qkv_rope_append(q, k, v, pos, torch.arange(t, device="cuda"), table, kp, vp).cpu().numpy()
    x = q.view(t, hq, d).cpu().numpy()
    for i in range(t):
        for h in range(hq):
            ref = O.rope(x[i, h][None], int(pos[i]), THETA)[0]
            size = np.hypot(x[i, h], np.roll(x[i, h], d // 2)).astype(np.float64)
            assert (np.abs(got[i, h] - ref) <= 2.0 ** -11 * np.abs(ref) + 2.0 ** -22 * size + 2.0 ** -25).all()


def test_append_past_32_bits():
    """A row beyond 2^32 elements of the pools."""
    hq, hkv, d, page = 2, 8, 128, 256
    n_pages = (1 << 32) // (hkv * page * d) + 2
    kp, vp = (torch.empty((n_pages, hkv, page, d), dtype=torch.float16, device="cuda") for _ in range(2))
    kp[-1], vp[-1], kp[:2], vp[:2] = 9.0, 9.0, 9.0, 9.0
    q, k, v, _ = _inputs(2, 2, hq, hkv, d, False)
    table = B.qdec_rope_table(8, d, THETA)
    slots = torch.tensor([n_pages * page - 1, 3], device="cuda")
    B.qkv_rope_append(q, k, v, torch.tensor([0, 0], dtype=torch.int32, device="cuda"), slots, table, kp, vp)
    assert torch.equal(kp[-1, :, -1].reshape(-1), k[0].half()) and torch.equal(vp[0, :, 3].reshape(-1), v[1].half())
    assert (kp[-1, :, :-1] == 9.0).all() and (kp[0, :, 4:] == 9.0).all() and (kp[1] == 9.0).all()
