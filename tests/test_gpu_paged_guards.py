"""qattn_paged_f16 writes its output and its workspace and nothing beside them:
both lie between guards, the workspace with exactly the bytes that it asks for."""

import math

import numpy as np
import pytest
import torch

from paper_2607_00501_amd import binding as B
from tests.test_gpu_paged_limits import _check, _inputs

pytestmark = pytest.mark.gpu

GUARD = 1 << 16
FILL = 0x5A


class _Between:
    """n bytes between two guards."""

    def __init__(self, n):
        self.n = n
        self.whole = torch.full((n + 2 * GUARD,), FILL, dtype=torch.uint8, device="cuda")
        self.inner = self.whole[GUARD:GUARD + n]

    def check(self):
        assert (self.whole[:GUARD] == FILL).all() and (self.whole[GUARD + self.n:] == FILL).all()


def _run(args, pad=3):
    """With `pad` rows of the output behind the last token."""
    q, k, v, tables, offsets, kv_lens, prefix = args
    t, hq, d = q.shape
    hkv, n = k.shape[1], tables.shape[0]
    rows = torch.cat([q, torch.full((pad, hq, d), float("nan"), dtype=q.dtype, device="cuda")])
    ws = _Between(B.qattn_paged_workspace_bytes(hq, hkv, d, n, t + pad, 0 if prefix is None else prefix.numel()))
    out = _Between((t + pad) * hq * d * 2)
    got = B.qattn_paged_f16(rows, k, v, tables, offsets, kv_lens, 1 / math.sqrt(d), prefix=prefix,
                            out=out.inner.view(torch.float16).view(t + pad, hq * d), workspace=ws.inner)
    ws.check()
    out.check()
    return got


HEADS = [(16, 8, 128), (32, 8, 64), (1, 1, 64), (128, 128, 64), (1024, 128, 64), (24, 8, 128), (128, 1, 128), (5, 1, 64)]


@pytest.mark.parametrize("prefix_pages", [0, 1, 40])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_batches_of_all_kinds(hq, hkv, d, prefix_pages):
    """Long and short requests, single tokens and prompts, as many parts as there are
    workers; and a few rows only."""
    rng = np.random.default_rng(hq + d)
    for n, longest, most_new in ((40 if hq < 200 else 6, 6000, 60), (3, 90000, 1), (1, 40, 1), (1, 700, 300)):
        new = [int(x) for x in rng.integers(1, most_new + 1, n)]
        kv = [t + 16 * prefix_pages + int(rng.integers(0, longest)) for t in new]
        args = _inputs(n, hq, hkv, d, 16, kv, new, prefix_pages)
        out = _run(args)
        t = sum(new)
        _check(args, out[:t], [0, t - 1], [0, hq - 1])
        assert (out[t:].view(torch.uint8) == FILL).all()


@pytest.mark.parametrize("prefix_pages", [0, 2])
def test_all_requests_and_tokens(prefix_pages):
    args = _inputs(9, 4, 2, 64, 16, [64 + 16 * prefix_pages] * 1024, [64 - 1] + [64] * 1022 + [61], prefix_pages)
    out = _run(args)
    t = int(args[4][-1])
    _check(args, out[:t], [0, 63, t - 1])
    assert (out[t:].view(torch.uint8) == FILL).all()


@pytest.mark.parametrize("offsets,kv_lens", [
    ([0, 10 ** 6, -5], [10 ** 9, -3]), ([2 ** 31 - 1, 0, 3], [2 ** 31 - 1, 64]), ([0, 0, 2 ** 31 - 1], [5, 5]),
    ([-(2 ** 31), 2, 1], [-(2 ** 31), 10 ** 9]), ([3, 2, 1], [64, 64]), ([1, 1, 1], [64, 64]), ([0, 3, 2], [0, 0])])
@pytest.mark.parametrize("prefix_pages", [0, 1])
@pytest.mark.parametrize("new", [[2, 1], [20, 30]])
def test_arrays_out_of_their_limits(offsets, kv_lens, prefix_pages, new):
    """Offsets that fall or pass the tokens, lengths below 0 or past the tables: held
    to their limits, whatever the rows then are."""
    args = list(_inputs(14, 4, 2, 64, 16, [50 + new[0], 60 + new[1]], new, prefix_pages))
    i32 = dict(dtype=torch.int32, device="cuda")
    bad = args[:4] + [torch.tensor(offsets, **i32), torch.tensor(kv_lens, **i32), args[6]]
    _run(bad)
    out = _run(args)
    _check(args, out[:sum(new)], range(sum(new)))
