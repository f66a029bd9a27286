"""Calls on another stream that leave their buffers to the binding, with the
current stream busy before them and taking memory behind them."""

import math

import pytest
import torch

from paper_2607_00501_amd import binding as B
from tests.test_gpu_paged_limits import _inputs

pytestmark = pytest.mark.gpu


def _busy(a):
    for _ in range(4):
        a = a @ a * 1e-3
    return a


@pytest.mark.parametrize("prefix_pages", [0, 3])
def test_calls_on_another_stream_with_their_own_buffers(prefix_pages):
    args = _inputs(41, 16, 8, 128, 64, [900, 4000, 300], [1, 90, 200], prefix_pages)
    q, k, v, tables, offsets, kv_lens, prefix = args
    logits = torch.randn((7, 40000), device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    lens, new = torch.tensor([5, 40, 0], **i32), torch.tensor([3, -1, 20], **i32)
    pages, ring, state = torch.arange(12, **i32).view(3, 4), torch.arange(12, 32, **i32), torch.tensor([0, 20], **i32)
    a = torch.randn((4096, 4096), device="cuda").half()

    def calls(stream=None):                                          # (a plan repeated does the same)
        out = B.qattn_paged_f16(q, k, v, tables, offsets, kv_lens, 1 / math.sqrt(128), prefix=prefix, stream=stream)
        plan = B.qkv_plan(lens, new, pages, ring, state, 16, 2000, stream=stream)
        return [out, B.qdec_argmax_rows(logits, stream=stream), plan.lens, plan.slots, plan.offsets]

    want = calls()
    side = torch.cuda.Stream()
    sizes = [t.numel() * t.element_size() for t in want]
    sizes.append(B.qattn_paged_workspace_bytes(16, 8, 128, 3, 291, prefix_pages))
    torch.cuda.synchronize()
    for turn in range(6):
        # Blocks of these sizes in use on the current stream, and free for the next allocation there.
        _busy(a)
        for n in sizes:
            torch.full((n,), turn, dtype=torch.uint8, device="cuda")
        with torch.cuda.stream(side):
            _busy(a)
        got = calls(side)
        for n in sizes * 2:                                          # blocks handed out again while the calls wait
            torch.full((n,), 255, dtype=torch.uint8, device="cuda")
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(x, y) for x, y in zip(got, want)), turn
        del got
