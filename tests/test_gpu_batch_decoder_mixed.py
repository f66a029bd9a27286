"""BatchDecoder: one captured step replayed between eager ones, in any order."""

import numpy as np
import pytest
import torch

from paper_2607_00501_amd.decoder import BatchDecoder
from tests.test_gpu_batch_decoder import TINY
from tests.test_gpu_decode import _model

pytestmark = pytest.mark.gpu

I32 = dict(dtype=torch.int32, device="cuda")


def _captured(dec, tokens, new, steps=1):
    """A graph of steps that feed the decoder's own tokens back to requests of `new`."""
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for _ in range(steps):
            tokens.copy_(dec.token)
            dec.step(tokens, new)
    return g


@pytest.mark.parametrize("steps", [1, 2])
@pytest.mark.parametrize("prefix", [0, 32])
def test_replays_and_eager_steps_in_any_order(steps, prefix):
    """Decode steps replayed from a graph, prompts that join and requests that end
    in eager steps between them, one or two at a time, against the same steps all
    launched one by one."""
    layers, emb, norm, head, _ = _model(TINY, 66)
    n = 3
    decs = [BatchDecoder(TINY, emb, layers, norm, head, n_req=n, n_pages=60, max_len=256, page_size=16, max_tokens=64)
            for _ in range(2)]
    ones, fed = torch.ones(n, **I32), [torch.zeros(n, **I32) for _ in range(2)]
    for d in decs:
        if prefix:
            d.share_prefix(torch.arange(1, 1 + prefix, **I32))
        d.step(torch.arange(5, 5 + 7, **I32), torch.tensor([5, 1, 1], **I32))
    g = _captured(decs[0], fed[0], ones, steps)
    rng = np.random.default_rng(steps)
    lens = [prefix + x for x in (5, 1, 1)]

    def count(new):
        return [0 if x < 0 else max(a, prefix) + x for a, x in zip(lens, new)]

    for turn in range(12):
        for _ in range(int(rng.integers(0, 3))):                     # replays
            g.replay()
            for _ in range(steps):
                fed[1].copy_(decs[1].token)
                decs[1].step(fed[1], ones)
                lens = count([1, 1, 1])
        for _ in range(int(rng.integers(0, 4))):                     # eager: one ends or has a prompt, others a few tokens
            new = [int(x) for x in rng.integers(0, 6, n)]
            new[int(rng.integers(0, n))] = -1 if rng.random() < 0.5 else 17
            tokens = torch.arange(1, 1 + max(1, sum(new) + 1), **I32) * 7 % 1000
            for d in decs:
                d.step(tokens, torch.tensor(new, **I32))
            lens = count(new)
        torch.cuda.synchronize()
        assert decs[0].plan.lens.tolist() == decs[1].plan.lens.tolist() == lens, turn
        assert decs[0].plan.ring[1].item() == decs[1].plan.ring[1].item()
        assert torch.equal(decs[0].logits, decs[1].logits) and torch.equal(decs[0].token, decs[1].token)
        pages = [p for i in range(n) for p in decs[0].tables[i, prefix // 16:-(-lens[i] // 16)].tolist()]
        assert len(set(pages)) == len(pages)                         # no page has two owners


def test_no_prefix_behind_a_captured_step():
    """The graph has none: its requests would begin without the prefix, and give its
    pages back when they end."""
    layers, emb, norm, head, _ = _model(TINY, 68)
    dec = BatchDecoder(TINY, emb, layers, norm, head, n_req=2, n_pages=20, max_len=128, page_size=16, max_tokens=32)
    ones, fed = torch.ones(2, **I32), torch.zeros(2, **I32)
    dec.step(fed, ones)
    dec.step(fed, -ones)                                             # (nothing is held)
    g = _captured(dec, fed, ones)
    with pytest.raises(ValueError, match="captured"):
        dec.share_prefix(torch.zeros(16, **I32))
    for _ in range(3):
        g.replay()
    assert dec.plan.lens.tolist() == [3, 3] and dec.prefix is None
