"""BatchDecoder: slots without new tokens keep what they would go on with."""

import pytest
import torch

from paper_2607_00501_amd.decoder import BatchDecoder
from tests.test_gpu_batch_decoder import D128, TINY
from tests.test_gpu_decode import _model

pytestmark = pytest.mark.gpu

I32 = dict(dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("cfg", [TINY, D128])
def test_idle_ended_and_refused_slots_keep_their_tokens(cfg):
    """A step leaves logits and token of every slot that has no new tokens in it,
    or whose tokens are refused, as they were (the first, the last, all between
    others), and slots that have never had any have token 0."""
    layers, emb, norm, head, _ = _model(cfg, 67)
    dec = BatchDecoder(cfg, emb, layers, norm, head, n_req=6, n_pages=6, max_len=64, page_size=16, max_tokens=40)
    dec.step(torch.arange(3, 3 + 12, **I32), torch.tensor([2, 5, 0, 1, 4, 0], **I32))
    assert dec.token[2].item() == dec.token[5].item() == 0
    # The sixth takes the two pages that are left, the second is refused when it needs another one.
    for new, kept in [([0, 1, 0, 0, 2, 0], [0, 2, 3, 5]), ([1, 0, 0, 0, 0, 17], [1, 2, 3, 4]),
                      ([0, 15, 0, 3, 0, 1], [0, 1, 2, 4]), ([-1, 0, 0, 1, 0, 0], [0, 1, 2, 4, 5])]:
        logits, token = dec.logits.clone(), dec.token.clone()
        dec.step(torch.arange(40, 40 + sum(max(x, 0) for x in new) + 3, **I32), torch.tensor(new, **I32))
        assert torch.equal(dec.logits[kept], logits[kept]) and torch.equal(dec.token[kept], token[kept]), new
        changed = [i for i in range(6) if i not in kept]
        assert all((dec.logits[i] != logits[i]).any() for i in changed), new
    assert dec.plan.refused.item() == 0 and dec.plan.ring[1].item() == 1
