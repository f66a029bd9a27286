"""BatchDecoder: the paged-cache entry points as they are used together.  Every
request's logits against the oracle's token-by-token decoder, whatever the
others do."""

import numpy as np
import pytest
import torch

from oracle import qmatmul_oracle as O
from paper_2607_00501_amd import binding as B
from paper_2607_00501_amd.decoder import BatchDecoder, DecoderConfig
from tests.helpers import MFMA_TOL, rel_err
from tests.test_gpu_decode import _model

pytestmark = pytest.mark.gpu

TINY = DecoderConfig(hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=64, inter=512, vocab=1000, layers=2, theta=1e4)
D128 = DecoderConfig(hidden=256, n_q_heads=6, n_kv_heads=2, head_dim=128, inter=256, vocab=500, layers=2, theta=1e4)


class _Oracle:
    """The oracle's decoder for one request."""

    def __init__(self, ref, cfg, max_len):
        self.ref, self.pos = ref, 0
        self.k = np.zeros((cfg.layers, cfg.n_kv_heads, max_len, cfg.head_dim))
        self.v = np.zeros_like(self.k)

    def feed(self, tokens):
        for t in tokens:
            logits = O.decode_step(self.ref, int(t), self.pos, self.k, self.v)
            self.pos += 1
        return logits


def _step(dec, fed, t_pad=0):
    """fed: request -> its new tokens, or None: it ends."""
    new = torch.zeros(dec.n_req, dtype=torch.int32)
    tokens = []
    for i in sorted(fed):
        new[i] = -1 if fed[i] is None else len(fed[i])
        tokens += fed[i] or []
    tokens += [0] * t_pad
    dec.step(torch.tensor(tokens, dtype=torch.int32, device="cuda"), new.cuda())


@pytest.mark.parametrize("cfg,interleave,qk_norm", [(TINY, True, False), (TINY, False, True), (D128, False, False)])
def test_requests_come_and_go(cfg, interleave, qk_norm):
    """Prompts, chunks of prompts and single tokens in one step, requests that end
    and slots that are taken again, fewer pages than everybody's longest: each
    request's logits are the oracle's at every step."""
    layers, emb, norm, head, ref = _model(cfg, 61, interleave=interleave, qk_norm=qk_norm)
    dec = BatchDecoder(cfg, emb, layers, norm, head, n_req=4, n_pages=9, max_len=64, page_size=16, max_tokens=64,
                       rope_rows_interleaved=interleave)
    rng = np.random.default_rng(0)
    some = lambda n: rng.integers(0, cfg.vocab, n).tolist()
    live = {}
    for fed, pad in [({0: some(13), 2: some(1)}, 0), ({0: some(1), 1: some(20), 2: some(17)}, 9),
                     ({0: some(1), 1: some(1), 2: some(1), 3: some(5)}, 0), ({0: some(1), 1: None, 3: some(30)}, 3),
                     ({0: None, 2: some(1), 3: some(1)}, 0), ({1: some(40), 2: some(2), 3: some(1)}, 0),
                     ({0: some(3), 1: some(1)}, 30)]:
        _step(dec, fed, pad)
        assert dec.plan.refused.item() == 0
        for i, tokens in fed.items():
            if tokens is None:
                del live[i]
                continue
            want = live.setdefault(i, _Oracle(ref, cfg, 64)).feed(tokens)
            got = dec.logits[i].cpu().numpy()
            assert rel_err(got, want) <= MFMA_TOL, (i, len(tokens))
            assert dec.token[i].item() == O.greedy_token(got)
    held = dec.plan.lens.tolist()
    assert held == [live[i].pos if i in live else 0 for i in range(4)]
    used = [p for i in range(4) for p in dec.tables[i, :-(-held[i] // 16)].tolist()]
    assert len(set(used)) == len(used) and dec.plan.ring[1].item() == 9 - len(used)


def test_shared_prefix_and_refusal():
    """A prefix run once serves every request; a request that finds no pages is
    refused and the others go on."""
    layers, emb, norm, head, ref = _model(TINY, 62)
    dec = BatchDecoder(TINY, emb, layers, norm, head, n_req=5, n_pages=7, max_len=128, page_size=16, max_tokens=48)
    rng = np.random.default_rng(1)
    prefix = rng.integers(0, 1000, 64).tolist()
    dec.share_prefix(torch.tensor(prefix, dtype=torch.int32, device="cuda"))     # 4 pages, in two steps
    first = _Oracle(ref, TINY, 128)
    first.feed(prefix)
    live = {}
    for fed, refused in [({0: [5, 6, 7], 2: [9]}, []), ({0: [1], 2: list(range(10)), 4: [3, 4]}, []),
                         ({0: [2] * 12, 1: [8], 4: [7]}, [1]), ({0: None, 2: [1], 4: [5]}, []), ({1: [8, 9], 2: [3]}, [])]:
        _step(dec, fed)
        assert dec.plan.refused.item() == len(refused)
        for i, tokens in fed.items():
            if tokens is None:
                live.pop(i)
            elif i not in refused:
                if i not in live:
                    live[i] = _Oracle(ref, TINY, 128)
                    live[i].k, live[i].v, live[i].pos = first.k.copy(), first.v.copy(), first.pos
                assert rel_err(dec.logits[i].cpu().numpy(), live[i].feed(tokens)) <= MFMA_TOL, (i, tokens)
            else:
                assert dec.plan.kv_lens[i].item() == 0
    with pytest.raises(ValueError):
        dec.share_prefix(torch.zeros(16, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        dec.step(torch.zeros(49, dtype=torch.int32, device="cuda"), torch.zeros(5, dtype=torch.int32, device="cuda"))


def test_replayed_steps_equal_eager_ones():
    """Two captured steps, the sampled tokens fed back on the device, replayed with
    eager work in between, against the same steps launched one by one."""
    layers, emb, norm, head, _ = _model(TINY, 63)
    decs = [BatchDecoder(TINY, emb, layers, norm, head, n_req=3, n_pages=40, max_len=200, page_size=16, max_tokens=64)
            for _ in range(2)]
    ones = torch.ones(3, dtype=torch.int32, device="cuda")
    prompts = torch.arange(3, 3 + 33, dtype=torch.int32, device="cuda")
    new = torch.tensor([20, 1, 12], dtype=torch.int32, device="cuda")
    tokens = [torch.zeros(3, dtype=torch.int32, device="cuda") for _ in range(2)]

    def one(i):
        tokens[i].copy_(decs[i].token)
        decs[i].step(tokens[i], ones)

    for d in decs:
        d.step(prompts, new)
        d.step(prompts[:3], ones)
    one(1)                                                   # (warms the second up)
    one(0)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        one(1)
        one(1)
    for _ in range(6):
        g.replay()
        one(0)
        one(0)
        torch.cuda.synchronize()
        assert torch.equal(decs[0].logits, decs[1].logits) and torch.equal(decs[0].token, decs[1].token)
        assert torch.equal(decs[0].plan.lens, decs[1].plan.lens)


def test_refused_steps_and_prefixes_change_nothing():
    """Wrong arguments, a prefix after a step, one whose pages are not there (its last
    part alone would find some): as if they had not been made."""
    layers, emb, norm, head, ref = _model(TINY, 64)
    dec = BatchDecoder(TINY, emb, layers, norm, head, n_req=2, n_pages=7, max_len=256, page_size=16, max_tokens=48)
    i32 = dict(dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        dec.share_prefix(torch.zeros(128, **i32))                    # 8 pages, parts of 3, 3 and 2
    _step(dec, {0: [5, 6, 7], 1: [8]})
    want = _Oracle(ref, TINY, 256)
    want.feed([5, 6, 7])
    for tokens, new in [(torch.zeros(2, **i32), torch.ones(3, **i32)),
                        (torch.zeros(2, **i32), torch.ones(2, dtype=torch.int64, device="cuda")),
                        (torch.zeros(2, **i32), torch.ones(2, dtype=torch.int32)),
                        (torch.zeros(2, dtype=torch.int32), torch.ones(2, **i32))]:
        with pytest.raises(ValueError):
            dec.step(tokens, new)
    with pytest.raises(ValueError):
        dec.share_prefix(torch.zeros(16, **i32))
    _step(dec, {0: [9]})
    assert dec.plan.lens.tolist() == [4, 1] and dec.plan.ring.tolist() == [2, 5]
    assert rel_err(dec.logits[0].cpu().numpy(), want.feed([9])) <= MFMA_TOL


def test_steps_on_another_stream():
    """A prefix in parts and steps, all on a stream of their own."""
    layers, emb, norm, head, _ = _model(TINY, 65)
    tokens = torch.arange(7, 7 + 96, dtype=torch.int32, device="cuda")
    new = torch.tensor([3, 0, 2], dtype=torch.int32, device="cuda")
    logits = []
    for stream in (None, torch.cuda.Stream()):
        dec = BatchDecoder(TINY, emb, layers, norm, head, n_req=3, n_pages=20, max_len=256, page_size=16, max_tokens=40)
        torch.cuda.synchronize()
        dec.share_prefix(tokens, stream=stream)
        dec.step(tokens[:5], new, stream=stream)
        torch.cuda.synchronize()
        assert dec.plan.lens.tolist() == [99, 96, 98]                # (all hold the prefix)
        logits.append(dec.logits[[0, 2]].clone())
    assert torch.equal(*logits)
