"""qattn_paged_f16 at its limits (heads, requests, tokens, long caches), over
random batches, with used workspaces and with two calls at once: rows taken
from the output against fp64 on the device."""

import math

import numpy as np
import pytest
import torch

from paper_2607_00501_amd import binding as B

pytestmark = pytest.mark.gpu


def _inputs(seed, hq, hkv, d, page, kv_lens, new, prefix_pages=0):
    """As a server holds them: every request's pages scattered over the pool, the
    prefix in one place."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    held = [-(-n // page) for n in kv_lens]
    own = [max(h - prefix_pages, 0) for h in held]
    n_pages = prefix_pages + sum(own) + 1
    ids = torch.randperm(n_pages, generator=g, device="cuda", dtype=torch.int32).cpu()
    tables = torch.full((len(kv_lens), max(held + [prefix_pages, 1])), -1, dtype=torch.int32)
    at = prefix_pages
    for i, h in enumerate(held):
        tables[i, :min(h, prefix_pages)] = ids[:min(h, prefix_pages)]
        tables[i, min(h, prefix_pages):h] = ids[at:at + own[i]]
        at += own[i]
    k, v = (torch.randn((n_pages, hkv, page, d), generator=g, device="cuda").half() for _ in range(2))
    offsets = torch.tensor([0] + np.cumsum(new).tolist(), dtype=torch.int32)
    q = torch.randn((int(offsets[-1]), hq, d), generator=g, device="cuda").half()
    prefix = ids[:prefix_pages].cuda() if prefix_pages else None
    return q, k, v, tables.cuda(), offsets.cuda(), torch.tensor(kv_lens, dtype=torch.int32, device="cuda"), prefix


def _check(args, out, rows, heads=None):
    """Rows (tokens) and query heads of out in fp64.  The bound: half a step of fp16
    for the output and for each weight, scores within 2^-12 of the weights, and
    fp32 sums over at most 2^12 MFMA steps one after the other, 2^-12 of
    size = sum w |v| again."""
    q, k, v, tables, offsets, kv_lens, _ = args
    _, hq, d = q.shape
    group, scale = hq // k.shape[1], float(np.float32(1 / math.sqrt(d)))
    off, lens = offsets.tolist(), kv_lens.tolist()
    out = out.view(q.shape).double()
    for t in rows:
        i = max(r for r in range(len(lens)) if off[r] <= t < off[r + 1])
        n = lens[i] - (off[i + 1] - off[i]) + t - off[i] + 1
        if n <= 0:
            assert not out[t].any()
            continue
        pages = tables[i, :-(-n // k.shape[2])].long()
        for h in (heads or range(hq)):
            kk, vv = (x[pages, h // group].reshape(-1, d)[:n].double() for x in (k, v))
            w = torch.softmax(scale * (kk * q[t, h].double()).sum(1), 0)[:, None]
            ref, size = (w * vv).sum(0), (w * vv.abs()).sum(0)
            bound = 2.0 ** -11 * ref.abs() + (2.0 ** -11 + 2.0 ** -11) * size + 2.0 ** -25
            worst = ((out[t, h] - ref).abs() / bound).max().item()
            assert worst <= 1.0, (t, h, n, worst)                     # (NaN: not)


def _run(args, **kw):
    q, k, v, tables, offsets, kv_lens, prefix = args
    return B.qattn_paged_f16(q, k, v, tables, offsets, kv_lens, 1 / math.sqrt(q.shape[2]), prefix=prefix, **kw)


@pytest.mark.parametrize("hq,hkv,d,kv_lens,new,prefix_pages", [
    (1024, 128, 64, [40, 3], [1, 2], 0), (1024, 8, 64, [70, 200], [1, 3], 1), (128, 128, 128, [130], [20], 0),
    (128, 128, 128, [130, 90], [1, 1], 2), (256, 2, 128, [50, 300], [40, 1], 0)])
def test_head_limits(hq, hkv, d, kv_lens, new, prefix_pages):
    args = _inputs(hq + d, hq, hkv, d, 32, kv_lens, new, prefix_pages)
    _check(args, _run(args), [0, sum(new) - 1], [0, 1, hq // 2, hq - 1])


@pytest.mark.parametrize("hq,hkv,d,new,prefix_pages", [
    (1, 1, 64, [1, 1], 0), (8, 2, 128, [1, 17], 0), (8, 2, 128, [1, 1], 700), (4, 1, 64, [60, 100], 500)])
def test_long_caches(hq, hkv, d, new, prefix_pages):
    """More keys than 2^18, over as many parts as there are workers."""
    args = _inputs(5, hq, hkv, d, 256, [300001, 180003], new, prefix_pages)
    _check(args, _run(args), sorted({0, new[0], sum(new) - 1}))


def test_one_prompt_of_all_tokens():
    args = _inputs(6, 2, 1, 64, 128, [65536], [65536])
    _check(args, _run(args), [0, 1, 63, 64, 127, 128, 4095, 30000, 65471, 65472, 65535])


@pytest.mark.parametrize("prefix_pages", [0, 6])
def test_all_requests_with_all_tokens(prefix_pages):
    """1,024 requests of 0 to 128 tokens, 65,536 in all."""
    rng = np.random.default_rng(7)
    new = rng.integers(0, 65, 1024)
    new[np.arange(512) * 2 + 1] = 128 - new[np.arange(512) * 2]
    kv = new + np.where(rng.random(1024) < 0.5, 0, rng.integers(0, 200, 1024))
    args = _inputs(8, 4, 2, 64, 16, [int(x) + 16 * prefix_pages for x in kv], new.tolist(), prefix_pages)
    assert int(args[4][-1]) == 65536
    _check(args, _run(args), [0, 65535] + rng.integers(0, 65536, 60).tolist())


@pytest.mark.parametrize("seed", range(12))
def test_random_batches(seed):
    """Lengths, new tokens, heads and pages over their ranges, short and long
    requests side by side; a workspace full of NaN, and the same bits again."""
    rng = np.random.default_rng(100 + seed)
    log_int = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    d, hkv, group, page = int(rng.choice([64, 128])), log_int(1, 9), log_int(1, 13), int(rng.choice([16, 32, 64, 128, 256]))
    prefix_pages = log_int(1, 3000) // page if seed % 2 else 0
    n = log_int(1, 90)
    new = [log_int(1, 700) if rng.random() < 0.2 else 1 for _ in range(n)]
    kv = [t + prefix_pages * page + (0 if rng.random() < 0.2 else log_int(1, 5000)) for t in new]
    args = _inputs(seed, hkv * group, hkv, d, page, kv, new, prefix_pages)
    ws = torch.full((B.qattn_paged_workspace_bytes(hkv * group, hkv, d, n, sum(new), prefix_pages),), 255,
                    dtype=torch.uint8, device="cuda")
    out = _run(args, workspace=ws)
    _check(args, out, {0, sum(new) - 1, *rng.integers(0, sum(new), 12).tolist()}, [0, hkv * group - 1])
    ws.fill_(127)
    assert torch.equal(_run(args, workspace=ws), out)


def test_two_calls_at_once():
    """Two streams, a workspace each."""
    both = [_inputs(30 + i, 16, 8, 128, 64, [3000 + 500 * i, 900], [1, 200], 3 * i) for i in range(2)]
    alone = [_run(args) for args in both]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.zeros_like(alone[i]) for _ in range(8)] for i in range(2)]
    ws = [torch.empty(B.qattn_paged_workspace_bytes(16, 8, 128, 2, 201, 3 * i), dtype=torch.uint8, device="cuda")
          for i in range(2)]
    torch.cuda.synchronize()
    for x in range(8):
        for i in range(2):
            _run(both[i], out=outs[i][x], workspace=ws[i], stream=streams[i])
    torch.cuda.synchronize()
    assert all(torch.equal(o, alone[i]) for i in range(2) for o in outs[i])


def test_prefix_pages_that_are_none():
    """Every row sees the prefix."""
    for bad in (-1, 2 ** 31 - 1):
        args = list(_inputs(9, 8, 4, 64, 16, [100, 70], [1, 40], 3))
        args[6] = args[6].clone()
        args[6][1] = bad
        assert torch.isnan(_run(args)).all()
