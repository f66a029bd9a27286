"""qattn_paged_f16 against fp64: ragged batches over scattered pages, a shared
prefix, prompts beside single tokens, what lies past a row's keys."""

import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as PO
from paper_2607_00501_amd import binding as B
from tests.paged_cases import assert_close, batch, on_gpu

pytestmark = pytest.mark.gpu


def _run(args, scale, **kw):
    q, k, v, tables, offsets, kv_lens, prefix = on_gpu(*args)
    return B.qattn_paged_f16(q, k, v, tables, offsets, kv_lens, scale, prefix=prefix, **kw)


def _check(args, scale=None, n_rows=None):
    q, k, v, tables, offsets, kv_lens, prefix = args
    t, hq, d = q.shape
    scale = 1 / math.sqrt(d) if scale is None else scale
    out = _run(args, scale).cpu().numpy().reshape(t, hq, d)
    ref, size = PO.paged_attention(q, k, v, tables, offsets, kv_lens, np.float32(scale), prefix)
    n = int(offsets[-1])
    assert_close(out[:n], ref[:n], size[:n], d)
    return out


# One token each: lengths around the 16-key tiles, the wavefronts' 32-key blocks,
# the 64-key split unit and the pages; every group size; both head dimensions.
@pytest.mark.parametrize("hq,hkv,d,page,kv_lens", [
    (1, 1, 64, 16, [1]), (16, 8, 128, 16, [1]), (8, 8, 64, 32, [2, 15, 16, 17]), (16, 8, 128, 16, [31, 32, 33, 1]),
    (24, 8, 128, 64, [63, 64, 65, 127, 128, 129]), (32, 8, 64, 256, [255, 256, 257, 5]),
    (40, 8, 64, 16, [100, 1, 700]), (6, 1, 128, 32, [1000]), (14, 2, 128, 128, [3000, 7]),
    (64, 8, 128, 16, [513, 40, 1]), (15, 1, 64, 16, [70, 300]), (16, 1, 128, 16, [90]), (17, 1, 64, 16, [50, 129]),
    (33, 1, 128, 32, [200]), (128, 1, 64, 16, [77]), (200, 2, 64, 16, [20, 300])])
def test_single_tokens(hq, hkv, d, page, kv_lens):
    _check(batch(hq + sum(kv_lens), hq, hkv, d, page, kv_lens, [1] * len(kv_lens)))


# Prompts, chunks after cached tokens and single tokens together.
@pytest.mark.parametrize("hq,hkv,d,page,kv_lens,new", [
    (4, 2, 64, 16, [5], [5]), (4, 2, 128, 16, [33, 1, 70], [33, 1, 20]), (8, 2, 64, 32, [40, 200], [39, 1]),
    (16, 8, 128, 64, [130, 64, 300], [129, 64, 2]), (3, 1, 64, 16, [257], [130]), (12, 4, 128, 128, [400, 9], [150, 9]),
    (2, 2, 64, 16, [16, 17, 15], [16, 17, 15]), (32, 8, 64, 16, [500], [260]), (5, 1, 128, 16, [64, 128], [64, 26]),
    (1, 1, 128, 32, [600, 3], [129, 3]), (6, 2, 64, 256, [700], [7])])
def test_prompts(hq, hkv, d, page, kv_lens, new):
    _check(batch(hq + sum(kv_lens), hq, hkv, d, page, kv_lens, new))


# A prefix that all share: as long as the requests, longer than some of them, in
# many pages; single tokens and prompts after it.
@pytest.mark.parametrize("hq,hkv,d,page,prefix_pages,kv_lens,new", [
    (4, 2, 64, 16, 1, [17], [1]), (4, 2, 64, 16, 2, [33, 32, 40], [1, 1, 1]),
    (16, 8, 128, 16, 5, [81, 90, 200, 80], [1, 1, 1, 1]), (8, 8, 64, 32, 3, [97, 300, 96], [1, 5, 1]),
    (24, 8, 128, 64, 4, [257, 256, 300, 700], [1, 1, 30, 100]), (14, 2, 64, 16, 9, [10, 150, 144, 1], [1, 6, 2, 1]),
    (16, 1, 128, 256, 2, [513, 600], [1, 1]), (64, 8, 128, 16, 20, [330] * 7, [1] * 7),
    (32, 8, 64, 128, 3, [400, 385, 20, 384], [16, 1, 20, 1]), (12, 4, 128, 16, 40, [700] * 40, [1] * 40)])
def test_shared_prefix(hq, hkv, d, page, prefix_pages, kv_lens, new):
    args = batch(sum(kv_lens), hq, hkv, d, page, kv_lens, new, prefix_pages=prefix_pages)
    out = _check(args)
    # The same batch without sharing reads the prefix from the tables.
    q, k, v, tables, offsets, lens, prefix = args
    ref, size = PO.paged_attention(q, k, v, tables, offsets, lens, np.float32(1 / math.sqrt(d)))
    assert_close(out, ref, size, d)
    _check((q, k, v, tables, offsets, lens, None))
    # With it, the tables' entries for the prefix are not read.
    blind = tables.copy()
    blind[:, :prefix_pages] = 10 ** 9
    assert np.array_equal(_check((q, k, v, blind, offsets, lens, prefix)), out)


def test_many_requests():
    """More requests than lanes: 16 a lane at most."""
    rng = np.random.default_rng(4)
    for n in (65, 300, 1024):
        kv_lens = rng.integers(1, 60, n).tolist()
        new = [int(min(x, rng.integers(0, 3))) for x in kv_lens]
        _check(batch(n, 2, 1, 64, 16, kv_lens, new))


def test_sharp_and_flat_softmax():
    for scale in (1.0, 1e-4):
        _check(batch(7, 16, 8, 64, 16, [900, 50], [1, 3]), scale)


def test_rows_without_keys_and_rows_behind_the_last():
    args = batch(2, 8, 4, 64, 16, [40, 0, 33, 0, 20], [1, 3, 2, 0, 20], pad=9)
    q, k, v, tables, offsets, kv_lens, _ = args
    for prefix in (None, tables[0, :1].copy()):
        out = torch.full((q.shape[0], 8 * 64), 5.0, dtype=torch.float16, device="cuda")
        dev = on_gpu(q, k, v, tables, offsets, kv_lens, prefix)
        B.qattn_paged_f16(*dev[:6], 0.125, prefix=dev[6], out=out)
        got = out.cpu().numpy().reshape(-1, 8, 64)
        ref, size = PO.paged_attention(q[:26], k, v, tables, offsets, kv_lens, np.float32(0.125), prefix)
        assert_close(got[:26], ref, size, 64)
        assert not got[1:4].any() and (got[26:] == 5.0).all()
    # More new tokens than keys (a refused part): the first rows see nothing.
    args = batch(3, 4, 2, 64, 16, [10], [14])
    out = _check(args)
    assert not out[:4].any() and out[4].any()


@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("d,new", [(64, 40), (128, 200), (128, 3), (64, 300)])
def test_values_that_a_row_does_not_see(value, d, new):
    """An infinite or NaN value (and NaN key) at the last positions of a prompt
    reaches the rows from there on and no earlier one."""
    n = new + 50
    args = list(batch(11, 4, 2, d, 16, [n, 30], [new, 1]))
    q, k, v, tables = args[:4]
    at = n - 2
    v[tables[0, at // 16], 1, at % 16, 3] = value
    k[tables[0, (n - 1) // 16], 0, (n - 1) % 16] = np.nan
    out = _check(tuple(args))
    assert np.isfinite(out[:new - 2]).all()
    assert not np.isfinite(out[new - 2, 2:, 3]).any() and np.isfinite(out[new - 2, :2]).all()
    assert np.isnan(out[new - 1, :2]).all() and np.isfinite(out[new]).all()


def test_scores_without_a_number():
    """Keys of the type's lowest value, infinite scores and all scores -infinity."""
    args = list(batch(12, 2, 1, 64, 16, [40, 40, 40, 40], [1, 1, 1, 1]))
    q, k, v, tables = args[:4]
    q[:] = np.abs(q) + np.float16(0.1)
    k[tables[0, 0], :, :16] = -65504                       # lowest value: weights 0
    k[tables[1, 0], :, 3] = -np.inf
    k[tables[2, :3]] = -np.inf                             # every score -inf: NaN, as softmax gives
    k[tables[3, 1], :, 2] = np.inf
    with np.errstate(invalid="ignore", over="ignore"):
        out = _check(tuple(args))
    assert np.isfinite(out[:2]).all() and np.isnan(out[2:]).all()


def test_pages_that_are_none():
    """A page id outside the pool makes the rows that see it NaN and touches no
    other request; ids past a request's keys are not looked at."""
    for bad in (-1, 10 ** 9, -(2 ** 31)):
        args = batch(13, 4, 2, 64, 16, [50, 60, 70], [1, 1, 1])
        q, k, v, tables, offsets, kv_lens, _ = args
        ref, size = PO.paged_attention(q, k, v, tables, offsets, kv_lens, np.float32(0.125))
        tables[1, 3] = bad
        tables[2, 5:] = bad
        out = _run(args, 0.125).cpu().numpy().reshape(3, 4, 64)
        assert np.isnan(out[1]).all()
        assert_close(out[[0, 2]], ref[[0, 2]], size[[0, 2]], 64)


def test_arrays_out_of_their_limits():
    """Offsets and lengths past the tokens and the tables are held to them."""
    args = batch(14, 4, 2, 64, 16, [50, 60], [2, 1])
    q, k, v, tables, offsets, kv_lens, _ = args
    _run((q, k, v, tables, np.array([0, 10 ** 6, -5], np.int32), np.array([10 ** 9, -3], np.int32), None), 0.1)
    _run((q, k, v, tables, np.array([2 ** 31 - 1, 0, 3], np.int32), np.array([2 ** 31 - 1, 64], np.int32),
          tables[0, :1].copy()), 0.1)
    _check(args)


def test_pools_past_32_bits():
    """Pages beyond 2^32 elements of the pools, both ends used by one request."""
    hq, hkv, d, page = 4, 8, 128, 256
    hq = 16
    n_pages = (1 << 32) // (hkv * page * d) + 3
    g = torch.Generator(device="cuda").manual_seed(1)
    kp, vp = (torch.empty((n_pages, hkv, page, d), dtype=torch.float16, device="cuda") for _ in range(2))
    ids = [n_pages - 1, 0, n_pages - 2]
    for pool in (kp, vp):
        for i in ids:
            pool[i] = torch.randn((hkv, page, d), generator=g, device="cuda").half()
    q = torch.randn((1, hq, d), generator=g, device="cuda").half()
    small = [x[torch.tensor(ids, device="cuda")].cpu().numpy() for x in (kp, vp)]
    ref, size = PO.paged_attention(q.cpu().numpy(), *small, [[0, 1, 2]], [0, 1], [700], np.float32(0.1))
    i32 = dict(dtype=torch.int32, device="cuda")
    for prefix in (None, torch.tensor(ids[:1], **i32)):
        out = B.qattn_paged_f16(q, kp, vp, torch.tensor([ids], **i32), torch.tensor([0, 1], **i32),
                                torch.tensor([700], **i32), 0.1, prefix=prefix)
        assert_close(out.cpu().numpy().reshape(1, hq, d), ref, size, d)


def test_deterministic_on_another_stream_and_in_replayed_graphs():
    """One captured call follows lengths and offsets that change between replays,
    its workspace filled with other bytes in between."""
    cases = [batch(s, 16, 8, 128, 16, kv, new, prefix_pages=4, pad=40 - sum(new)) for s, kv, new in (
        (21, [70, 900, 65, 100], [1, 1, 1, 1]), (22, [64, 65, 500, 0], [0, 1, 36, 2]), (23, [700, 80, 80, 80], [10, 10, 10, 10]))]
    n_pages = max(c[1].shape[0] for c in cases)
    width = max(c[3].shape[1] for c in cases)
    dev = [torch.zeros((40, 16, 128), dtype=torch.float16, device="cuda")]
    dev += [torch.zeros((n_pages, 8, 16, 128), dtype=torch.float16, device="cuda") for _ in range(2)]
    dev += [torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((4, width), (5,), (4,), (4,))]
    ws = torch.empty(B.qattn_paged_workspace_bytes(16, 8, 128, 4, 40, 4), dtype=torch.uint8, device="cuda")
    out = torch.zeros((40, 16 * 128), dtype=torch.float16, device="cuda")
    call = lambda: B.qattn_paged_f16(*dev[:6], 0.09, prefix=dev[6], out=out, workspace=ws)

    def load(c):
        for t, x in zip(dev, on_gpu(*c)):
            t[tuple(slice(n) for n in x.shape)] = x

    load(cases[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for c in cases * 2:
        load(c)
        ws.fill_(0xFF)
        out.zero_()
        call()
        eager = out.clone()
        out.zero_()
        ws.fill_(0x7F)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        n = int(c[4][-1])
        ref, size = PO.paged_attention(c[0][:n], c[1], c[2], c[3], c[4], c[5], np.float32(0.09), c[6])
        assert_close(out[:n].cpu().numpy().reshape(n, 16, 128), ref, size, 128)


def test_workspace_is_checked():
    args = on_gpu(*batch(30, 4, 2, 64, 16, [50], [1]))
    small = torch.empty(B.qattn_paged_workspace_bytes(4, 2, 64, 1, 1) - 1, dtype=torch.uint8, device="cuda")
    with pytest.raises(B.QmError) as e:
        B.qattn_paged_f16(*args[:6], 0.1, workspace=small)
    assert e.value.status == 6
