"""Batches over a paged cache for the tests: random pages, poisoned places that
no request sees, and the bound that an fp16 attention output has to keep."""

import numpy as np
import torch


def batch(seed, hq, hkv, d, page, kv_lens, new, prefix_pages=0, poison=np.nan, pad=0, spare=2, same_prefix=True):
    """(q, k_pages, v_pages, tables, offsets, kv_lens, prefix) as numpy arrays.
    Every place of the pools that is not a request's key is `poison`.  kv_lens 0:
    a request without keys (its new tokens are rows that see nothing)."""
    rng = np.random.default_rng(seed)
    n = len(kv_lens)
    held = [-(-x // page) for x in kv_lens]
    width = max(held + [prefix_pages, 1]) + 1
    own = [max(h - prefix_pages, 0) for h in held]
    n_pages = prefix_pages + sum(own) + spare
    ids = rng.permutation(n_pages)
    shared = ids[:prefix_pages]
    tables = np.full((n, width), -7, np.int32)
    at = prefix_pages
    k = rng.standard_normal((n_pages, hkv, page, d)).astype(np.float16)
    v = rng.standard_normal((n_pages, hkv, page, d)).astype(np.float16)
    seen = np.zeros((n_pages, page), bool)
    for i in range(n):
        table = list(shared[:held[i]]) + list(ids[at:at + own[i]])
        at += own[i]
        tables[i, :held[i]] = table
        for p in range(held[i]):
            seen[table[p], :min(page, kv_lens[i] - p * page)] = True
    hidden = np.broadcast_to(~seen[:, None, :, None], k.shape)
    k[hidden] = poison
    v[hidden] = poison
    offsets = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    q = rng.standard_normal((int(offsets[-1]) + pad, hq, d)).astype(np.float16)
    return (q, k, v, tables, offsets, np.asarray(kv_lens, np.int32),
            shared.astype(np.int32) if prefix_pages and same_prefix else None)


def on_gpu(*arrays):
    return [None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in arrays]


def assert_close(out, ref, size, d):
    """fp16 result against fp64.  Half a step of fp16 (2^-11 relative, 2^-25 below
    the normal range) for the output; half a step for each weight, 2^-11 of
    size = sum w |v|; the scores' sums of d products in fp32 and the exponentials,
    at most d x 2^-24 of sum |q k| scale, which for unit normal q, k and scale
    1/sqrt(d) is below sqrt(d) x 0.8 = 9.1 (d = 128): another 2^-13.4 of size, taken as 2^-12."""
    out, ref, size = (np.asarray(x, np.float64) for x in (out, ref, size))
    assert np.array_equal(np.isnan(out), np.isnan(ref))
    ok = np.isfinite(ref)
    assert np.array_equal(out[~ok & ~np.isnan(ref)], ref[~ok & ~np.isnan(ref)])
    err = np.abs(out - np.where(ok, ref, 0))[ok]
    bound = (2.0 ** -11 * np.abs(ref) + (2.0 ** -11 + 2.0 ** -12) * size + 2.0 ** -25)[ok]
    worst = (err / bound).max() if err.size else 0.0
    assert worst <= 1.0, worst
