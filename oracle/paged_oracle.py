"""CPU oracle of batched serving over a paged KV cache (TEST INFRASTRUCTURE):
the definitions restated with Python integers and numpy in fp64, request by
request, without tiles, splits or sharing."""

import numpy as np


def plan_step(lens, new_lens, tables, free_ring, ring, page, max_tokens, prefix_pages=0):
    """One step's page tables, slots, positions and lengths.  lens, new_lens,
    free_ring, ring: lists; tables: list of lists.  Returns a dict of lists;
    the arguments are not changed."""
    tables, free_ring = [list(t) for t in tables], list(free_ring)
    n_pages, width = len(free_ring), len(tables[0])
    head, count = ring
    if not (0 <= head < n_pages and 0 <= count <= n_pages):
        head = count = 0
    out = dict(lens=[], kv_lens=[], offsets=[0], positions=[-1] * max_tokens, slots=[-1] * max_tokens)
    wanted = taken = refused = start = 0
    back = []
    old = [list(t) for t in tables]
    for i, (length, new) in enumerate(zip(lens, new_lens)):
        sane = 0 <= length <= width * page
        length = max(length, prefix_pages * page) if sane else length
        have = -(-length // page) if sane else 0
        if new < 0:
            if sane:
                back += old[i][prefix_pages:max(prefix_pages, have)]
            out["lens"].append(0 if sane else length)
            out["kv_lens"].append(0)
            out["offsets"].append(min(start, max_tokens))
            continue
        fits = sane and length + new <= width * page and start + new <= max_tokens
        need = -(-(length + new) // page) - have if fits else 0
        wanted += need
        if fits and (need == 0 or wanted <= count):
            for j in range(need):
                tables[i][have + j] = free_ring[(head + wanted - need + j) % n_pages]
            taken += need
            for j in range(new):
                p = length + j
                out["positions"][start + j] = p
                out["slots"][start + j] = tables[i][p // page] * page + p % page
            out["lens"].append(length + new)
            out["kv_lens"].append(length + new)
        else:
            refused += 1
            out["lens"].append(length)
            out["kv_lens"].append(0)
        start += new
        out["offsets"].append(min(start, max_tokens))
    back = back[:n_pages - count]
    for j, page_id in enumerate(back):
        free_ring[(head + count + j) % n_pages] = page_id
    out.update(tables=tables, free_ring=free_ring, ring=[(head + taken) % n_pages, count - taken + len(back)],
               refused=[refused])
    return out


def paged_attention(q, k_pages, v_pages, tables, offsets, kv_lens, scale, prefix=None):
    """(out, weight): out fp64 [tokens][Hq][D]; weight[t][h][d] = sum_p w_p |v_p|,
    the size that rounding errors of the weights scale with.  q [tokens][Hq][D];
    pools [n_pages][Hkv][page][D]; prefix: page ids that replace the first
    entries of every table."""
    tokens, hq, d = q.shape
    _, hkv, page, _ = k_pages.shape
    out = np.zeros((tokens, hq, d))
    size = np.zeros((tokens, hq, d))
    for i in range(len(kv_lens)):
        new = offsets[i + 1] - offsets[i]
        for j in range(new):
            t = offsets[i] + j
            n = kv_lens[i] - new + j + 1
            if n <= 0:
                continue
            ids = list(tables[i][:-(-n // page)])
            if prefix is not None:
                ids[:len(prefix)] = list(prefix)[:len(ids)]
            k = np.concatenate([k_pages[p] for p in ids], axis=1)[:, :n].astype(np.float64)
            v = np.concatenate([v_pages[p] for p in ids], axis=1)[:, :n].astype(np.float64)
            for h in range(hq):
                g = h // (hq // hkv)
                s = (k[g] @ q[t, h].astype(np.float64)) * float(scale)
                w = np.exp(s - s.max())
                w /= w.sum()
                with np.errstate(invalid="ignore"):
                    out[t, h] = w @ v[g]
                    size[t, h] = w @ np.abs(v[g])
    return out, size
