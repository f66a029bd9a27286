"""Operators of batched serving over a paged KV cache, with their plain forms:

  plan    page tables, slots, positions and lengths of one step of a batch,
          from the requests' lengths and a ring of free pages (qkv_plan)
  append  rotary embedding of the batch's queries and keys, keys and values
          into the cache pages at the slots (qkv_rope_append)
  attend  attention of the batch over its pages, with the pages of a prefix
          that all requests share read once for all of them (qattn_paged_f16)
  greedy  the index of the largest logit of every row (qdec_argmax_rows)

A cache is two pools fp16 [n_pages][kv heads][page][head dim].  Request i's
token at position p is in page tables[i][p // page], row p % page.  The
tokens of a batch lie one after the other, request i's at offsets[i] ..
offsets[i + 1] - 1, and are the last of its kv_lens[i] cached ones.

`own` chooses between the plain forms (elementary torch operations in fp32
and integers) and the library's calls.
"""

import math
import random

import torch

own = False

DEV = "cuda"
EPS = 1e-6
THETA = 5e5
# (query heads, KV heads, head dimension): the decoders of this repository,
# the attention tests' largest group, a model without grouping, a small one.
HEADS = [(16, 8, 128), (32, 8, 64), (24, 8, 128), (64, 8, 128), (8, 8, 64), (14, 2, 128)]


def listed():
    return [
        # The plan of the smallest step: one sequence generates one token.
        dict(name="plan_one", op="plan", n=1, page=16, max_pages=256, ctx_lo=700, ctx_hi=700, new_lo=1, new_hi=1,
             done=0, prefix=0, spare=64, pad=0, short=False),
        # An ordinary decode step: 200 sequences, some of them ended, two prefix pages shared.
        dict(name="plan_decode_200", op="plan", n=200, page=32, max_pages=512, ctx_lo=1, ctx_hi=9000, new_lo=1,
             new_hi=1, done=5, prefix=64, spare=3000, pad=56, short=False),
        # The largest step: 1,000 requests with 3 to 117 new tokens each, about 60,000 in all.
        dict(name="plan_prompts_1000", op="plan", n=1000, page=16, max_pages=1024, ctx_lo=1, ctx_hi=12000, new_lo=3,
             new_hi=117, done=3, prefix=0, spare=20000, pad=1000, short=False),
        # One token's queries, keys and values, with per-head norms (the Qwen3 layer).
        dict(name="append_one", op="append", hq=16, hkv=8, d=128, page=16, tokens=1, pad=0, max_len=4096, norm=True,
             interleaved=False),
        # A batch of prompts, 6,000 tokens in buffers for 6,144, rows of W_q and W_k interleaved.
        dict(name="append_prompts_6000", op="append", hq=24, hkv=8, d=128, page=64, tokens=6000, pad=144,
             max_len=16384, norm=False, interleaved=True),
        # Greedy sampling of a handful of sequences over a small vocabulary.
        dict(name="greedy_5", op="greedy", rows=5, vocab=32001),
        # Greedy sampling of a large batch over the largest vocabulary of this repository's models.
        dict(name="greedy_200", op="greedy", rows=200, vocab=151936),
        # One sequence's single token at an ordinary position: the smallest call, where latency counts.
        dict(name="attend_one_700", op="attend", hq=16, hkv=8, d=128, page=16, n=1, ctx_lo=700, ctx_hi=700, new_lo=1,
             new_hi=1, prefix=0),
        # A ragged decode batch: 48 sequences of 200 to 20,000 tokens, no shared prefix.
        dict(name="attend_ragged_48", op="attend", hq=16, hkv=8, d=128, page=64, n=48, ctx_lo=200, ctx_hi=20000,
             new_lo=1, new_hi=1, prefix=0),
        # A decode batch of 61 sequences after one system prompt of 4,096 tokens, heads of 64.
        dict(name="attend_prefix_61", op="attend", hq=32, hkv=8, d=64, page=16, n=61, ctx_lo=1, ctx_hi=900, new_lo=1,
             new_hi=1, prefix=4096),
        # Prompt chunks of odd lengths beside single tokens: 9 requests, 1 to 1,900 new tokens each.
        dict(name="attend_prompts_9", op="attend", hq=32, hkv=8, d=64, page=32, n=9, ctx_lo=1, ctx_hi=3000, new_lo=1,
             new_hi=1900, prefix=0),
        # The largest: 250 sequences that share a document of 16,384 tokens.
        dict(name="attend_prefix_250", op="attend", hq=24, hkv=8, d=128, page=64, n=250, ctx_lo=1, ctx_hi=2000,
             new_lo=1, new_hi=1, prefix=16384),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    most = max(_cost(c) for c in listed())
    op = rng.choice(["plan", "append", "greedy", "attend", "attend", "attend", "attend", "attend"])
    page = rng.choice([16, 32, 64, 128, 256])
    if op == "greedy":
        vocab = _log_int(rng, 1000, 160000)
        return dict(op=op, rows=_log_int(rng, 1, min(400, 31000000 // vocab)), vocab=vocab)
    if op == "append":
        hq, hkv, d = rng.choice(HEADS)
        norm = rng.random() < 0.4
        return dict(op=op, hq=hq, hkv=hkv, d=d, page=page, tokens=_log_int(rng, 1, 6000),
                    pad=rng.choice([0, 0, 1, 7, 100]), max_len=_log_int(rng, 512, 16384), norm=norm,
                    interleaved=not norm and rng.random() < 0.5)
    if op == "plan":
        new_hi = rng.choice([1, 1, _log_int(rng, 2, 4000)])
        n = _log_int(rng, 1, min(1000, 60000 // new_hi))
        ctx_hi = _log_int(rng, 1, 12000)
        prefix = page * rng.choice([0, 0, 1, 5])
        return dict(op=op, n=n, page=page, max_pages=(prefix + ctx_hi + new_hi) // page + 1 + rng.randrange(0, 20),
                    ctx_lo=rng.choice([0, 1]), ctx_hi=ctx_hi, new_lo=rng.choice([0, 1]), new_hi=new_hi,
                    done=rng.choice([0, 3, 10]), prefix=prefix, spare=rng.randrange(0, 3000),
                    pad=rng.choice([0, 5, 300]), short=rng.random() < 0.2)
    while True:
        hq, hkv, d = rng.choice(HEADS)
        n = _log_int(rng, 1, 250)
        new_hi = rng.choice([1, 1, 1, _log_int(rng, 2, 2000)])
        prefix = rng.choice([0, 0, page * _log_int(rng, 1, max(1, 16384 // page))])
        ctx_hi = _log_int(rng, 1, 60000)
        case = dict(op=op, hq=hq, hkv=hkv, d=d, page=page, n=n, ctx_lo=rng.choice([0, 1, max(1, ctx_hi // 50)]),
                    ctx_hi=ctx_hi, new_lo=1, new_hi=new_hi, prefix=prefix)
        ctx, new = _lengths(case)
        longest = max(c + t for c, t in zip(ctx, new))
        if _cost(case) <= most and n * longest * hkv * d <= 10 ** 9 and n * new_hi * hq * (longest + prefix) <= 10 ** 9:
            return case


# ---------------------------------------------------------------- the inputs


def _spread(lo, hi, n):
    """n lengths from lo to hi, by their logarithm where that spans much."""
    if n == 1:
        return [hi]
    if lo >= 1 and hi > 10 * lo:
        return [min(hi, int(round(lo * (hi / lo) ** (i / (n - 1))))) for i in range(n)]
    return [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _lengths(case):
    """Per request: cached tokens beyond the prefix, and new tokens (-1: it has ended)."""
    ctx, new = (_spread(case[a + "_lo"], case[a + "_hi"], case["n"]) for a in ("ctx", "new"))
    fixed = random.Random(5)
    fixed.shuffle(ctx)
    if case.get("done"):                                   # per cent of the requests, which have ended
        new = [-1 if fixed.randrange(100) < case["done"] else t for t in new]
    return ctx, new


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEV)


def _rope_table(max_len, d):
    """(cos, sin) of p * theta^(-2i/d) as fp32 [max_len][d/2][2]."""
    freq = THETA ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device=DEV) / d)
    a = torch.arange(max_len, dtype=torch.float64, device=DEV)[:, None] * freq
    return torch.stack([a.cos(), a.sin()], dim=-1).float()


def prepare(case, seed):
    rng = random.Random(seed)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(shape, dtype=torch.float16):
        return torch.randn(shape, generator=g, device=DEV, dtype=dtype)

    if case["op"] == "greedy":
        return dict(case=case, logits=normal((case["rows"], case["vocab"]), torch.float32) * 3)
    if case["op"] == "append":
        hq, hkv, d, page, t, pad = (case[x] for x in ("hq", "hkv", "d", "page", "tokens", "pad"))
        n_pages = -(-t // page) + 8
        slots = torch.randperm(n_pages * page, generator=g, device=DEV)[:t]
        pos = torch.randint(0, case["max_len"], (t,), generator=g, device=DEV, dtype=torch.int32)
        none = _ints([-1] * pad)
        gains = [(1 + 0.1 * normal(d, torch.float32)).half() for _ in range(2)] if case["norm"] else [None, None]
        return dict(case=case, q=normal((t + pad, hq * d), torch.float32), k=normal((t + pad, hkv * d), torch.float32),
                    v=normal((t + pad, hkv * d), torch.float32), positions=torch.cat([pos, none]),
                    slots=torch.cat([slots, none.long()]), table=_rope_table(case["max_len"], d),
                    k_pages=normal((n_pages, hkv, page, d)), v_pages=normal((n_pages, hkv, page, d)),
                    q_norm=gains[0], k_norm=gains[1], q_out=torch.zeros((t + pad, hq, d), dtype=torch.float16, device=DEV))

    n, page, prefix = case["n"], case["page"], case["prefix"]
    ctx, new = _lengths(case)
    order = list(range(n))
    rng.shuffle(order)
    ctx, new = [ctx[i] for i in order], [new[i] for i in order]
    pp = prefix // page
    if case["op"] == "plan":
        lens = [prefix + c for c in ctx]
        held = [-(-l // page) for l in lens]
        need = sum(-(-(l + t) // page) - h for l, t, h in zip(lens, new, held) if t > 0)
        count = need // 2 if case["short"] else need + case["spare"]
        owned = sum(h - pp for h in held)
        n_pages = pp + owned + count + 3
        ids = list(range(n_pages))
        rng.shuffle(ids)
        tables, at = [], pp
        for h in held:
            tables.append(ids[:pp] + ids[at:at + h - pp] + [-1] * (case["max_pages"] - h))
            at += h - pp
        head = rng.randrange(n_pages)
        ring = [-1] * n_pages
        for j in range(count):
            ring[(head + j) % n_pages] = ids[at + j]
        return dict(case=case, lens=_ints(lens), new_lens=_ints(new), tables=_ints(tables), free_ring=_ints(ring),
                    ring=_ints([head, count]), max_tokens=max(1, sum(max(t, 0) for t in new) + case["pad"]))
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    held = [-(-(prefix + c + t) // page) for c, t in zip(ctx, new)]
    n_pages = pp + sum(h - pp for h in held) + 3
    ids = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    wide = max(held) + 1
    idl = ids.tolist()
    tables, at = [], pp
    for h in held:
        tables.append(idl[:pp] + idl[at:at + h - pp] + [-1] * (wide - h))
        at += h - pp
    offsets = [0]
    for t in new:
        offsets.append(offsets[-1] + t)
    kp, vp = normal((n_pages, hkv, page, d)), normal((n_pages, hkv, page, d))
    return dict(case=case, q=normal((offsets[-1], hq, d)), k_pages=kp, v_pages=vp, tables=_ints(tables),
                prefix=ids[:pp].clone() if pp else None, offsets=_ints(offsets),
                kv_lens=_ints([prefix + c + t for c, t in zip(ctx, new)]), scale=1 / math.sqrt(d),
                tokens=offsets[-1], most_new=max(new), most_own=max(c + t for c, t in zip(ctx, new)))


# ------------------------------------------------------------------ one pass


def run(state):
    return (_library if own else _plain)[state["case"]["op"]](state)


def _plain_plan(s):
    case, page = s["case"], s["case"]["page"]
    n, width = s["tables"].shape
    n_pages, pp, cap = s["free_ring"].numel(), case["prefix"] // page, s["max_tokens"]
    lens, new, ring = s["lens"].long(), s["new_lens"].long(), s["free_ring"]
    head, count = s["ring"][0].long(), s["ring"][1].long()
    sane = (lens >= 0) & (lens <= width * page)
    active, add = new >= 0, new.clamp(min=0)
    end = add.cumsum(0)
    fits = active & sane & (lens + add <= width * page) & (end <= cap)
    have = (lens + page - 1) // page
    need = torch.where(fits, (lens + add + page - 1) // page - have, 0)
    upto = need.cumsum(0)
    granted = fits & ((need == 0) | (upto <= count))
    given, first = torch.where(granted, need, 0), upto - need
    total = lens + add
    col = torch.arange(width, device=DEV)[None]
    fresh = ring[(head + first[:, None] + col - have[:, None]) % n_pages]
    mine = (col >= have[:, None]) & (col < (have + given)[:, None])
    back = torch.where(~active & sane, (have - pp).clamp(min=0), 0)
    taken, room = given.sum(), n_pages - count
    upto_back = back.cumsum(0).clamp(max=room)
    rank = (back.cumsum(0) - back)[:, None] + col - pp
    freed = (col >= pp) & (col < (pp + back)[:, None]) & (rank < room)
    to = torch.where(freed, (head + count + rank) % n_pages, n_pages)
    ring_ext = torch.cat([ring, ring[:1]])
    ring_ext[to] = s["tables"]
    ring.copy_(ring_ext[:n_pages])
    s["tables"].copy_(torch.where(mine, fresh, s["tables"]))
    offsets = torch.cat([end.new_zeros(1), end]).clamp(max=cap)
    t = torch.arange(cap, device=DEV)
    i = (torch.searchsorted(offsets, t, right=True) - 1).clamp(max=n - 1)
    there = (t < offsets[-1]) & granted[i]
    pos = lens[i] + t - offsets[i]
    slot = s["tables"][i, (pos // page).clamp(0, width - 1)].long() * page + pos % page
    return dict(tables=s["tables"], free_ring=ring,
                lens=torch.where(active, torch.where(granted, total, lens), torch.where(sane, 0, lens)).int(),
                kv_lens=torch.where(granted, total, 0).int(), offsets=offsets.int(),
                positions=torch.where(there, pos, -1).int(), slots=torch.where(there, slot, -1),
                ring=torch.stack([(head + taken) % n_pages, count - taken + upto_back[-1]]).int(),
                refused=(active & ~granted).sum().int()[None])


def _plain_append(s):
    case = s["case"]
    hq, hkv, d, page, t = (case[x] for x in ("hq", "hkv", "d", "page", "tokens"))
    cs = s["table"][s["positions"][:t].long()][:, None]
    cos, sin = cs[..., 0], cs[..., 1]

    def rotated(x, heads, gain):
        x = x[:t].view(t, heads, d)
        if case["interleaved"]:
            x = torch.cat([x[..., 0::2], x[..., 1::2]], dim=-1)
        if gain is not None:
            x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * gain.float()
        a, b = x[..., :d // 2], x[..., d // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1).half()

    at, row = s["slots"][:t] // page, s["slots"][:t] % page
    s["q_out"][:t] = rotated(s["q"], hq, s["q_norm"])
    s["k_pages"][at, :, row] = rotated(s["k"], hkv, s["k_norm"])
    s["v_pages"][at, :, row] = s["v"][:t].view(t, hkv, d).half()
    return dict(q=s["q_out"], k_pages=s["k_pages"], v_pages=s["v_pages"])


def _plain_greedy(s):
    x = s["logits"]
    number = ~x.isnan()
    top = torch.where(number, x, -math.inf).amax(1, keepdim=True)
    at = torch.where(number & (x == top), torch.arange(x.shape[1], device=DEV), x.shape[1]).amin(1)
    return torch.where(at < x.shape[1], at, 0).int()


def _plain_attend(s):
    case = s["case"]
    hq, hkv, d, page, n, prefix = (case[x] for x in ("hq", "hkv", "d", "page", "n", "prefix"))
    t, group = s["most_new"], hq // hkv
    start, new = s["offsets"][:-1].long(), s["offsets"].diff().long()
    # Queries padded to the most new tokens: [n][kv head][token, query head of the group][d].
    j = torch.arange(t, device=DEV)
    q = s["q"][(start[:, None] + j).clamp(max=s["tokens"] - 1)].float().view(n, t, hkv, group, d)
    q = q.permute(0, 2, 1, 3, 4).reshape(n, hkv, t * group, d)
    seen = (s["kv_lens"].long() - new)[:, None] + j + 1                       # keys that a token attends to
    # The requests' own keys and values, padded to the most: [n][kv head][key][d].
    pos = prefix + torch.arange(s["most_own"], device=DEV)
    at = s["tables"][:, (pos // page).clamp(max=s["tables"].shape[1] - 1)].long().clamp(min=0)
    k, v = (x[at, :, pos % page].float().permute(0, 2, 1, 3).contiguous() for x in (s["k_pages"], s["v_pages"]))
    score = torch.matmul(q, k.transpose(-1, -2).contiguous()) * s["scale"]
    score = score.view(n, hkv, t, group, -1).masked_fill(~(pos < seen[..., None])[:, None, :, None], -math.inf)
    if prefix:
        kp, vp = (x[s["prefix"].long()].float().transpose(0, 1).reshape(hkv, prefix, d)
                  for x in (s["k_pages"], s["v_pages"]))
        flat = q.transpose(0, 1).reshape(hkv, n * t * group, d)
        shared = torch.matmul(flat, kp.transpose(-1, -2).contiguous()) * s["scale"]
        shared = shared.view(hkv, n, t, group, prefix).transpose(0, 1)
        score = torch.cat([score, shared.masked_fill(~(torch.arange(prefix, device=DEV) < seen[..., None])
                                                     [:, None, :, None], -math.inf)], dim=-1)
    p = (score - score.amax(-1, keepdim=True)).exp()
    p = p / p.sum(-1, keepdim=True)
    o = torch.matmul(p[..., :pos.numel()].reshape(n, hkv, t * group, -1), v)
    if prefix:
        o = o + torch.matmul(p[..., pos.numel():].transpose(0, 1).reshape(hkv, n * t * group, prefix), vp
                             ).view(hkv, n, t * group, d).transpose(0, 1)
    o = o.view(n, hkv, t, group, d).permute(0, 2, 1, 3, 4).reshape(n, t, hq * d)
    request = torch.repeat_interleave(torch.arange(n, device=DEV), new, output_size=s["tokens"])
    return o[request, torch.arange(s["tokens"], device=DEV) - start[request]].half()


def _own_plan(s):
    from paper_2607_00501_amd import binding as B
    p = s["out"] = B.qkv_plan(s["lens"], s["new_lens"], s["tables"], s["free_ring"], s["ring"], s["case"]["page"],
                              s["max_tokens"], prefix_pages=s["case"]["prefix"] // s["case"]["page"],
                              out=s.get("out"))
    return dict(tables=s["tables"], free_ring=s["free_ring"], lens=p.lens, kv_lens=p.kv_lens, offsets=p.offsets,
                positions=p.positions, slots=p.slots, ring=p.ring, refused=p.refused)


def _own_append(s):
    from paper_2607_00501_amd import binding as B
    q = B.qkv_rope_append(s["q"], s["k"], s["v"], s["positions"], s["slots"], s["table"], s["k_pages"], s["v_pages"],
                          interleaved=s["case"]["interleaved"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS,
                          q_out=s["q_out"])
    return dict(q=q, k_pages=s["k_pages"], v_pages=s["v_pages"])


def _own_greedy(s):
    from paper_2607_00501_amd import binding as B
    if "workspace" not in s:
        s["workspace"] = torch.empty(B.qdec_argmax_rows_workspace_bytes(s["case"]["rows"]), dtype=torch.uint8, device=DEV)
    s["out"] = B.qdec_argmax_rows(s["logits"], out=s.get("out"), workspace=s["workspace"])
    return s["out"]


def _own_attend(s):
    from paper_2607_00501_amd import binding as B
    if "workspace" not in s:
        nb = B.qattn_paged_workspace_bytes(s["case"]["hq"], s["case"]["hkv"], s["case"]["d"], s["case"]["n"],
                                           s["tokens"], s["case"]["prefix"] // s["case"]["page"])
        s["workspace"] = torch.empty(max(nb, 16), dtype=torch.uint8, device=DEV)
    s["out"] = B.qattn_paged_f16(s["q"], s["k_pages"], s["v_pages"], s["tables"], s["offsets"], s["kv_lens"],
                                 s["scale"], prefix=s["prefix"], out=s.get("out"), workspace=s["workspace"])
    return s["out"]


_plain = dict(plan=_plain_plan, append=_plain_append, greedy=_plain_greedy, attend=_plain_attend)
_library = dict(plan=_own_plan, append=_own_append, greedy=_own_greedy, attend=_own_attend)


# ------------------------------------------------- what a pass cannot do without


def work(case):
    if case["op"] == "greedy":
        return dict(bytes=4 * case["rows"] * (case["vocab"] + 1), flops=case["rows"] * case["vocab"])
    if case["op"] == "append":
        hq, hkv, d, t = (case[x] for x in ("hq", "hkv", "d", "tokens"))
        return dict(bytes=t * ((hq + 2 * hkv) * d * (4 + 2) + 4 * d + 12), flops=t * (hq + hkv) * d * 3)
    ctx, new = _lengths(case)
    if case["op"] == "plan":
        # Lengths in and out, offsets; a position and a slot per token, and the page table entry it is read
        # from or written to once per page; the pages that go to and from the ring.
        pages = sum((case["prefix"] + c + t) // case["page"] - (case["prefix"] + c) // case["page"] + 1
                    for c, t in zip(ctx, new) if t > 0)
        tokens = sum(max(t, 0) for t in new)
        return dict(bytes=20 * case["n"] + 12 * (tokens + case["pad"]) + 8 * pages, flops=10 * tokens)
    hq, hkv, d, prefix = (case[x] for x in ("hq", "hkv", "d", "prefix"))
    rows = prefix + sum(c + t for c, t in zip(ctx, new))
    pairs = sum(t * (prefix + c) + t * (t + 1) // 2 for c, t in zip(ctx, new))
    return dict(bytes=4 * rows * hkv * d + 4 * sum(new) * hq * d + 4 * (rows // case["page"] + 2 * case["n"]),
                flops=4 * pairs * hq * d)


# ------------------------------------------------------- the definition, in 64 bits


def exact(case, seed):
    if case["op"] in ("plan", "greedy"):
        return None                                        # whole numbers
    s = prepare(case, seed)
    if case["op"] == "append":
        hq, hkv, d, page, t = (case[x] for x in ("hq", "hkv", "d", "page", "tokens"))
        i = torch.arange(d // 2, device=DEV)
        low, high = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + d // 2)
        turn = torch.view_as_complex(s["table"].double())[s["positions"][:t].long()].unsqueeze(1)

        def turned(x, heads, gain):
            x = x[:t].double().view(t, heads, d)
            z = torch.complex(x[..., low], x[..., high])
            if gain is not None:
                z = z / (z.abs().square().sum(-1, keepdim=True) / d + EPS).sqrt()
                z = torch.complex(z.real * gain[:d // 2].double(), z.imag * gain[d // 2:].double())
            z = z * turn
            return torch.cat([z.real, z.imag], dim=-1)

        q, k, v = s["q_out"].double(), s["k_pages"].double(), s["v_pages"].double()
        q[:t] = turned(s["q"], hq, s["q_norm"])
        kt, slots = turned(s["k"], hkv, s["k_norm"]), s["slots"][:t]
        for pool, rows in ((k, kt), (v, s["v"][:t].double().view(t, hkv, d))):
            flat = pool.transpose(1, 2).reshape(-1, hkv, d)  # rows in the order of the slots
            flat[slots] = rows
            pool.copy_(flat.view(-1, page, hkv, d).transpose(1, 2))
        return dict(q=q, k_pages=k, v_pages=v)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    pairs = work(case)["flops"] // (4 * hq * d)
    if pairs * hq > 3e9:
        return None
    out = torch.empty((s["tokens"], hq * d), dtype=torch.float64, device=DEV)
    offsets, lens = s["offsets"].tolist(), s["kv_lens"].tolist()
    for i in range(case["n"]):
        pages = s["tables"][i, :-(-lens[i] // case["page"])].long()
        k, v = (x[pages].double().transpose(0, 1).reshape(hkv, -1, d)[:, :lens[i]] for x in (s["k_pages"], s["v_pages"]))
        for h in range(hq):
            kh, vh = k[h // (hq // hkv)], v[h // (hq // hkv)]
            for a in range(offsets[i], offsets[i + 1], 512):
                b = min(a + 512, offsets[i + 1])
                last = torch.arange(a, b, device=DEV)[:, None] - offsets[i + 1] + lens[i]
                z = (s["q"][a:b, h].double() @ kh.T * s["scale"]).masked_fill(
                    torch.arange(lens[i], device=DEV) > last, -math.inf)
                out[a:b, h * d:(h + 1) * d] = torch.softmax(z, dim=1) @ vh
    return out
