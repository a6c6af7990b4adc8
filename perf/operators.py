"""The paged key-value cache's operators: what they compute, on what they are measured.

Three operators of a language model that answers token by token (the multimodal
model that conditions an editing pipeline is one), over a cache of pages:

  append  the new tokens' keys and values go to their places in the pages, and
          their accumulated attention weights start at zero
  attend  attention of one new token per sequence over its cached tokens, with
          grouped heads, the logsumexp, and the weight that each cached token
          got from this softmax added to its accumulated weight
  evict   of each head's cached tokens the first few, the last few and those of
          the largest accumulated weights are kept, in order, in fresh pages

A cache is a pool of pages [pages, page tokens, KV heads, d] (any strides, d
contiguous), a table of page numbers per sequence, and lengths.  ``own`` False:
the plain forms; True: the calls a program makes of the library.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(name, op, dtype, B, H, Hkv, d, page, max_len, layout, spread, **more):
    return dict(name=name, op=op, dtype=dtype, B=B, H=H, Hkv=Hkv, d=d, page=page, max_len=max_len,
                layout=layout, spread=spread, **more)


def listed():
    return [
        # one conversation a few hundred tokens in: launches and latency
        _case("attend_one", "attend", "bf16", 1, 24, 8, 128, 16, 517, "tokens", 0.0, score=True),
        # a served batch of uneven conversations, an idle slot among them
        _case("attend_batch", "attend", "bf16", 48, 32, 8, 128, 16, 4096, "heads", 0.9, score=True),
        # the same without any use for the weights (no eviction planned)
        _case("attend_plain", "attend", "bf16", 48, 32, 8, 128, 16, 4096, "heads", 0.9, score=False),
        # one long document, all of the device for one token
        _case("attend_long", "attend", "bf16", 1, 32, 4, 128, 64, 131072, "tokens", 0.0, score=True),
        # every head has keys and values of its own, short rows
        _case("attend_heads", "attend", "bf16", 40, 24, 24, 64, 32, 1500, "joint", 0.7, score=True),
        # full precision, for validation runs
        _case("attend_f32", "attend", "f32", 6, 16, 4, 96, 16, 1023, "tokens", 0.5, score=True),
        # one step of a served batch: a token for each sequence
        _case("append_step", "append", "bf16", 64, 32, 8, 128, 16, 384, "tokens", 0.8, new=1),
        # a batch of prompts, all of their tokens at once
        _case("append_prompts", "append", "bf16", 12, 32, 8, 128, 16, 4100, "heads", 0.8, new=4000),
        # one conversation's cache is halved
        _case("evict_one", "evict", "bf16", 1, 24, 8, 128, 16, 1024, "tokens", 0.0, keep=512, sinks=4,
              recent=64),
        # a served batch, uneven: the short ones keep all they have
        _case("evict_batch", "evict", "bf16", 24, 32, 8, 128, 16, 4096, "heads", 0.9, keep=1024, sinks=4,
              recent=128),
        # a long document is cut to an eighth
        _case("evict_long", "evict", "bf16", 1, 32, 8, 128, 64, 131072, "tokens", 0.0, keep=16384,
              sinks=16, recent=1024),
        # full precision, odd sizes
        _case("evict_f32", "evict", "f32", 5, 8, 2, 80, 24, 777, "joint", 0.5, keep=301, sinks=1,
              recent=33),
    ]


# -------------------------------------------------------------------- draw --
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST_BYTES = 400e6   # of keys and values moved: below the largest listed case's


def draw(rng):
    op = rng.choice(["attend", "attend", "append", "evict"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    d = rng.choice([64, 80, 96, 128, 128, 256])
    Hkv = rng.choice([1, 2, 3, 4, 8, 8, 16, 24])
    H = Hkv * rng.choice([1, 2, 3, 4, 4, 6, 8, 12, 16, 24] if Hkv <= 8 else [1, 2, 4])
    page = rng.choice([8, 16, 16, 24, 32, 64, 128])
    B = _log(rng, 1, 96)
    width = Hkv * d * 2 * (2 if dtype == "bf16" else 4) * (1 if op == "attend" else 2)
    most = max(16, min(8192 if op == "append" else 131072, int(MOST_BYTES / (width * B))))
    max_len = _log(rng, 1, most)
    c = dict(op=op, dtype=dtype, B=B, H=H, Hkv=Hkv, d=d, page=page, max_len=max_len,
             layout=rng.choice(["tokens", "heads", "joint"]),
             spread=rng.choice([0.0, 0.5, 0.9]))
    if op == "attend":
        c["score"] = rng.random() < 0.7
    elif op == "append":
        c["new"] = rng.choice([1, _log(rng, 1, max_len)])
    else:
        c["keep"] = _log(rng, 1, max_len)
        c["sinks"] = rng.randint(0, min(16, c["keep"] // 4))
        c["recent"] = rng.randint(0, c["keep"] // 4)
    return c


# ----------------------------------------------------------------- prepare --
def _lens(c):
    """The sequences' lengths: the first is the longest, the others spread down
    to (1 - spread) of it; in a batch of 16 and more one slot is idle."""
    B, n = c["B"], c["max_len"]
    out = [max(1, int(n * (1.0 - c["spread"] * ((i * 0.6180339887498949) % 1.0)))) for i in range(B)]
    out[0] = n
    if B >= 16:
        out[B // 2] = 0
    return out


def _new(c):
    """New tokens per sequence (an append): the last of each length."""
    return [min(n, max(1, int(c["new"] * n / c["max_len"]))) if n else 0 for n in _lens(c)]


def _pool(c, pages, dt):
    """Keys' and values' pages, seen as [pages, page, Hkv, d]."""
    P, H, d = c["page"], c["Hkv"], c["d"]
    if c["layout"] == "tokens":
        return (torch.zeros(pages, P, H, d, dtype=dt, device=DEV),
                torch.zeros(pages, P, H, d, dtype=dt, device=DEV))
    if c["layout"] == "heads":
        return (torch.zeros(pages, H, P, d, dtype=dt, device=DEV).transpose(1, 2),
                torch.zeros(pages, H, P, d, dtype=dt, device=DEV).transpose(1, 2))
    both = torch.zeros(pages, 2, P, H, d, dtype=dt, device=DEV)
    return both[:, 0], both[:, 1]


def _table(lens, page, wide, gen):
    """Page numbers in no order (-1: none) and how many pages there are."""
    used = -(-torch.tensor(lens, device=DEV) // page)
    total = max(1, int(used.sum()))
    order = torch.randperm(total, generator=gen, device=DEV).to(torch.int32)
    j = torch.arange(wide, device=DEV)
    at = order[((used.cumsum(0) - used)[:, None] + j).clamp_max(total - 1)]
    return at.masked_fill_(j >= used[:, None], -1), total


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    dt = TYPES[c["dtype"]]
    B, H, Hkv, d, page, n = c["B"], c["H"], c["Hkv"], c["d"], c["page"], c["max_len"]
    wide = -(-n // page)
    lens = _lens(c)
    table, pages = _table(lens, page, wide, gen)
    k, v = _pool(c, pages, dt)
    for t in (k, v):
        t.copy_(torch.randn(pages, page, Hkv, d, dtype=dt, device=DEV, generator=gen))
    s = dict(c=c, k=k, v=v, table=table, lens=torch.tensor(lens, dtype=torch.int32, device=DEV))
    # accumulated weights as decoding leaves them: a few heavy tokens, a long
    # tail, and many that got the same rounded weight or none
    u = torch.rand(B, Hkv, n, device=DEV, generator=gen)
    acc = torch.exp(-9.0 * u) * 8.0
    s["acc"] = torch.where(u > 0.75, (acc * 4096.0).round() / 4096.0, acc)
    if c["op"] == "attend":
        q = torch.randn(B, H, d, device=DEV, generator=gen)
        # the first token of a sequence draws attention, as in trained models
        heads = q.view(B, Hkv, H // Hkv, d).mean(2)
        first = table[:, 0].long()
        live = first >= 0
        pull = heads / heads.norm(dim=-1, keepdim=True).clamp_min(1e-6) * math.sqrt(d) * 0.5
        k[first[live], 0] += pull[live].to(dt)
        s.update(q=(2.0 * q).to(dt), o=torch.empty(B, H, d, dtype=dt, device=DEV),
                 lse=torch.empty(B, H, device=DEV), scale=1.0 / math.sqrt(d))
    elif c["op"] == "append":
        new = _new(c)
        cu = [0]
        for x in new:
            cu.append(cu[-1] + x)
        s.update(cu=torch.tensor(cu, dtype=torch.int32, device=DEV),
                 k_new=torch.randn(cu[-1], Hkv, d, dtype=dt, device=DEV, generator=gen),
                 v_new=torch.randn(cu[-1], Hkv, d, dtype=dt, device=DEV, generator=gen))
    else:
        keep = c["keep"]
        kept = [min(x, keep) for x in lens]
        to, pages_to = _table(kept, page, -(-keep // page), gen)
        k2, v2 = _pool(c, pages_to, dt)
        s.update(to=to, k2=k2, v2=v2, lens2=torch.zeros(B, dtype=torch.int32, device=DEV),
                 acc2=torch.zeros(B, Hkv, keep, device=DEV),
                 idx=torch.empty(B, Hkv, keep, dtype=torch.int32, device=DEV))
    s["plan"] = {}   # the library's descriptors of these buffers, made at the first pass
    return s


# --------------------------------------------------------------------- run --
def run(state):
    return _RUN[state["c"]["op"]](state)


def _cache(s, which="src"):
    """The library's descriptor of the cache: made once and kept, as a program
    keeps it beside the buffers."""
    got = s["plan"].get(which)
    if got is None:
        import paper_2608_17995_gb300 as av
        if which == "src":
            got = av.KVCache(s["k"], s["v"], s["table"], s["lens"], acc=s["acc"],
                             max_len=s["c"]["max_len"])
        else:
            got = av.KVCache(s["k2"], s["v2"], s["to"], s["lens2"], acc=s["acc2"],
                             max_len=s["c"]["keep"])
        s["plan"][which] = got
    return got


def _rows(pool, table, n):
    """[B, n, Hkv, d] of the pages' tokens, in order, in 32 bits."""
    got = pool[table.clamp_min(0).long()]
    return got.reshape(table.shape[0], -1, pool.shape[2], pool.shape[3])[:, :n].float()


def _attend(s):
    c = s["c"]
    score = c["score"]
    if own:
        import paper_2608_17995_gb300 as av
        av.avits_cache_attention(_cache(s), s["q"], s["scale"], s["o"], lse=s["lse"],
                                 weight=1.0 if score else None)
    else:
        B, H, Hkv, d, n = c["B"], c["H"], c["Hkv"], c["d"], c["max_len"]
        live = torch.arange(n, device=DEV)[None, :] < s["lens"][:, None]          # [B, n]
        k = _rows(s["k"], s["table"], n).masked_fill_(~live[:, :, None, None], 0.0)
        q = s["q"].float().view(B, Hkv, H // Hkv, d) * s["scale"]
        x = torch.matmul(q, k.permute(0, 2, 3, 1))                                 # [B, Hkv, G, n]
        del k
        x = x.masked_fill_(~live[:, None, None, :], -math.inf)
        top = x.amax(-1, keepdim=True).clamp_min(-3.0e38)
        p = torch.exp(x - top)
        total = p.sum(-1, keepdim=True)
        p = p / torch.where(total > 0, total, torch.ones_like(total))
        v = _rows(s["v"], s["table"], n).masked_fill_(~live[:, :, None, None], 0.0)
        o = torch.matmul(p, v.permute(0, 2, 1, 3))
        s["o"].copy_(o.reshape(B, H, d))
        s["lse"].copy_((torch.log(total) + top).reshape(B, H))
        if score:
            s["acc"] += p.mean(2)
    return {"o": s["o"], "lse": s["lse"], "acc": s["acc"]} if score else {"o": s["o"], "lse": s["lse"]}


def _append(s):
    if own:
        import paper_2608_17995_gb300 as av
        av.avits_cache_append(_cache(s), s["k_new"], s["v_new"], s["cu"])
    else:
        page, T = s["c"]["page"], s["k_new"].shape[0]
        t = torch.arange(T, device=DEV)
        cu = s["cu"].long()
        b = torch.searchsorted(cu[1:], t, right=True)
        at = s["lens"].long()[b] - (cu[b + 1] - t)                                 # place in its sequence
        p = s["table"].long()[b, at // page]
        s["k"][p, at % page] = s["k_new"]
        s["v"][p, at % page] = s["v_new"]
        s["acc"][b, :, at] = 0.0
    return {"k": s["k"], "v": s["v"], "acc": s["acc"]}


def _evict(s):
    c = s["c"]
    keep, sinks, recent = c["keep"], c["sinks"], c["recent"]
    if own:
        import paper_2608_17995_gb300 as av
        av.avits_cache_evict(_cache(s), _cache(s, "dst"), keep, sinks, recent, keep_idx=s["idx"])
    else:
        n, page = c["max_len"], c["page"]
        j = torch.arange(n, device=DEV)
        lens = s["lens"].long()[:, None, None]                                     # [B, 1, 1]
        x = torch.where((j < sinks) | (j >= lens - recent), math.inf, s["acc"])
        x = torch.where(j < lens, x, -math.inf)
        # largest first, equal ones by their index
        first = torch.sort(x, dim=-1, descending=True, stable=True).indices[..., :keep]
        first = torch.where(torch.arange(keep, device=DEV) < lens, first, n)       # n: none
        first = torch.sort(first, dim=-1).values
        some = first < n
        got = first.clamp_max(n - 1)                                               # [B, Hkv, keep]
        b = torch.arange(c["B"], device=DEV)[:, None, None].expand_as(got)
        h = torch.arange(c["Hkv"], device=DEV)[None, :, None].expand_as(got)
        r = torch.arange(keep, device=DEV).expand_as(got)
        b, h, r, got = b[some], h[some], r[some], got[some]
        src = s["table"].long()[b, got // page]
        dst = s["to"].long()[b, r // page]
        s["k2"][dst, r % page, h] = s["k"][src, got % page, h]
        s["v2"][dst, r % page, h] = s["v"][src, got % page, h]
        s["acc2"][b, h, r] = s["acc"][b, h, got]
        s["idx"].copy_(torch.where(some, first, -1))
        s["lens2"].copy_(s["lens"].clamp_max(keep))
    return {"k": s["k2"], "v": s["v2"], "acc": s["acc2"], "idx": s["idx"], "lens": s["lens2"]}


_RUN = {"attend": _attend, "append": _append, "evict": _evict}


# -------------------------------------------------------------------- work --
def work(case):
    c = case
    lens = _lens(c)
    total, es = sum(lens), 2 if c["dtype"] == "bf16" else 4
    token = 2 * c["Hkv"] * c["d"] * es                       # one token's keys and values
    book = 4 * c["B"] + 4 * sum(-(-x // c["page"]) for x in lens)
    if c["op"] == "attend":
        b = total * token + book + 2 * c["B"] * c["H"] * c["d"] * es + 4 * c["B"] * c["H"]
        b += 8 * total * c["Hkv"] if c["score"] else 0
        return {"bytes": b, "flops": 4.0 * total * c["H"] * c["d"]}
    if c["op"] == "append":
        new = sum(_new(c))
        return {"bytes": new * (2 * token + 4 * c["Hkv"]) + 8 * c["B"] + 4 * new // c["page"],
                "flops": 0.0}
    kept = [min(x, c["keep"]) for x in lens]
    cut = sum(x for x in lens if x > c["keep"])
    b = sum(kept) * (2 * token + 4 * c["Hkv"]) + 4 * c["Hkv"] * (cut + sum(kept) - c["keep"] * sum(
        x > c["keep"] for x in lens)) + 4 * c["B"] * c["Hkv"] * c["keep"] + 2 * book
    return {"bytes": b, "flops": 0.0}


# ------------------------------------------------------------------- exact --
def exact(case, seed):
    """From the definitions, one sequence at a time, in 64 bits."""
    s = prepare(case, seed)
    c = case
    page, H, Hkv = c["page"], c["H"], c["Hkv"]
    G = H // Hkv
    lens, table = s["lens"].tolist(), s["table"].tolist()
    acc = s["acc"].double()
    if c["op"] == "attend":
        o = torch.zeros(c["B"], H, c["d"], dtype=torch.float64, device=DEV)
        lse = torch.full((c["B"], H), -math.inf, dtype=torch.float64, device=DEV)
        for b, n in enumerate(lens):
            if n == 0:
                continue
            at = torch.tensor(table[b][:-(-n // page)], device=DEV)
            for h in range(Hkv):
                k = s["k"][at][:, :, h].flatten(0, 1)[:n].double()
                v = s["v"][at][:, :, h].flatten(0, 1)[:n].double()
                x = s["q"][b, h * G:(h + 1) * G].double() @ k.T / math.sqrt(c["d"])
                z = torch.logsumexp(x, -1)
                p = torch.exp(x - z[:, None])
                lse[b, h * G:(h + 1) * G] = z
                o[b, h * G:(h + 1) * G] = p @ v
                acc[b, h, :n] += p.sum(0) / G
        return {"o": o, "lse": lse, "acc": acc} if c["score"] else {"o": o, "lse": lse}
    if c["op"] == "append":
        k, v, cu = s["k"].double(), s["v"].double(), s["cu"].tolist()
        for b, n in enumerate(lens):
            x = cu[b + 1] - cu[b]
            if x == 0:
                continue
            place = torch.arange(n - x, n, device=DEV)
            p = s["table"][b].long()[torch.div(place, page, rounding_mode="floor")]
            k[p, place % page] = s["k_new"][cu[b]:cu[b + 1]].double()
            v[p, place % page] = s["v_new"][cu[b]:cu[b + 1]].double()
            acc[b, :, n - x:n] = 0.0
        return {"k": k, "v": v, "acc": acc}
    keep, sinks, recent = c["keep"], c["sinks"], c["recent"]
    k2, v2, acc2 = s["k2"].double(), s["v2"].double(), s["acc2"].double()
    idx = torch.full((c["B"], Hkv, keep), -1, dtype=torch.int32, device=DEV)
    for b, n in enumerate(lens):
        if n == 0:
            continue
        m = min(n, keep)
        src = torch.tensor(table[b][:-(-n // page)], device=DEV)
        dst = s["to"][b].long()
        for h in range(Hkv):
            if n <= keep:
                chosen = torch.arange(n, device=DEV)
            else:
                mid = torch.arange(sinks, n - recent, device=DEV)
                # a stable ascending sort of the negated weights: ties by index
                by = torch.sort(-acc[b, h, sinks:n - recent], stable=True).indices
                chosen = torch.cat([torch.arange(sinks, device=DEV),
                                    mid[by[:keep - sinks - recent]].sort().values,
                                    torch.arange(n - recent, n, device=DEV)])
            r = torch.arange(m, device=DEV)
            p = dst[torch.div(r, page, rounding_mode="floor")]
            k2[p, r % page, h] = s["k"][src][:, :, h].flatten(0, 1)[chosen].double()
            v2[p, r % page, h] = s["v"][src][:, :, h].flatten(0, 1)[chosen].double()
            acc2[b, h, :m] = acc[b, h, chosen]
            idx[b, h, :m] = chosen.to(torch.int32)
    return {"k": k2, "v": v2, "acc": acc2, "idx": idx,
            "lens": torch.tensor([min(x, keep) for x in lens], dtype=torch.int32, device=DEV)}
