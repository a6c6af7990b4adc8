"""A served batch's step around a paged key-value cache: what its operators
compute, on what they are measured.

  plan    what a step does to the sequences' lengths (new tokens, cut ones,
          finished sequences) becomes page numbers taken from and given back to
          a list of free pages, the block tables, and a place for every new row
  rotate  queries and keys after their projection: the norm of each head and the
          rotation by the token's position (one axis, or the rows and columns of
          an image), in one pass
  append  the same for a step's new tokens, keys and values going straight to
          their places in the pages
  shared  attention of one new token per sequence over a prefix that its group
          has in common and the sequence's own cached tokens

``own`` False: the plain forms; True: the calls a program makes of the library.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def _plan(name, B, page, max_len, new, done, cut, spread, spare):
    return dict(name=name, op="plan", B=B, page=page, max_len=max_len, new=new, done=done, cut=cut,
                spread=spread, spare=spare)


def _rotate(name, dtype, B, N, H, Hkv, d, rot, axes, interleaved, norm, layout, base=10000.0,
            scaling="none", factor=1.0, far=0):
    return dict(name=name, op="rotate", dtype=dtype, B=B, N=N, H=H, Hkv=Hkv, d=d, rot=rot, axes=axes,
                interleaved=interleaved, norm=norm, layout=layout, base=base, scaling=scaling,
                factor=factor, far=far)


def _append(name, dtype, B, H, Hkv, d, rot, page, max_len, new, spread, layout, interleaved=False,
            norm=True, base=1000000.0, scaling="none", factor=1.0):
    return dict(name=name, op="append", dtype=dtype, B=B, H=H, Hkv=Hkv, d=d, rot=rot, page=page,
                max_len=max_len, new=new, spread=spread, layout=layout, interleaved=interleaved,
                norm=norm, base=base, scaling=scaling, factor=factor, axes=1)


def _shared(name, dtype, B, groups, H, Hkv, d, page, prefix, max_len, spread, layout):
    return dict(name=name, op="shared", dtype=dtype, B=B, groups=groups, H=H, Hkv=Hkv, d=d, page=page,
                prefix=prefix, max_len=max_len, spread=spread, layout=layout)


def listed():
    return [
        # one decoding step of a served batch: a token each, a few sequences end, a few
        # lose drafted tokens that were not taken
        _plan("plan_step", 256, 16, 4096, 1, 0.05, 0.1, 0.9, 1.0),
        # a batch of prompts is let in, and there are pages for most of it
        _plan("plan_prompts", 96, 16, 4096, 2048, 0.1, 0.0, 0.8, 0.7),
        # an image's tokens on a 64 x 64 grid, positions by row and column
        _rotate("rotate_image", "bf16", 1, 4096, 24, 24, 128, 128, 2, True, True, "heads"),
        # a batch of prompts, grouped heads, half of each head turned
        _rotate("rotate_half", "bf16", 5, 1733, 32, 8, 96, 48, 1, False, True, "joint", base=500000.0),
        # full precision at far positions, frequencies stretched part by part
        _rotate("rotate_f32", "f32", 2, 777, 16, 4, 80, 80, 1, False, True, "tokens", base=500000.0,
                scaling="parts", factor=16.0, far=900000),
        # one decoding step of a served batch
        _append("append_turned", "bf16", 64, 32, 8, 128, 128, 16, 4096, 1, 0.8, "tokens"),
        # a batch of prompts, all of their tokens at once
        _append("append_turned_prompts", "bf16", 12, 32, 8, 128, 64, 16, 4100, 4000, 0.8, "heads",
                interleaved=True),
        # a few conversations on one short instruction: launches and latency
        _shared("shared_few", "bf16", 8, 1, 32, 8, 128, 16, 517, 96, 0.5, "tokens"),
        # a served batch on one long instruction with its documents
        _shared("shared_batch", "bf16", 64, 1, 32, 8, 128, 16, 8192, 512, 0.9, "heads"),
        # several instructions of uneven lengths, a group of sequences on each
        _shared("shared_groups", "bf16", 96, 12, 24, 8, 128, 64, 3001, 700, 0.9, "tokens"),
        # many samples of one long document: products bound it
        _shared("shared_many", "bf16", 128, 1, 32, 4, 128, 64, 32768, 300, 0.5, "tokens"),
        # full precision, odd sizes
        _shared("shared_f32", "f32", 10, 2, 16, 4, 96, 24, 1023, 77, 0.5, "joint"),
    ]


# -------------------------------------------------------------------- draw --
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _turn(rng, c):
    c["rot"] = rng.choice([c["d"], c["d"], c["d"] // 2, c["d"] // 4 // 2 * 2])
    c["interleaved"] = rng.random() < 0.5
    c["norm"] = rng.random() < 0.8
    c["base"] = rng.choice([10000.0, 500000.0, 1000000.0])
    c["scaling"] = rng.choice(["none", "none", "linear", "base", "parts"])
    c["factor"] = 1.0 if c["scaling"] == "none" else rng.choice([2.0, 8.0, 32.0])


def draw(rng):
    op = rng.choice(["plan", "rotate", "append", "shared", "shared"])
    if op == "plan":
        B = _log(rng, 1, 2000)
        max_len = _log(rng, 1, 16384)
        new = rng.choice([1, min(max_len, _log(rng, 1, max(1, min(4096, 200000 // B))))])
        return dict(op=op, B=B, page=rng.choice([1, 8, 16, 16, 24, 64, 128]), max_len=max_len, new=new,
                    done=rng.choice([0.0, 0.05, 0.3]), cut=rng.choice([0.0, 0.1]),
                    spread=rng.choice([0.0, 0.5, 0.9]), spare=rng.choice([1.0, 1.0, 0.5]))
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    d = rng.choice([64, 72, 80, 96, 128, 128, 256])
    Hkv = rng.choice([1, 2, 3, 4, 8, 8, 16])
    H = Hkv * rng.choice([1, 2, 3, 4, 4, 6, 8])
    c = dict(op=op, dtype=dtype, H=H, Hkv=Hkv, d=d)
    es = 2 if dtype == "bf16" else 4
    if op == "rotate":
        most = max(1, int(60e6 / ((H + Hkv) * d * es)))      # below the largest listed case's
        B = min(most, rng.choice([1, 1, 2, 5, 16]))
        c.update(B=B, N=_log(rng, 1, max(1, most // B)), axes=rng.choice([1, 1, 2, 3]),
                 layout=rng.choice(["tokens", "heads", "joint"]), far=rng.choice([0, 0, 100000, 900000]))
        _turn(rng, c)
        return c
    c.update(page=rng.choice([8, 16, 16, 24, 32, 64, 128]), spread=rng.choice([0.0, 0.5, 0.9]),
             layout=rng.choice(["tokens", "heads", "joint"]))
    if op == "append":
        most = max(16, int(120e6 / ((H + 2 * Hkv) * d * es)))
        B = _log(rng, 1, 96)
        c.update(B=B, max_len=_log(rng, 1, max(1, min(8192, most // B))), axes=1)
        c["new"] = rng.choice([1, _log(rng, 1, c["max_len"])])
        _turn(rng, c)
        return c
    # the products of the largest listed case, less in full precision
    flops = 6e10 if dtype == "bf16" and d <= 128 else 6e9
    B = _log(rng, 1, 160)
    groups = min(B, rng.choice([1, 1, 2, 3, 8, 24]))
    prefix = _log(rng, 1, max(1, min(65536, int(flops / (4 * B * H * d)),
                                    int(300e6 / (2 * groups * Hkv * d * es)))))
    c.update(B=B, groups=groups, prefix=prefix,
             max_len=_log(rng, 1, max(1, min(4096, int(100e6 / (2 * B * Hkv * d * es))))))
    return c


# ----------------------------------------------------------------- prepare --
def _golden(i):
    return (i * 0.6180339887498949) % 1.0


def _lens(c):
    """Lengths: the first is the longest, the others spread down to (1 - spread)
    of it; in a batch of 16 and more one slot is idle."""
    n = c["max_len"]
    out = [max(1, int(n * (1.0 - c["spread"] * _golden(i)))) for i in range(c["B"])]
    out[0] = n
    if c["B"] >= 16:
        out[c["B"] // 2] = 0
    return out


def _new(c):
    """New tokens per sequence (an append): the last of each length."""
    return [min(n, max(1, int(c["new"] * n / c["max_len"]))) if n else 0 for n in _lens(c)]


def _steps(c):
    """Lengths before a plan and their changes: finished sequences give all back, a
    few lose up to 7 tokens, prompts start from nothing, the others go on."""
    n, fresh, lens, change = c["max_len"], c["new"] > 1, [], []
    for i in range(c["B"]):
        u, x = _golden(i * 7 + 3), max(1, int(n * (1.0 - c["spread"] * _golden(i))))
        new = max(1, int(c["new"] * (1.0 - c["spread"] * _golden(i + 1))))
        if u < c["done"]:
            lens.append(x)
            change.append(-x)
        elif u < c["done"] + c["cut"]:
            lens.append(x)
            change.append(-(1 + i % 7))
        elif fresh:
            lens.append(0)
            change.append(new)
        else:
            lens.append(min(x, n - 1))
            change.append(1 if i % 17 != 16 else 0)
    return lens, change


def _members(c):
    """Sequences of each group, in order: about as many, some more, some fewer."""
    B, g = c["B"], c["groups"]
    at = sorted(min(B, max(0, round(B * (i + 0.5 * (_golden(i) - 0.5)) / g))) for i in range(1, g))
    edges = [0] + at + [B]
    return [edges[i + 1] - edges[i] for i in range(g)]


def _prefixes(c):
    p = [max(1, int(c["prefix"] * (1.0 - 0.8 * _golden(i)))) for i in range(c["groups"])]
    p[0] = c["prefix"]
    return p


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


def _table(lens, page, wide, gen, pages=None):
    """Page numbers in no order (-1: none), how many pages are used, the others."""
    used = -(-torch.tensor(lens, device=DEV) // page)
    total = int(used.sum())
    order = torch.randperm(max(1, total if pages is None else pages), generator=gen,
                           device=DEV).to(torch.int32)
    j = torch.arange(wide, device=DEV)
    at = order[((used.cumsum(0) - used)[:, None] + j).clamp_max(order.numel() - 1)]
    return at.masked_fill_(j >= used[:, None], -1), order.numel(), order[total:]


def _sections(c):
    """Pairs that turn by each axis of the position: equal parts, the first one with
    what is left over."""
    n, a = c["rot"] // 2, c["axes"]
    return [n - (a - 1) * (n // a)] + [n // a] * (a - 1)


LOW, HIGH, TRAINED = 1.0, 4.0, 8192      # of frequencies that are stretched part by part


def _frequencies(c):
    """Radians per position of each pair.  One axis: base^(-2i/rot); several: each
    axis has a ladder of its own over its part."""
    out = []
    for n in _sections(c):
        width = 2 * n
        base = c["base"]
        if c["scaling"] == "base" and width > 2:
            base *= c["factor"] ** (width / (width - 2))
        for i in range(n):
            f = base ** (-2.0 * i / width)
            if c["scaling"] == "linear":
                f /= c["factor"]
            elif c["scaling"] == "parts":
                keep = min(1.0, max(0.0, (TRAINED * f / (2 * math.pi) - LOW) / (HIGH - LOW)))
                f = keep * f + (1.0 - keep) * f / c["factor"]
            out.append(f)
    return out


def _magnitude(c):
    return 0.1 * math.log(c["factor"]) + 1.0 if c["scaling"] == "parts" else 1.0


def _views(c, lead, dt, gen):
    """Queries, keys and values of the tokens `lead`, as projections leave them:
    parts of one buffer or three of their own."""
    H, Hkv, d = c["H"], c["Hkv"], c["d"]
    if c["layout"] == "joint":
        x = torch.randn(*lead, H + 2 * Hkv, d, device=DEV, generator=gen)
        x = (x * (1.0 + torch.rand(H + 2 * Hkv, 1, device=DEV, generator=gen) * 3.0)).to(dt)
        return x[..., :H, :], x[..., H:H + Hkv, :], x[..., H + Hkv:, :]
    return tuple((torch.randn(*lead, h, d, device=DEV, generator=gen) *
                  (1.0 + torch.rand(h, 1, device=DEV, generator=gen) * 3.0)).to(dt)
                 for h in (H, Hkv, Hkv))


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    s = _PREPARE[c["op"]](c, gen)
    s["c"] = c
    s["plan"] = {}   # the library's descriptors of these buffers, made at the first pass
    return s


def _weights(c, dt, gen):
    if not c["norm"]:
        return None, None
    return tuple((1.0 + 0.2 * torch.randn(c["d"], device=DEV, generator=gen)).to(dt) for _ in range(2))


def _turning(c, s, dt, gen):
    s["wq"], s["wk"] = _weights(c, dt, gen)
    s["freq"] = torch.tensor(_frequencies(c), dtype=torch.float64, device=DEV)
    s["axis"] = torch.repeat_interleave(torch.arange(c["axes"], device=DEV),
                                        torch.tensor(_sections(c), device=DEV))
    return s


def _prepare_plan(c, gen):
    lens, change = _steps(c)
    page, n = c["page"], c["max_len"]
    wide = -(-n // page)
    used = sum(-(-x // page) for x in lens)
    need = sum(-(-max(0, x + y) // page) - -(-x // page) for x, y in zip(lens, change) if y > 0)
    spare = max(0, int(need * c["spare"])) + (3 if c["spare"] >= 1.0 else 0)
    table, pages, rest = _table(lens, page, wide, gen, used + spare)
    free = torch.zeros(pages, dtype=torch.int32, device=DEV)
    free[:rest.numel()] = rest
    rows = sum(x for x in change if x > 0)
    T = -(-max(rows, 1) // 8) * 8         # the rows of a step come in eights
    z = dict(device=DEV)
    kv = torch.zeros(2, pages, page, 1, 8, dtype=torch.bfloat16, **z)
    # a few sequences lie at other places than their changes say: seeds differ
    turn = torch.randperm(c["B"], generator=gen, device=DEV)
    lens_t = torch.tensor(lens, dtype=torch.int32, **z)[turn]
    return dict(k=kv[0], v=kv[1], table=table[turn].contiguous(), lens=lens_t,
                change=torch.tensor(change, dtype=torch.int32, **z)[turn],
                base=torch.randint(0, 4096, (c["B"],), generator=gen, dtype=torch.int32, **z),
                lens1=torch.zeros(c["B"], dtype=torch.int32, **z), free=free,
                count=torch.tensor([rest.numel()], dtype=torch.int32, **z),
                count1=torch.zeros(1, dtype=torch.int32, **z),
                cu=torch.zeros(c["B"] + 1, dtype=torch.int32, **z),
                slot=torch.zeros(T, dtype=torch.int64, **z),
                seq=torch.zeros(T, dtype=torch.int32, **z), place=torch.zeros(T, dtype=torch.int32, **z),
                pos=torch.zeros(T, dtype=torch.int32, **z))


def _prepare_rotate(c, gen):
    dt, B, N, H, Hkv, d = TYPES[c["dtype"]], c["B"], c["N"], c["H"], c["Hkv"], c["d"]
    q, k, _ = _views(c, (B, N), dt, gen)
    if c["axes"] == 1:
        start = torch.randint(0, c["far"] + 1, (B, 1), generator=gen, device=DEV)
        pos = (start + torch.arange(N, device=DEV)).to(torch.int32)[..., None].contiguous()
    else:            # rows and columns of a grid, and an image's number before them
        wide = max(1, math.isqrt(N))
        i = torch.arange(N, device=DEV)
        grid = torch.stack([i * 0 + 1, i // wide, i % wide][-c["axes"]:], -1).to(torch.int32)
        pos = grid[torch.stack([torch.randperm(N, generator=gen, device=DEV) for _ in range(B)])]
    if c["layout"] == "heads":         # the order in which the attention reads, behind 7 other tokens
        qo = torch.zeros(B, H, N + 7, d, dtype=dt, device=DEV).transpose(1, 2)[:, 7:]
        ko = torch.zeros(B, Hkv, N + 7, d, dtype=dt, device=DEV).transpose(1, 2)[:, 7:]
    else:
        qo = torch.zeros(B, N, H, d, dtype=dt, device=DEV)
        ko = torch.zeros(B, N, Hkv, d, dtype=dt, device=DEV)
    return _turning(c, dict(q=q, k_in=k, pos=pos, qo=qo, ko=ko), dt, gen)


def _prepare_append(c, gen):
    dt, page, n = TYPES[c["dtype"]], c["page"], c["max_len"]
    lens, new = _lens(c), _new(c)
    table, pages, _ = _table(lens, page, -(-n // page), gen)
    k, v = _pool(c, pages, dt)
    seq = [b for b, x in enumerate(new) for _ in range(x)]
    place = [lens[b] - x + i for b, x in enumerate(new) for i in range(x)]
    T = len(seq)
    seq = torch.tensor(seq, device=DEV)
    place = torch.tensor(place, device=DEV)
    slot = table[seq, place // page].long() * page + place % page
    if T >= 4:
        slot[T // 3] = -1                 # one row is padding
    q, k_new, v_new = _views(c, (T,), dt, gen)
    start = torch.randint(0, 3000, (c["B"],), generator=gen, device=DEV)
    s = dict(k=k, v=v, table=table, lens=torch.tensor(lens, dtype=torch.int32, device=DEV), slot=slot,
             pos=(start[seq] + place).to(torch.int32), q=q, k_new=k_new, v_new=v_new,
             qo=torch.zeros(T, c["H"], c["d"], dtype=dt, device=DEV))
    return _turning(c, s, dt, gen)


def _prepare_shared(c, gen):
    dt, page, B, Hkv, H, d = TYPES[c["dtype"]], c["page"], c["B"], c["Hkv"], c["H"], c["d"]
    lens, pre, size = _lens(c), _prefixes(c), _members(c)
    wide, wide_p = -(-c["max_len"] // page), -(-c["prefix"] // page)
    both, pages, _ = _table(pre + lens, page, max(wide, wide_p), gen)
    k, v = _pool(c, pages, dt)
    for t in (k, v):
        t.copy_(torch.randn(pages, page, Hkv, d, dtype=dt, device=DEV, generator=gen))
    q = torch.randn(B, H, d, device=DEV, generator=gen)
    group = [g for g, m in enumerate(size) for _ in range(m)]
    start = [0]
    for m in size:
        start.append(start[-1] + m)
    # the first token of a prefix draws attention, as in trained models
    head = torch.zeros(c["groups"], H, d, device=DEV).index_add_(
        0, torch.tensor(group, device=DEV), q)
    head = head.view(c["groups"], Hkv, H // Hkv, d).mean(2)
    first = both[:c["groups"], 0].long()
    k[first, 0] += (head / head.norm(dim=-1, keepdim=True).clamp_min(1e-6) * math.sqrt(d) * 0.5).to(dt)
    z = dict(device=DEV)
    return dict(k=k, v=v, table=both[c["groups"]:, :wide].contiguous(),
                table_p=both[:c["groups"], :wide_p].contiguous(),
                lens=torch.tensor(lens, dtype=torch.int32, **z),
                lens_p=torch.tensor(pre, dtype=torch.int32, **z),
                start=torch.tensor(start, dtype=torch.int32, **z), q=(2.0 * q).to(dt),
                o=torch.zeros(B, H, d, dtype=dt, **z), lse=torch.zeros(B, H, **z),
                scale=1.0 / math.sqrt(d))


_PREPARE = {"plan": _prepare_plan, "rotate": _prepare_rotate, "append": _prepare_append,
            "shared": _prepare_shared}


# --------------------------------------------------------------------- run --
def run(state):
    return _RUN[state["c"]["op"]](state)


def _cache(s):
    """The library's descriptor of the cache: made once and kept, as a program
    keeps it beside the buffers."""
    got = s["plan"].get("cache")
    if got is None:
        import paper_2608_17995_gb300 as av
        lens = s["lens1"] if s["c"]["op"] == "plan" else s["lens"]
        got = s["plan"]["cache"] = av.KVCache(s["k"], s["v"], s["table"], lens,
                                              max_len=s["c"]["max_len"])
    return got


def _rotary(s):
    got = s["plan"].get("rotary")
    if got is None:
        import paper_2608_17995_gb300 as av
        c = s["c"]
        got = s["plan"]["rotary"] = av.Rotary(
            c["rot"], base=c["base"], sections=_sections(c), interleaved=c["interleaved"],
            scaling=c["scaling"], factor=c["factor"], original_len=TRAINED, low=LOW, high=HIGH,
            magnitude=_magnitude(c), device=DEV)
    return got


def _run_plan(s):
    if own:
        import paper_2608_17995_gb300 as av
        av.avits_cache_plan(_cache(s), s["change"], s["free"], s["count"], s["cu"], s["slot"], s["seq"],
                            s["place"], pos=s["pos"], pos_base=s["base"], lens=s["lens"],
                            free_out=s["count1"])
    else:
        c = s["c"]
        page, T, cap = c["page"], s["slot"].numel(), s["free"].numel()
        n0, d = s["lens"].long(), s["change"].long()
        n1 = (n0 + d).clamp_min(0)
        rows = d.clamp_min(0)
        cum = rows.cumsum(0)
        p0, p1 = (n0 + page - 1) // page, (n1 + page - 1) // page
        fits = (d <= 0) | ((n1 <= c["max_len"]) & (cum <= T))
        need = torch.where(fits, (p1 - p0).clamp_min(0), 0)
        back = (p0 - p1).clamp_min(0)
        avail = s["count"].long() + back.sum()
        upto = need.cumsum(0)
        ok = fits & ((need == 0) | (upto <= avail))
        # pages that are given back go behind the free ones, in order
        j = torch.arange(s["table"].shape[1], device=DEV)
        give = (j >= p1[:, None]) & (j < p0[:, None])
        rank = (give.reshape(-1).cumsum(0) - 1).view_as(give)
        free = torch.cat([s["free"], s["free"][:1]])
        free.scatter_(0, torch.where(give, s["count"] + rank, cap).reshape(-1), s["table"].reshape(-1))
        free = free[:cap]
        # and pages are taken from their end
        take = ok[:, None] & (j >= p0[:, None]) & (j < p1[:, None])
        rank = (upto - need)[:, None] + j - p0[:, None]
        s["table"].copy_(torch.where(take, free[(avail - 1 - rank).clamp(0, cap - 1)], s["table"]))
        s["free"].copy_(free)
        s["count1"].copy_(avail - torch.where(ok, need, 0).sum())
        s["lens1"].copy_(torch.where(ok, n1, n0))
        s["cu"][1:].copy_(cum.clamp_max(T))
        t = torch.arange(T, device=DEV)
        b = torch.searchsorted(cum, t, right=True).clamp_max(c["B"] - 1)
        here = (t < cum[-1]) & ok[b]
        at = n0[b] + t - (cum - rows)[b]
        slot = s["table"][b, (at // page).clamp(0, j.numel() - 1)].long() * page + at % page
        s["slot"].copy_(torch.where(here, slot, -1))
        s["seq"].copy_(torch.where(here, b, -1))
        s["place"].copy_(torch.where(here, at, -1))
        s["pos"].copy_(torch.where(here, at + s["base"][b], -1))
    return {"table": s["table"], "lens": s["lens1"], "free": s["free"], "count": s["count1"],
            "cu": s["cu"], "slot": s["slot"], "seq": s["seq"], "place": s["place"], "pos": s["pos"]}


def _turned(s, x, w, pos):
    """Norm and rotation in 32 bits (angles in 64): x [..., heads, d], pos [..., axes]."""
    c = s["c"]
    y = x.float()
    if c["norm"]:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * w.float()
    angle = pos.double()[..., s["axis"]] * s["freq"]
    m, half = _magnitude(c), c["rot"] // 2
    cos = (torch.cos(angle) * m).float()[..., None, :]
    sin = (torch.sin(angle) * m).float()[..., None, :]
    out = y.clone()
    if c["interleaved"]:
        a, b = y[..., 0:c["rot"]:2], y[..., 1:c["rot"]:2]
        out[..., 0:c["rot"]:2] = a * cos - b * sin
        out[..., 1:c["rot"]:2] = b * cos + a * sin
    else:
        a, b = y[..., :half], y[..., half:c["rot"]]
        out[..., :half] = a * cos - b * sin
        out[..., half:c["rot"]] = b * cos + a * sin
    return out


def _run_rotate(s):
    if own:
        import paper_2608_17995_gb300 as av
        av.avits_norm_rotate(_rotary(s), s["pos"], s["q"], s["qo"], k=s["k_in"], k_out=s["ko"],
                             q_weight=s["wq"], k_weight=s["wk"], norm=s["c"]["norm"], eps=EPS)
    else:
        s["qo"].copy_(_turned(s, s["q"], s["wq"], s["pos"]))
        s["ko"].copy_(_turned(s, s["k_in"], s["wk"], s["pos"]))
    return {"q": s["qo"], "k": s["ko"]}


def _run_append(s):
    if own:
        import paper_2608_17995_gb300 as av
        av.avits_cache_append_rotated(_cache(s), _rotary(s), s["pos"], s["slot"], s["q"], s["qo"],
                                      s["k_new"], s["v_new"], q_weight=s["wq"], k_weight=s["wk"],
                                      norm=s["c"]["norm"], eps=EPS)
    else:
        page = s["c"]["page"]
        live = s["slot"] >= 0
        # a padding row goes where the row before it (or behind it) goes too
        t = torch.arange(live.numel(), device=DEV)
        src = torch.where(live, t, torch.where(t > 0, t - 1, t + 1).clamp_max(live.numel() - 1))
        at = s["slot"][src]
        some = at >= 0
        at = at.clamp_min(0)
        p, i = at // page, at % page
        pos = s["pos"][:, None]
        k = _turned(s, s["k_new"], s["wk"], pos).to(s["k"].dtype)[src]
        q = _turned(s, s["q"], s["wq"], pos).to(s["qo"].dtype)
        w = some[:, None, None]
        s["k"][p, i] = torch.where(w, k, s["k"][p, i])
        s["v"][p, i] = torch.where(w, s["v_new"][src], s["v"][p, i])
        s["qo"].copy_(torch.where(live[:, None, None], q, s["qo"]))
    return {"q": s["qo"], "k": s["k"], "v": s["v"]}


def _rows(pool, table, n):
    """[B, n, Hkv, d] of the pages' tokens, in order, in 32 bits."""
    got = pool[table.clamp_min(0).long()]
    return got.reshape(table.shape[0], -1, pool.shape[2], pool.shape[3])[:, :n].float()


def _run_shared(s):
    c = s["c"]
    if own:
        import paper_2608_17995_gb300 as av
        prefix = s["plan"].get("prefix")
        if prefix is None:
            prefix = s["plan"]["prefix"] = av.KVCache(s["k"], s["v"], s["table_p"], s["lens_p"],
                                                      max_len=c["prefix"])
        av.avits_cache_attention_shared(_cache(s), prefix, s["start"], s["q"], s["scale"], s["o"],
                                        lse=s["lse"])
        return {"o": s["o"], "lse": s["lse"]}
    B, H, Hkv, d, n = c["B"], c["H"], c["Hkv"], c["d"], c["max_len"]
    G = H // Hkv
    q = s["q"].float().view(B, Hkv, G, d) * s["scale"]
    # the own tokens
    live = torch.arange(n, device=DEV)[None, :] < s["lens"][:, None]
    k = _rows(s["k"], s["table"], n).masked_fill_(~live[:, :, None, None], 0.0)
    x = torch.matmul(q, k.permute(0, 2, 3, 1)).masked_fill_(~live[:, None, None, :], -math.inf)
    top = x.amax(-1, keepdim=True)
    k = _rows(s["v"], s["table"], n).masked_fill_(~live[:, :, None, None], 0.0)
    # the groups' prefixes, one product for all that share them
    at, tops, parts = 0, [], []
    for g, m in enumerate(_members(c)):
        if m == 0:
            continue
        P = _prefixes(c)[g]
        kp = _rows(s["k"], s["table_p"][g:g + 1], P)[0].permute(1, 2, 0)            # [Hkv, d, P]
        qp = q[at:at + m].permute(1, 0, 2, 3).reshape(Hkv, m * G, d)
        parts.append(torch.matmul(qp, kp).view(Hkv, m, G, P))
        tops.append(parts[-1].amax(-1, keepdim=True).permute(1, 0, 2, 3))
        at += m
    top = torch.maximum(top, torch.cat(tops))
    e = torch.exp(x.sub_(top))
    total, o = e.sum(-1, keepdim=True), torch.matmul(e, k.permute(0, 2, 1, 3))
    at, sums, outs = 0, [], []
    i = 0
    for g, m in enumerate(_members(c)):
        if m == 0:
            continue
        P = _prefixes(c)[g]
        e = torch.exp(parts[i].sub_(top[at:at + m].permute(1, 0, 2, 3)))
        vp = _rows(s["v"], s["table_p"][g:g + 1], P)[0].permute(1, 0, 2)            # [Hkv, P, d]
        sums.append(e.sum(-1, keepdim=True).permute(1, 0, 2, 3))
        outs.append(torch.matmul(e.view(Hkv, m * G, P), vp).view(Hkv, m, G, d).permute(1, 0, 2, 3))
        at += m
        i += 1
    total = total + torch.cat(sums)
    s["o"].copy_(((o + torch.cat(outs)) / total).reshape(B, H, d))
    s["lse"].copy_((torch.log(total) + top).reshape(B, H))
    return {"o": s["o"], "lse": s["lse"]}


_RUN = {"plan": _run_plan, "rotate": _run_rotate, "append": _run_append, "shared": _run_shared}


# -------------------------------------------------------------------- work --
def work(case):
    c = case
    if c["op"] == "plan":
        lens, change = _steps(c)
        page = c["page"]
        moved = sum(abs(-(-max(0, x + y) // page) - -(-x // page)) for x, y in zip(lens, change))
        rows = sum(y for y in change if y > 0)
        return {"bytes": 20 * c["B"] + 8 * moved + 20 * rows, "flops": 0.0}
    es = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "rotate":
        vals = c["B"] * c["N"] * (c["H"] + c["Hkv"]) * c["d"]
        return {"bytes": 2 * vals * es + 4 * c["B"] * c["N"] * c["axes"], "flops": 7.0 * vals}
    if c["op"] == "append":
        T = sum(_new(c))
        vals = T * (c["H"] + c["Hkv"]) * c["d"]
        return {"bytes": 2 * (vals + T * c["Hkv"] * c["d"]) * es + 12 * T, "flops": 7.0 * vals}
    lens, pre, size = _lens(c), _prefixes(c), _members(c)
    token = 2 * c["Hkv"] * c["d"] * es
    read = sum(lens) + sum(p for p, m in zip(pre, size) if m)
    pairs = sum(lens) + sum(p * m for p, m in zip(pre, size))
    return {"bytes": read * (token + 4.0 / c["page"]) + 2 * c["B"] * c["H"] * c["d"] * es +
            4 * c["B"] * c["H"], "flops": 4.0 * pairs * c["H"] * c["d"]}


# ------------------------------------------------------------------- exact --
def exact(case, seed):
    """From the definitions, in 64 bits, one sequence (or token row) at a time."""
    s = prepare(case, seed)
    return _EXACT[case["op"]](case, s)


def _exact_plan(c, s):
    page, T = c["page"], s["slot"].numel()
    lens, change, base = s["lens"].tolist(), s["change"].tolist(), s["base"].tolist()
    table, free, n_free = s["table"].tolist(), s["free"].tolist(), int(s["count"])
    for b, (n, y) in enumerate(zip(lens, change)):
        if y < 0:
            for j in range(-(-max(0, n + y) // page), -(-n // page)):
                free[n_free] = table[b][j]
                n_free += 1
    left, wanted, cu = n_free, 0, [0]
    slot, seq, place, pos = [-1] * T, [-1] * T, [-1] * T, [-1] * T
    for b, (n, y) in enumerate(zip(lens, change)):
        at = cu[-1]
        cu.append(at + max(0, y))
        if y < 0:
            lens[b] = max(0, n + y)
            continue
        cols = range(-(-n // page), -(-(n + y) // page))
        if n + y > c["max_len"] or cu[-1] > T:
            continue
        wanted += len(cols)
        if len(cols) and wanted > left:
            continue
        for j in cols:
            n_free -= 1
            table[b][j] = free[n_free]
        lens[b] = n + y
        for i in range(y):
            j = n + i
            slot[at + i] = table[b][j // page] * page + j % page
            seq[at + i], place[at + i], pos[at + i] = b, j, j + base[b]
    i32 = dict(dtype=torch.int32, device=DEV)
    return {"table": torch.tensor(table, **i32).view_as(s["table"]), "lens": torch.tensor(lens, **i32),
            "free": torch.tensor(free, **i32), "count": torch.tensor([n_free], **i32),
            "cu": torch.tensor([min(x, T) for x in cu], **i32),
            "slot": torch.tensor(slot, dtype=torch.int64, device=DEV), "seq": torch.tensor(seq, **i32),
            "place": torch.tensor(place, **i32), "pos": torch.tensor(pos, **i32)}


def _exact_turn(c, s, x, w, pos):
    """One head at a time as complex numbers; x [rows, heads, d], pos [rows, axes]."""
    x = x.double()
    out = torch.empty_like(x)
    phase = pos.double()[:, s["axis"]] * s["freq"]
    unit = torch.polar(torch.full_like(phase, _magnitude(c)), phase)
    r = c["rot"]
    for h in range(x.shape[1]):
        y = x[:, h]
        if c["norm"]:
            y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / c["d"] + EPS) * w.double()
        if c["interleaved"]:
            z = torch.view_as_complex(y[:, :r].reshape(-1, r // 2, 2).contiguous()) * unit
            turned = torch.view_as_real(z).reshape(-1, r)
        else:
            z = torch.complex(y[:, :r // 2].contiguous(), y[:, r // 2:r].contiguous()) * unit
            turned = torch.cat([z.real, z.imag], -1)
        out[:, h] = torch.cat([turned, y[:, r:]], -1)
    return out


def _exact_rotate(c, s):
    flat = s["pos"].reshape(-1, c["axes"])
    return {n: _exact_turn(c, s, x.reshape(-1, *x.shape[2:]), w, flat).view(x.shape)
            for n, x, w in (("q", s["q"], s["wq"]), ("k", s["k_in"], s["wk"]))}


def _exact_append(c, s):
    pos = s["pos"][:, None]
    q, k = (_exact_turn(c, s, x, w, pos) for x, w in ((s["q"], s["wq"]), (s["k_new"], s["wk"])))
    live = s["slot"] >= 0
    qo, kp, vp = s["qo"].double(), s["k"].double(), s["v"].double()
    qo[live] = q[live]
    at = s["slot"][live]
    p, i = torch.div(at, c["page"], rounding_mode="floor"), at % c["page"]
    kp[p, i] = k[live]
    vp[p, i] = s["v_new"][live].double()
    return {"q": qo, "k": kp, "v": vp}


def _exact_shared(c, s):
    H, Hkv, page = c["H"], c["Hkv"], c["page"]
    G = H // Hkv
    lens, pre, start = s["lens"].tolist(), s["lens_p"].tolist(), s["start"].tolist()
    o = torch.zeros(c["B"], H, c["d"], dtype=torch.float64, device=DEV)
    lse = torch.zeros(c["B"], H, dtype=torch.float64, device=DEV)

    def tokens(pool, row, n, h):
        return pool[row[:-(-n // page)].long(), :, h].flatten(0, 1)[:n].double()

    for g, n_p in enumerate(pre):
        if start[g] == start[g + 1]:
            continue
        for h in range(Hkv):
            kp, vp = (tokens(t, s["table_p"][g], n_p, h) for t in (s["k"], s["v"]))
            for b in range(start[g], start[g + 1]):
                k, v = (tokens(t, s["table"][b], lens[b], h) for t in (s["k"], s["v"]))
                k, v = torch.cat([kp, k]), torch.cat([vp, v])
                x = s["q"][b, h * G:(h + 1) * G].double() @ k.T / math.sqrt(c["d"])
                z = torch.logsumexp(x, -1)
                lse[b, h * G:(h + 1) * G] = z
                o[b, h * G:(h + 1) * G] = torch.exp(x - z[:, None]) @ v
    return {"o": o, "lse": lse}


_EXACT = {"plan": _exact_plan, "rotate": _exact_rotate, "append": _exact_append, "shared": _exact_shared}
