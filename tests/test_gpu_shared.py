"""GPU parity of the attention over shared prefixes against the oracle (numpy
fp64, one sequence at a time over its prefix and its own tokens).

Tolerances: those of the cache attention (test_gpu_cache.py), with n the keys of
both, and 2^-16 of sum_j w_j |v_j| for bf16 weights in two parts: the first is cut
to 8 bits, the rest, below 2^-7 of the weight, is rounded by 2^-9 of itself.  Joining
up to a few hundred parts adds 2^-23 per part and is within n 2^-23.
"""
import math
import threading

import numpy as np
import pytest

import oracle.cache as oc
from test_gpu_cache import DEV, _dt, _torch, av, make_pool  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


class World:
    """Prefixes and own tokens in one pool (or two), NaN wherever no token lies."""

    def __init__(self, av, dtype, size, pre, lens, H, Hkv, d, page, layout="tokens", page_p=None,
                 seed=0, std=2.0, before=0, max_len=None, max_pre=None):
        t = _torch()
        rng = np.random.default_rng(seed)
        g = t.Generator(device=DEV)
        g.manual_seed(seed)
        self.av, self.dtype, self.H, self.Hkv, self.d = av, dtype, H, Hkv, d
        self.size, self.pre, self.lens, self.B = list(size), list(pre), list(lens), len(lens)
        self.start = [before]
        for m in size:
            self.start.append(self.start[-1] + m)
        assert self.start[-1] <= self.B

        def fill(lens, page, max_len):
            used = [-(-n // page) for n in lens]
            order = rng.permutation(sum(used) + 2).astype(np.int32)
            table = np.full((len(lens), max(1, -(-max_len // page))), -1, np.int32)
            pools = make_pool(layout, len(order), page, Hkv, d, _dt(dtype))
            at = 0
            for b, n in enumerate(used):
                table[b, :n] = order[at:at + n]
                at += n
                if n:
                    place = t.arange(lens[b], device=DEV)
                    p = t.from_numpy(table[b].astype(np.int64)).to(DEV)[place // page]
                    for pool in pools:
                        pool[p, place % page] = t.randn(lens[b], Hkv, d, device=DEV, generator=g).to(_dt(dtype))
            tab, ln = t.from_numpy(table).to(DEV), t.tensor(lens, dtype=t.int32, device=DEV)
            return av.KVCache(pools[0], pools[1], tab, ln, max_len=max_len)

        self.cache = fill(lens, page, max_len or max(max(lens), 1))
        self.prefix = fill(pre, page_p or page, max_pre or max(max(pre), 1))
        self.q = (std * t.randn(self.B, H, d, device=DEV, generator=g)).to(_dt(dtype))
        self.scale = 1.0 / math.sqrt(d)
        self.group = t.tensor(self.start, dtype=t.int32, device=DEV)

    def rows(self, cache, b, n):
        tab = cache.block_table[b].cpu().numpy()
        return [oc.pages_to_rows(p.float().cpu().numpy(), tab, n) for p in (cache.k_pages, cache.v_pages)]

    def group_of(self, b):
        for g in range(len(self.size)):
            if self.start[g] <= b < self.start[g + 1]:
                return g
        return -1

    def outputs(self):
        t = _torch()
        return (t.full((self.B, self.H, self.d), 7.0, dtype=_dt(self.dtype), device=DEV),
                t.full((self.B, self.H), 7.0, device=DEV))

    def run(self, status=0, **kw):
        o, lse = self.outputs()
        self.av.avits_cache_attention_shared(self.cache, self.prefix, self.group, self.q, self.scale, o,
                                             lse=lse, **kw)
        assert self.av.avits_device_status() == status
        return o, lse

    def keys(self, b, shared, pre):
        k, v = self.rows(self.cache, b, self.lens[b])
        g = self.group_of(b) if shared else -1
        if g >= 0:
            k, v = np.concatenate([pre[g][0], k], 1), np.concatenate([pre[g][1], v], 1)
        return k, v

    def check(self, o, lse, shared=True, seqs=None, keys=None):
        d, eps_t = self.d, 2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -24
        q = self.q.float().cpu().numpy().astype(np.float64)
        got_o, got_l = o.float().cpu().numpy(), lse.cpu().numpy()
        pre = None if keys else {g: self.rows(self.prefix, g, n) for g, n in enumerate(self.pre)}
        for b in range(self.B) if seqs is None else seqs:
            k, v = keys(b) if keys else self.keys(b, shared, pre)
            n = k.shape[1]
            if n == 0:
                assert not got_o[b].any() and np.all(np.isneginf(got_l[b])), b
                continue
            want, wl, _ = oc.cache_attention(q[b], k, v, self.scale)
            G = self.H // self.Hkv
            X = self.scale * np.max(np.einsum("hgd,hnd->hgn", np.abs(q[b]).reshape(self.Hkv, G, d),
                                              np.abs(k).astype(np.float64)))
            dx = X * (d + 8) * 2.0 ** -23
            eps = 2 * dx + n * 2.0 ** -23 + 2.0 ** -21
            av, _, _ = oc.cache_attention(q[b], k, np.abs(v), self.scale)
            tol = (eps + n * 2.0 ** -23 + (2.0 ** -16 if self.dtype == "bf16" else 0)) * av
            tol = tol + eps_t * (np.abs(want) + tol) + 1e-30
            assert np.all(np.abs(got_o[b] - want) <= tol), (b, np.max(np.abs(got_o[b] - want) / tol))
            assert np.all(np.abs(got_l[b] - wl) <= dx + n * 2.0 ** -23 + 2.0 ** -22 * (1 + np.abs(wl))), b


CASES = [   # sizes, prefixes, own lengths, H, Hkv, d, page, layout
    ([1], [1], [1], 1, 1, 64, 16, "tokens"),
    ([3], [37], [5, 0, 70], 8, 2, 128, 16, "tokens"),
    ([2, 0, 3], [200, 50, 9], [3, 1, 30, 2, 17], 6, 3, 64, 8, "heads"),
    ([17, 2], [300, 129], [1 + 3 * i for i in range(19)], 16, 2, 96, 24, "joint"),
    ([33], [513], [i % 7 for i in range(33)], 8, 2, 128, 32, "heads"),
    ([70], [1000], [4] * 70, 4, 4, 80, 64, "tokens"),
    ([40, 41], [257, 640], [9] * 81, 4, 1, 128, 128, "tokens"),
    ([5], [77], [3, 9, 1, 0, 2], 16, 1, 256, 16, "tokens"),
    ([4, 4], [31, 64], [2] * 8, 6, 2, 72, 5, "joint"),
    ([1] * 30, [3 + i for i in range(30)], [i for i in range(30)], 8, 8, 64, 16, "tokens"),
    ([2], [5], [600, 900], 40, 1, 64, 16, "heads"),
    ([3, 3], [0, 40], [0, 2, 5, 0, 1, 0], 4, 2, 128, 16, "tokens"),
    # by parts: prefixes too long for one launch, on the tensor cores or (page, width, type) not
    ([3], [4200], [5, 0, 70], 8, 2, 128, 16, "tokens"),
    ([2, 0, 3], [5000, 50, 9], [3, 1, 30, 2, 17], 6, 3, 64, 8, "heads"),
    ([19, 1], [4100, 6000], [1 + 60 * i for i in range(20)], 16, 2, 96, 24, "joint"),
    ([4, 4], [4310, 64], [2] * 8, 6, 2, 72, 5, "joint"),
    ([5], [4177], [3, 9, 1, 0, 1500], 16, 1, 256, 16, "tokens"),
    ([2, 2], [4500, 4096], [600, 9000, 0, 16], 40, 1, 64, 16, "heads"),
    ([40, 41], [4257, 640], [9] * 81, 4, 1, 128, 128, "tokens"),
    ([3, 2], [0, 4400], [0, 3, 0, 0, 4], 4, 2, 80, 48, "tokens"),
    # more groups than lanes of a warp, some of them empty
    ([i % 4 for i in range(75)], [(i * 37) % 200 for i in range(75)], [(5 * i) % 30 for i in range(111)], 12, 6,
     64, 16, "tokens"),
    ([3, 1] * 35, [(i * 53) % 90 for i in range(70)], [i % 9 for i in range(140)], 24, 8, 80, 24, "heads"),
    # and where they are many
    ([90, 60], [70, 3], [i % 40 for i in range(150)], 8, 8, 64, 16, "heads"),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES)
def test_shared(av, dtype, case):
    size, pre, lens, H, Hkv, d, page, layout = case
    w = World(av, dtype, size, pre, lens, H, Hkv, d, page, layout)
    w.check(*w.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_prefix(av, dtype):
    """Many parts to a prefix, and the caches' page sizes differ."""
    w = World(av, dtype, [7, 30], [20000, 3000], [100] * 37, 8, 2, 128, 16, page_p=64, seed=2)
    w.check(*w.run(), seqs=[0, 6, 7, 20, 36])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("std", [0.0, 30.0])
def test_flat_and_steep(av, dtype, std):
    w = World(av, dtype, [20, 1], [700, 90], [33] * 21, 8, 2, 64, 16, std=std, seed=5)
    w.check(*w.run())


def test_many_rows(av):
    """More query heads of one group than a block of rows, borders inside a sequence."""
    w = World(av, "bf16", [130, 3], [400, 64], [(7 * i) % 50 for i in range(133)], 15, 3, 64, 16, seed=1)
    w.check(*w.run())


def test_sequences_of_no_group(av):
    w = World(av, "bf16", [2, 2], [50, 60], [3, 4, 0, 6, 7, 0, 9], 8, 2, 64, 16, before=1)
    o, lse = w.run()
    w.check(o, lse)
    assert np.isfinite(lse.cpu().numpy()).sum() == 6 * 8        # sequence 5 has no token at all


def test_long_max_len(av):
    """Bounds far above the lengths."""
    w = World(av, "bf16", [3], [100], [5, 0, 9], 8, 2, 128, 16, max_len=5000, max_pre=40000)
    w.check(*w.run())
    w = World(av, "f32", [3], [100], [5, 0, 9], 8, 2, 128, 16, max_len=5000, max_pre=40000)
    w.check(*w.run())


@pytest.mark.parametrize("start", [[0, 3, 2], [-1, 2, 4], [0, 2, 99], [2, 1, 1]])
def test_groups_that_do_not_rise(av, start):
    """Refused on the device: no sequence has a prefix."""
    w = World(av, "bf16", [2, 2], [50, 60], [3, 4, 5, 6], 8, 2, 64, 16)
    w.group.copy_(_torch().tensor(start, dtype=_torch().int32))
    w.check(*w.run(status=7), shared=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 24, 5])
def test_bad_pages_and_lengths(av, dtype, page):
    """A page number outside the pool masks its tokens; a length past max_len is cut."""
    t = _torch()
    w = World(av, dtype, [3, 2], [100, 130], [20, 9, 40, 3, 8], 8, 2, 64, page, seed=4)
    w.prefix.block_table[0, 1] = -1
    w.prefix.block_table[1, 0] = 1 << 20
    w.cache.block_table[2, 0] = w.cache.k_pages.shape[0]
    w.prefix.lens[1] = 1 << 20
    o, lse = w.run(status=7)

    def keys(b):
        """Without the tokens of those pages."""
        g = w.group_of(b)
        gone = {0: range(page, 2 * page), 1: range(page)}[g]
        pre = [x[:, [j for j in range(w.pre[g]) if j not in gone]] for x in take(w.prefix, g, w.pre[g])]
        own = [x[:, page if b == 2 else 0:] for x in take(w.cache, b, w.lens[b])]
        return [np.concatenate(x, 1) for x in zip(pre, own)]

    w.check(o, lse, keys=keys)


def take(cache, b, n):
    """Tokens of a row whose table may hold numbers outside the pool (they read page 0)."""
    tab = cache.block_table[b].cpu().numpy().copy()
    tab[(tab < 0) | (tab >= cache.k_pages.shape[0])] = 0
    return [oc.pages_to_rows(p.float().cpu().numpy(), tab, n) for p in (cache.k_pages, cache.v_pages)]


@pytest.mark.parametrize("page", [16, 5])
def test_infinite_values(av, page):
    """An infinite value makes its column infinite in all heads that see it, and no other."""
    t = _torch()
    w = World(av, "bf16", [4, 1], [150, 20], [6] * 5, 8, 2, 64, page, std=1.0, seed=3)
    pg = int(w.prefix.block_table[0, 33 // page])
    w.prefix.v_pages[pg, 33 % page, 1, 5] = float("inf")
    w.prefix.v_pages[pg, 33 % page, 1, 6] = float("-inf")
    w.prefix.v_pages[pg, 33 % page, 0, 7] = float("nan")
    o, _ = w.run()
    o = o.float().cpu().numpy()
    assert np.all(np.isposinf(o[:4, 4:, 5])) and np.all(np.isneginf(o[:4, 4:, 6]))
    assert np.all(np.isnan(o[:4, :4, 7]))
    bad = np.zeros_like(o, bool)
    bad[:4, 4:, 5:7] = True
    bad[:4, :4, 7] = True
    assert np.all(np.isfinite(o[~bad]))


def test_a_workspace_of_any_content(av):
    t = _torch()
    w = World(av, "bf16", [20, 5], [700, 90], [33] * 25, 8, 2, 128, 16, seed=6)
    need = av.avits_cache_attention_shared_workspace(w.cache, w.prefix, 8)
    first = w.run()
    for fill in (0, 255, 127):
        ws = t.full((need,), fill, dtype=t.uint8, device=DEV)
        o, lse = w.run(workspace=ws)
        assert t.equal(o, first[0]) and t.equal(lse, first[1])
    with pytest.raises(av.AvitsError):
        w.run(workspace=ws[:need - 16])
    with pytest.raises(ValueError):
        w.run(workspace=t.zeros(2 * need, dtype=t.uint8, device=DEV)[::2])
    w.check(*first)


def test_calls_in_a_row(av):
    """Without waiting between them, other calls among them, in a graph and on streams."""
    t = _torch()
    worlds = [World(av, "bf16", [20, 5], [700, 90], [33] * 25, 8, 2, 128, 16, seed=s) for s in range(3)]
    first = [w.run() for w in worlds]
    outs = [w.outputs() for w in worlds]

    def all_of(stream=None):
        for w, (o, lse) in zip(worlds, outs):
            av.avits_cache_attention_shared(w.cache, w.prefix, w.group, w.q, w.scale, o, lse=lse,
                                            stream=stream)

    def same():
        t.cuda.synchronize()
        for (o, lse), (fo, fl) in zip(outs, first):
            assert t.equal(o, fo) and t.equal(lse, fl)
            o.zero_()
            lse.zero_()
        t.cuda.synchronize()

    all_of()
    all_of()
    same()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        all_of()
    t.cuda.synchronize()
    [o.zero_() for o, _ in outs]
    graph.replay()
    graph.replay()
    same()
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    all_of(side)
    same()
    threads = [threading.Thread(target=all_of, args=(t.cuda.Stream(),)) for _ in range(3)]
    [x.start() for x in threads]
    [x.join() for x in threads]
    same()


def test_strided_queries(av):
    """Queries and outputs as parts of larger buffers, at odd offsets too."""
    t = _torch()
    w = World(av, "bf16", [6, 2], [100, 30], [9] * 8, 8, 2, 64, 16, seed=7)
    first = w.run()
    buf = t.zeros(8, 8, 200, dtype=t.bfloat16, device=DEV)
    out = t.full((8, 8, 200), 3.0, dtype=t.bfloat16, device=DEV)
    buf[..., 3:67] = w.q
    lse = t.empty(8, 8, device=DEV)
    av.avits_cache_attention_shared(w.cache, w.prefix, w.group, buf[..., 3:67], w.scale, out[..., 101:165],
                                    lse=lse)
    assert av.avits_device_status() == 0
    assert t.equal(out[..., 101:165], first[0]) and t.equal(lse, first[1])
    assert t.all(out[..., :101] == 3) and t.all(out[..., 165:] == 3)


def test_uneven_groups(av):
    """One group of many rows among small ones: two row tiles to a CTA, the second empty."""
    w = World(av, "bf16", [200, 1, 1], [500, 4200, 64], [3] * 202, 6, 2, 128, 16, seed=8)
    w.check(*w.run(), seqs=[0, 1, 41, 42, 43, 85, 86, 127, 128, 199, 200, 201])
    w = World(av, "bf16", [100], [4500], [1] * 100, 8, 2, 64, 8, seed=9)
    w.check(*w.run(), seqs=[0, 31, 32, 33, 63, 64, 65, 99])


@pytest.mark.parametrize("dtype,H,Hkv,d,page", [("bf16", 8, 8, 64, 16), ("bf16", 32, 8, 128, 16),
                                               ("bf16", 40, 4, 80, 24), ("bf16", 8, 8, 256, 16),
                                               ("f32", 8, 8, 96, 24), ("f32", 40, 4, 128, 5)])
def test_long_own_tokens(av, dtype, H, Hkv, d, page):
    """Own tokens on one line of tiles: sequences that may be long, and many of them."""
    lens = [(7 * i) % 40 for i in range(80)]
    lens[0], lens[33], lens[79] = 2500, 2111, 300
    w = World(av, dtype, [50, 0, 28], [1500, 8, 333], lens, H, Hkv, d, page, before=1, seed=13)
    first = w.run()
    w.check(*first, seqs=[0, 1, 2, 33, 40, 49, 50, 51, 77, 78, 79])
    again = w.run()
    assert _torch().equal(first[0], again[0]) and _torch().equal(first[1], again[1])


def pairs_of_tiles(av, size, pre, lens, H, Hkv, d, page, **kw):
    """Long own tokens by the bound, so that a prefix's rows go by two tiles to a CTA."""
    return World(av, "bf16", size, pre, lens, H, Hkv, d, page, max_len=(152 << 10) // (len(lens) * Hkv) + 1, **kw)


@pytest.mark.parametrize("size,pre,lens,H,Hkv,d,page,seqs", [
    ([200, 1, 1], [500, 4200, 64], [3] * 202, 6, 2, 128, 16, [0, 1, 41, 42, 43, 85, 86, 127, 128, 199, 200, 201]),
    ([100], [4500], [1] * 100, 8, 2, 64, 8, [0, 31, 32, 33, 63, 64, 65, 99]),
    ([64, 60], [1500, 0], [(5 * i) % 90 for i in range(124)], 12, 3, 80, 24, [0, 1, 2, 21, 42, 63, 64, 65, 123]),
    ([0, 130], [70, 1999], [0] * 130, 16, 8, 128, 64, [0, 1, 63, 64, 65, 127, 128, 129]),
])
def test_pairs_of_row_tiles(av, size, pre, lens, H, Hkv, d, page, seqs):
    w = pairs_of_tiles(av, size, pre, lens, H, Hkv, d, page, seed=8)
    first = w.run()
    w.check(*first, seqs=seqs)
    again = w.run()
    assert _torch().equal(first[0], again[0]) and _torch().equal(first[1], again[1])


def test_odd_values_in_pairs_of_row_tiles(av):
    """Infinite values, page numbers outside the pool and logits that rise along the keys."""
    t = _torch()
    w = pairs_of_tiles(av, [64], [4400], [6] * 64, 8, 2, 64, 16, std=1.0, seed=3)
    w.prefix.v_pages[int(w.prefix.block_table[0, 4399 // 16]), 4399 % 16, 1, 5] = float("inf")
    o = w.run()[0].float().cpu().numpy()
    assert np.all(np.isposinf(o[:, 4:, 5])) and np.isfinite(o).sum() == o.size - 64 * 4
    w = pairs_of_tiles(av, [64], [4300], [20] * 64, 8, 2, 128, 24, seed=4)
    w.prefix.block_table[0, 1] = -1
    w.prefix.block_table[0, 100] = 1 << 20
    o, lse = w.run(status=7)
    gone = {c * 24 + i for c in (1, 100) for i in range(24)}

    def keys(b):
        pre = [x[:, [j for j in range(4300) if j not in gone]] for x in take(w.prefix, 0, 4300)]
        return [np.concatenate(x, 1) for x in zip(pre, take(w.cache, b, w.lens[b]))]

    w.check(o, lse, keys=keys, seqs=[0, 31, 32, 33, 63])
    w = pairs_of_tiles(av, [30, 34], [2500, 2500], [10] * 64, 12, 2, 128, 16, std=1.0, seed=12)
    for g in range(2):
        place = t.arange(2500, device=DEV)
        pg = w.prefix.block_table[g].long()[place // 16]
        scale = (0.2 + 40.0 * (place % 1500) / 1500).to(t.bfloat16)[:, None, None]
        w.prefix.k_pages[pg, place % 16] = (w.prefix.k_pages[pg, place % 16] * scale)
    w.check(*w.run(), seqs=[0, 17, 29, 30, 63])


def test_infinite_values_by_parts(av):
    """As above where the prefix is on the tensor cores: of either part of a group's rows."""
    w = World(av, "bf16", [70], [4400], [6] * 70, 8, 2, 64, 16, std=1.0, seed=3)
    pg = int(w.prefix.block_table[0, 4399 // 16])
    w.prefix.v_pages[pg, 4399 % 16, 1, 5] = float("inf")
    w.prefix.v_pages[int(w.prefix.block_table[0, 0]), 3, 0, 7] = float("-inf")
    o, _ = w.run()
    o = o.float().cpu().numpy()
    assert np.all(np.isposinf(o[:, 4:, 5])) and np.all(np.isneginf(o[:, :4, 7]))
    bad = np.zeros_like(o, bool)
    bad[:, 4:, 5] = True
    bad[:, :4, 7] = True
    assert np.all(np.isfinite(o[~bad]))


@pytest.mark.parametrize("page", [16, 24])
def test_bad_pages_by_parts(av, page):
    """Numbers outside the pool in a prefix on the tensor cores: those tokens are masked."""
    w = World(av, "bf16", [40, 2], [4300, 130], [20] * 42, 8, 2, 64, page, seed=4)
    w.prefix.block_table[0, 1] = -1
    w.prefix.block_table[0, 100] = 1 << 20
    w.prefix.block_table[1, 0] = -5
    o, lse = w.run(status=7)

    def keys(b):
        g = w.group_of(b)
        gone = {c * page + i for c in ((1, 100) if g == 0 else (0,)) for i in range(page)}
        pre = [x[:, [j for j in range(w.pre[g]) if j not in gone]] for x in take(w.prefix, g, w.pre[g])]
        return [np.concatenate(x, 1) for x in zip(pre, take(w.cache, b, w.lens[b]))]

    w.check(o, lse, keys=keys, seqs=[0, 20, 39, 40, 41])


def test_steep_by_parts(av):
    """Logits that rise along the keys: the reference moves and O is rescaled."""
    t = _torch()
    w = World(av, "bf16", [50, 40], [4500, 4500], [10] * 90, 8, 2, 128, 16, std=1.0, seed=12)
    for g in range(2):
        place = t.arange(4500, device=DEV)
        pg = w.prefix.block_table[g].long()[place // 16]
        scale = (0.2 + 40.0 * (place % 1500) / 1500).to(t.bfloat16)[:, None, None]
        w.prefix.k_pages[pg, place % 16] = (w.prefix.k_pages[pg, place % 16] * scale)
    w.check(*w.run(), seqs=[0, 17, 49, 50, 89])


def test_refused_by_the_binding(av):
    t = _torch()
    w = World(av, "bf16", [2, 1], [20, 9], [3, 4, 5], 8, 2, 64, 16)
    f = World(av, "f32", [2, 1], [20, 9], [3, 4, 5], 8, 2, 64, 16)
    n = World(av, "bf16", [2, 1], [20, 9], [3, 4, 5], 8, 4, 64, 16)
    o, lse = w.outputs()

    def call(cache=w.cache, prefix=w.prefix, group=w.group, q=w.q, o=o, **kw):
        av.avits_cache_attention_shared(cache, prefix, group, q, w.scale, o, **kw)

    for bad in (dict(q=w.q[:2]), dict(o=o[:, :4]), dict(q=w.q[..., :32]), dict(group=w.group[:2]),
                dict(group=w.group.long()), dict(prefix=n.prefix), dict(lse=lse[:2]),
                dict(lse=lse.half()), dict(q=w.q.cpu()), dict(q=w.q.transpose(1, 2))):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(prefix=f.prefix), dict(q=f.q), dict(o=o.float())):
        with pytest.raises(TypeError):
            call(**bad)
    with pytest.raises(av.AvitsError):
        call(q=w.q[:, :7], o=o[:, :7])               # heads no multiple of Hkv
    with pytest.raises(av.AvitsError):
        call(o=o[:1].expand(3, 8, 64))
