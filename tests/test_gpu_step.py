"""GPU parity of the calls around the paged cache (plan of pages, norm and
rotation, append by slots) against the oracle (numpy fp64, plain loops).

Plans are whole numbers and exact, the memory that a call leaves alone included.
Rotation, from the arithmetic of the kernel, for a pair (a, b) after the norm:
  y       mean of d squares in fp32 (d 2^-24 relative, half of it in the root), rsqrt
          2^-22, three products 2^-24 each: e_y = (d / 2 + 12) 2^-24 of |y|
  angle   fp32 of half turns: 2^-25, times pi, one product more: 2^-22
  cos,sin bf16: 2^-21 by the fast functions in [-pi, pi] (documented 2^-21.41), fp32: 2 ulp,
          2^-23; times the magnitude m, 2^-24
  out     (|a| + |b|) m (e_y + 2^-22 + trig + 2^-23), two products and a sum, then one
          rounding: 2^-9 |out| (bf16), 2^-25 (fp32); held below with twice that.
"""
import threading

import numpy as np
import pytest

import oracle.step as os_

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def av():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2608_17995_gb300 as av
    av.build()
    av.lib()
    assert av.avits_device_status() == 0
    return av


def _torch():
    import torch
    return torch


def _dt(name):
    t = _torch()
    return t.bfloat16 if name == "bf16" else t.float32


# -------------------------------------------------------------------- plan --
class Pages:
    """The buffers of a plan, and the oracle's answer."""

    def __init__(self, av, lens, change, page, max_len, spare, T=None, seed=0, base=True, extra=0):
        t = _torch()
        rng = np.random.default_rng(seed)
        self.av, self.B = av, len(lens)
        cols = -(-max_len // page)
        used = [-(-min(max(n, 0), max_len) // page) for n in lens]
        self.pages = max(1, sum(used) + spare + extra)
        order = rng.permutation(self.pages).astype(np.int32)
        self.table = np.full((self.B, cols + 1), -7, np.int32)
        at = 0
        for b, n in enumerate(used):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.free = np.full(self.pages, -9, np.int32)
        self.free[:spare] = order[at:at + spare]
        self.spare, self.lens, self.change = spare, np.array(lens, np.int32), np.array(change, np.int32)
        rows = int(sum(max(c, 0) for c in change))
        self.T = rows + 3 if T is None else T
        self.base = rng.integers(0, 99, self.B).astype(np.int32) if base else None
        self.page, self.max_len = page, max_len
        kv = t.zeros(2, self.pages, page, 1, 8, dtype=t.bfloat16, device=DEV)
        self.d = {n: t.from_numpy(getattr(self, n).copy()).to(DEV) for n in ("table", "free", "lens",
                                                                            "change")}
        self.d["base"] = None if self.base is None else t.from_numpy(self.base).to(DEV)
        i32 = dict(dtype=t.int32, device=DEV)
        self.d["count"] = t.tensor([spare], **i32)
        self.d["cu"] = t.full((self.B + 1,), 77, **i32)
        self.d["slots"] = t.full((self.T,), 77, dtype=t.int64, device=DEV)
        for n in ("seq", "place", "pos"):
            self.d[n] = t.full((self.T,), 77, **i32)
        # one more column than the lengths can use: never touched
        self.cache = av.KVCache(kv[0], kv[1], self.d["table"], self.d["lens"], max_len=max_len)

    def call(self, **kw):
        d = self.d
        a = dict(pos=d["pos"], pos_base=d["base"])
        a.update(kw)
        self.av.avits_cache_plan(self.cache, d["change"], d["free"], d["count"], d["cu"], d["slots"],
                                 d["seq"], d["place"], **a)

    def check(self, bad=False):
        want = os_.cache_plan(self.lens.tolist(), self.change.tolist(), self.table.tolist(),
                              self.free.tolist(), self.spare, self.page, self.max_len, self.pages,
                              self.T, None if self.base is None else self.base.tolist())
        assert want["bad"] == bad
        assert self.av.avits_device_status() == (7 if bad else 0)
        for n in ("lens", "table", "free", "cu", "slots", "seq", "place", "pos"):
            assert np.array_equal(self.d[n].cpu().numpy(), want[n]), n
        assert self.d["count"].tolist() == [want["count"]]


def steps(B, max_len, seed, fresh=0.2):
    """Lengths and changes of all kinds: going on, new, cut, done, idle."""
    rng = np.random.default_rng(seed)
    lens, change = [], []
    for _ in range(B):
        n = int(rng.integers(0, max_len + 1))
        kind = rng.random()
        if kind < 0.4:
            c = min(1, max_len - n)
        elif kind < 0.5:
            c = 0
        elif kind < 0.5 + fresh:
            n, c = 0, int(rng.integers(1, max_len + 1))
        elif kind < 0.85:
            c = -int(rng.integers(1, 9))
        else:
            c = -n
        lens.append(n)
        change.append(c)
    return lens, change


@pytest.mark.parametrize("B,page,max_len", [
    (1, 16, 100), (7, 1, 9), (31, 8, 64), (256, 16, 513), (300, 24, 1000), (1024, 16, 40),
    (1025, 16, 40), (3000, 5, 33), (40, 128, 1 << 14), (3, 1 << 20, 5000)])
def test_plan(av, B, page, max_len):
    lens, change = steps(B, max_len, B + page)
    need = sum(max(0, -(-(n + c) // page) - -(-n // page)) for n, c in zip(lens, change) if c > 0)
    p = Pages(av, lens, change, page, max_len, need + 2, seed=B)
    p.call()
    p.check()


@pytest.mark.parametrize("T", [0, 1, 4096, 4097])
def test_plan_rows(av, T):
    """The step's rows end at T, before it, or behind it: those sequences stay."""
    change = [1, 3000, -2, 1090, 5, 0, 2]
    lens = [0, 17, 40, 0, 11, 3, 15]
    p = Pages(av, lens, change, 16, 4000, 400, T=T, seed=T)
    p.call()
    p.check(bad=T < 4101)


@pytest.mark.parametrize("spare,extra", [(0, 0), (1, 0), (3, 9), (7, 1)])
def test_plan_short_of_pages(av, spare, extra):
    lens, change = steps(90, 200, 5)
    p = Pages(av, lens, change, 16, 200, spare, extra=extra, seed=spare)
    p.call()
    p.check(bad=True)


@pytest.mark.parametrize("B,seed", [(3, 0), (700, 1), (2100, 2)])
def test_plan_many_rows(av, B, seed):
    """Rows that a kernel of their own writes, among long runs of sequences without any."""
    rng = np.random.default_rng(seed)
    lens, change = [0] * B, [0] * B
    for b in list(rng.integers(0, B, 40)) + [0, B - 1]:
        lens[b], change[b] = int(rng.integers(0, 50)), int(rng.integers(1, 900))
    lens[1], change[1] = 4000, -3900
    lens[B // 2], change[B // 2] = 5000, 9000
    p = Pages(av, lens, change, 16, 14000, 4000, seed=seed)
    assert p.T > 8192 + 3
    p.call()
    p.check()


def test_plan_many_rows_without_room(av):
    """The same where a prompt finds no pages: its rows are padding."""
    p = Pages(av, [0, 10, 0, 7], [9000, 1, 5000, 1], 16, 10000, 400, T=14010)
    p.call()
    p.check(bad=True)


def test_plan_takes_pages_given_back_behind(av):
    """The pages come from a sequence later in the batch; without positions."""
    p = Pages(av, [4, 12], [8, -12], 4, 12, 0, base=False)
    p.call()
    p.check()


@pytest.mark.parametrize("lens,change,max_len", [
    ([-1, 3], [1, 1], 8), ([9, 3], [-9, 1], 8), ([8, 3], [1, 1], 8), ([3, 2], [1 << 30, 1], 8),
    ([3, 2], [-(1 << 31), 1], 8), ([0, 0], [(1 << 31) - 1] * 2, 8)])
def test_plan_lengths_out_of_range(av, lens, change, max_len):
    p = Pages(av, lens, change, 4, max_len, 4, T=6)
    p.call()
    p.check(bad=not all(0 <= n <= max_len and n + c <= max_len for n, c in zip(lens, change)))


@pytest.mark.parametrize("count,want", [(-3, 0), (99, 4)])
def test_plan_count_out_of_range(av, count, want):
    p = Pages(av, [2, 0], [-2, 0], 4, 8, 3, T=2)
    p.d["count"].fill_(count)
    p.free[3:] = 0
    p.d["free"].copy_(_torch().from_numpy(p.free))
    p.spare = count
    p.call()
    p.check(bad=True)


def test_plan_pages_out_of_range(av):
    """A bad number in the list, and one in the table: rows without a slot."""
    p = Pages(av, [3, 6], [3, 1], 4, 8, 2)
    p.free[1] = 1000
    p.table[1, 1] = -1
    p.d["free"].copy_(_torch().from_numpy(p.free))
    p.d["table"].copy_(_torch().from_numpy(p.table))
    p.call()
    p.check(bad=True)


def test_plan_beside_other_outputs(av):
    """lens and count apart from the outputs: the call can be made again."""
    t = _torch()
    lens, change = steps(50, 300, 8)
    p = Pages(av, lens, change, 16, 300, 600, seed=3)
    old, out = p.d["lens"].clone(), t.zeros(1, dtype=t.int32, device=DEV)
    count = p.d["count"]
    for _ in range(3):
        p.d["lens"].fill_(5)
        p.call(lens=old, free_out=out)
    assert count.tolist() == [p.spare]
    p.d["count"] = out
    p.check()


def test_plan_in_a_graph(av):
    """A decoding loop's steps, replayed: lengths go on in place; and on a stream of its own."""
    t = _torch()
    p = Pages(av, [0, 5, 15], [1, 1, 1], 16, 64, 9, T=8)
    p.call()
    assert av.avits_device_status() == 0
    g = t.cuda.CUDAGraph()
    with t.cuda.graph(g):
        p.call()
    for _ in range(20):
        g.replay()
    t.cuda.synchronize()
    assert p.d["lens"].tolist() == [21, 26, 36] and p.d["count"].tolist() == [9 - 2 - 1 - 2]
    assert p.d["place"].tolist() == [20, 25, 35] + [-1] * 5
    owned = [p.d["table"][b, :-(-n // 16)].tolist() for b, n in enumerate(p.d["lens"].tolist())]
    left = p.d["free"][:4].tolist()
    assert len(set(sum(owned, left))) == 4 + 2 + 2 + 3
    side = t.cuda.Stream()
    p.call(stream=side)
    side.synchronize()
    assert p.d["lens"].tolist() == [22, 27, 37]


def test_plan_refused_by_the_binding(av):
    t = _torch()
    p = Pages(av, [1, 2], [1, 1], 4, 8, 4)
    d = p.d

    def call(**kw):
        a = dict(change=d["change"], free=d["free"], count=d["count"], cu=d["cu"], slots=d["slots"],
                 seq=d["seq"], place=d["place"])
        more = {n: kw.pop(n) for n in ("pos", "pos_base", "lens", "free_out") if n in kw}
        a.update(kw)
        av.avits_cache_plan(p.cache, *a.values(), **more)

    for bad in (dict(change=d["change"][:1]), dict(change=d["change"].long()), dict(cu=d["cu"][:2]),
                dict(free=d["free"][:1]), dict(slots=d["slots"].int()), dict(seq=d["seq"][1:]),
                dict(place=d["place"].cpu()), dict(pos=d["pos"][1:]), dict(pos_base=d["base"]),
                dict(pos=d["pos"], pos_base=d["base"][:1]), dict(lens=d["lens"][::2]),
                dict(free_out=t.zeros(2, dtype=t.int32, device=DEV))):
        with pytest.raises(ValueError):
            call(**bad)
    assert d["lens"].tolist() == [1, 2]


# ---------------------------------------------------------- norm, rotation --
def tolerance(want_a, dt, d, m, norm):
    """want_a: |a| + |b| of each value's pair."""
    e_y = (d / 2 + 12) * 2.0 ** -24 if norm else 0.0
    trig = 2.0 ** -21 if dt == "bf16" else 2.0 ** -23
    return 2 * want_a * m * (e_y + 2.0 ** -22 + trig + 2.0 ** -23)


def close(got, x, pos, freq, sections, inter, w, norm, m, dt, eps=1e-6):
    """got against the oracle's turn of x [..., heads, d]."""
    x = x.float().cpu().numpy()
    wn = None if w is None else w.float().cpu().numpy()
    a = (x, pos, freq, sections, inter, wn, norm, eps, m)
    want = os_.norm_rotate(*a)
    d, half = x.shape[-1], len(freq)
    y = np.abs(os_.norm_rotate(x, pos, freq * 0, sections, inter, wn, norm, eps, 1.0))
    size = y.copy()
    if inter:
        size[..., 0:2 * half:2] += y[..., 1:2 * half:2]
        size[..., 1:2 * half:2] += y[..., 0:2 * half:2]
    else:
        size[..., :half] += y[..., half:2 * half]
        size[..., half:2 * half] += y[..., :half]
    tol = tolerance(size, dt, d, max(1.0, m), norm)
    tol += 2 * (2.0 ** -9 if dt == "bf16" else 2.0 ** -25) * (np.abs(want) + tol) + 1e-38
    got = got.float().cpu().numpy()
    assert np.all(np.abs(got - want) <= tol), np.max(np.abs(got - want) / tol)


def data(dt, shape, seed):
    t = _torch()
    g = t.Generator(device=DEV)
    g.manual_seed(seed)
    return (3 * t.randn(*shape, device=DEV, generator=g)).to(_dt(dt))


ROTATIONS = [   # B, N, H, Hkv, d, rot, sections, interleaved
    (1, 1, 1, 0, 64, 64, None, False), (2, 5, 4, 2, 128, 128, None, False),
    (2, 5, 4, 2, 128, 128, None, True), (1, 33, 3, 3, 96, 48, None, False),
    (1, 33, 3, 3, 96, 48, None, True), (3, 7, 5, 1, 80, 20, None, False),
    (3, 7, 5, 1, 80, 20, None, True), (1, 9, 2, 1, 72, 36, None, False), (1, 9, 2, 2, 72, 72, None, True),
    (2, 3, 7, 2, 256, 256, None, False), (2, 3, 2, 2, 256, 2, None, True),
    (1, 50, 6, 6, 128, 128, [8, 28, 28], True), (2, 20, 4, 4, 64, 64, [16, 16], False),
    (1, 6, 2, 1, 64, 32, [0, 3, 13, 0], True), (1, 4, 2, 1, 8, 8, None, False), (1, 4, 2, 1, 16, 4, None, True),
    (1, 5, 40, 8, 64, 0, None, False), (1, 3000, 2, 1, 64, 32, None, False), (2, 77, 1, 1, 24, 10, None, False),
    # halves that are whole numbers of 8 and 4 bytes only, of none, and of rows too wide for those
    (2, 9, 5, 2, 72, 72, None, False), (1, 40, 3, 1, 72, 18, None, False), (3, 5, 2, 2, 96, 24, [4, 8], False),
    (1, 6, 3, 1, 256, 20, None, False), (1, 6, 3, 1, 256, 24, None, False), (2, 3, 17, 5, 248, 124, None, False)]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("case", ROTATIONS)
def test_norm_rotate(av, dt, case):
    t = _torch()
    B, N, H, Hkv, d, rot, sections, inter = case
    parts = sections or [rot // 2]
    freq = np.concatenate([os_.frequencies(2 * n, 10000.0) for n in parts if n] or [np.zeros(0)])
    rotary = av.Rotary(rot, sections=sections, interleaved=inter, magnitude=1.25)
    rng = np.random.default_rng(N)
    pos = rng.integers(-5, 200000, size=(B, N, len(parts))).astype(np.int32)
    q, k = data(dt, (B, N, H, d), 1), data(dt, (B, N, Hkv, d), 2) if Hkv else None
    wq, wk = data(dt, (d,), 3), data(dt, (d,), 4)
    p = t.from_numpy(pos).to(DEV)
    for norm, weights in ((True, True), (True, False), (False, False)):
        qo = t.full_like(q, 7)
        ko = None if k is None else t.full_like(k, 7)
        w = (wq, wk) if weights else (None, None)
        av.avits_norm_rotate(rotary, p, q, qo, k=k, k_out=ko, q_weight=w[0], k_weight=w[1], norm=norm)
        assert av.avits_device_status() == 0
        close(qo, q, pos, freq, parts, inter, w[0], norm, 1.25, dt)
        if Hkv:
            close(ko, k, pos, freq, parts, inter, w[1], norm, 1.25, dt)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
def test_rotate_far_positions(av, dt, inter):
    """At the integers' ends and with frequencies just below half a turn."""
    t = _torch()
    pos = np.array([2 ** 31 - 1, -2 ** 31, 10 ** 9 + 7, 16777217, 0], np.int32)
    freq = os_.frequencies(64, 500000.0)
    # fp64 has far positions' angles to p 2^-53: 2^-22 turns
    rotary = av.Rotary(64, base=500000.0, interleaved=inter)
    x = data(dt, (5, 3, 64), 9)
    out = t.empty_like(x)
    av.avits_norm_rotate(rotary, t.from_numpy(pos).to(DEV), x, out, norm=False)
    # the table's frequencies, exactly: whole numbers of 2^-64 turns, products in integers
    table = [int(v) % (1 << 64) for v in rotary.freq.tolist()]
    turns = np.array([[(f * int(p)) % (1 << 64) / 2.0 ** 64 for f in table] for p in pos])
    one = np.ones((5, 1))
    got = out.float().cpu().numpy()
    for i in range(32):
        a, b = (2 * i, 2 * i + 1) if inter else (i, i + 32)
        y = x[..., [a, b]].float().cpu().numpy().astype(np.float64)
        z = (y[..., 0] + 1j * y[..., 1]) * np.exp(2j * np.pi * turns[:, i:i + 1] * one)
        size = np.abs(y).sum(-1)
        for j, w in ((a, z.real), (b, z.imag)):
            tol = tolerance(size, dt, 64, 1.0, False)
            tol = tol + 2 * (2.0 ** -9 if dt == "bf16" else 2.0 ** -25) * (np.abs(w) + tol)
            assert np.all(np.abs(got[..., j] - w) <= tol)
    assert np.allclose([f / 2.0 ** 64 for f in table], freq / (2 * np.pi), rtol=1e-12, atol=2.0 ** -63)


def test_rotate_views(av):
    """Parts of a joint projection in place; outputs as the attention reads them, behind
    other rows that stay; positions shared by the batch; without a batch axis."""
    t = _torch()
    B, N, H, Hkv, d = 2, 11, 6, 2, 64
    x = data("bf16", (B, N, H + 2 * Hkv, d), 5)
    keep = x.clone()
    q, k = x[:, :, :H], x[:, :, H:H + Hkv]
    pos = t.arange(N, dtype=t.int32, device=DEV)
    freq, rotary = os_.frequencies(64, 10000.0), av.Rotary(64)
    out = t.full((B, H, N + 5, d), 7.0, dtype=t.bfloat16, device=DEV)
    av.avits_norm_rotate(rotary, pos, q, out.transpose(1, 2)[:, 5:])
    p3 = np.broadcast_to(np.arange(N)[None, :, None], (B, N, 1))
    close(out.transpose(1, 2)[:, 5:], q, p3, freq, [32], False, None, True, 1.0, "bf16")
    assert t.all(out[:, :, :5] == 7)
    av.avits_norm_rotate(rotary, pos[:, None], q, q, k=k, k_out=k)
    assert t.equal(x[:, :, :H], out.transpose(1, 2)[:, 5:])
    assert t.equal(x[:, :, H + Hkv:], keep[:, :, H + Hkv:])
    close(k, keep[:, :, H:H + Hkv], p3, freq, [32], False, None, True, 1.0, "bf16")
    alone = t.empty(N, H, d, dtype=t.bfloat16, device=DEV)
    av.avits_norm_rotate(rotary, pos, keep[1, :, :H], alone)
    assert t.equal(alone, x[1, :, :H])


def test_rotary_is_fixed(av):
    r = av.Rotary(64)
    with pytest.raises(AttributeError):
        r.freq = r.freq + 1


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rot,inter", [(32, False), (32, True), (36, False)])
def test_rotate_infinities_with_norm(av, dt, rot, inter):
    """A row with an infinity is NaN there and zero elsewhere, as the formula gives; the
    others do not see it."""
    t = _torch()
    x = data(dt, (3, 2, 72), 3)
    x[1, 0, 71] = float("inf")
    out = t.empty_like(x)
    av.avits_norm_rotate(av.Rotary(rot, interleaved=inter), t.tensor([3, 4, 5], dtype=t.int32, device=DEV),
                         x, out)
    assert t.isnan(out[1, 0, 71]) and not out[1, 0, :71].any()
    out[1, 0] = 0
    assert t.isfinite(out).all() and out[1, 1].any() and out[2].any()


def test_rotate_joint_ladder(av):
    """One ladder of frequencies whose parts turn by several axes."""
    t = _torch()
    rotary = av.Rotary(48, base=500.0, sections=[8, 16], joint=True, scaling="parts", factor=4.0,
                       original_len=100, low=1.0, high=8.0)
    x = data("f32", (1, 9, 3, 64), 1)
    pos = np.random.default_rng(0).integers(0, 50, size=(1, 9, 2)).astype(np.int32)
    out = t.empty_like(x)
    av.avits_norm_rotate(rotary, t.from_numpy(pos).to(DEV), x, out)
    freq = os_.frequencies(48, 500.0, "parts", 4.0, 100, 1.0, 8.0)
    close(out, x, pos, freq, [8, 16], False, None, True, 1.0, "f32")


def test_rotate_infinities_stay_in_their_pair(av):
    t = _torch()
    for inter in (False, True):
        for d, rot in ((64, 32), (72, 36)):
            x = data("f32", (2, 1, d), 3)
            x[0, 0, d - 1] = float("inf")            # of the rest
            x[1, 0, 0] = float("nan")                # of pair 0
            out = t.empty_like(x)
            av.avits_norm_rotate(av.Rotary(rot, interleaved=inter), t.tensor([3, 4], dtype=t.int32,
                                                                             device=DEV), x, out, norm=False)
            assert t.isfinite(out[0, 0, :d - 1]).all() and t.isinf(out[0, 0, d - 1])
            pair = [0, 1] if inter else [0, rot // 2]
            rest = [i for i in range(d) if i not in pair]
            assert t.isnan(out[1, 0, pair]).all() and t.isfinite(out[1, 0, rest]).all()


def test_rotate_refused_by_the_binding(av):
    t = _torch()
    r, r2 = av.Rotary(64), av.Rotary(64, sections=[16, 16])
    q, k = data("bf16", (2, 4, 3, 64), 1), data("bf16", (2, 4, 1, 64), 2)
    p, o, ko = t.zeros(2, 4, dtype=t.int32, device=DEV), t.empty_like(q), t.empty_like(k)
    w = t.ones(64, dtype=t.bfloat16, device=DEV)
    bad = [lambda: av.avits_norm_rotate(r, p[:, :3], q, o), lambda: av.avits_norm_rotate(r, p.long(), q, o),
           lambda: av.avits_norm_rotate(r, None, q, o), lambda: av.avits_norm_rotate(r2, p, q, o),
           lambda: av.avits_norm_rotate(r2, t.zeros(2, 4, 4, dtype=t.int32, device=DEV)[..., ::2], q, o),
           lambda: av.avits_norm_rotate(r, p, q, o[:1]), lambda: av.avits_norm_rotate(r, p, q, o, k=k),
           lambda: av.avits_norm_rotate(r, p, q, o, k=k[:, :3], k_out=ko[:, :3]),
           lambda: av.avits_norm_rotate(r, p, q, o, q_weight=w[:32]),
           lambda: av.avits_norm_rotate(r, p, q, o, q_weight=w.float()),
           lambda: av.avits_norm_rotate(r, p, q[0, 0], o[0, 0]),
           lambda: av.avits_norm_rotate(r, p, q.cpu(), o),
           lambda: av.avits_norm_rotate(r, p, q.transpose(2, 3), o.transpose(2, 3))]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: av.avits_norm_rotate(r, p, q, o.float()),
              lambda: av.avits_norm_rotate(r, p, q.half(), o.half()),
              lambda: av.avits_norm_rotate(r, p, q, o, k=k.float(), k_out=ko)):
        with pytest.raises(TypeError):
            f()
    with pytest.raises(av.AvitsError):       # rows over one another
        av.avits_norm_rotate(r, p, q, o[:1].expand(2, 4, 3, 64))
    with pytest.raises(av.AvitsError):       # head offsets of no 16 bytes
        av.avits_norm_rotate(av.Rotary(4), p, q[..., 4:12], o[..., 4:12])


# ------------------------------------------------------------------ append --
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["tokens", "heads", "joint"])
@pytest.mark.parametrize("T,H,Hkv,d,page,rot,inter", [
    (1, 8, 2, 128, 16, 128, False), (37, 6, 3, 96, 24, 48, True), (500, 4, 4, 64, 8, 20, False),
    (3, 24, 24, 256, 5, 256, False), (64, 3, 1, 72, 16, 72, True)])
def test_append(av, dt, layout, T, H, Hkv, d, page, rot, inter):
    from test_gpu_cache import make_pool
    t = _torch()
    pages = -(-T // page) + 3
    k, v = make_pool(layout, pages, page, Hkv, d, _dt(dt), fill=7.0)
    rng = np.random.default_rng(T)
    slot = rng.permutation(pages * page)[:T].astype(np.int64)
    slot[T // 2] = slot[T // 2] if T < 3 else -1 - T // 2          # padding
    seq, place = np.arange(T) % 2, np.arange(T) // 2
    acc = t.full((2, Hkv, T + 4), 5.0, device=DEV)
    table = t.zeros(2, pages, dtype=t.int32, device=DEV)
    cache = av.KVCache(k, v, table, t.zeros(2, dtype=t.int32, device=DEV), acc=acc,
                       max_len=min(T + 4, pages * page))
    q, kn, vn = data(dt, (T, H, d), 1), data(dt, (T, Hkv, d), 2), data(dt, (T, Hkv, d), 3)
    w = data(dt, (d,), 4)
    pos = rng.integers(0, 5000, size=(T, 1)).astype(np.int32)
    out = t.full_like(q, 9)
    put = lambda a: t.from_numpy(a).to(DEV)
    av.avits_cache_append_rotated(cache, av.Rotary(rot, interleaved=inter), put(pos), put(slot), q, out, kn,
                                  vn, k_weight=w, seq=put(seq.astype(np.int32)),
                                  place=put(place.astype(np.int32)))
    assert av.avits_device_status() == 0
    freq, live = os_.frequencies(rot, 10000.0), slot >= 0
    lt = put(live)
    close(out[lt], q[lt], pos[live], freq, [rot // 2], inter, None, True, 1.0, dt)
    assert t.all(out[~lt] == 9)
    rows = put(slot[live])
    close(k[rows // page, rows % page], kn[lt], pos[live], freq, [rot // 2], inter, w, True, 1.0, dt)
    assert t.equal(v[rows // page, rows % page], vn[lt])
    other = t.ones(pages * page, dtype=t.bool, device=DEV)
    other[rows] = False
    idx = other.nonzero()[:, 0]
    for pool in (k, v):
        assert t.all(pool[idx // page, idx % page] == 7)
    want = np.full((2, Hkv, T + 4), 5.0, np.float32)
    want[seq[live], :, place[live]] = 0
    assert np.array_equal(acc.cpu().numpy(), want)


def test_append_bad_slots(av):
    """A slot past the pool, and a token out of acc: nothing of it is written there."""
    t = _torch()
    kv = t.full((2, 3, 4, 1, 8), 7.0, device=DEV)
    acc = t.full((1, 1, 12), 5.0, device=DEV)
    lens = t.zeros(1, dtype=t.int32, device=DEV)
    cache = av.KVCache(kv[0], kv[1], t.zeros(1, 3, dtype=t.int32, device=DEV), lens, acc=acc)
    x = t.ones(3, 1, 8, device=DEV)
    i32 = lambda *a: t.tensor(a, dtype=t.int32, device=DEV)
    out = t.zeros_like(x)
    args = (av.Rotary(0), None, t.tensor([12, 1, 1 << 40], device=DEV), x, out, x, x)
    av.avits_cache_append_rotated(cache, *args, norm=False, seq=i32(0, 0, 0), place=i32(2, 3, 4))
    assert av.avits_device_status() == 7
    assert out[:, 0, 0].tolist() == [0, 1, 0] and kv[:, 0, 1].eq(1).all() and kv.eq(1).sum() == 16
    assert acc[0, 0].tolist() == [5, 5, 5, 0] + [5] * 8
    av.avits_cache_append_rotated(cache, *args[:2], t.tensor([0, 1, 2], device=DEV), *args[3:], norm=False,
                                  seq=i32(0, 1, -1), place=i32(12, 0, 0))
    assert av.avits_device_status() == 7
    assert acc[0, 0].tolist() == [5, 5, 5, 0] + [5] * 8 and kv[:, 0, :3].eq(1).all()


def test_append_slots_past_32_bits(av):
    """Pages so many and large that slots pass 2^31: 2.1e9 places of one narrow head."""
    t = _torch()
    page, pages = 1 << 20, 2050
    kv = t.empty(2, pages, page, 1, 8, dtype=t.bfloat16, device=DEV)      # 69 GB
    lens = t.zeros(1, dtype=t.int32, device=DEV)
    cache = av.KVCache(kv[0], kv[1], t.zeros(1, 1, dtype=t.int32, device=DEV), lens)
    last = pages * page - 1
    slots = t.tensor([last, 0, last - page], device=DEV)
    x = data("bf16", (3, 1, 8), 1)
    out = t.empty_like(x)
    av.avits_cache_append_rotated(cache, av.Rotary(0), None, slots, x, out, x, x, norm=False)
    assert av.avits_device_status() == 0
    for i, s in enumerate(slots.tolist()):
        assert t.equal(kv[:, s // page, s % page], x[i].expand(2, 1, 8))
    assert t.equal(out, x)


def test_append_refused_by_the_binding(av):
    t = _torch()
    kv = t.zeros(2, 3, 4, 2, 64, dtype=t.bfloat16, device=DEV)
    lens, table = t.zeros(1, dtype=t.int32, device=DEV), t.zeros(1, 3, dtype=t.int32, device=DEV)
    plain = av.KVCache(kv[0], kv[1], table, lens)
    weighed = av.KVCache(kv[0], kv[1], table, lens, acc=t.zeros(1, 2, 12, device=DEV))
    q, x = data("bf16", (5, 4, 64), 1), data("bf16", (5, 2, 64), 2)
    o, slots, pos = t.empty_like(q), t.zeros(5, dtype=t.int64, device=DEV), t.zeros(5, dtype=t.int32,
                                                                                  device=DEV)
    r = av.Rotary(64)

    def call(cache=plain, rotary=r, pos=pos, slots=slots, q=q, o=o, k=x, v=x, **kw):
        av.avits_cache_append_rotated(cache, rotary, pos, slots, q, o, k, v, **kw)

    for bad in (dict(q=q[:4]), dict(o=o[..., :32]), dict(k=x[:, :1]), dict(v=x[:4]), dict(slots=slots.int()),
                dict(slots=slots[:4]), dict(pos=pos[:4]), dict(pos=pos.long()), dict(cache=weighed),
                dict(cache=weighed, seq=pos), dict(seq=pos, place=pos.long()), dict(q=q.cpu()),
                dict(q_weight=pos)):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(TypeError):
        call(k=x.float())
    with pytest.raises(av.AvitsError):
        call(norm=False, q_weight=t.ones(64, dtype=t.bfloat16, device=DEV))


def test_step_of_a_batch(av):
    """Plan, append by its slots and the attention over the result, on a stream of its
    own and as a replayed graph, against the plain append of the same tokens."""
    t = _torch()
    B, H, Hkv, d, page, max_len = 5, 8, 2, 64, 16, 96
    lens0 = [0, 15, 16, 40, 60]
    rng = np.random.default_rng(0)
    pages = 64
    order = rng.permutation(pages).astype(np.int32)
    table = np.full((B, 6), -1, np.int32)
    at = 0
    for b, n in enumerate(lens0):
        table[b, :-(-n // page)] = order[at:at - (-n // page)]
        at += -(-n // page)
    kv = data("bf16", (2, pages, page, Hkv, d), 1)
    plain_kv = kv.clone()
    i32 = dict(dtype=t.int32, device=DEV)
    put = lambda a: t.from_numpy(np.ascontiguousarray(a)).to(DEV)
    lens, tab = t.tensor(lens0, **i32), put(table)
    free = t.zeros(pages, **i32)
    free[:pages - at] = put(order[at:])
    count = t.tensor([pages - at], **i32)
    change = t.tensor([3, 1, 1, -40, 1], **i32)
    cu, T = t.zeros(B + 1, **i32), 8
    slots = t.zeros(T, dtype=t.int64, device=DEV)
    seq, place = t.zeros(T, **i32), t.zeros(T, **i32)
    cache = av.KVCache(kv[0], kv[1], tab, lens, max_len=max_len)
    q, k, v = data("bf16", (T, H, d), 2), data("bf16", (T, Hkv, d), 3), data("bf16", (T, Hkv, d), 4)
    qo, rotary = t.zeros_like(q), av.Rotary(64)
    o, rows = t.zeros(B, H, d, dtype=t.bfloat16, device=DEV), t.tensor([2, 3, 4, 0, 5], device=DEV)
    keep = [x.clone() for x in (lens, tab, free, count)]

    def step():
        av.avits_cache_plan(cache, change, free, count, cu, slots, seq, place)
        av.avits_cache_append_rotated(cache, rotary, place, slots, q, qo, k, v)
        av.avits_cache_attention(cache, qo[rows], 0.125, o)

    step()
    assert av.avits_device_status() == 0
    n = lens.tolist()
    assert n == [3, 16, 17, 0, 61]
    first = o.clone()
    # the same by the other calls: rotated rows, appended by lengths
    ko = t.empty_like(k)
    av.avits_norm_rotate(rotary, place, q, t.empty_like(q), k=k, k_out=ko)
    twin = av.KVCache(plain_kv[0], plain_kv[1], tab, lens, max_len=max_len)
    av.avits_cache_append(twin, ko, v, cu)
    o2 = t.zeros_like(o)
    av.avits_cache_attention(twin, qo[rows], 0.125, o2)
    assert av.avits_device_status() == 0 and t.equal(first, o2) and t.equal(kv, plain_kv)
    for x, y in zip((lens, tab, free, count), keep):
        x.copy_(y)
    g = t.cuda.CUDAGraph()
    with t.cuda.graph(g):
        step()
    o.zero_()
    g.replay()
    t.cuda.synchronize()
    assert t.equal(o, first) and lens.tolist() == n and av.avits_device_status() == 0


def test_threads_and_streams(av):
    """Calls from several threads on streams of their own give what one gives."""
    t = _torch()
    x, rotary = data("bf16", (700, 4, 64), 1), av.Rotary(64)
    pos = t.arange(700, dtype=t.int32, device=DEV)
    want = t.empty_like(x)
    av.avits_norm_rotate(rotary, pos, x, want)
    t.cuda.synchronize()
    outs = [t.zeros_like(x) for _ in range(4)]
    streams = [t.cuda.Stream() for _ in outs]
    t.cuda.synchronize()

    def work(o, s):
        for _ in range(10):
            av.avits_norm_rotate(rotary, pos, x, o, stream=s)

    threads = [threading.Thread(target=work, args=a) for a in zip(outs, streams)]
    [h.start() for h in threads]
    [h.join() for h in threads]
    t.cuda.synchronize()
    assert all(t.equal(o, want) for o in outs)
