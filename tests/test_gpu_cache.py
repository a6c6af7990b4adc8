"""GPU parity of the paged key-value cache's operators against the oracle
(numpy fp64, one sequence at a time).

Tolerances, from the arithmetic of the kernels.  With X the largest
scale * sum_i |q_i k_i| of a call, n the largest length and d the head width:
  logits  fp32 sums of d products: |dx| <= X (d + 4) 2^-23 (a tensor-core sum
          may cut instead of round, hence a whole step per addition), times
          log2(e) and back, two more roundings of x: X 2^-22.
  lse     dx, a sum of n positive terms in fp32 (n 2^-24 relative, ex2 adds
          2^-22) and the final log: 2^-22 (1 + |lse|).
  weights eps = 2 dx + n 2^-23 + 2^-21 relative (numerator and lse).
  o       eps sum_j w_j |v_j|, 2^-17 of the same for the bf16 weights in two
          parts (8 + 8 bits and a sign), and the sum over j, n 2^-23 of it;
          then one rounding to the type: 2^-8 |o| (bf16), 2^-24 |o| (fp32).
  acc     eps w, and one fp32 addition: 2^-24 (|acc| + w).
Everything copied (pages, kept weights, places) is exact.
"""
import math
import threading

import numpy as np
import pytest

import oracle.cache as oc

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


def make_pool(layout, pages, page, Hkv, d, dt, fill=float("nan")):
    t = _torch()
    if layout == "tokens":
        return [t.full((pages, page, Hkv, d), fill, dtype=dt, device=DEV) for _ in range(2)]
    if layout == "heads":
        return [t.full((pages, Hkv, page, d), fill, dtype=dt, device=DEV).transpose(1, 2)
                for _ in range(2)]
    both = t.full((pages, 2, page, Hkv, d), fill, dtype=dt, device=DEV)
    return [both[:, 0], both[:, 1]]


class World:
    """A cache with NaN wherever no token lies, its contents on the host, and
    the queries.  Two pages belong to nobody."""

    def __init__(self, av, dtype, lens, H, Hkv, d, page, layout="tokens", seed=0, max_len=None,
                 std=2.0, acc=True):
        t = _torch()
        rng = np.random.default_rng(seed)
        self.av, self.dtype, self.lens_l, self.H, self.Hkv, self.d = av, dtype, list(lens), H, Hkv, d
        self.page, self.B = page, len(lens)
        dt = _dt(dtype)
        self.max_len = max_len or max(max(lens), 1)
        used = [-(-n // page) for n in lens]
        order = rng.permutation(sum(used) + 2)
        table = np.full((self.B, -(-self.max_len // page)), -1, np.int32)
        at = 0
        for b, n in enumerate(used):
            table[b, :n] = order[at:at + n]
            at += n
        self.k_pages, self.v_pages = make_pool(layout, len(order), page, Hkv, d, dt)
        g = t.Generator(device=DEV)
        g.manual_seed(seed)
        for b, n in enumerate(lens):
            if n == 0:
                continue
            place = t.arange(n, device=DEV)
            p = t.from_numpy(table[b].astype(np.int64)).to(DEV)[place // page]
            for pool in (self.k_pages, self.v_pages):
                pool[p, place % page] = t.randn(n, Hkv, d, device=DEV, generator=g).to(dt)
        self.table = t.from_numpy(table).to(DEV)
        self.lens = t.tensor(lens, dtype=t.int32, device=DEV)
        self.acc = t.rand(self.B, Hkv, self.max_len, device=DEV, generator=g) if acc else None
        self.q = (std * t.randn(self.B, H, d, device=DEV, generator=g)).to(dt)
        self.scale = 1.0 / math.sqrt(d)
        self.cache = av.KVCache(self.k_pages, self.v_pages, self.table, self.lens, acc=self.acc,
                                max_len=self.max_len)

    def rows(self, b, n=None):
        n = self.lens_l[b] if n is None else n
        tab = self.table[b].cpu().numpy()
        return [oc.pages_to_rows(p.float().cpu().numpy(), tab, n) for p in (self.k_pages, self.v_pages)]

    def outputs(self):
        t = _torch()
        return (t.full((self.B, self.H, self.d), 7.0, dtype=_dt(self.dtype), device=DEV),
                t.full((self.B, self.H), 7.0, device=DEV))

    def check(self, o, lse, acc0=None, weight=None, accumulate=True, lens=None):
        d, eps_t = self.d, 2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -24
        lens = self.lens_l if lens is None else lens
        q = self.q.float().cpu().numpy().astype(np.float64)
        got_o, got_l = o.float().cpu().numpy(), None if lse is None else lse.cpu().numpy()
        got_a = None if weight is None else self.acc.cpu().numpy()
        for b, n in enumerate(lens):
            k, v = self.rows(b, n)
            want, wl, w = oc.cache_attention(q[b], k, v, self.scale)
            if n == 0:
                assert not got_o[b].any(), b
                assert got_l is None or np.all(np.isneginf(got_l[b])), b
            else:
                G = self.H // self.Hkv
                X = self.scale * np.max(np.einsum("hgd,hnd->hgn", np.abs(q[b]).reshape(self.Hkv, G, d),
                                                  np.abs(k).astype(np.float64)))
                dx = X * (d + 8) * 2.0 ** -23
                eps = 2 * dx + n * 2.0 ** -23 + 2.0 ** -21
                av, _, _ = oc.cache_attention(q[b], k, np.abs(v), self.scale)
                tol = (eps + n * 2.0 ** -23 + (2.0 ** -17 if self.dtype == "bf16" else 0)) * av
                tol = tol + eps_t * (np.abs(want) + tol) + 1e-30
                assert np.all(np.abs(got_o[b] - want) <= tol), (b, np.max(np.abs(got_o[b] - want) / tol))
                if got_l is not None:
                    assert np.all(np.abs(got_l[b] - wl) <= dx + n * 2.0 ** -23 +
                                  2.0 ** -22 * (1 + np.abs(wl))), b
            if weight is not None:
                old = acc0[b] if accumulate else np.zeros_like(acc0[b])
                if n:
                    ref = old[:, :n] + weight * w
                    tol = eps * weight * w + 2.0 ** -23 * (np.abs(old[:, :n]) + weight * w) + 1e-30
                    assert np.all(np.abs(got_a[b, :, :n] - ref) <= tol), b
                assert np.array_equal(got_a[b, :, n:], acc0[b][:, n:]), b   # left as they were


def run_attention(w, weight=None, accumulate=True, lse=True, **kw):
    o, l = w.outputs()
    w.av.avits_cache_attention(w.cache, w.q, w.scale, o, lse=l if lse else None, weight=weight,
                               accumulate=accumulate, **kw)
    assert w.av.avits_device_status() == 0
    return o, l if lse else None


SHAPES = [  # dtype, lens, H, Hkv, d, page, layout
    ("bf16", [1], 1, 1, 64, 16, "tokens"),
    ("bf16", [517], 24, 8, 128, 16, "tokens"),
    ("bf16", [0, 1, 15, 16, 17, 31, 32, 33, 64, 65, 0], 6, 2, 64, 16, "heads"),
    ("bf16", [300, 1, 0, 129], 14, 2, 128, 24, "joint"),        # G 7, pages of 24
    ("bf16", [100, 63], 9, 1, 80, 8, "tokens"),                 # G 9: two row tiles
    ("bf16", [100, 250], 32, 2, 96, 1, "heads"),                # G 16, pages of one token
    ("bf16", [77, 400], 24, 1, 256, 3, "tokens"),               # G 24, pages of 3
    ("bf16", [90], 35, 1, 8, 16, "tokens"),                     # G 35: two groups of rows
    ("bf16", [40, 70], 200, 2, 136, 7, "joint"),                # G 100
    ("bf16", [33] * 70, 4, 4, 64, 32, "tokens"),                # one head each, G 1
    ("bf16", [5000, 12, 1900], 16, 4, 128, 64, "heads"),
    ("bf16", [50, 0, 300], 256, 1, 64, 16, "tokens"),           # the largest group
    ("bf16", [5, 999, 1001], 8, 2, 128, 1000, "heads"),         # long pages
    ("f32", [1], 2, 2, 4, 16, "tokens"),
    ("f32", [50, 131], 256, 1, 128, 8, "joint"),
    ("f32", [0, 1, 15, 16, 17, 33], 6, 2, 64, 16, "heads"),
    ("f32", [300, 129], 14, 2, 128, 24, "joint"),
    ("f32", [100, 250], 16, 1, 100, 5, "tokens"),
    ("f32", [77, 400], 24, 1, 256, 3, "heads"),
    ("f32", [40, 70], 80, 1, 200, 8, "tokens"),                 # G 80: three groups of rows
    ("f32", [2000, 1], 4, 4, 96, 16, "joint"),
]


@pytest.mark.parametrize("bound", [None, 6000])      # of the lengths: one launch, or two
@pytest.mark.parametrize("score", [False, True])
@pytest.mark.parametrize("dtype,lens,H,Hkv,d,page,layout", SHAPES)
def test_attention(av, dtype, lens, H, Hkv, d, page, layout, score, bound):
    w = World(av, dtype, lens, H, Hkv, d, page, layout, seed=len(lens) + H + d, max_len=bound)
    assert bound is None or av.avits_cache_attention_workspace(w.cache, H, score) > 0
    acc0 = w.acc.cpu().numpy()
    o, lse = run_attention(w, weight=0.75 if score else None)
    w.check(o, lse, acc0, 0.75 if score else None)
    if not score:
        assert np.array_equal(w.acc.cpu().numpy(), acc0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_one_long_sequence(av, dtype):
    """Split over all SMs and joined."""
    w = World(av, dtype, [70001], 4, 1, 64, 16, seed=1)
    acc0 = w.acc.cpu().numpy()
    o, lse = run_attention(w, weight=1.0)
    w.check(o, lse, acc0, 1.0)


@pytest.mark.parametrize("bound", [None, 6000])
def test_attention_more_sequences_than_threads(av, bound):
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 90, 333).tolist()
    w = World(av, "bf16", lens, 4, 2, 64, 16, "heads", seed=5, max_len=bound)
    acc0 = w.acc.cpu().numpy()
    o, lse = run_attention(w, weight=1.0)
    w.check(o, lse, acc0, 1.0)


@pytest.mark.parametrize("dtype,H", [("bf16", 8), ("bf16", 64), ("f32", 8)])
def test_attention_one_long_among_many_short(av, dtype, H):
    """Many units, one of them in more pieces than the others have keys."""
    w = World(av, dtype, [50] * 60 + [20011] + [7] * 60, H, 2, 64, 16, seed=12)
    acc0 = w.acc.cpu().numpy()
    o, lse = run_attention(w, weight=1.0)
    w.check(o, lse, acc0, 1.0)


def test_attention_pages_that_share_memory(av):
    """A stride of zero between pages (every page the same one): no TMA map has
    it, the rows come by 16-byte copies."""
    t = _torch()
    w = World(av, "bf16", [100, 40], 4, 2, 64, 16, seed=13)
    for i in range(2):
        n = w.lens_l[i]
        w.table[i, :-(-n // 16)] = w.table[0, 0]
    k, v = (p[int(w.table[0, 0])][None].expand(w.k_pages.shape) for p in (w.k_pages, w.v_pages))
    flat = av.KVCache(k, v, w.table, w.lens, acc=w.acc, max_len=w.max_len)
    (oa, la), (ob, lb) = w.outputs(), w.outputs()
    av.avits_cache_attention(flat, w.q, w.scale, oa, lse=la)
    av.avits_cache_attention(w.cache, w.q, w.scale, ob, lse=lb)
    assert av.avits_device_status() == 0
    w.check(oa, la)
    assert t.equal(oa, ob) and t.equal(la, lb)      # the same products in the same order


@pytest.mark.parametrize("bound", [None, 6000])
def test_calls_in_a_row_without_waiting(av, bound):
    """append -> attention -> eviction -> attention, each reading what the one
    before wrote, many times over: the bits of a run that waits each time."""
    t = _torch()
    B, H, Hkv, d, page, keep = 3, 8, 2, 64, 16, 40
    lens = [90, 33, 64]

    def run(wait):
        w = World(av, "bf16", lens, H, Hkv, d, page, seed=14, max_len=bound)
        g = t.Generator(device=DEV)
        g.manual_seed(15)
        k2, v2 = make_pool("tokens", B * 3, page, Hkv, d, t.bfloat16, fill=0.0)
        dst = av.KVCache(k2, v2, t.arange(B * 3, dtype=t.int32, device=DEV).view(B, 3),
                         t.zeros(B, dtype=t.int32, device=DEV),
                         acc=t.zeros(B, Hkv, 48, device=DEV), max_len=48)
        cu = t.arange(B + 1, dtype=t.int32, device=DEV)
        kn = t.randn(20, B, Hkv, d, device=DEV, generator=g).bfloat16()
        idx = t.empty(B, Hkv, keep, dtype=t.int32, device=DEV)
        q = w.q
        out = []
        for r in range(20):
            o, o2 = t.empty_like(q), t.empty_like(q)
            av.avits_cache_append(w.cache, kn[r], kn[19 - r], cu)
            if wait:
                t.cuda.synchronize()
            av.avits_cache_attention(w.cache, q, w.scale, o, weight=1.0)
            if wait:
                t.cuda.synchronize()
            av.avits_cache_evict(w.cache, dst, keep, 4, 8, idx)
            if wait:
                t.cuda.synchronize()
            av.avits_cache_attention(dst, q, w.scale, o2, weight=1.0)
            if wait:
                t.cuda.synchronize()
            out += [o, o2, idx.clone(), dst.acc.clone(), w.acc.clone()]
        t.cuda.synchronize()
        return out

    for a, b in zip(run(True), run(False)):
        assert t.equal(a, b)
    assert av.avits_device_status() == 0


def test_attention_no_token_at_all(av):
    w = World(av, "bf16", [0, 0, 0], 4, 2, 64, 16, max_len=50)
    acc0 = w.acc.cpu().numpy()
    o, lse = run_attention(w, weight=1.0)
    w.check(o, lse, acc0, 1.0)


def test_attention_weights_written(av):
    """accumulate=False: below the length the old weight is gone, past it kept."""
    w = World(av, "bf16", [100, 0, 31], 8, 2, 64, 16, max_len=200)
    acc0 = w.acc.cpu().numpy()
    o, lse = run_attention(w, weight=2.0, accumulate=False, lse=False)
    w.check(o, None, acc0, 2.0, accumulate=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_steep_logits(av, dtype):
    """Logits of some hundreds: one key takes all, the running maximum moves."""
    w = World(av, dtype, [700, 90], 8, 2, 128, 16, std=300.0, seed=9)
    acc0 = w.acc.cpu().numpy()
    o, lse = run_attention(w, weight=1.0)
    assert np.isfinite(o.float().cpu().numpy()).all()
    w.check(o, lse, acc0, 1.0)


def test_attention_nan_and_infinite_inputs(av):
    """A NaN value reaches the outputs of its own head and sequence only; an
    infinite value where the weight is not zero does."""
    t = _torch()
    w = World(av, "bf16", [40, 40], 4, 2, 64, 16, seed=2)
    o0, l0 = run_attention(w)
    p = int(w.table[0, 1])
    w.k_pages[p, 3, 1, 5] = float("nan")
    o, lse = run_attention(w, weight=1.0)
    assert t.isnan(o[0, 2:]).all() and t.isnan(lse[0, 2:]).all()
    assert t.equal(o[0, :2], o0[0, :2]) and t.equal(o[1], o0[1])
    assert t.isnan(w.acc[0, 1, :40]).all() and not t.isnan(w.acc[0, 0]).any()
    w.k_pages[p, 3, 1, 5] = 0.0
    w.v_pages[p, 3, 1, 5] = float("inf")
    o, lse = run_attention(w)
    assert t.isinf(o[0, 2:, 5]).all() and t.isfinite(o[0, 2:, :5]).all()
    w.q[1] = float("nan")
    o, lse = run_attention(w)
    assert t.isnan(o[1]).all() and t.isnan(lse[1]).all() and t.isfinite(o[0, :2]).all()


def test_attention_nan_over_a_split_row(av):
    """Every logit NaN in a row whose pieces are joined."""
    t = _torch()
    w = World(av, "bf16", [9000], 4, 1, 64, 16, seed=2)
    w.q[0, 1] = float("nan")
    o, lse = run_attention(w, weight=1.0)
    assert t.isnan(o[0, 1]).all() and t.isnan(lse[0, 1])
    assert t.isfinite(o[0, [0, 2, 3]]).all() and t.isnan(w.acc[0, 0]).all()


def test_attention_strided_queries_and_outputs(av):
    t = _torch()
    w = World(av, "bf16", [100, 37], 8, 2, 64, 16, seed=3)
    wide = t.zeros(2, 8, 3 * 64 + 3, dtype=t.bfloat16, device=DEV)
    wide[..., 65:129] = w.q
    w.q = wide[..., 65:129]                      # odd offset, a fused projection's view
    out = t.full((8, 2, 70), 7.0, dtype=t.bfloat16, device=DEV)
    o = out.transpose(0, 1)[..., 3:67]
    lse = t.empty(2, 8, device=DEV)
    av.avits_cache_attention(w.cache, w.q, w.scale, o, lse=lse)
    assert av.avits_device_status() == 0
    w.check(o, lse)
    assert (out[..., :3] == 7).all() and (out[..., 67:] == 7).all()


def test_attention_same_bits_again(av):
    w = World(av, "bf16", [3000, 100, 0, 900], 16, 2, 128, 16, seed=4)
    acc0 = w.acc.clone()
    o, lse = run_attention(w, weight=1.0)
    acc1 = w.acc.clone()
    for _ in range(3):
        w.acc.copy_(acc0)
        o2, lse2 = run_attention(w, weight=1.0)
        t = _torch()
        assert t.equal(o, o2) and t.equal(lse, lse2) and t.equal(acc1, w.acc)


def test_attention_shared_pages(av):
    """Sequences of one common prompt: the same pages in several rows."""
    w = World(av, "bf16", [64, 64, 64], 8, 2, 64, 16, seed=6)
    w.table[1] = w.table[0]
    w.table[2, :2] = w.table[0, :2]
    acc0 = w.acc.cpu().numpy()
    o, lse = run_attention(w, weight=1.0)
    w.check(o, lse, acc0, 1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_pages_out_of_range(av, dtype):
    """A page number outside the pool: reported, its tokens are as masked and
    the other sequences are right."""
    t = _torch()
    w = World(av, dtype, [48, 40, 20], 4, 2, 64, 16, seed=7)
    good = w.table.clone()
    w.table[0, 1] = w.k_pages.shape[0]
    w.table[2, :] = -5
    w.acc.zero_()
    o, lse = w.outputs()
    av.avits_cache_attention(w.cache, w.q, w.scale, o, lse=lse, weight=1.0)
    assert av.avits_device_status() == 7
    assert av.avits_device_status() == 0
    assert not o[2].any() and t.isneginf(lse[2]).all() and not w.acc[2].any()
    assert not w.acc[0, :, 16:32].any()
    w.table.copy_(good)
    k, v = w.rows(0)
    some = np.r_[0:16, 32:48]
    want, wl, _ = oc.cache_attention(w.q[0].float().cpu().numpy(), k[:, some], v[:, some], w.scale)
    assert np.allclose(o[0].float().cpu().numpy(), want, rtol=1e-2, atol=1e-2)
    assert np.allclose(lse[0].cpu().numpy(), wl, atol=1e-4)
    w.lens_l = [0, 40, 0]
    q = w.q.clone()
    w.check(t.where(t.tensor([False, True, False], device=DEV)[:, None, None], o, 0),
            t.where(t.tensor([False, True, False], device=DEV)[:, None], lse, -math.inf))
    assert t.equal(q, w.q)


def test_attention_length_out_of_range(av):
    """Lengths outside [0, max_len] are cut to it and reported."""
    w = World(av, "bf16", [48, 40], 4, 2, 64, 16, seed=8, max_len=48)
    w.lens.copy_(_torch().tensor([1000, -3], dtype=_torch().int32))
    o, lse = w.outputs()
    acc0 = w.acc.cpu().numpy()
    av.avits_cache_attention(w.cache, w.q, w.scale, o, lse=lse, weight=1.0)
    assert av.avits_device_status() == 7
    w.check(o, lse, acc0, 1.0, lens=[48, 0])


def far_pool(pages, page, Hkv, d, dt, stride):
    """Pages whose distance in memory passes 2^31 elements."""
    t = _torch()
    both = []
    for _ in range(2):
        flat = t.empty((pages - 1) * stride + page * Hkv * d, dtype=dt, device=DEV)
        both.append(flat.as_strided((pages, page, Hkv, d), (stride, Hkv * d, d, 1)))
    return both


def test_offsets_past_32_bits(av):
    """A pool of more than 2^32 bytes and elements per tensor: append, attend
    and evict through page offsets that 32 bits do not hold."""
    t = _torch()
    page, Hkv, d, stride = 16, 2, 64, 3 * 2 ** 29 + 64
    k, v = far_pool(4, page, Hkv, d, t.bfloat16, stride)
    table = t.tensor([[3, 0]], dtype=t.int32, device=DEV)
    lens = t.tensor([30], dtype=t.int32, device=DEV)
    cache = av.KVCache(k, v, table, lens, acc=t.rand(1, Hkv, 32, device=DEV), max_len=30)
    kn, vn = (t.randn(30, Hkv, d, device=DEV).bfloat16() for _ in range(2))
    av.avits_cache_append(cache, kn, vn, t.tensor([0, 30], dtype=t.int32, device=DEV))
    assert t.equal(k[3], kn[:16]) and t.equal(v[0, :14], vn[16:])
    q = t.randn(1, 4, d, device=DEV).bfloat16()
    o, lse = t.empty_like(q), t.empty(1, 4, device=DEV)
    av.avits_cache_attention(cache, q, 0.125, o, lse=lse, weight=1.0)
    want, wl, _ = oc.cache_attention(q[0].float().cpu().numpy(),
                                     kn.float().cpu().numpy().transpose(1, 0, 2),
                                     vn.float().cpu().numpy().transpose(1, 0, 2), 0.125)
    assert np.allclose(o[0].float().cpu().numpy(), want, atol=2e-2)
    assert np.allclose(lse[0].cpu().numpy(), wl, atol=1e-4)
    dst = av.KVCache(k, v, t.tensor([[2]], dtype=t.int32, device=DEV),
                     t.zeros(1, dtype=t.int32, device=DEV), acc=t.zeros(1, Hkv, 16, device=DEV))
    idx = t.empty(1, Hkv, 12, dtype=t.int32, device=DEV)
    av.avits_cache_evict(cache, dst, 12, 2, 3, idx)
    assert av.avits_device_status() == 0
    for h in range(Hkv):
        assert t.equal(k[2, :12, h], kn[idx[0, h].long(), h])
        assert t.equal(v[2, :12, h], vn[idx[0, h].long(), h])


# ----------------------------------------------------------------- append --
@pytest.mark.parametrize("dtype,page,layout,d,Hkv", [
    ("bf16", 16, "tokens", 128, 8), ("bf16", 7, "heads", 80, 3), ("f32", 24, "joint", 100, 2),
    ("bf16", 1, "tokens", 8, 1), ("f32", 16, "heads", 256, 40)])
@pytest.mark.parametrize("B", [1, 5, 40, 1100])
def test_append(av, dtype, page, layout, d, Hkv, B):
    """Uneven new tokens, some sequences without any: exactly the places below
    each length are written, nothing else."""
    if B == 1100 and Hkv > 8:
        B = 300
    t = _torch()
    rng = np.random.default_rng(B + d)
    old = rng.integers(0, 20, B)
    new = rng.choice([0, 1, 1, 2, 9], B)
    lens = (old + new).tolist()
    w = World(av, dtype, lens, Hkv, Hkv, d, page, layout, seed=B)
    want_k, want_v, want_a = w.k_pages.clone(), w.v_pages.clone(), w.acc.clone()
    cu = np.concatenate([[0], np.cumsum(new)])
    T = int(cu[-1]) + 3                                  # rows that belong to nobody
    kn, vn = (t.randn(T, Hkv, 2 * d, device=DEV).to(_dt(dtype))[..., :d] for _ in range(2))
    place = np.concatenate([np.arange(n, n + x) for n, x in zip(old, new)]).astype(np.int64)
    b = np.repeat(np.arange(B), new)
    tab = w.table.cpu().numpy()
    if len(b):
        p = t.from_numpy(tab[b, place // page].astype(np.int64)).to(DEV)
        s = t.from_numpy(place % page).to(DEV)
        want_k[p, s] = kn[:len(b)]
        want_v[p, s] = vn[:len(b)]
        want_a[t.from_numpy(b).to(DEV), :, t.from_numpy(place).to(DEV)] = 0.0
    av.avits_cache_append(w.cache, kn, vn, t.from_numpy(cu.astype(np.int32)).to(DEV))
    assert av.avits_device_status() == 0
    for got, want in ((w.k_pages, want_k), (w.v_pages, want_v), (w.acc, want_a)):
        assert t.equal(got.nan_to_num(nan=-77.0), want.nan_to_num(nan=-77.0))


def test_append_nothing_and_more_than_fits(av):
    t = _torch()
    w = World(av, "bf16", [10, 4], 2, 2, 64, 16, acc=False)
    before = w.k_pages.clone()
    none = t.empty(0, 2, 64, dtype=t.bfloat16, device=DEV)
    av.avits_cache_append(w.cache, none, none, t.zeros(3, dtype=t.int32, device=DEV))
    assert t.equal(before.nan_to_num(nan=5.0), w.k_pages.nan_to_num(nan=5.0))
    # 6 tokens for a sequence of 4: the last 4 are stored, the rest reported
    kn = t.randn(6, 2, 64, device=DEV).bfloat16()
    av.avits_cache_append(w.cache, kn, kn, t.tensor([0, 0, 6], dtype=t.int32, device=DEV))
    assert av.avits_device_status() == 7
    p = int(w.table[1, 0])
    assert t.equal(w.k_pages[p, :4], kn[2:]) and t.equal(w.v_pages[p, :4], kn[2:])
    assert t.isnan(w.k_pages[p, 4:]).all()


def test_append_page_out_of_range(av):
    t = _torch()
    w = World(av, "bf16", [20, 4], 2, 2, 64, 16)
    w.table[0, 1] = 99
    before = w.k_pages.clone()
    kn = t.randn(3, 2, 64, device=DEV).bfloat16()
    av.avits_cache_append(w.cache, kn, kn, t.tensor([0, 2, 3], dtype=t.int32, device=DEV))
    assert av.avits_device_status() == 7
    before[int(w.table[1, 0]), 3] = kn[2]
    assert t.equal(before.nan_to_num(nan=5.0), w.k_pages.nan_to_num(nan=5.0))


# ------------------------------------------------------------------ evict --
def run_evict(av, w, keep, sinks, recent, page2=None, layout2="tokens", acc=None):
    t = _torch()
    page2 = page2 or w.page
    if acc is not None:
        w.acc.copy_(acc)
    cols = -(-keep // page2)
    k2, v2 = make_pool(layout2, w.B * cols + 1, page2, w.Hkv, w.d, _dt(w.dtype))
    perm = np.random.default_rng(1).permutation(w.B * cols + 1)[:w.B * cols]
    table2 = t.from_numpy(perm.reshape(w.B, cols).astype(np.int32)).to(DEV)
    lens2 = t.full((w.B,), 9, dtype=t.int32, device=DEV)
    acc2 = t.full((w.B, w.Hkv, keep + 3), -1.0, device=DEV)
    dst = av.KVCache(k2, v2, table2, lens2, acc=acc2, max_len=keep)
    idx = t.full((w.B, w.Hkv, keep), 123, dtype=t.int32, device=DEV)
    av.avits_cache_evict(w.cache, dst, keep, sinks, recent, idx)
    return dst, idx


def check_evict(w, dst, idx, keep, sinks, recent):
    a, got = w.acc.cpu().numpy(), idx.cpu().numpy()
    acc2, lens2 = dst.acc.cpu().numpy(), dst.lens.cpu().numpy()
    tab2 = dst.block_table.cpu().numpy()
    k2, v2 = dst.k_pages.float().cpu().numpy(), dst.v_pages.float().cpu().numpy()
    assert lens2.tolist() == [min(n, keep) for n in w.lens_l]
    for b, n in enumerate(w.lens_l):
        m = min(n, keep)
        k, v = w.rows(b)
        rk, rv = oc.pages_to_rows(k2, tab2[b], m), oc.pages_to_rows(v2, tab2[b], m)
        for h in range(w.Hkv):
            want = oc.cache_keep(a[b, h, :n], keep, sinks, recent)
            assert np.array_equal(got[b, h, :m], want), (b, h)
            assert (got[b, h, m:] == -1).all()
            assert np.array_equal(acc2[b, h, :m], a[b, h, want], equal_nan=True)
            assert (acc2[b, h, m:] == -1).all()                     # left as they were
            assert np.array_equal(rk[h], k[h, want]) and np.array_equal(rv[h], v[h, want])
    filled = sum(min(n, keep) for n in w.lens_l) * w.Hkv * w.d
    assert int((~np.isnan(k2)).sum()) == int((~np.isnan(v2)).sum()) == filled   # nothing else


@pytest.mark.parametrize("dtype,lens,Hkv,d,page,layout,keep,sinks,recent,page2,layout2", [
    ("bf16", [100], 2, 128, 16, "tokens", 40, 4, 10, 16, "tokens"),
    ("bf16", [0, 1, 39, 40, 41, 500, 77], 3, 64, 16, "heads", 40, 0, 0, 8, "joint"),
    ("bf16", [700, 20], 2, 80, 7, "joint", 100, 40, 60, 24, "heads"),   # nothing to choose
    ("bf16", [5000, 4097], 2, 8, 64, "tokens", 1, 0, 0, 1, "tokens"),
    ("bf16", [5000, 1], 1, 8, 64, "tokens", 4999, 1, 1, 16, "tokens"),
    ("f32", [300, 9], 2, 100, 24, "joint", 64, 3, 5, 10, "heads"),
    ("f32", [129], 40, 256, 16, "heads", 33, 1, 1, 16, "tokens"),
])
def test_evict(av, dtype, lens, Hkv, d, page, layout, keep, sinks, recent, page2, layout2):
    w = World(av, dtype, lens, Hkv, Hkv, d, page, layout, seed=keep)
    dst, idx = run_evict(av, w, keep, sinks, recent, page2, layout2)
    assert av.avits_device_status() == 0
    check_evict(w, dst, idx, keep, sinks, recent)


@pytest.mark.parametrize("n", [4096, 4097, 8192, 20000, 33333])
def test_evict_ties_over_the_whole_row(av, n):
    """Few values, so that the threshold's ties spread over the CTAs of a row;
    zeros of both signs, infinities and NaN among them."""
    t = _torch()
    w = World(av, "bf16", [n, n - 5], 2, 2, 8, 64, seed=n)
    g = t.Generator(device=DEV)
    g.manual_seed(n)
    vals = t.tensor([0.0, -0.0, 0.5, 1.0, -1.0, float("inf"), -float("inf"), float("nan")], device=DEV)
    acc = vals[t.randint(0, 8, w.acc.shape, device=DEV, generator=g)]
    for keep in (n // 4, n // 2, n - 7):
        dst, idx = run_evict(av, w, keep, 3, 11, acc=acc)
        assert av.avits_device_status() == 0
        check_evict(w, dst, idx, keep, 3, 11)
    w.acc.zero_()                                       # all equal
    dst, idx = run_evict(av, w, n // 3, 0, 0)
    check_evict(w, dst, idx, n // 3, 0, 0)


def test_evict_row_read_again(av):
    """So long a row that a thread's keys do not fit its registers: every digit reads
    the row again."""
    w = World(av, "bf16", [400001], 1, 1, 8, 256, seed=1)
    dst, idx = run_evict(av, w, 1000, 5, 5)
    assert av.avits_device_status() == 0
    check_evict(w, dst, idx, 1000, 5, 5)


def test_evict_into_the_same_pool(av):
    """Source and kept tokens in one pool, by two tables."""
    t = _torch()
    w = World(av, "bf16", [64, 50], 2, 2, 64, 16, seed=3)
    k, v = (t.cat([p, t.full_like(p[:4], float("nan"))]) for p in (w.k_pages, w.v_pages))
    base = w.k_pages.shape[0]
    src = av.KVCache(k, v, w.table, w.lens, acc=w.acc)
    table2 = t.arange(base, base + 4, dtype=t.int32, device=DEV).view(2, 2)
    dst = av.KVCache(k, v, table2, t.zeros(2, dtype=t.int32, device=DEV),
                     acc=t.full((2, 2, 35), -1.0, device=DEV), max_len=32)
    idx = t.empty(2, 2, 32, dtype=t.int32, device=DEV)
    av.avits_cache_evict(src, dst, 32, 4, 8, idx)
    assert av.avits_device_status() == 0
    assert t.equal(k[:base].nan_to_num(nan=9.0), w.k_pages.nan_to_num(nan=9.0))
    for b in range(2):
        for h in range(2):
            want = oc.cache_keep(w.acc[b, h, :w.lens_l[b]].cpu().numpy(), 32, 4, 8)
            assert idx[b, h].tolist() == want.tolist()
            rows = k[table2[b].long()].flatten(0, 1)[:32, h]
            assert np.array_equal(rows.float().cpu().numpy(), w.rows(b)[0][h, want])


def test_evict_pages_out_of_range(av):
    """Reported; what has a page on both sides is copied."""
    t = _torch()
    w = World(av, "bf16", [64, 64], 1, 1, 64, 16, seed=3)
    w.acc.copy_(t.arange(64, 0, -1, device=DEV).float().expand_as(w.acc))
    w.table[0, 0] = 1000
    dst, idx = run_evict(av, w, 32, 0, 0)
    assert av.avits_device_status() == 7
    assert idx[0, 0].tolist() == idx[1, 0].tolist() == list(range(32))
    got = dst.k_pages[dst.block_table[1].long()].flatten(0, 1)
    assert np.array_equal(got[:, 0].float().cpu().numpy(), w.rows(1)[0][0, :32])
    assert t.isnan(dst.k_pages[int(dst.block_table[0, 0])]).all()
    assert not t.isnan(dst.k_pages[int(dst.block_table[0, 1])]).any()


# ------------------------------------------------- streams, graphs, threads --
def test_calls_on_another_stream(av):
    """stream= given while another one is current: the default workspace goes
    with the stream that uses it."""
    t = _torch()
    w = World(av, "bf16", [3000, 10], 8, 2, 64, 16, seed=11)
    o, lse = w.outputs()
    s = t.cuda.Stream()
    s.wait_stream(t.cuda.current_stream())
    acc0 = w.acc.cpu().numpy()
    av.avits_cache_attention(w.cache, w.q, w.scale, o, lse=lse, weight=1.0, stream=s)
    s.synchronize()
    w.check(o, lse, acc0, 1.0)


def test_two_streams_at_once(av):
    t = _torch()
    ws = [World(av, "bf16", [6000, 500], 8, 2, 64, 16, seed=20 + i) for i in range(2)]
    outs = [w.outputs() for w in ws]
    acc0 = [w.acc.cpu().numpy() for w in ws]
    streams = [t.cuda.Stream() for _ in ws]
    t.cuda.synchronize()
    for r in range(10):
        for w, (o, lse), s in zip(ws, outs, streams):
            with t.cuda.stream(s):
                av.avits_cache_attention(w.cache, w.q, w.scale, o, lse=lse, weight=1.0,
                                         accumulate=False)
    t.cuda.synchronize()
    for w, (o, lse), a in zip(ws, outs, acc0):
        w.check(o, lse, a, 1.0, accumulate=False)


def test_threads_on_one_stream(av):
    t = _torch()
    ws = [World(av, "bf16", [6000, 500], 8, 2, 64, 16, seed=30 + i) for i in range(3)]
    outs = [w.outputs() for w in ws]
    acc0 = [w.acc.cpu().numpy() for w in ws]

    def work(w, o, lse):
        for _ in range(40):
            av.avits_cache_attention(w.cache, w.q, w.scale, o, lse=lse, weight=1.0,
                                     accumulate=False)

    threads = [threading.Thread(target=work, args=(w, *o)) for w, o in zip(ws, outs)]
    [x.start() for x in threads]
    [x.join() for x in threads]
    t.cuda.synchronize()
    for w, (o, lse), a in zip(ws, outs, acc0):
        w.check(o, lse, a, 1.0, accumulate=False)


def test_two_graphs_replayed_at_once(av):
    """Each captured call has a workspace of its own."""
    t = _torch()
    ws = [World(av, "bf16", [6000, 500], 8, 2, 64, 16, seed=40 + i) for i in range(2)]
    outs = [w.outputs() for w in ws]
    acc0 = [w.acc.cpu().numpy() for w in ws]
    graphs = []
    side = t.cuda.Stream()
    for w, (o, lse) in zip(ws, outs):
        run = lambda: av.avits_cache_attention(w.cache, w.q, w.scale, o, lse=lse, weight=1.0,
                                               accumulate=False)
        side.wait_stream(t.cuda.current_stream())
        with t.cuda.stream(side):
            run()
        t.cuda.current_stream().wait_stream(side)
        g = t.cuda.CUDAGraph()
        with t.cuda.graph(g):
            run()
        graphs.append(g)
        o.zero_()
    t.cuda.synchronize()
    for _ in range(10):
        for g, s in zip(graphs, (t.cuda.Stream(), t.cuda.Stream())):
            with t.cuda.stream(s):
                g.replay()
    t.cuda.synchronize()
    for w, (o, lse), a in zip(ws, outs, acc0):
        w.check(o, lse, a, 1.0, accumulate=False)


def test_growing_workspace(av):
    """A larger call after a smaller one, on one stream without waiting."""
    small = World(av, "bf16", [20], 4, 2, 64, 16, seed=50)
    large = World(av, "bf16", [9000, 800], 16, 2, 128, 16, seed=51)
    a0, b0 = small.acc.cpu().numpy(), large.acc.cpu().numpy()
    oa, ob, oc_ = small.outputs(), large.outputs(), small.outputs()
    for w, (o, lse) in ((small, oa), (large, ob), (small, oc_)):
        av.avits_cache_attention(w.cache, w.q, w.scale, o, lse=lse, weight=1.0, accumulate=False)
    _torch().cuda.synchronize()
    small.check(*oa, a0, 1.0, accumulate=False)
    small.check(*oc_, a0, 1.0, accumulate=False)
    large.check(*ob, b0, 1.0, accumulate=False)


def test_binding_refusals_on_the_device(av):
    t = _torch()
    w = World(av, "bf16", [20, 9], 4, 2, 64, 16)
    o, lse = w.outputs()
    att = av.avits_cache_attention
    with pytest.raises(ValueError):
        att(w.cache, w.q[:1], w.scale, o[:1])
    with pytest.raises(ValueError):
        att(w.cache, w.q, w.scale, o[:, :2])
    with pytest.raises(TypeError):
        att(w.cache, w.q.float(), w.scale, o)
    with pytest.raises(ValueError):
        att(w.cache, w.q, w.scale, o, lse=lse.double())
    with pytest.raises(ValueError):
        att(w.cache, w.q, w.scale, o.cpu())
    with pytest.raises(av.AvitsError):
        att(w.cache, w.q[:, :3], w.scale, o[:, :3])               # 3 heads over 2
    with pytest.raises(av.AvitsError):
        att(w.cache, w.q, 0.0, o)
    long = World(av, "bf16", [20, 9], 4, 2, 64, 16, max_len=20000)      # one that needs some
    assert av.avits_cache_attention_workspace(long.cache, 4, True) > 16
    with pytest.raises(av.AvitsError):
        att(long.cache, long.q, w.scale, o, workspace=t.empty(16, dtype=t.uint8, device=DEV))
    with pytest.raises(ValueError):                                 # one byte, many times
        att(long.cache, long.q, w.scale, o,
            workspace=t.empty(1, dtype=t.uint8, device=DEV).expand(1 << 24))
    plain = av.KVCache(w.k_pages, w.v_pages, w.table, w.lens)
    with pytest.raises(ValueError):
        att(plain, w.q, w.scale, o, weight=1.0)
    kn = t.zeros(2, 2, 64, dtype=t.bfloat16, device=DEV)
    cu = t.tensor([0, 1, 2], dtype=t.int32, device=DEV)
    with pytest.raises(ValueError):
        av.avits_cache_append(w.cache, kn[:, :1], kn[:, :1], cu)
    with pytest.raises(ValueError):
        av.avits_cache_append(w.cache, kn, kn, cu.long())
    with pytest.raises(ValueError):
        av.avits_cache_append(w.cache, kn, kn, cu[:2])
    with pytest.raises(TypeError):
        av.avits_cache_append(w.cache, kn.float(), kn.float(), cu)
    with pytest.raises(av.AvitsError):                              # rows not on 16 bytes
        odd = t.zeros(2, 2, 65, dtype=t.bfloat16, device=DEV)[..., :64]
        av.avits_cache_append(w.cache, odd, odd, cu)
    idx = t.zeros(2, 2, 8, dtype=t.int32, device=DEV)
    with pytest.raises(ValueError):
        av.avits_cache_evict(w.cache, plain, 8, 1, 1, idx)
    with pytest.raises(av.AvitsError):                              # into itself
        av.avits_cache_evict(w.cache, w.cache, 8, 1, 1, idx)
    with pytest.raises(ValueError):
        av.avits_cache_evict(w.cache, w.cache, 9, 1, 1, idx)
    assert av.avits_device_status() == 0


# -------------------------------------------------------------- all of it --
@pytest.mark.parametrize("captured", [False, True])
def test_prompt_decode_evict_decode(av, captured):
    """Prompts in, decoding steps that add up the weights, eviction, and more
    steps on what was kept, against the oracle run on rows of its own.  The
    kept sets are compared where the oracle's weights decide them by more than
    the fp32 sums can be off."""
    t = _torch()
    B, H, Hkv, d, page, cap, keep = 3, 8, 2, 64, 16, 96, 40
    g = t.Generator(device=DEV)
    g.manual_seed(77)
    prompts = [70, 1, 33]
    pages = B * (cap // page)
    k, v = make_pool("heads", 2 * pages, page, Hkv, d, t.bfloat16)
    order = t.randperm(2 * pages, device=DEV, generator=g).to(t.int32)
    acc = [t.full((B, Hkv, cap), float("nan"), device=DEV) for _ in range(2)]
    lens = [t.zeros(B, dtype=t.int32, device=DEV) for _ in range(2)]
    caches = [av.KVCache(k, v, order[i * pages:(i + 1) * pages].view(B, -1), lens[i], acc=acc[i])
              for i in range(2)]
    idx = t.empty(B, Hkv, keep, dtype=t.int32, device=DEV)
    host = [[[np.zeros((0, d)) for _ in range(Hkv)] for _ in range(B)] for _ in range(2)]  # k, v rows
    hacc = [[np.zeros(0) for _ in range(Hkv)] for _ in range(B)]

    def feed(cache, counts, capture):
        T = sum(counts)
        kn = t.randn(T, Hkv, d, device=DEV, generator=g).bfloat16()
        vn = t.randn(T, Hkv, d, device=DEV, generator=g).bfloat16()
        q = (2 * t.randn(B, H, d, device=DEV, generator=g)).bfloat16()
        cu = t.tensor(np.cumsum([0] + counts), dtype=t.int32, device=DEV)
        o, lse = t.empty_like(q), t.empty(B, H, device=DEV)
        n = t.tensor(counts, dtype=t.int32, device=DEV)

        def step():
            cache.lens.add_(n)
            av.avits_cache_append(cache, kn, vn, cu)
            av.avits_cache_attention(cache, q, 0.125, o, lse=lse, weight=1.0)

        if capture:
            graph = t.cuda.CUDAGraph()
            t.cuda.synchronize()
            with t.cuda.graph(graph):
                step()
            graph.replay()
        else:
            step()
        t.cuda.synchronize()
        at = 0
        for b, c in enumerate(counts):
            for h in range(Hkv):
                for which, rows in ((0, kn), (1, vn)):
                    host[which][b][h] = np.vstack([host[which][b][h],
                                                   rows[at:at + c, h].float().cpu().numpy()])
                hacc[b][h] = np.concatenate([hacc[b][h], np.zeros(c)])
            at += c
            want, wl, w = oc.cache_attention(q[b].float().cpu().numpy(),
                                             np.stack(host[0][b]), np.stack(host[1][b]), 0.125)
            assert np.allclose(o[b].float().cpu().numpy(), want, rtol=2 ** -8, atol=1e-4), b
            assert np.allclose(lse[b].cpu().numpy(), wl, atol=1e-4), b
            for h in range(Hkv):
                hacc[b][h] = hacc[b][h] + w[h]
                got = cache.acc[b, h, :len(hacc[b][h])].cpu().numpy()
                assert np.allclose(got, hacc[b][h], rtol=1e-4, atol=1e-7), (b, h)

    feed(caches[0], prompts, False)
    for _ in range(6):
        feed(caches[0], [1, 1, 1], captured)
    av.avits_cache_evict(caches[0], caches[1], keep, 4, 8, idx)
    assert av.avits_device_status() == 0
    assert lens[1].tolist() == [40, 7, 39]
    for b in range(B):
        for h in range(Hkv):
            n = len(hacc[b][h])
            got = idx[b, h, :min(n, keep)].cpu().numpy()
            # the kernel's own weights decide; they are the oracle's up to rounding
            mine = oc.cache_keep(caches[0].acc[b, h, :n].cpu().numpy(), keep, 4, 8)
            assert np.array_equal(got, mine)
            if n > keep:
                rest = np.setdiff1d(np.arange(4, n - 8), got)
                inner = got[(got >= 4) & (got < n - 8)]
                assert hacc[b][h][inner].min() >= hacc[b][h][rest].max() - 1e-4
            for which in range(2):
                host[which][b][h] = host[which][b][h][got]
            hacc[b][h] = hacc[b][h][got]
    for _ in range(5):
        feed(caches[1], [1, 0, 1], captured)
    assert av.avits_device_status() == 0
