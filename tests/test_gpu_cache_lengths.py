"""Appends and evictions of sequences whose length is outside [0, max_len]: what
they write is what the description says, all else is left as it was."""
import numpy as np
import pytest

import oracle.cache as oc
from test_gpu_cache import DEV, World, _torch, av, make_pool  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def same(a, b):
    return _torch().equal(a.nan_to_num(nan=-77.0), b.nan_to_num(nan=-77.0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("length,new", [(49, 1), (50, 4), (60, 3), (48 + 7, 55), (2 ** 31 - 1, 2),
                                        (-1, 1), (-2 ** 31, 2)])
def test_append_past_the_capacity(av, dtype, length, new):
    """New token i of a sequence has the place length - new + i: places from
    max_len on, and below 0, are left out and reported, and the tokens that were
    cached keep their keys, values and weights."""
    t = _torch()
    cap = 48
    w = World(av, dtype, [cap, 20], 2, 2, 64, 16, max_len=cap)
    want_k, want_v, want_a = w.k_pages.clone(), w.v_pages.clone(), w.acc.clone()
    w.lens.copy_(t.tensor([length, 20], dtype=t.int32))
    kn, vn = (t.randn(new + 1, 2, 64, device=DEV).to(w.k_pages.dtype) for _ in range(2))
    places = [(0, length - new + i, i) for i in range(new)] + [(1, 19, new)]
    for b, j, row in places:
        if 0 <= j < cap and (b == 1 or length >= 0):
            p, s = int(w.table[b, j // 16]), j % 16
            want_k[p, s], want_v[p, s], want_a[b, :, j] = kn[row], vn[row], 0.0
    av.avits_cache_append(w.cache, kn, vn, t.tensor([0, new, new + 1], dtype=t.int32, device=DEV))
    assert av.avits_device_status() == 7
    assert same(w.k_pages, want_k) and same(w.v_pages, want_v) and same(w.acc, want_a)


def test_evict_of_lengths_out_of_range(av):
    """A length is cut to [0, max_len] and reported."""
    t = _torch()
    cap, keep = 48, 20
    w = World(av, "bf16", [cap, cap, cap, 30], 2, 2, 64, 16, max_len=cap)
    w.lens.copy_(t.tensor([49, -3, 2 ** 31 - 1, 30], dtype=t.int32))
    k2, v2 = make_pool("tokens", 8, 16, 2, 64, t.bfloat16)
    dst = av.KVCache(k2, v2, t.arange(8, dtype=t.int32, device=DEV).view(4, 2),
                     t.full((4,), 9, dtype=t.int32, device=DEV),
                     acc=t.full((4, 2, keep), -1.0, device=DEV), max_len=keep)
    idx = t.empty(4, 2, keep, dtype=t.int32, device=DEV)
    av.avits_cache_evict(w.cache, dst, keep, 2, 3, idx)
    assert av.avits_device_status() == 7
    assert dst.lens.tolist() == [keep, 0, keep, keep]
    a = w.acc.cpu().numpy()
    for b, n in enumerate((cap, 0, cap, 30)):
        k, _ = w.rows(b, n)
        for h in range(2):
            want = oc.cache_keep(a[b, h, :n], keep, 2, 3)
            assert idx[b, h].tolist() == want.tolist() + [-1] * (keep - len(want))
            rows = k2[dst.block_table[b].long()].flatten(0, 1)[:len(want), h]
            assert np.array_equal(rows.float().cpu().numpy(), k[h, want])
            assert (dst.acc[b, h, len(want):] == -1).all()
    assert t.isnan(k2[2:4]).all()                       # the empty sequence's pages


def test_append_of_the_most_tokens(av):
    """T = 2^31 - 1 rows, one row seen so many times; three belong to sequences."""
    t = _torch()
    w = World(av, "bf16", [5, 2], 2, 2, 64, 16)
    want_k, want_v = w.k_pages.clone(), w.v_pages.clone()
    kn, vn = (t.randn(1, 2, 64, device=DEV).bfloat16() for _ in range(2))
    for b, j in ((0, 3), (0, 4), (1, 1)):
        p = int(w.table[b, 0])
        want_k[p, j], want_v[p, j] = kn[0], vn[0]
    av.avits_cache_append(w.cache, kn.expand(2 ** 31 - 1, 2, 64), vn.expand(2 ** 31 - 1, 2, 64),
                          t.tensor([0, 2, 3], dtype=t.int32, device=DEV))
    assert av.avits_device_status() == 0
    assert same(w.k_pages, want_k) and same(w.v_pages, want_v)
