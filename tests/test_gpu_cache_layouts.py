"""Cache calls that write rows in unusual orders: taken as long as no two meet."""
import itertools

import numpy as np
import pytest

from test_gpu_cache import DEV, World, _torch, av  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("osb,osh", [(64, 2 * 64), (3 * 64, 2 * 64), (70, 2 * 70), (8 * 64, 64)])
def test_outputs_between_one_another(av, osb, osh):
    t = _torch()
    w = World(av, "bf16", [100, 37], 8, 2, 64, 16, seed=3)
    flat = t.full((osb + 7 * osh + 64 + 9,), 7.0, dtype=t.bfloat16, device=DEV)
    o = flat.as_strided((2, 8, 64), (osb, osh, 1))
    lse = t.empty(2, 8, device=DEV)
    av.avits_cache_attention(w.cache, w.q, w.scale, o, lse=lse)
    assert av.avits_device_status() == 0
    w.check(o, lse)
    assert int((flat == 7).sum()) == flat.numel() - 2 * 8 * 64


@pytest.mark.parametrize("order", list(itertools.permutations(range(3))))
def test_append_into_every_order_of_axes(av, order):
    """Pools whose pages, places and heads lie in any order, the weights' rows too."""
    t = _torch()
    pages, page, Hkv, d, B = 5, 8, 3, 40, 2
    shape = [(pages, page, Hkv)[i] for i in order]
    back = [order.index(i) for i in range(3)]
    k, v = (t.zeros(*shape, d, dtype=t.bfloat16, device=DEV).permute(*back, 3) for _ in range(2))
    acc = t.ones(Hkv, B, 20, device=DEV).transpose(0, 1)
    table = t.tensor([[4, 1, 0], [2, 3, -1]], dtype=t.int32, device=DEV)
    cache = av.KVCache(k, v, table, t.tensor([19, 16], dtype=t.int32, device=DEV), acc=acc, max_len=20)
    kn, vn = (t.randn(35, Hkv, d, device=DEV).bfloat16() for _ in range(2))
    av.avits_cache_append(cache, kn, vn, t.tensor([0, 19, 35], dtype=t.int32, device=DEV))
    assert av.avits_device_status() == 0
    for pool, new in ((k, kn), (v, vn)):
        got = pool[table[0].long()].flatten(0, 1)[:19], pool[table[1, :2].long()].flatten(0, 1)
        assert t.equal(got[0], new[:19]) and t.equal(got[1], new[19:])
        assert int((pool != 0).sum()) == int((new != 0).sum())
    want = np.ones((B, Hkv, 20))
    want[0, :, :19] = want[1, :, :16] = 0
    assert np.array_equal(acc.cpu().numpy(), want)


def test_refused_before_anything_is_written(av):
    t = _torch()
    w = World(av, "bf16", [30, 20], 8, 2, 64, 16, seed=4)
    flat = t.full((8 * 64 + 64,), 7.0, dtype=t.bfloat16, device=DEV)
    with pytest.raises(av.AvitsError):          # both sequences' heads shifted by one
        av.avits_cache_attention(w.cache, w.q, w.scale, flat.as_strided((2, 8, 64), (64, 64, 1)))
    same = w.k_pages[:1].expand(w.k_pages.shape)
    shared = av.KVCache(same, w.v_pages, w.table, w.lens, max_len=w.max_len)
    kn = t.ones(2, 2, 64, dtype=t.bfloat16, device=DEV)
    cu = t.tensor([0, 1, 2], dtype=t.int32, device=DEV)
    before = w.k_pages.nan_to_num(nan=-77.0)
    with pytest.raises(av.AvitsError):          # every page the same memory
        av.avits_cache_append(shared, kn, kn, cu)
    with pytest.raises(av.AvitsError):          # keys and values the same memory
        av.avits_cache_append(av.KVCache(w.k_pages, w.k_pages, w.table, w.lens), kn, kn, cu)
    assert (flat == 7).all() and t.equal(before, w.k_pages.nan_to_num(nan=-77.0))
    assert av.avits_device_status() == 0
