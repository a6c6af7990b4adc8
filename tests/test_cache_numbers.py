"""Numbers that the C interface holds in 32 bits: the binding refuses larger ones
instead of passing what is left of them."""
import pytest
import torch

import paper_2608_17995_gb300 as av
from test_cache_host import _DeviceTensor, tensors

PAST = 1 << 32


def cache(**change):
    a = tensors()
    a.update(change)
    more = {k: a.pop(k) for k in list(a) if k == "max_len"}
    return av.KVCache(**{k: t if t is None else _DeviceTensor(t) for k, t in a.items()}, **more)


def huge_pages(cols):
    """Pages of 2^20 tokens, all of them the same one."""
    one = torch.zeros(1, 1, 2, 16, dtype=torch.bfloat16).expand(1, 1 << 20, 2, 16)
    return dict(k_pages=one, v_pages=one, acc=None,
                block_table=torch.zeros(2, cols, dtype=torch.int32))


def test_capacity_of_the_table():
    for cols in (4097, 2048):                 # 2^32 + 2^20 tokens, 2^31
        with pytest.raises(ValueError, match="max_len"):
            cache(**huge_pages(cols))
    c = cache(**huge_pages(4097), max_len=1 << 30)      # a bound that fits may be given
    assert c.max_len == c._struct.max_len == 1 << 30
    c = cache(**huge_pages(2047))
    assert c.max_len == c._struct.max_len == 2047 << 20


def test_pages_and_places():
    one = torch.zeros(1, 1, 2, 16, dtype=torch.bfloat16)
    for shape in ((PAST + 6, 4, 2, 16), (6, PAST + 4, 2, 16), (6, 4, PAST + 2, 16)):
        pool = one[:, :, :1].expand(*shape)
        with pytest.raises(ValueError):
            cache(k_pages=pool, v_pages=pool, acc=None, max_len=8)


def test_new_tokens():
    c = cache()
    rows = _DeviceTensor(torch.zeros(1, 2, 16, dtype=torch.bfloat16).expand(PAST + 1, 2, 16))
    cu = _DeviceTensor(torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="tokens"):
        av.avits_cache_append(c, rows, rows, cu)


@pytest.mark.parametrize("sinks,recent", [(PAST + 1, 1), (1, PAST), (-PAST, 0), (1 << 31, 0),
                                          (0, -(1 << 33))])
def test_kept_ends(sinks, recent):
    src, dst = cache(), cache()
    idx = _DeviceTensor(torch.zeros(2, 2, 8, dtype=torch.int32))
    with pytest.raises(ValueError, match="sinks"):
        av.avits_cache_evict(src, dst, 8, sinks, recent, idx)


def test_heads():
    av.build()
    c = cache(**huge_pages(2), max_len=1 << 20)
    assert av.avits_cache_attention_workspace(c, 8, True) > 0
    assert av.avits_cache_attention_workspace(c, PAST + 8, True) == 0     # no such size
