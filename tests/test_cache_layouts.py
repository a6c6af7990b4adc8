"""Layouts that the cache calls refuse or take, without a GPU: rows that a call
writes may be in any order in memory but not over one another.  A layout that is
taken shows by a later refusal (UNSUPPORTED) that the call is given on purpose, so
that nothing is launched here."""
import ctypes
import itertools

import numpy as np
import pytest

import paper_2608_17995_gb300 as av
from test_cache_host import INVALID, P, UNSUPPORTED, struct


@pytest.fixture(scope="module")
def lib():
    av.build()
    return av.lib()


def over(width, dims):
    """Whether two rows of `width` of a view with these (extent, stride) meet."""
    starts = np.zeros(1, np.int64)
    for n, s in dims:
        starts = (starts[:, None] + np.arange(n) * s).ravel()
    starts.sort()
    return bool((np.diff(starts) < width).any())


@pytest.mark.parametrize("B,H,osb,osh", [
    (3, 8, 3 * 64, 2 * 64),             # head 3 of one sequence, head 0 of the next one but one
    (2, 8, 8 * 64 - 1, 64), (2, 8, 64, 2 * 64 - 1), (2, 8, 64, 64), (3, 8, 64 * 5, 128),
    (2, 8, 65, 128), (3, 256, 255 * 64, 64), (5, 8, 100, 420), (64, 8, 64, 63 * 64)])
def test_output_rows(lib, B, H, osb, osh):
    """(What is taken: the GPU tests, and the pages' rows below.)"""
    assert over(64, [(B, osb), (H, osh)])
    s = struct(B=B, Hkv=1, acc=None)
    assert lib.avits_cache_attention(ctypes.addressof(s), P, H, 64 * H, 64, 0.1, P, osb, osh, None,
                                     0, 1.0, P, 1 << 40, None) == INVALID


WEIGHTS = [  # B, Hkv, acc_sb, acc_sh (max_len 100)
    (3, 2, 200, 100), (3, 2, 100, 300), (3, 2, 250, 120), (1, 2, 0, 100), (3, 1, 100, 0),
    (3, 2, 100, 100), (3, 2, 199, 100), (2, 3, 300, 150), (2, 4, 100, 200), (2, 3, 150, 100)]


@pytest.mark.parametrize("B,Hkv,sb,sh", WEIGHTS)
def test_weight_rows(lib, B, Hkv, sb, sh):
    """Where they are written: in an append, an attention with weights and in the
    cache that an eviction fills."""
    want = INVALID if over(100, [(B, sb), (Hkv, sh)]) else UNSUPPORTED
    st, sp = Hkv * 64, 16 * Hkv * 64
    where = dict(k_sh=64, k_st=st, k_sp=sp, v_sh=64, v_st=st, v_sp=sp)
    s = struct(B=B, Hkv=Hkv, acc_sb=sb, acc_sh=sh, **where)
    ref = ctypes.addressof(s)
    if want == INVALID:
        for mode in (1, 2):
            assert lib.avits_cache_attention(ref, P, 2 * Hkv, 128 * Hkv, 64, 0.1, P, 128 * Hkv, 64,
                                             None, mode, 1.0, P, 1 << 40, None) == INVALID
    # new rows off 16 bytes: UNSUPPORTED
    assert lib.avits_cache_append(ref, P + 4, P, 4, P, 64 * Hkv, 64, 64 * Hkv, 64, None) == want


def test_weight_rows_of_an_eviction(lib):
    # so many rows to keep that the copy's blocks have no index: UNSUPPORTED
    big = dict(B=1 << 20, max_len=1 << 14, table_sb=1 << 10, num_pages=1 << 30)
    src = struct(acc_sb=2 << 14, acc_sh=1 << 14, **big)
    for sb, sh, want in ((2 << 14, 1 << 14, UNSUPPORTED), (1 << 14, 1 << 34, UNSUPPORTED),
                         (1 << 14, 1 << 14, INVALID), ((2 << 14) - 1, 1 << 14, INVALID)):
        dst = struct(lens=P + 64, acc=P + 64, acc_sb=sb, acc_sh=sh, **big)
        assert lib.avits_cache_evict(ctypes.addressof(src), ctypes.addressof(dst), 1 << 14, 2, 3, P,
                                     None) == want


PAGES = [  # strides of page, token, head (20 pages of 16 tokens, 2 heads of 64)
    (2048, 128, 64), (2048, 64, 1024), (4096, 256, 128), (64, 20 * 128, 20 * 64),
    (2048, 128, 20 * 2048), (128, 20 * 128, 64),
    (0, 128, 64), (2048, 0, 64), (2048, 128, 0), (2040, 128, 64), (2048, 64, 64),
    (64, 128, 64), (2048, 120, 64), (1024, 64, 512)]


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("strides", PAGES)
def test_page_rows(lib, strides, which):
    want = INVALID if over(64, list(zip((20, 16, 2), strides))) else UNSUPPORTED
    s = struct(v_pages=P + (1 << 20), **dict(zip((which + "_sp", which + "_st", which + "_sh"), strides)))
    assert lib.avits_cache_append(ctypes.addressof(s), P + 4, P, 4, P, 128, 64, 128, 64, None) == want
    big = dict(B=1 << 20, max_len=1 << 14, table_sb=1 << 10, acc_sb=2 << 14, acc_sh=1 << 14)
    src, dst = struct(**big), struct(lens=P + 64, acc=P + 64, v_pages=P + (1 << 20), **big)
    for name, x in zip(("_sp", "_st", "_sh"), strides):
        setattr(dst, which + name, x)
    assert lib.avits_cache_evict(ctypes.addressof(src), ctypes.addressof(dst), 1 << 14, 2, 3, P,
                                 None) == want


def test_keys_and_values_in_one_place(lib):
    """A pool that is written cannot be both."""
    s = struct(v_pages=P)
    ref = ctypes.addressof(s)
    assert lib.avits_cache_append(ref, P, P, 4, P, 128, 64, 128, 64, None) == INVALID
    src, dst = struct(), struct(lens=P + 64, acc=P + 64)
    assert lib.avits_cache_evict(ctypes.addressof(src), ctypes.addressof(dst), 10, 2, 3, P,
                                 None) == INVALID


def test_page_rows_of_every_order(lib):
    """The six orders of a dense pool's axes, whole and cut in steps of 2."""
    n = dict(zip("pth", (20, 16, 2)))
    for order in itertools.permutations("pth"):
        for step in (1, 2):
            st, at = {}, 64 * step
            for a in reversed(order):
                st[a], at = at, at * n[a] * step
            s = struct(v_pages=P + (1 << 20), k_sp=st["p"], k_st=st["t"], k_sh=st["h"])
            assert lib.avits_cache_append(ctypes.addressof(s), P + 4, P, 4, P, 128, 64, 128, 64,
                                          None) == UNSUPPORTED


def test_page_rows_of_many_layouts(lib):
    rng = np.random.default_rng(1)
    seen = [0, 0]
    for _ in range(3000):
        n = [int(x) for x in rng.integers(1, 9, 3)]
        d = int(rng.choice([8, 16, 64]))
        st = [d * int(rng.choice([1, n[0], n[1], n[0] * n[1], n[1] * n[2], int(rng.integers(1, 100))]))
              for _ in range(3)]
        bad = over(d, list(zip(n, st)))
        seen[bad] += 1
        s = struct(v_pages=P + (1 << 20), acc=None, d=d, num_pages=n[0], page_size=n[1], Hkv=n[2],
                   k_sp=st[0], k_st=st[1], k_sh=st[2], v_sp=st[0], v_st=st[1], v_sh=st[2])
        assert lib.avits_cache_append(ctypes.addressof(s), P + 4, P, 4, P, 64 * d, d, 64 * d, d,
                                      None) == (INVALID if bad else UNSUPPORTED), (d, n, st)
    assert min(seen) > 500
