"""The calls around the paged cache without a GPU: the oracle's pins, the
frequencies, and what the library and its binding refuse before anything is launched."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest

import oracle.step as os_
import paper_2608_17995_gb300 as av
from test_cache_host import BAD, INVALID, UNSUPPORTED, P, struct

W = 1 << 16          # another 16-byte aligned address


@pytest.fixture(scope="module")
def lib():
    av.build()
    return av.lib()


# ------------------------------------------------------------ oracle pins --
def test_oracle_plan_by_hand():
    got = os_.cache_plan([3, 4, 7, 0], [1, 2, -7, 3], [[9, -1], [5, -1], [6, 2], [-1, -1]],
                         [8, 1, 0, 0, 0, 0, 0, 0, 0, 0], 2, 4, 8, 10, 7, base=[10, 0, 0, 100])
    # pages 6, 2 come back behind 8, 1; sequence 1 takes 2, sequence 3 takes 6
    assert got["free"][:4].tolist() == [8, 1, 6, 2] and got["count"] == 2
    assert got["lens"].tolist() == [4, 6, 0, 3] and not got["bad"]
    assert got["table"].tolist() == [[9, -1], [5, 2], [6, 2], [6, -1]]
    assert got["cu"].tolist() == [0, 1, 3, 3, 6]
    assert got["slots"].tolist() == [39, 8, 9, 24, 25, 26, -1]
    assert got["seq"].tolist() == [0, 1, 1, 3, 3, 3, -1]
    assert got["place"].tolist() == [3, 4, 5, 0, 1, 2, -1]
    assert got["pos"].tolist() == [13, 4, 5, 100, 101, 102, -1]


def test_oracle_plan_without_room():
    got = os_.cache_plan([0, 3, 0], [9, 1, 4], [[-1] * 3] * 3, [4, 7] + [0] * 6, 2, 4, 12, 8, 14)
    assert got["lens"].tolist() == [0, 4, 0] and got["count"] == 2 and got["bad"]
    assert got["seq"].tolist() == [-1] * 9 + [1] + [-1] * 4


def test_oracle_rotation_is_one():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(5, 2, 12))
    pos = rng.integers(-9, 9, size=(5, 2))
    f = os_.frequencies(8, 100.0)
    for inter in (False, True):
        y = os_.norm_rotate(x, pos, f, [1, 3], inter, norm=False, magnitude=2.0)
        assert np.allclose((y[..., :8] ** 2).sum(-1), 4 * (x[..., :8] ** 2).sum(-1))
        assert np.array_equal(y[..., 8:], x[..., 8:])
    # a quarter turn by hand
    y = os_.norm_rotate(np.array([[[1.0, 2.0]]]), [[1]], [math.pi / 2], [1], True, norm=False)
    assert np.allclose(y, [[[-2.0, 1.0]]])
    z = os_.norm_rotate(np.full((1, 1, 4), 3.0), [[0]], [1.0], [1], True, weight=[1, 2, 3, 4], eps=0)
    assert np.allclose(z, [[[1, 2, 3, 4]]])


# ------------------------------------------------------------- frequencies --
@pytest.mark.parametrize("width,base,scaling,kw", [
    (128, 10000.0, "none", {}), (2, 10000.0, "none", {}), (64, 500000.0, "linear", dict(factor=8.0)),
    (96, 10000.0, "base", dict(factor=4.0)), (2, 10000.0, "base", dict(factor=4.0)),
    (128, 500000.0, "parts", dict(factor=16.0, original_len=8192, low=1.0, high=4.0)),
    (256, 1.0, "none", {})])
def test_frequencies(lib, width, base, scaling, kw):
    got = (ctypes.c_uint64 * (width // 2))()
    a = dict(factor=1.0, original_len=0.0, low=1.0, high=32.0)
    a.update(kw)
    assert lib.avits_rotary_frequencies(width, base, av._SCALINGS[scaling], a["factor"],
                                        a["original_len"], a["low"], a["high"],
                                        ctypes.addressof(got)) == 0
    want = os_.frequencies(width, base, scaling, **kw) / (2 * math.pi)
    # a power and a few products in 64 bits
    assert np.allclose([x / 2.0 ** 64 for x in got], want, rtol=1e-13, atol=2.0 ** -63)


@pytest.mark.parametrize("bad", [
    dict(width=0), dict(width=3), dict(width=258), dict(base=0.0), dict(base=-1.0),
    dict(base=float("inf")), dict(base=float("nan")), dict(scaling=4), dict(scaling=-1),
    dict(scaling=1, factor=0.5), dict(scaling=1, factor=float("nan")),
    dict(scaling=3, original_len=0.0), dict(scaling=3, original_len=4.0, low=2.0, high=2.0),
    dict(base=1e-9)])           # half a turn and more per position
def test_frequencies_refused(lib, bad):
    a = dict(width=8, base=100.0, scaling=0, factor=2.0, original_len=0.0, low=1.0, high=32.0)
    a.update(bad)
    out = (ctypes.c_uint64 * 128)(*([7] * 128))
    assert lib.avits_rotary_frequencies(*a.values(), ctypes.addressof(out)) == INVALID
    assert lib.avits_rotary_frequencies(8, 100.0, 0, 1.0, 0.0, 1.0, 2.0, None) == INVALID
    assert list(out) == [7] * 128


# ------------------------------------------------------- the C entry points --
def rotary(**kw):
    a = dict(freq=P, rot=64, interleaved=0, axes=1, sections=(ctypes.c_int32 * 4)(32),
             magnitude=1.0)
    a.update(kw)
    if not isinstance(a["sections"], ctypes.Array):
        a["sections"] = (ctypes.c_int32 * 4)(*a["sections"])
    return av._RotaryStruct(**a)


def plan(lib, s, **kw):
    a = dict(lens=P, change=P, free=P, count=P, out=P, T=8, cu=P, slots=P, seq=P, place=P, pos=None,
             base=None)
    a.update(kw)
    return lib.avits_cache_plan(s and ctypes.addressof(s), *a.values(), None)


@pytest.mark.parametrize("bad,code", [x for x in BAD if "acc" not in str(x[0])])
def test_plan_caches_refused(lib, bad, code):
    assert plan(lib, struct(acc=None, **bad)) == code


@pytest.mark.parametrize("bad,code", [
    (dict(lens=None), INVALID), (dict(change=None), INVALID), (dict(free=None), INVALID),
    (dict(count=None), INVALID), (dict(out=None), INVALID), (dict(cu=None), INVALID),
    (dict(slots=None), INVALID), (dict(seq=None), INVALID), (dict(place=None), INVALID),
    (dict(T=-1), INVALID), (dict(T=(1 << 30) + 1), UNSUPPORTED)])
def test_plan_refused(lib, bad, code):
    assert plan(lib, struct(), **bad) == code


def test_plan_rows_that_meet(lib):
    assert plan(lib, struct(table_sb=6)) == INVALID       # 100 tokens in pages of 16: 7 columns
    assert plan(lib, None) == INVALID


def rotate(lib, r, **kw):
    a = dict(dt=1, B=2, N=3, d=64, pos=P, pos_sb=0, pos_sn=1, q=P, H=4, q_str=(768, 256, 64), qo=W,
             qo_str=(768, 256, 64), k=2 * P, Hkv=2, k_str=(384, 128, 64), ko=2 * W,
             ko_str=(384, 128, 64), norm=1, wq=None, wk=None, eps=1e-6)
    a.update(kw)
    for x in ("q_str", "qo_str", "k_str", "ko_str"):
        if a[x] is not None:
            a[x] = (ctypes.c_int64 * 3)(*a[x])
    return lib.avits_norm_rotate(r and ctypes.addressof(r), *a.values(), None)


@pytest.mark.parametrize("bad,code", [
    (dict(dt=2), INVALID), (dict(B=0), INVALID), (dict(N=0), INVALID), (dict(d=0), INVALID),
    (dict(H=0), INVALID), (dict(Hkv=-1), INVALID), (dict(q=None), INVALID), (dict(qo=None), INVALID),
    (dict(q_str=None), INVALID), (dict(k=None), INVALID), (dict(Hkv=0), INVALID),
    (dict(ko=None), INVALID), (dict(ko_str=None), INVALID), (dict(pos=None), INVALID),
    (dict(pos_sn=-1), INVALID), (dict(q_str=(768, -256, 64)), INVALID),
    (dict(qo_str=(768, 256, 32)), INVALID),                  # rows over one another
    (dict(ko_str=(128, 128, 64)), INVALID), (dict(qo=P, qo_str=(1024, 256, 64)), INVALID),
    (dict(qo=2 * P), INVALID), (dict(ko=P), INVALID), (dict(ko=W), INVALID),
    (dict(norm=0, wq=P), INVALID), (dict(norm=0, wk=P), INVALID), (dict(eps=-1.0), INVALID),
    (dict(eps=float("nan")), INVALID),
    (dict(d=264, q_str=(2112, 528, 264)), UNSUPPORTED), (dict(d=68), UNSUPPORTED),
    (dict(q=P + 8), UNSUPPORTED), (dict(q_str=(768, 252, 64)), UNSUPPORTED),
    (dict(ko=W + 2), UNSUPPORTED), (dict(wq=P + 8), UNSUPPORTED), (dict(N=1 << 30), UNSUPPORTED)])
def test_rotate_refused(lib, bad, code):
    assert rotate(lib, rotary(), **bad) == code


BAD_ROTARY = [dict(freq=None), dict(rot=63), dict(rot=-2), dict(rot=66), dict(axes=0), dict(axes=5),
              dict(sections=(31,)), dict(sections=(33, -1), axes=2), dict(magnitude=float("nan")),
              dict(magnitude=float("inf"))]


@pytest.mark.parametrize("bad", BAD_ROTARY)
def test_rotary_refused(lib, bad):
    assert rotate(lib, rotary(**bad)) == INVALID
    assert append(lib, struct(**GOOD), rotary(**bad)) == INVALID
    assert rotate(lib, None) == INVALID


def append(lib, s, r, **kw):
    a = dict(T=5, pos=P, pos_st=1, slots=P, seq=P, place=P, q=P, H=4, q_st=256, q_sh=64, qo=W, qo_st=256,
             qo_sh=64, k=2 * P, k_st=128, k_sh=64, v=3 * P, v_st=128, v_sh=64, norm=1, wq=None, wk=None,
             eps=1e-6)
    a.update(kw)
    return lib.avits_cache_append_rotated(s and ctypes.addressof(s), r and ctypes.addressof(r),
                                          *a.values(), None)


@pytest.mark.parametrize("bad,code", BAD)
def test_append_caches_refused(lib, bad, code):
    assert append(lib, struct(**bad), rotary(rot=0)) == code


GOOD = dict(k_pages=4 * W, v_pages=5 * W)


@pytest.mark.parametrize("bad,code", [
    (dict(T=-1), INVALID), (dict(H=0), INVALID), (dict(slots=None), INVALID), (dict(q=None), INVALID),
    (dict(qo=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID),
    (dict(pos=None), INVALID), (dict(seq=None), INVALID), (dict(place=None), INVALID),
    (dict(q_st=-1), INVALID), (dict(v_sh=-64), INVALID), (dict(pos_st=-1), INVALID),
    (dict(qo_sh=32), INVALID), (dict(qo=P, qo_st=512), INVALID), (dict(qo=2 * P), INVALID),
    (dict(qo=3 * P), INVALID), (dict(qo=4 * W), INVALID), (dict(norm=0, wk=P), INVALID),
    (dict(eps=float("inf")), INVALID), (dict(T=(1 << 30) + 1), UNSUPPORTED),
    (dict(q=P + 8), UNSUPPORTED), (dict(k_st=132), UNSUPPORTED), (dict(wk=P + 2), UNSUPPORTED)])
def test_append_refused(lib, bad, code):
    assert append(lib, struct(**GOOD), rotary(), **bad) == code


def test_append_of_nothing(lib):
    assert append(lib, struct(**GOOD), rotary(), T=0, slots=None, q=None, qo=None, k=None, v=None,
                  pos=None, seq=None, place=None) == 0


def test_append_pages_that_meet(lib):
    assert append(lib, struct(k_pages=4 * W, v_pages=4 * W), rotary()) == INVALID
    assert append(lib, struct(**GOOD, k_st=64), rotary()) == INVALID


# ------------------------------------------------------------- the binding --
def test_rotary_struct_matches_the_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    names = [n for n, _ in av._RotaryStruct._fields_]
    src = tmp_path / "offsets.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "avits.h"\nint main(void) {\n'
                   '  printf("%zu\\n", sizeof(avits_rotary));\n' +
                   "".join('  printf("%%zu %%zu\\n", offsetof(avits_rotary, %s), '
                           'sizeof(((avits_rotary*)0)->%s));\n' % (n, n) for n in names) +
                   "  return 0;\n}\n")
    exe = str(tmp_path / "offsets")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.check_call([cc, str(src), "-I" + os.path.join(root, "include"), "-o", exe])
    out = subprocess.check_output([exe], text=True).split("\n")
    assert int(out[0]) == ctypes.sizeof(av._RotaryStruct)
    for n, line in zip(names, out[1:]):
        field = getattr(av._RotaryStruct, n)
        assert [field.offset, field.size] == [int(x) for x in line.split()], n


@pytest.mark.parametrize("kw", [dict(rot=7), dict(rot=258), dict(rot=-2), dict(rot=8, sections=[3]),
                                dict(rot=8, sections=[1] * 5), dict(rot=8, sections=[5, -1]),
                                dict(rot=8, scaling="other")])
def test_binding_refuses_rotaries(kw):
    with pytest.raises(ValueError):
        av.Rotary(device="cpu", **kw)


# -------------------------------------------------------- shared prefixes --
def shared(lib, c, p, **kw):
    a = dict(start=P, q=P, H=8, q_sb=512, q_sh=64, scale=0.1, o=P, o_sb=512, o_sh=64, lse=None, ws=P,
             ws_bytes=1 << 40)
    a.update(kw)
    at = lambda s: s and ctypes.addressof(s)
    return lib.avits_cache_attention_shared(at(c), at(p), *a.values(), None)


@pytest.mark.parametrize("bad,code", BAD)
def test_shared_caches_refused(lib, bad, code):
    good, s = struct(), struct(**bad)
    assert shared(lib, s, good) == code and shared(lib, good, s) == code
    at = ctypes.addressof
    assert lib.avits_cache_attention_shared_workspace(at(s), at(good), 8) == 0
    assert lib.avits_cache_attention_shared_workspace(at(good), at(s), 8) == 0


@pytest.mark.parametrize("bad,code", [
    (dict(start=None), INVALID), (dict(q=None), INVALID), (dict(o=None), INVALID), (dict(H=0), INVALID),
    (dict(H=7), INVALID), (dict(q_sb=-1), INVALID), (dict(o_sh=-64), INVALID), (dict(scale=0.0), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(o_sh=32), INVALID),
    (dict(o_sb=64), INVALID), (dict(ws=None), INVALID), (dict(ws=P + 8), INVALID),
    (dict(ws_bytes=16), INVALID), (dict(H=2 * 257, o_sb=2 * 257 * 64), UNSUPPORTED)])
def test_shared_refused(lib, bad, code):
    assert shared(lib, struct(), struct(B=2), **bad) == code


@pytest.mark.parametrize("other", [dict(dt=0), dict(Hkv=4, acc=None), dict(d=32)])
def test_shared_caches_that_differ(lib, other):
    assert shared(lib, struct(), struct(**other)) == INVALID


def test_shared_sizes(lib):
    at = ctypes.addressof
    long = struct(max_len=1 << 29, acc=None)
    assert shared(lib, struct(B=1 << 20, acc=None), long) == UNSUPPORTED
    assert lib.avits_cache_attention_shared_workspace(at(struct()), at(struct()), 9) == 0


# ------------------------------------------------- arguments in an array --
def test_packed_calls(lib):
    """The same answers as the calls themselves give, for refused and empty ones."""
    call = lib.avits_call_packed
    c, r = struct(**GOOD), rotary()
    cp, rp = ctypes.addressof(c), ctypes.addressof(r)
    # an append of nothing, one of something refused, a size past 32 bits
    a = [cp, rp, 0, P, 1, P, P, P, P, 4, 256, 64, W, 256, 64, 2 * P, 128, 64, 3 * P, 128, 64, 1, 0, 0, 1e-6, 0]
    assert call(2, av._APPEND_ROTATED(*a)) == 0
    for at, bad, code in ((2, -1, INVALID), (2, 1 << 32, INVALID), (9, 0, INVALID), (9, (1 << 32) + 4, INVALID),
                          (22, P + 8, UNSUPPORTED), (24, -1.0, INVALID), (4, -1, INVALID)):
        b = list(a)
        b[2] = 5
        b[at] = bad
        assert call(2, av._APPEND_ROTATED(*b)) == code, at
    p = [cp, P, P, P, P, P, 8, P, P, P, P, 0, 0, 0]
    for at, bad in ((0, 0), (1, 0), (6, -1), (6, 1 << 33), (8, 0)):
        b = list(p)
        b[at] = bad
        assert call(0, av._PLAN(*b)) == INVALID, at
    s = (ctypes.c_int64 * 3)(768, 256, 64)
    sa = ctypes.addressof(s)
    q = [rp, 1, 2, 3, 64, P, 0, 1, P, 4, sa, W, sa, 0, 0, 0, 0, 0, 1, 0, 0, 1e-6, 0]
    for at, bad, code in ((1, 2, INVALID), (2, 0, INVALID), (9, 1 << 40, INVALID), (8, P + 8, UNSUPPORTED),
                          (21, float("nan"), INVALID), (13, P, INVALID)):
        b = list(q)
        b[at] = bad
        assert call(1, av._ROTATE(*b)) == code, at
    h = [cp, cp, P, P, 8, 512, 64, 0.1, P, 512, 64, 0, P, 1 << 40, 0]
    for at, bad, code in ((2, 0, INVALID), (4, 7, INVALID), (7, 0.0, INVALID), (13, 16, INVALID),
                          (13, -1, INVALID), (12, 0, INVALID)):
        b = list(h)
        b[at] = bad
        assert call(3, av._SHARED(*b)) == code, at
    assert call(4, av._PLAN(*p)) == INVALID and call(-1, av._PLAN(*p)) == INVALID
    assert call(0, None) == INVALID
