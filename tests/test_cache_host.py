"""The paged key-value cache without a GPU: the oracle's pins, and the calls
that the library and its binding refuse before anything is launched."""
import ctypes

import numpy as np
import pytest
import torch

import oracle.cache as oc
import paper_2608_17995_gb300 as av

INVALID, UNSUPPORTED = 1, 2


@pytest.fixture(scope="module")
def lib():
    av.build()
    return av.lib()


def test_struct_matches_the_header():
    assert ctypes.sizeof(av._CacheStruct) == 5 * 8 + 9 * 8 + 7 * 4 + 4


# ------------------------------------------------------------ oracle pins --
def test_oracle_uniform_attention():
    """q = 0: every key gets 1/n, o is the mean of the values, lse = log n."""
    v = np.arange(2 * 5 * 4, dtype=np.float64).reshape(2, 5, 4)
    o, lse, w = oc.cache_attention(np.zeros((6, 4)), np.ones((2, 5, 4)), v, 0.5)
    assert np.allclose(o.reshape(2, 3, 4), v.mean(1)[:, None])
    assert np.allclose(lse, np.log(5)) and np.allclose(w, 0.2)


def test_oracle_against_brute_force():
    rng = np.random.default_rng(3)
    q, k, v = rng.normal(size=(4, 8)), rng.normal(size=(2, 7, 8)), rng.normal(size=(2, 7, 8))
    o, lse, w = oc.cache_attention(q, k, v, 0.3)
    mean = np.zeros((2, 7))
    for h in range(4):
        x = [0.3 * sum(q[h, i] * k[h // 2, j, i] for i in range(8)) for j in range(7)]
        z = sum(np.exp(t) for t in x)
        assert abs(lse[h] - np.log(z)) < 1e-12
        p = np.exp(x) / z
        assert np.allclose(o[h], sum(p[j] * v[h // 2, j] for j in range(7)))
        mean[h // 2] += p / 2
    assert np.allclose(w, mean) and np.allclose(w.sum(1), 1)


def test_oracle_empty_sequence():
    o, lse, w = oc.cache_attention(np.ones((2, 4)), np.zeros((1, 0, 4)), np.zeros((1, 0, 4)), 1.0)
    assert not o.any() and np.all(np.isneginf(lse)) and w.shape == (1, 0)


@pytest.mark.parametrize("acc,keep,sinks,recent,want", [
    ([5, 1, 3, 3, 3, 0], 4, 1, 1, [0, 2, 3, 5]),            # ties: the lower places
    ([0, 0, 0, 0], 2, 0, 0, [0, 1]),
    ([9, 9, 9], 3, 0, 0, [0, 1, 2]),                        # n <= keep
    ([], 3, 1, 1, []),
    ([0, 7, 1, 8, 0], 3, 2, 1, [0, 1, 4]),                  # nothing left to choose
    ([np.nan, -np.inf, np.nan, -1], 2, 0, 0, [1, 3]),       # NaN below -inf
    ([-0.0, 0.0, -0.0], 1, 0, 0, [0]),                      # equal
    ([1, 2, 3, 4], 1, 0, 1, [3]),
])
def test_oracle_kept_places(acc, keep, sinks, recent, want):
    assert oc.cache_keep(np.array(acc, np.float32), keep, sinks, recent).tolist() == want


def test_oracle_pages():
    pages = np.arange(5 * 2 * 1 * 1).reshape(5, 2, 1, 1)
    assert oc.pages_to_rows(pages, [4, 0, -1], 3)[0, :, 0].tolist() == [8, 9, 0]
    assert oc.pages_to_rows(pages, [-1], 0).shape == (1, 0, 1)


# ------------------------------------------------------- the C entry points --
P = 4096   # a 16-byte aligned address; nothing is launched with it


def struct(**kw):
    a = dict(k_pages=P, v_pages=P, block_table=P, lens=P, acc=P, k_sp=16 * 2 * 64, k_st=2 * 64,
             k_sh=64, v_sp=16 * 2 * 64, v_st=2 * 64, v_sh=64, table_sb=8, acc_sb=2 * 100,
             acc_sh=100, dt=1, B=3, Hkv=2, d=64, num_pages=20, page_size=16, max_len=100)
    a.update(kw)
    s = av._CacheStruct(**a)
    return s


BAD = [(dict(k_pages=None), INVALID), (dict(v_pages=None), INVALID),
       (dict(block_table=None), INVALID), (dict(lens=None), INVALID), (dict(dt=2), INVALID),
       (dict(B=0), INVALID), (dict(Hkv=0), INVALID), (dict(d=0), INVALID),
       (dict(num_pages=0), INVALID), (dict(page_size=0), INVALID), (dict(max_len=0), INVALID),
       (dict(k_st=-128), INVALID), (dict(v_sp=-1), INVALID), (dict(table_sb=-1), INVALID),
       (dict(acc_sh=99), INVALID), (dict(acc_sb=99), INVALID),
       (dict(d=264), UNSUPPORTED), (dict(d=60), UNSUPPORTED),
       (dict(k_pages=P + 8), UNSUPPORTED), (dict(v_pages=P + 2), UNSUPPORTED),
       (dict(k_st=132), UNSUPPORTED), (dict(v_sh=68), UNSUPPORTED),
       (dict(dt=0, v_sp=2050), UNSUPPORTED), (dict(max_len=(1 << 30) + 1, acc=None), UNSUPPORTED)]


@pytest.mark.parametrize("bad,code", BAD)
def test_cache_descriptions_refused(lib, bad, code):
    s = struct(**bad)
    ref = ctypes.addressof(s)
    assert lib.avits_cache_append(ref, P, P, 4, P, 128, 64, 128, 64, None) == code
    assert lib.avits_cache_attention_workspace(ref, 8, 0) == 0
    assert lib.avits_cache_attention(ref, P, 8, 512, 64, 0.1, P, 512, 64, None, 0, 1.0, P,
                                     1 << 40, None) == code
    good = struct(lens=P + 64, acc=P + 64)
    assert lib.avits_cache_evict(ref, ctypes.addressof(good), 10, 1, 1, P, None) == code
    assert lib.avits_cache_evict(ctypes.addressof(good), ref, 10, 1, 1, P, None) == code


def test_append_refusals(lib):
    s = struct()
    ref = ctypes.addressof(s)

    def call(T=4, k=P, v=P, cu=P, kst=128, ksh=64, vst=128, vsh=64, c=ref):
        return lib.avits_cache_append(c, k, v, T, cu, kst, ksh, vst, vsh, None)

    assert call(c=None) == INVALID
    assert call(T=-1) == INVALID
    assert call(k=None) == INVALID and call(v=None) == INVALID and call(cu=None) == INVALID
    assert call(kst=-128) == INVALID
    assert call(k=P + 4) == UNSUPPORTED
    assert call(vst=130) == UNSUPPORTED
    assert call(T=0, k=None, v=None) == 0      # nothing to do, nothing launched


def test_attention_refusals(lib):
    # long enough to need a workspace
    s = struct(max_len=100000, table_sb=6250, acc_sb=2 * 100000, acc_sh=100000)
    ref = ctypes.addressof(s)
    need = lib.avits_cache_attention_workspace(ref, 8, 2)
    assert need > lib.avits_cache_attention_workspace(ref, 8, 0) > 0
    short = struct()                                                # one launch, no workspace
    assert lib.avits_cache_attention_workspace(ctypes.addressof(short), 8, 2) == 0
    assert lib.avits_cache_attention_workspace(ref, 7, 0) == 0      # not a multiple of Hkv
    assert lib.avits_cache_attention_workspace(ref, 8, 3) == 0

    def call(q=P, H=8, qsb=512, qsh=64, scale=0.1, o=P, osb=512, osh=64, mode=2, ws=P, wsb=None,
             c=ref):
        return lib.avits_cache_attention(c, q, H, qsb, qsh, scale, o, osb, osh, None, mode, 1.0,
                                         ws, need if wsb is None else wsb, None)

    assert call(q=None) == INVALID and call(o=None) == INVALID
    assert call(H=0) == INVALID and call(H=7) == INVALID
    assert call(qsb=-1) == INVALID and call(osh=-1) == INVALID
    assert call(osh=63) == INVALID and call(osb=0) == INVALID       # rows of o over one another
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        assert call(scale=bad) == INVALID
    assert call(mode=3) == INVALID and call(mode=-1) == INVALID
    assert call(ws=None) == INVALID and call(ws=P + 8) == INVALID
    assert call(wsb=need - 1) == INVALID
    assert call(H=2 * 257) == UNSUPPORTED
    without = struct(acc=None)
    assert call(c=ctypes.addressof(without)) == INVALID
    huge = struct(B=1 << 20, Hkv=8, max_len=1 << 20, acc=None)
    assert lib.avits_cache_attention(ctypes.addressof(huge), P, 8, 512, 64, 0.1, P, 512, 64, None,
                                     0, 1.0, P, 1 << 40, None) == UNSUPPORTED


def test_evict_refusals(lib):
    src, dst = struct(), struct(lens=P + 64, acc=P + 64, max_len=50)

    def call(keep=10, sinks=2, recent=3, idx=P, s=src, d=dst):
        return lib.avits_cache_evict(s and ctypes.addressof(s), d and ctypes.addressof(d), keep,
                                     sinks, recent, idx, None)

    assert call(s=None) == INVALID and call(d=None) == INVALID and call(idx=None) == INVALID
    assert call(keep=0) == INVALID and call(sinks=-1) == INVALID and call(recent=-1) == INVALID
    assert call(keep=4) == INVALID and call(sinks=2**31 - 1, recent=2**31 - 1) == INVALID
    assert call(keep=51) == INVALID                               # more than dst holds
    assert call(s=struct(acc=None)) == INVALID
    assert call(d=struct(acc=None, lens=P + 64)) == INVALID
    assert call(d=struct(lens=P + 64)) == INVALID                 # the same acc
    assert call(d=struct(acc=P + 64)) == INVALID                  # the same lens
    for other in (dict(dt=0), dict(B=2), dict(Hkv=1), dict(d=56)):
        assert call(d=struct(lens=P + 64, acc=P + 64, **other)) == INVALID


# ------------------------------------------------------------- the binding --
def tensors(B=2, pages=6, page=4, Hkv=2, d=16, cols=3, dt=torch.bfloat16):
    return dict(k_pages=torch.zeros(pages, page, Hkv, d, dtype=dt),
                v_pages=torch.zeros(pages, page, Hkv, d, dtype=dt),
                block_table=torch.zeros(B, cols, dtype=torch.int32),
                lens=torch.zeros(B, dtype=torch.int32), acc=torch.zeros(B, Hkv, cols * page))


@pytest.mark.parametrize("change", [
    dict(k_pages=torch.zeros(6, 4, 2, dtype=torch.bfloat16)),
    dict(v_pages=torch.zeros(6, 4, 2, 8, dtype=torch.bfloat16)),
    dict(k_pages=torch.zeros(6, 4, 2, 32, dtype=torch.bfloat16)[..., ::2]),
    dict(block_table=torch.zeros(2, 3)),
    dict(block_table=torch.zeros(2, 6, dtype=torch.int32)[:, ::2]),
    dict(lens=torch.zeros(3, dtype=torch.int32)),
    dict(lens=torch.zeros(2, dtype=torch.int64)),
    dict(acc=torch.zeros(2, 2, 11)),
    dict(acc=torch.zeros(2, 3, 12)),
    dict(acc=torch.zeros(2, 2, 12, dtype=torch.float64)),
    dict(acc=torch.zeros(2, 2, 24)[..., ::2]),
    dict(max_len=13), dict(max_len=0),
])
def test_binding_refuses_descriptions(change):
    a = tensors()
    a.update(change)
    with pytest.raises(ValueError):
        av.KVCache(**a)


def test_binding_refuses_types_and_host_tensors():
    a = tensors()
    with pytest.raises(TypeError):
        av.KVCache(**dict(a, v_pages=a["v_pages"].float()))
    with pytest.raises(TypeError):
        av.KVCache(**tensors(dt=torch.float16))
    with pytest.raises(ValueError, match="device tensor"):
        av.KVCache(**a)


class _DeviceTensor:
    """A stand-in for a device tensor where there is no device."""

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    is_cuda = True

    def get_device(self):
        return 0


def test_binding_description_is_fixed():
    c = av.KVCache(**{k: _DeviceTensor(t) for k, t in tensors().items()})
    with pytest.raises(AttributeError):
        c.lens = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(AttributeError):
        c.max_len = 4
    with pytest.raises(AttributeError):
        c.another = 1
    assert c.max_len == 12
