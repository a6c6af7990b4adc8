"""What the binding of the calls around the cache hands to the library, without a GPU."""
import ctypes
import struct
import types

import torch

import paper_2608_17995_gb300 as av


def rotary(call):
    """A Rotary on the CPU whose foreign call is `call`."""
    return types.SimpleNamespace(rot=0, axes=1, device=torch.device("cpu"), _index=-1, _ref=0,
                                 int32=torch.int32, codes={torch.bfloat16: av.BF16}, _call=call)


def test_strides_live_until_the_call(monkeypatch):
    """Other threads may look up any number of other strides between this call's look-up and
    the library's reading of them."""
    wide = torch.empty(1 << 16, dtype=torch.bfloat16)
    seen = []

    def others(*_):
        for i in range(1100):
            av._heads_of(wide.as_strided((2, 3, 4, 8), (1000 + i, 100 + i, 8, 1)), "other")
        return 0

    def call(which, args):
        a = struct.unpack("=21qdq", args)
        seen.extend(tuple((ctypes.c_int64 * 3).from_address(a[i])) for i in (10, 12, 15, 17))
        return 0

    monkeypatch.setattr(av, "_rotary_stream", others)
    want = [(701, 97, 16), (702, 98, 24), (703, 99, 32), (704, 101, 40)]
    q, qo, k, ko = (wide.as_strided((2, 3, 2, 8), (*s, 1)) for s in want)
    av.avits_norm_rotate(rotary(call), None, q, qo, k=k, k_out=ko)
    assert seen == want
    seen.clear()
    alone = wide.as_strided((3, 2, 8), (97, 16, 1))
    av.avits_norm_rotate(rotary(lambda which, args: call_of_q(args, seen)), None, alone, alone)
    assert seen == [(0, 97, 16)] * 2


def call_of_q(args, seen):
    a = struct.unpack("=21qdq", args)
    assert (a[13], a[15], a[16], a[17]) == (0, 0, 0, 0)      # no keys: no strides of theirs
    seen.extend(tuple((ctypes.c_int64 * 3).from_address(a[i])) for i in (10, 12))
    return 0


def test_workspace_sizes_kept_are_few(monkeypatch):
    """A program that makes a prefix per length does not grow what a cache keeps."""
    asked = []

    def need(cache, prefix, H):
        asked.append(prefix.n)
        return 16 * prefix.n + H

    monkeypatch.setattr(av, "avits_cache_attention_shared_workspace", need)
    cache = types.SimpleNamespace(_shared_need={})
    prefixes = [types.SimpleNamespace(n=n, _shape=n.to_bytes(4, "little")) for n in range(1000)]
    for p in prefixes:
        for H in (8, 8, 40):
            assert av._shared_bytes(cache, p, H) == 16 * p.n + H
    assert len(cache._shared_need) <= 64
    assert len(asked) == 2000                  # the second of the same was kept
