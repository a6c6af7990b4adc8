"""Cache attention over values that are infinite or NaN.

A softmax weight above 2^-126 is positive in 32 bits, so that a key whose value is
+inf (-inf) in a column gives +inf (-inf) there, infinities of both signs give NaN,
and every other column is, bit for bit, what it is without them: columns of O are
sums of their own.  No tolerance.  The logits here are N(0, 2^2), far from 2^-126.
"""
import numpy as np
import pytest

from test_gpu_cache import World, _torch, av, run_attention  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu
INF = float("inf")

# dtype, H, Hkv, d, page: each number of rows to a unit, by TMA and by 16-byte copies
UNITS = [("bf16", 1, 1, 64, 16), ("bf16", 16, 2, 128, 16), ("bf16", 6, 2, 256, 24),
         ("bf16", 16, 1, 64, 8), ("bf16", 24, 2, 128, 16), ("bf16", 16, 1, 256, 3),
         ("bf16", 24, 1, 64, 16), ("bf16", 32, 1, 128, 5), ("bf16", 40, 1, 128, 16),
         ("f32", 4, 2, 64, 16), ("f32", 8, 1, 128, 16), ("f32", 12, 1, 256, 3)]
LENS = list(range(1, 34)) + [0, 300, 77]


def place_of(w, b, j):
    return int(w.table[b, j // w.page]), j % w.page


@pytest.mark.parametrize("bound", [None, 6000])      # of the lengths: one launch, or two
@pytest.mark.parametrize("dtype,H,Hkv,d,page", UNITS)
def test_infinite_values(av, dtype, H, Hkv, d, page, bound):
    t = _torch()
    w = World(av, dtype, LENS, H, Hkv, d, page, seed=H + d, max_len=bound)
    acc0 = w.acc.clone()
    o0, lse0 = run_attention(w, weight=1.0)
    acc1 = w.acc.clone()
    rng = np.random.default_rng(H * d)
    want = o0.clone()
    G = H // Hkv
    for b, n in enumerate(LENS):
        for hk in range(Hkv if n else 0):
            cols = rng.choice(d, 4, replace=False)
            heads = slice(hk * G, (hk + 1) * G)
            for col, value in zip(cols, (INF, -INF)):
                p, s = place_of(w, b, int(rng.integers(n)))
                w.v_pages[p, s, hk, int(col)] = value
                want[b, heads, int(col)] = value
            if n < 2:
                continue
            # both signs, and a NaN
            i, j = rng.choice(n, 2, replace=False)
            for at, value in ((i, INF), (j, -INF)):
                p, s = place_of(w, b, int(at))
                w.v_pages[p, s, hk, int(cols[2])] = value
            p, s = place_of(w, b, int(i))
            w.v_pages[p, s, hk, int(cols[3])] = float("nan")
            want[b, heads, [int(cols[2]), int(cols[3])]] = float("nan")
    w.acc.copy_(acc0)
    o, lse = run_attention(w, weight=1.0)
    assert t.equal(t.isnan(o), t.isnan(want))
    assert t.equal(o.nan_to_num(nan=7.0, posinf=INF, neginf=-INF),
                   want.nan_to_num(nan=7.0, posinf=INF, neginf=-INF))
    assert t.equal(lse, lse0) and t.equal(w.acc, acc1)      # of the keys alone


@pytest.mark.parametrize("dtype,H", [("bf16", 8), ("bf16", 16), ("bf16", 32), ("f32", 8)])
def test_one_infinite_value_in_a_split_row(av, dtype, H):
    """A row whose pieces are joined, the infinity in the first, a middle or the last
    piece; a place that takes part in no sequence may hold anything."""
    t = _torch()
    w = World(av, dtype, [9001], H, 1, 64, 16, seed=H)
    o0, _ = run_attention(w)
    for j in (0, 4444, 9000):
        p, s = place_of(w, 0, j)
        old = w.v_pages[p, s, 0, 9].clone()
        w.v_pages[p, s, 0, 9] = -INF
        o, _ = run_attention(w)
        want = o0.clone()
        want[:, :, 9] = -INF
        assert t.equal(o, want), j
        w.v_pages[p, s, 0, 9] = old
