"""Cache attention where the logsumexp is large: the softmax is still normalised.

All logits lie at 2^19, where one step of fp32 is 2^-4 (also after the factor
log2 e), so that a weight taken as exp2(x - lse) with a rounded lse would be off by up
to 2 per cent.  With the values all one, o = 1; the weights of a row sum to one.

Tolerance.  o is sum p / sum p over the same fp32 p >= 0, and the weights are such
p times one reciprocal.  Any order of n positive fp32 terms is off by n 2^-24
relative, a tensor-core sum, which may cut, by twice that, in numerator and
denominator: below n 2^-22 together.  Each exponential has 2^-22; a term carries one
and one for each rise of the maximum since it came and for each joining of parts:
at most 63 tiles to a warp (2000 keys in tiles of 8 over 4 warps) and 5 + 2.  So
(n + 72) 2^-22, for bf16 also 2^-17 of o for weights in two parts and half a step
of o, 2^-8.  Differences of logits are multiples of 2^-4 below 2^20: exact.
"""
import numpy as np
import pytest

from test_gpu_cache import World, _torch, av, run_attention  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bound", [None, 6000])      # of the lengths: one launch, or two
@pytest.mark.parametrize("dtype,H,Hkv,d,page", [
    ("bf16", 8, 2, 64, 16), ("bf16", 16, 1, 128, 16), ("bf16", 40, 1, 64, 5),
    ("f32", 4, 2, 64, 16), ("f32", 8, 1, 128, 7), ("f32", 20, 1, 64, 8)])
def test_steep_rows_are_normalised(av, dtype, H, Hkv, d, page, bound):
    t = _torch()
    lens = [2000, 33, 1, 0, 513, 700]
    w = World(av, dtype, lens, H, Hkv, d, page, seed=d + H, max_len=bound)
    w.q[..., 0] = 2.0 ** 12
    w.k_pages[..., 0] = 2.0 ** 10
    w.v_pages.masked_fill_(~t.isnan(w.v_pages), 1.0)
    w.scale = 0.125
    o, lse = run_attention(w, weight=1.0, accumulate=False)
    acc = w.acc.double().cpu().numpy()
    got = o.double().cpu().numpy()
    for b, n in enumerate(lens):
        if n == 0:
            continue
        tol = (n + 72) * 2.0 ** -22
        assert np.all(np.abs(acc[b, :, :n].sum(-1) - 1.0) <= tol), b
        if dtype == "bf16":
            tol += 2.0 ** -17 + 2.0 ** -8
        assert np.all(np.abs(got[b] - 1.0) <= tol), b
        assert np.all(np.abs(lse[b].cpu().numpy() - 2.0 ** 19) < 2.0 ** 12), b


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_long_steep_row_is_normalised(av, dtype):
    """Over all SMs: more pieces to a row than one thread joins.  The sum of 20000
    terms is off by less than its bound for n, above; the pieces are shorter."""
    t = _torch()
    n = 20000
    w = World(av, dtype, [n], 4, 1, 64, 16, seed=3)
    w.q[..., 0] = 2.0 ** 12
    w.k_pages[..., 0] = 2.0 ** 10
    w.v_pages.masked_fill_(~t.isnan(w.v_pages), 1.0)
    w.scale = 0.125
    o, _ = run_attention(w, weight=1.0, accumulate=False)
    tol = (n + 72) * 2.0 ** -22
    assert abs(float(w.acc.double().sum()) - 1.0) <= tol
    assert float((o.double() - 1.0).abs().max()) <= tol + (2.0 ** -7 if dtype == "bf16" else 0)
