"""GPU parity of shared prefixes by two row tiles to a CTA, at sizes of each side of the rule
that takes them: own tokens by their bound, whole and uneven pieces, widths (tolerances and
oracle of test_gpu_shared)."""
import numpy as np
import pytest

from test_gpu_cache import av  # noqa: F401 (a fixture)
from test_gpu_shared import World, _torch, take

pytestmark = pytest.mark.gpu


def keys(av, n, size, pre, lens, H, Hkv, d, page, **kw):
    """n keys of own tokens to an SM, by the bound on their lengths."""
    sms = _torch().cuda.get_device_properties(0).multi_processor_count
    most = max(max(lens), -(-n * sms // (len(lens) * Hkv)))
    return World(av, "bf16", size, pre, lens, H, Hkv, d, page, max_len=most, **kw)


@pytest.mark.parametrize("n", [500, 1000, 1600, 2100])
@pytest.mark.parametrize("size,pre,lens,H,Hkv,d,page,seqs", [
    # one prefix in pieces that run into the next unit, that end with one, and in many
    ([64], [2000], [(5 * i) % 90 for i in range(64)], 32, 8, 128, 16, [0, 31, 32, 63]),
    ([64], [4000], [(7 * i) % 50 for i in range(64)], 32, 4, 128, 64, [0, 15, 16, 31, 32, 63]),
    ([70], [8192], [3] * 70, 30, 3, 96, 32, [0, 24, 25, 26, 50, 51, 69]),
    ([128], [4400], [2 + i % 5 for i in range(128)], 16, 4, 64, 16, [0, 31, 32, 63, 64, 65, 127]),
    ([128], [600], [2 + i % 5 for i in range(128)], 16, 4, 64, 8, [0, 31, 32, 63, 64, 65, 127]),
    # several prefixes, and sequences of none
    ([64, 0, 62], [2100, 50, 900], [(3 * i) % 40 for i in range(130)], 8, 2, 128, 24, [0, 1, 63, 64, 65, 127, 128, 129]),
])
def test_either_side_of_the_rule(av, size, pre, lens, H, Hkv, d, page, seqs, n):
    w = keys(av, n, size, pre, lens, H, Hkv, d, page, seed=n)
    first = w.run()
    w.check(*first, seqs=seqs)
    again = w.run()
    assert _torch().equal(first[0], again[0]) and _torch().equal(first[1], again[1])


def test_odd_values_of_width_64(av):
    """Infinite values and page numbers outside the pool, two row tiles of width 64."""
    w = keys(av, 2100, [64], [4400], [6] * 64, 8, 2, 64, 16, std=1.0, seed=3)
    w.prefix.v_pages[int(w.prefix.block_table[0, 4399 // 16]), 4399 % 16, 1, 5] = float("inf")
    o = w.run()[0].float().cpu().numpy()
    assert np.all(np.isposinf(o[:, 4:, 5])) and np.isfinite(o).sum() == o.size - 64 * 4
    w = keys(av, 2100, [64], [4300], [20] * 64, 8, 2, 64, 24, seed=4)
    w.prefix.block_table[0, 1] = -1
    w.prefix.block_table[0, 100] = 1 << 20
    o, lse = w.run(status=7)
    gone = {c * 24 + i for c in (1, 100) for i in range(24)}

    def there(b):
        pre = [x[:, [j for j in range(4300) if j not in gone]] for x in take(w.prefix, 0, 4300)]
        return [np.concatenate(x, 1) for x in zip(pre, take(w.cache, b, w.lens[b]))]

    w.check(o, lse, keys=there, seqs=[0, 31, 32, 33, 63])
