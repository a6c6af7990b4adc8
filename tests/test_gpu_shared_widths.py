"""GPU parity of shared prefixes at narrow and odd widths, each form of the call (tolerances and
oracle of test_gpu_shared)."""
import pytest

from test_gpu_cache import av  # noqa: F401 (a fixture)
from test_gpu_shared import World

pytestmark = pytest.mark.gpu

FORMS = [   # sizes, prefixes, own lengths, H, Hkv, page: one launch, parts, a line of own tokens, pages of 5
    ([3, 2], [60, 9], [5, 0, 70, 1, 2], 8, 2, 16),
    ([20, 3], [4200, 5000], [(5 * i) % 33 for i in range(23)], 16, 2, 16),
    ([20, 3], [4200, 90], [(5 * i) % 33 for i in range(22)] + [2600], 12, 4, 8),
    ([3, 2], [4200, 9], [5, 0, 70, 1, 2], 130, 2, 5),
]


@pytest.mark.parametrize("dtype,d", [("bf16", 8), ("bf16", 24), ("bf16", 40), ("bf16", 136), ("bf16", 248),
                                     ("f32", 4), ("f32", 12), ("f32", 68), ("f32", 252)])
@pytest.mark.parametrize("size,pre,lens,H,Hkv,page", FORMS)
def test_widths(av, dtype, d, size, pre, lens, H, Hkv, page):
    w = World(av, dtype, size, pre, lens, H, Hkv, d, page, seed=d)
    w.check(*w.run())
