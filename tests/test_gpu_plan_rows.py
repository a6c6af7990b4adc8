"""Plans of steps with few rows, which the call's first kernel writes itself: batches of
many warps and of more sequences than threads, at both sides of the border to the second
kernel.  Whole numbers, exact, memory left alone included (test_gpu_step.Pages)."""
import numpy as np
import pytest

from test_gpu_step import Pages, av  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def few(B, ones, max_len, seed, long=()):
    """Lengths and changes of a batch: `long` new tokens for a few sequences, one for each of
    `ones` more, the rest idle, cut or done."""
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, max_len + 1, B)
    change = np.zeros(B, np.int64)
    order = rng.permutation(B)
    assert len(long) + ones <= B
    change[order[:len(long)]] = long
    change[order[len(long):len(long) + ones]] = 1
    for b in order[len(long) + ones:]:
        kind = rng.random()
        change[b] = 0 if kind < 0.3 else -int(rng.integers(1, 40)) if kind < 0.7 else -lens[b]
    return lens.tolist(), change.tolist()


def pages_needed(lens, change, page):
    return sum(max(0, -(-(n + c) // page) - -(-n // page)) for n, c in zip(lens, change) if c > 0)


BATCHES = [   # B, sequences of one new token, page, new tokens of a few more
    (256, 200, 16, ()), (256, 256, 16, ()), (256, 180, 16, (9, 40, 33, 1, 8)), (256, 170, 1, (9, 3, 2)),
    (511, 400, 16, (64,)), (1024, 500, 16, ()), (1024, 386, 8, (100, 9, 17)), (1025, 499, 16, (12,)),
    (1025, 20, 16, ()), (2100, 400, 16, (9, 33, 70)), (2100, 300, 2, (5, 8, 9)), (5000, 250, 64, (200, 10)),
    (20, 9, 16, (96, 97, 32, 31, 33, 8, 9, 7, 2, 3, 60)), (2, 1, 16, (499,)), (16, 9, 16, (300, 90, 100, 13)),
    (17, 0, 24, (60,) * 14 + (58,)), (33, 0, 5, (16,) * 32), (300, 4, 16, (4,) * 290), (128, 1, 16, (8,) * 126 + (15,)),
]


@pytest.mark.parametrize("short", [False, True])
@pytest.mark.parametrize("B,ones,page,long", BATCHES)
def test_plan_few_rows(av, B, ones, page, long, short):
    lens, change = few(B, ones, 300 if B < 1000 else 120, B + ones, long)
    need = pages_needed(lens, change, page)
    spare = need + 3
    if short:                    # some find no pages, and none come back
        change = [max(c, 0) for c in change]
        spare = need // 2
    p = Pages(av, lens, change, page, max(n + max(c, 0) for n, c in zip(lens, change)), spare,
              T=sum(max(c, 0) for c in change) + B % 3, seed=B)
    p.call()
    p.check(bad=short)


@pytest.mark.parametrize("T", [256, 511, 512, 513, 1023, 1024, 1025, 2047, 2048, 2049])
@pytest.mark.parametrize("B", [1, 7, 64, 256, 1030])
def test_plan_at_the_borders(av, B, T):
    """T rows exactly, one less than the step has, and more."""
    each = [T // B + (i < T % B) for i in range(B)]
    lens = [(37 * i) % 90 for i in range(B)]
    for more in (0, -1, 5):
        p = Pages(av, lens, each, 16, 90 + T // B + 1, pages_needed(lens, each, 16) + 1, T=T + more, seed=B + T)
        p.call()
        p.check(bad=more < 0)


def test_plan_one_long_among_many(av):
    """A prompt among decoding sequences: its rows are most of the step's."""
    lens, change = [(13 * i) % 200 for i in range(256)], [1] * 256
    lens[100], change[100] = 0, 700
    p = Pages(av, lens, change, 16, 1000, pages_needed(lens, change, 16) + 2, T=1000)
    p.call()
    p.check()
