"""A served batch's step around the cache from its definitions, numpy fp64 and plain loops."""
import math

import numpy as np


def cache_plan(lens, change, table, free, count, page, max_len, num_pages, T, base=None):
    """Lists in, a dict of arrays out; `free` and `table` are not changed in place."""
    lens, table, free = list(lens), [list(r) for r in table], list(free)
    n_free = min(max(count, 0), num_pages)
    bad = n_free != count

    def pages(n):
        return -(-n // page)

    def in_range(n, c):
        return 0 <= n <= max_len and n + c <= max_len

    for b, (n, c) in enumerate(zip(lens, change)):
        if c < 0 and in_range(n, c):
            for j in range(pages(max(0, n + c)), pages(n)):
                if n_free < num_pages:
                    free[n_free] = table[b][j]
                    n_free += 1
                else:
                    bad = True
    left = n_free
    asked, cu = 0, [0]
    slots, seq, place, pos = [-1] * T, [-1] * T, [-1] * T, [-1] * T
    for b, (n, c) in enumerate(zip(list(lens), change)):
        first = cu[-1]
        cu.append(first + max(c, 0))
        if not in_range(n, c):
            bad = True
            continue
        if c <= 0:
            lens[b] = max(0, n + c)
            continue
        if cu[-1] > T:
            bad = True
            continue
        cols = range(pages(n), pages(n + c))
        asked += len(cols)
        if len(cols) and asked > left:
            bad = True
            continue
        for j in cols:
            n_free -= 1
            table[b][j] = free[n_free]
        lens[b] = n + c
        for i in range(c):
            j = n + i
            p = table[b][j // page]
            if 0 <= p < num_pages:
                slots[first + i] = p * page + j % page
            else:
                bad = True
            seq[first + i], place[first + i] = b, j
            pos[first + i] = j + (0 if base is None else base[b])
    return dict(lens=np.array(lens, np.int32), table=np.array(table, np.int32),
                free=np.array(free, np.int32), count=n_free,
                cu=np.array([min(x, T) for x in cu], np.int32), slots=np.array(slots, np.int64),
                seq=np.array(seq, np.int32), place=np.array(place, np.int32),
                pos=np.array(pos, np.int32), bad=bad)


def frequencies(width, base, scaling="none", factor=1.0, original_len=0.0, low=1.0, high=32.0):
    """Radians per position of each pair of a ladder of width/2."""
    if scaling == "base" and width > 2:
        base = base * factor ** (width / (width - 2))
    out = []
    for i in range(width // 2):
        f = base ** (-2.0 * i / width)
        if scaling == "linear":
            f /= factor
        if scaling == "parts":
            g = min(1.0, max(0.0, (original_len * f / (2 * math.pi) - low) / (high - low)))
            f = g * f + (1.0 - g) * f / factor
        out.append(f)
    return np.array(out)


def norm_rotate(x, pos, freq, sections, interleaved, weight=None, norm=True, eps=1e-6,
                magnitude=1.0):
    """x [..., heads, d], pos [..., axes] -> the same in fp64; freq of rot/2 pairs."""
    x = np.asarray(x, np.float64)
    d, half = x.shape[-1], len(freq)
    y = x
    if norm:
        y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        if weight is not None:
            y = y * np.asarray(weight, np.float64)
    out = y.copy()
    i = 0
    for axis, n in enumerate(sections):
        for _ in range(n):
            t = np.asarray(pos, np.float64)[..., axis] * freq[i]
            turn = (magnitude * np.exp(1j * t))[..., None]
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            z = (y[..., a] + 1j * y[..., b]) * turn
            out[..., a], out[..., b] = z.real, z.imag
            i += 1
    assert i == half and d >= 2 * half
    return out
