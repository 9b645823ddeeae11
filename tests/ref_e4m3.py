"""The e4m3 and e2m1 formats and the rounding numbers of 8-bit optimizer states, in numpy (tests only; written from the
formats' definitions and from include/hsadmm.h)."""
import numpy as np


def _e4m3():
    v = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = np.ldexp(1 + m / 8, e - 7) if e else np.ldexp(m / 8, -6)
        v[c] = np.nan if (e == 15 and m == 7) else (-x if c >> 7 else x)
    return v


E4M3 = _e4m3()
E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])


def grid_step(y, least=-6, bits=3):
    """The step of a floating format's values next to |y| (2^least its smallest normal, `bits` bits after the point)."""
    with np.errstate(divide="ignore"):
        e = np.where(y == 0, least, np.maximum(np.frexp(y)[1] - 1, least))
    return np.ldexp(1.0, e - bits)


def round_down_on_grid(y, u):
    """floor(y / step + u) step on e4m3's grid, for y >= 0."""
    s = grid_step(y)
    return np.floor(y / s + u) * s


def nearest_code(y, fmt):
    """Codes of the nearest values, ties to even (fmt: 0 e4m3, 1 e2m1), for |y| within the format's range."""
    s = grid_step(np.abs(y), *((-6, 3) if fmt == 0 else (0, 1)))
    q = np.rint(np.abs(y) / s) * s
    table = E4M3[:127] if fmt == 0 else E2M1[:8]
    code = np.searchsorted(table, q)
    assert np.array_equal(table[code], q)
    return (code + np.signbit(y) * (128 if fmt == 0 else 8)).astype(np.uint8)


def rounding_numbers(n, R, noise, first=0):
    """u of every element of an arena from element `first` (a multiple of 4) on, per replica."""
    m1, m2, m3, full = 0x6A09E667, 0xBB67AE85, 0x3C6EF373, 0xFFFFFFFF
    four = np.arange(first // 4, (first + n + 3) // 4, dtype=np.uint64)
    out = np.zeros((R, 4 * four.size))
    for r in range(R):
        x = ((four & np.uint64(full)) + (four >> np.uint64(32)) * np.uint64(m3) + np.uint64(noise + r * m3)) & np.uint64(full)
        x = (x * np.uint64(m1)) & np.uint64(full)
        x = ((x ^ (x >> np.uint64(16))) * np.uint64(m2)) & np.uint64(full)
        x = x ^ (x >> np.uint64(15))
        for i, k in enumerate((1, m1, m2, m3)):
            out[r, i::4] = (((x * np.uint64(k)) & np.uint64(full)) >> np.uint64(12)) * 2.0 ** -20
    return out[:, :n]
