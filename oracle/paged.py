"""A cache in pages of 8-bit entries in 64 bits, from its definition: e4m3 bytes, a power of two as the scale of 16 entries of a head, places in a page."""
import numpy as np

BLOCK = 16
LEAST = 2.0 ** -120


def e4m3(x):
    """x rounded to the nearest e4m3 value (OCP: 3 bits behind the leading one down to 2^-6, steps of 2^-9 below, 448 the largest), ties to even."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(x)
    e = np.floor(np.log2(np.maximum(a, 2.0 ** -6)))
    step = 2.0 ** (e - 3)
    with np.errstate(invalid="ignore"):
        return np.where(np.isfinite(x), np.copysign(np.minimum(np.rint(a / step) * step, 448.0), x), np.nan)


def e4m3_byte(x):
    """The byte of an e4m3 value."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(x)
    e = np.floor(np.log2(np.maximum(a, 2.0 ** -6)))
    normal = a >= 2.0 ** -6
    with np.errstate(invalid="ignore"):
        code = np.where(normal, (e + 7) * 8 + (a / 2.0 ** e - 1) * 8, a * 2.0 ** 9)
        code = np.where(np.isnan(x), 0x7f, code)
        return code.astype(np.uint8) | np.where(np.signbit(x) & ~np.isnan(x), 0x80, 0).astype(np.uint8)


def scale_for(x):
    """The least power of two s >= 2^-120 with |x| <= 448 s for every finite x."""
    x = np.abs(np.asarray(x, dtype=np.float64))
    most = float(np.max(np.where(np.isfinite(x), x, 0.0), initial=0.0))
    s = LEAST
    while 448.0 * s < most:
        s *= 2.0
    return s


class Sequence:
    """Entries of one sequence, keys or values: [head][entry][d] e4m3 values and a scale for every block of a head."""

    def __init__(self, heads, d):
        self.values, self.scales = np.zeros((heads, 0, d)), np.zeros((heads, 0))

    def __len__(self):
        return self.values.shape[1]

    def append(self, rows, keep=None):
        """rows: [n, head, d]; entries from `keep` on are dropped first."""
        n, heads, _ = rows.shape
        if n == 0:
            return
        start = len(self) if keep is None else keep
        self.values = np.concatenate([self.values[:, :start], np.zeros((heads, n, rows.shape[2]))], axis=1)
        blocks = -(-(start + n) // BLOCK)
        scales = np.zeros((heads, blocks))
        scales[:, :-(-start // BLOCK)] = self.scales[:, :-(-start // BLOCK)]
        self.scales = scales
        for h in range(heads):
            for b in range(start // BLOCK, blocks):
                lo, hi = max(start, b * BLOCK), min(start + n, (b + 1) * BLOCK)
                new = rows[lo - start:hi - start, h]
                old = scales[h, b] if lo > b * BLOCK else 0.0
                scales[h, b] = max(old, scale_for(new))
                if lo > b * BLOCK:
                    self.values[h, b * BLOCK:lo] = e4m3(self.values[h, b * BLOCK:lo] * old / scales[h, b])
                self.values[h, lo:hi] = e4m3(new / scales[h, b])

    def numbers(self):
        """[entry, head, d]"""
        return (self.values * np.repeat(self.scales, BLOCK, axis=1)[:, :len(self), None]).transpose(1, 0, 2)


def key_place(row, x, d):
    return (row // 4) * 4 * d + (x // 64) * 256 + (row % 4) * 64 + x % 64


def value_place(row, x, d):
    return (row // 4) * 4 * d + 4 * x + row % 4
