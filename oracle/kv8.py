"""The 8-bit paged cache in numpy fp64, from its definition: an element is an e4m3 number (4 exponent bits of bias 7, 3 mantissa
bits, largest 448, NaN = 0x7f / 0xff) times the scale of its (page, kv head)."""
import numpy as np

from . import ops

# magnitudes of the codes 0 .. 126 in ascending order: m 2^-9, then (1 + m / 8) 2^(e - 7)
MAGNITUDES = np.array([m * 2.0 ** -9 for m in range(8)] + [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)])[:127]
LARGEST = 448.0
LEAST_EXP = -117
MOST = 1.875 * 2.0 ** 127        # finite elements beyond it are stored as it is: the next number is 2^128, in bf16 and fp32 infinite


def decode(codes):
    c = np.asarray(codes, dtype=np.uint8)
    v = np.append(MAGNITUDES, np.nan)[c & 0x7F]
    return np.where(c & 0x80, -v, v)


def encode(x):
    """nearest number, ties to the even code; what is no finite number is NaN"""
    x = np.asarray(x, dtype=np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    assert np.all(a <= LARGEST * (1 + 1e-6))
    mid = (MAGNITUDES[1:] + MAGNITUDES[:-1]) / 2
    lo, hi = np.searchsorted(mid, a, side="left"), np.searchsorted(mid, a, side="right")   # differ at a tie
    c = np.where(lo % 2 == 0, lo, hi).astype(np.uint8)
    c = np.where(np.isfinite(x), c, 0x7F).astype(np.uint8)
    return c | np.where(np.signbit(x) & np.isfinite(x), 0x80, 0).astype(np.uint8)


def scale_for(amax):
    """the least power of two from 2^-117 on that keeps amax within 448"""
    e = LEAST_EXP
    while amax > LARGEST * 2.0 ** e:
        e += 1
    return 2.0 ** e


class Cache8:
    """codes [pages, positions, nkv, d], scales [pages, nkv] of K and V"""

    def __init__(self, num_pages, page_size, nkv, d):
        self.page_size, self.nkv, self.d = page_size, nkv, d
        self.codes = {n: np.zeros((num_pages, page_size, nkv, d), dtype=np.uint8) for n in "kv"}
        self.scale = {n: np.zeros((num_pages, nkv)) for n in "kv"}

    def append(self, pages, start, k, v):
        """rows [n, nkv d] (keys after rotation) at positions start .. of the sequence that holds `pages`"""
        n, ps = len(k), self.page_size
        p = start
        while p < start + n:
            m = min(ps - p % ps, start + n - p)
            page, at = int(pages[p // ps]), p % ps
            for name, rows in (("k", k), ("v", v)):
                new = np.asarray(rows[p - start:p - start + m], dtype=np.float64).reshape(m, self.nkv, self.d)
                for h in range(self.nkv):
                    x = np.where(np.isfinite(new[:, h]), np.clip(new[:, h], -MOST, MOST), new[:, h])
                    s = scale_for(np.max(np.abs(x), where=np.isfinite(x), initial=0.0))
                    old = self.scale[name][page, h]
                    codes = self.codes[name][page, :, h]
                    if at and old >= s:
                        s = old
                    elif at:
                        codes[...] = encode(decode(codes) * (old / s))
                    codes[at:at + m] = encode(x / s)
                    self.scale[name][page, h] = s
            p += m

    def rows(self, name, pages, n):
        """the first n rows [n, nkv d] of a sequence"""
        p = np.arange(n)
        pg = np.asarray(pages, dtype=np.int64)[p // self.page_size]
        x = decode(self.codes[name][pg, p % self.page_size]) * self.scale[name][pg][:, :, None]
        return x.reshape(n, -1)

    def attention(self, q, start, pages, n_q_heads):
        """(out, lse) of the queries at positions start .. of the sequence"""
        end = start + len(q)
        return ops.attention(q, np.arange(start, end), self.rows("k", pages, end), self.rows("v", pages, end), n_q_heads, self.nkv, self.d)
