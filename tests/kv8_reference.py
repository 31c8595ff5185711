"""64-bit reference of the 8-bit KV cache, one sequence at a time (numpy)."""
import numpy as np

TOP = {"int8": 127.0, "fp8": 448.0}


def e4m3_value(code):
    """Values of e4m3 code bytes: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7F and 0xFF are NaN."""
    c = np.asarray(code, np.uint8).astype(np.int64)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where((c & 0x7F) == 0x7F, np.nan, v)
    return np.where(c & 0x80, -v, v)


def value(code, fmt):
    return np.asarray(code).view(np.int8).astype(np.float64) if fmt == "int8" else e4m3_value(code)


_E4M3 = np.sort(np.unique(e4m3_value(np.arange(127))))         # the magnitudes, 0 .. 448


def nearest(y, fmt):
    """y (|y| <= 127 or 448) to the nearest value of a code, ties to the even one."""
    if fmt == "int8":
        return np.rint(y)
    a = np.abs(y)
    hi = np.searchsorted(_E4M3, a)                              # first magnitude >= a
    lo = np.maximum(hi - 1, 0)
    down, up = a - _E4M3[lo], _E4M3[hi] - a
    take_lo = (down < up) | ((down == up) & (lo % 2 == 0))      # neighbours alternate in the last mantissa bit
    return np.copysign(np.where(take_lo, _E4M3[lo], _E4M3[hi]), y)


def exponent(amax, fmt):
    """The smallest b in 1..254 with amax <= TOP 2^(b - 127)."""
    if not np.isfinite(amax):
        return 255
    b = 1
    while amax > TOP[fmt] * 2.0 ** (b - 127):
        b += 1
    return b


class Cache:
    """Pages of values: val [page][head][slot][dim] (multiples of the page's scale) and exponent bytes."""

    def __init__(self, n_pages, hkv, hd, fmt):
        self.fmt, self.hkv, self.hd = fmt, hkv, hd
        self.val = np.zeros((n_pages, hkv, 16, hd))
        self.exp = np.zeros((n_pages, hkv), np.int64)

    def write(self, x, table, start):
        """x [tokens][head][dim] at positions start.. of a page table (-1: no page)."""
        for pg in range(start // 16, -(-(start + len(x)) // 16)):
            if pg >= len(table) or not 0 <= table[pg] < len(self.val):
                continue
            s0, s1 = max(0, start - 16 * pg), min(16, start + len(x) - 16 * pg)
            for h in range(self.hkv):
                new = x[16 * pg + s0 - start:16 * pg + s1 - start, h].astype(np.float64)
                b = exponent(np.max(np.abs(new)) if np.all(np.isfinite(new)) else np.inf, self.fmt)
                if s0 > 0:
                    b = max(b, int(self.exp[table[pg], h]))
                scale = 2.0 ** (b - 127)
                page = self.val[table[pg], h]
                if b == 255:
                    page[s0:s1] = 0.0
                else:
                    page[:s0] = nearest(page[:s0] / scale, self.fmt) * scale
                    page[s0:s1] = nearest(new / scale, self.fmt) * scale
                self.exp[table[pg], h] = b

    def read(self, table, start, n):
        out = np.zeros((n, self.hkv, self.hd))
        for t in range(n):
            pg, slot = (start + t) // 16, (start + t) % 16
            if pg < len(table) and 0 <= table[pg] < len(self.val):
                out[t] = np.where((self.exp[table[pg]] == 255)[:, None], np.nan, self.val[table[pg], :, slot])
        return out


def attention(q, k, v, present, ctx, scale):
    """q [n][Hq][hd] are the last n of ctx tokens; k, v [>= ctx][Hkv][hd]; present [>= ctx] says which positions have
    a page.  Rows that see nothing are 0."""
    n, hq, hd = q.shape
    group = hq // k.shape[1]
    out = np.zeros((n, hq, hd))
    for t in range(n):
        seen = np.flatnonzero(present[:max(0, ctx - n + t + 1)])
        if not len(seen):
            continue
        for h in range(hq):
            s = scale * (k[seen, h // group] @ q[t, h].astype(np.float64))
            p = np.exp(s - np.max(s))
            out[t, h] = (p / p.sum()) @ v[seen, h // group]
    return out
