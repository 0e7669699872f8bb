"""Plain forms of the 8-bit cache, in numpy, written from the formulas of include/conduit.h.

Codes are bytes (sign, 4 exponent bits, 3 of the mantissa); rotated keys come from fp32 operations rounded
one by one, so codes are compared bit for bit.
"""

import numpy as np

E_LO, E_HI, NAN = -40, 119, 0x7F
f32 = np.float32


def _table():
    b = np.arange(128)
    power, part = b >> 3, b & 7
    x = np.where(power > 0, (8 + part) * 2.0 ** (power - 10.0), part * 2.0 ** -9)
    x[127] = np.nan
    return np.concatenate([x, -x])


TABLE = _table()


def encode(x):
    """The bytes of the nearest codes of float64 x, |x| <= 448 2^0 or beyond (then +-448); half to even."""
    x = np.asarray(x, dtype=np.float64)
    size = np.minimum(np.abs(x), 448.0)
    bad = np.isnan(size)
    size = np.where(bad, 0.0, size)
    _, e = np.frexp(np.maximum(size, 2.0 ** -6))  # size in [2^(e-1), 2^e)
    step = np.ldexp(1.0, e - 4)
    r = np.rint(size / step) * step
    at = np.searchsorted(TABLE[:127], r)
    return np.where(bad, NAN, at + np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def exponent(top):
    """Least e with top <= 448 2^e, within the range of a scale."""
    if top == 0:
        return E_LO
    f, x = np.frexp(np.float64(top))
    return int(np.clip(x - 9 + (2 * f > 1.75), E_LO, E_HI))


def rotate32(x, pos, table, axis, layout="halves"):
    """fp32 rows [T, H, d] turned by int positions [A, T], each operation rounded."""
    x = np.array(x, dtype=f32)
    half = len(axis)
    p = np.arange(half)
    cs = np.asarray(table, dtype=f32)[np.asarray(pos)[np.asarray(axis)].T, p]  # [T, pairs, 2]
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    i, j = (p, p + half) if layout == "halves" else (2 * p, 2 * p + 1)
    a, b = x[..., i], x[..., j]
    y = x.copy()
    with np.errstate(invalid="ignore"):
        y[..., i] = (a * c).astype(f32) - (b * s).astype(f32)
        y[..., j] = (b * c).astype(f32) + (a * s).astype(f32)
    return y


class Blocks:
    """Blocks of one layer, request and head, K or V: codes [tokens, d] (bytes) and an exponent for each 16."""

    def __init__(self, capacity, d):
        n = -(-capacity // 16)
        self.codes = np.zeros((16 * n, d), dtype=np.uint8)
        self.exp = [None] * n
        self.held = np.zeros(16 * n, dtype=bool)  # tokens that were ever written

    def append(self, begin, rows, ok=None):
        """fp32 rows become tokens begin .. ; ok: those that are written."""
        ok = np.ones(len(rows), dtype=bool) if ok is None else np.asarray(ok)
        for b in range(begin // 16, (begin + len(rows) - 1) // 16 + 1):
            at = [j for j in range(max(begin, 16 * b), min(begin + len(rows), 16 * b + 16)) if ok[j - begin]]
            if not at:
                continue
            x = np.array([rows[j - begin] for j in at], dtype=np.float64)
            x[~np.isfinite(x)] = np.nan
            fin = np.abs(x[np.isfinite(x)])
            e = exponent(fin.max() if fin.size else 0.0)
            old = slice(16 * b, max(16 * b, begin))
            if begin > 16 * b:
                was = self.exp[b] if self.exp[b] is not None else E_LO
                e = max(e, was)
                if e > was:
                    self.codes[old] = encode(TABLE[self.codes[old]] * 2.0 ** (was - e))
            self.exp[b] = e
            self.codes[at] = encode(x * 2.0 ** -float(e))
            self.held[at] = True

    def values(self, n):
        e = np.repeat([0 if x is None else x for x in self.exp], 16)[:n, None].astype(np.float64)
        return TABLE[self.codes[:n]] * 2.0 ** e


def put_block(rec, k, v, b, held=None):
    """Writes block b of the Blocks k and v into the bytes rec [32 d + 16]; `held` tokens alone."""
    d = k.codes.shape[1]
    held = k.held[16 * b:16 * b + 16] if held is None else held
    t = np.arange(16)[held][:, None]
    i = np.arange(d)[None, :]
    rec[t // 8 * 8 * d + i // 16 * 128 + t % 8 * 16 + i % 16] = k.codes[16 * b:16 * b + 16][held]
    rec[16 * d + i * 16 + t % 8 // 2 * 4 + t // 8 * 2 + t % 2] = v.codes[16 * b:16 * b + 16][held]
    if k.exp[b] is not None:
        rec[32 * d:32 * d + 8] = np.array([2.0 ** k.exp[b], 2.0 ** v.exp[b]], dtype="<f4").view(np.uint8)
