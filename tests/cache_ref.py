"""Plain 64-bit definitions of rotary positions and of the growing 8-bit cache (numpy, one element or one row at a time where that is the clearer form).
They share nothing with the library."""
import math

import numpy as np

D = 128


def e4m3_value(code):
    """Values of E4M3 codes (OCP: bias 7, largest 448, 0x7f and 0xff are NaN)."""
    code = np.asarray(code).astype(np.int64)
    e, m = (code >> 3) & 15, code & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * np.exp2(e - 10.0))
    v = np.where((code & 0x7f) == 0x7f, np.nan, v)
    return np.where(code & 0x80, -v, v)


_VALUES = e4m3_value(np.arange(0x7f))                  # ascending


def e4m3_code(x):
    """Codes of the nearest values, ties to the even code, of |x| <= 448 and NaN: by search in the table of values."""
    x = np.asarray(x, np.float64)
    a = np.abs(x)
    hi = np.minimum(np.searchsorted(_VALUES, a, side="left"), 0x7e)
    lo = np.maximum(hi - 1, 0)
    up, down = _VALUES[hi] - a, a - _VALUES[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(a == _VALUES[hi], hi, code)
    code = np.where(np.isfinite(x), code, 0x7f)
    return (code | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def scale_of(x):
    """The smallest power of two s >= 2^-100 with |x| <= 448 s for the finite x."""
    a = np.abs(x[np.isfinite(x)])
    a = float(a.max()) if a.size else 0.0
    s = 2.0 ** -100
    while a > 448.0 * s:
        s *= 2.0
    return s


def rotary(x, pos, inv_freq, rot, interleaved, mscale):
    """x [n][heads][D] float64."""
    y = x.copy()
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        for t in range(x.shape[0]):
            angle = math.fmod(float(pos[t]) * float(inv_freq[i]), 2 * math.pi)
            c, s = mscale * math.cos(angle), mscale * math.sin(angle)
            y[t, :, a], y[t, :, b] = x[t, :, a] * c - x[t, :, b] * s, x[t, :, b] * c + x[t, :, a] * s
    return y


class Cache:
    """Codes [2][L][H][T][D], scales [2][L][H][NS], gathered weights [L][H][T]; index 0 is K, 1 is V."""

    def __init__(self, cu, L, H, block):
        self.cu, self.L, self.H, self.block, self.B, self.T = list(map(int, cu)), L, H, block, len(cu) - 1, int(cu[-1])
        self.ns = self.T // block + self.B
        self.codes = np.zeros((2, L, H, self.T, D), np.uint8)
        self.scale = np.ones((2, L, H, self.ns))
        self.acc = np.zeros((L, H, self.T))

    def slot(self, b, row):
        return self.cu[b] // self.block + b + row // self.block

    def rows(self, kv, l, h, b, rows):
        """Values of rows of a sequence."""
        rows = np.asarray(rows, np.int64)
        return e4m3_value(self.codes[kv, l, h, self.cu[b] + rows]) * self.scale[kv, l, h, self.slot(b, rows)][:, None]

    def append(self, l, b, h, held, k, v):
        """k, v [m][D] float64 behind `held` rows."""
        m = min(len(k), self.cu[b + 1] - self.cu[b] - held)
        for kv, x in enumerate((k, v)):
            for first in range(held // self.block * self.block, held + m, self.block):
                lo, hi = max(first, held), min(first + self.block, held + m)
                new, at, old = x[lo - held: hi - held], self.slot(b, first), None
                s = scale_of(new)
                if first < held:
                    old = self.scale[kv, l, h, at]
                    s = max(s, old)
                    if s > old:
                        c = self.codes[kv, l, h, self.cu[b] + first: self.cu[b] + held]
                        self.codes[kv, l, h, self.cu[b] + first: self.cu[b] + held] = e4m3_code(e4m3_value(c) * (old / s))
                self.scale[kv, l, h, at] = s
                self.codes[kv, l, h, self.cu[b] + lo: self.cu[b] + hi] = e4m3_code(np.where(np.isfinite(new), new / s, np.copysign(np.nan, new)))
        self.acc[l, h, self.cu[b] + held: self.cu[b] + held + m] = 0.0

    def compact(self, l, b, h, idx, out=None):
        """Rows idx become the first ones (of `out`, another cache of the same layout, or of this one)."""
        out, n = out or self, self.cu[b + 1] - self.cu[b]
        idx = np.asarray(idx, np.int64)
        ok = (idx >= 0) & (idx < n)
        src = np.where(ok, idx, 0)
        for kv in range(2):
            codes = np.where(ok[:, None], self.codes[kv, l, h, self.cu[b] + src], 0)
            scale = np.where(ok, self.scale[kv, l, h, self.slot(b, src)], 2.0 ** -100)
            for first in range(0, len(idx), self.block):
                part = slice(first, min(first + self.block, len(idx)))
                s = scale[part].max()
                f = (scale[part] / s)[:, None]
                out.codes[kv, l, h, self.cu[b] + first: self.cu[b] + part.stop] = np.where(f == 1, codes[part], e4m3_code(e4m3_value(codes[part]) * f))
                out.scale[kv, l, h, self.slot(b, first)] = s
        acc = np.where(ok, self.acc[l, h, self.cu[b] + src], 0.0)
        out.acc[l, h, self.cu[b]: self.cu[b] + len(idx)] = acc


def attend(q, K, V):
    """One query group [G][D] over rows [n][D]: out, lse, weights [G][n], and the largest sum of |products| of a logit."""
    G, n = q.shape[0], K.shape[0]
    if n == 0:
        return np.zeros((G, D)), np.full(G, -np.inf), np.zeros((G, 0)), 0.0
    with np.errstate(invalid="ignore", over="ignore"):
        x = q @ K.T / math.sqrt(D)
        m = x.max(axis=1, keepdims=True)
        e = np.exp(x - m)
        z = e.sum(axis=1, keepdims=True)
        p = e / z
        out = np.stack([(p[g][:, None] * V).sum(axis=0) for g in range(G)])
    return out, (m + np.log(z))[:, 0], p, float(np.nanmax(np.abs(q) @ np.abs(K).T)) / math.sqrt(D)


def evict(acc, keep, sink, recent):
    """Rows that stay, ascending."""
    n = len(acc)
    if n <= keep:
        return np.arange(n)
    rest = np.arange(sink, n - recent)
    a = acc[rest]
    order = rest[np.lexsort((rest, -np.where(np.isnan(a), 0, a) + 0.0, np.isnan(a)))]
    return np.sort(np.concatenate([np.arange(sink), np.arange(n - recent, n), order[: keep - sink - recent]])).astype(np.int64)
