"""The attention block's operators in 64 bits, plain numpy and loops, for the tests."""
import math

import numpy as np

B = 64
Q = {"e4m3": 448.0, "int8": 127.0}


def _e4m3_table():
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = (1 + m / 8) * 2.0 ** (e - 7) if e else m * 2.0 ** -9
        out[c] = -v if c & 128 else v
    out[0x7F] = out[0xFF] = np.nan
    return out


E4M3 = _e4m3_table()
_GRID = E4M3[:0x7F]                      # the non-negative values, ascending


def decode(codes, fmt):
    codes = np.asarray(codes, dtype=np.uint8)
    return codes.view(np.int8).astype(np.float64) if fmt == "int8" else E4M3[codes]


def nearest(x, fmt):
    """x (already divided by the scale) as the nearest representable value, ties to even, clamped."""
    x = np.clip(np.asarray(x, dtype=np.float64), -Q[fmt], Q[fmt])
    if fmt == "int8":
        return np.rint(x)
    a = np.abs(x)
    hi = np.clip(np.searchsorted(_GRID, a), 1, len(_GRID) - 1)
    lo = hi - 1
    dl, dh = a - _GRID[lo], _GRID[hi] - a
    up = (dh < dl) | ((dh == dl) & (hi % 2 == 0))
    return np.copysign(np.where(up, _GRID[hi], _GRID[lo]), x)


def scale_of(x, fmt):
    """Least power of two s >= 2^-64 with |x| <= Q s over the finite x."""
    x = np.abs(np.asarray(x, dtype=np.float64))
    top = float(np.max(x[np.isfinite(x)], initial=0.0))
    e = -64
    if top > 0:
        e = max(e, math.frexp(top / Q[fmt])[1] - 2)
        while top > Q[fmt] * 2.0 ** e:
            e += 1
    return 2.0 ** e


class Cache:
    """A copy of a cache on the host: data uint8 [P, H, 2, 64, D], scales, mass."""

    def __init__(self, data, scales, mass, fmt):
        self.data, self.scales, self.fmt = np.array(data), np.array(scales), fmt
        self.mass = None if mass is None else np.array(mass)

    def values(self, page, h, j, slots=slice(None)):
        return decode(self.data[page, h, j, slots], self.fmt) * np.float64(self.scales[page, h, j])

    def put(self, page, h, j, slot, scaled):
        """Codes of values already divided by the scale (nearest() of them)."""
        v = nearest(scaled, self.fmt)
        if self.fmt == "int8":
            self.data[page, h, j, slot] = v.astype(np.int8).view(np.uint8)
        else:
            c = np.searchsorted(_GRID, np.abs(v)).astype(np.uint8)
            self.data[page, h, j, slot] = c | np.where(np.signbit(v), 128, 0).astype(np.uint8)

    def sequence(self, table, length):
        """K and V [H, length, D] of the tokens; a bad page's are NaN."""
        P, H, _, _, D = self.data.shape
        out = np.full((2, H, length, D), np.nan)
        for t0 in range(0, length, B):
            p, n = int(table[t0 // B]), min(B, length - t0)
            if 0 <= p < P:
                for h in range(H):
                    for j in (0, 1):
                        out[j, h, t0:t0 + n] = self.values(p, h, j, slice(0, n))
        return out

    def append(self, table, lens, cu, k, v):
        """k, v [rows, H, D] float64 (bf16 values); returns the status bits."""
        P, H, _, _, D = self.data.shape
        status = 0
        for i, length in enumerate(lens):
            n = cu[i + 1] - cu[i]
            start = length - n
            for b in range(start // B, -(-length // B) if n else 0):
                p = int(table[i][b])
                if not 0 <= p < P:
                    status |= 1
                    continue
                lo, hi = max(start - b * B, 0), min(length - b * B, B)
                r = cu[i] + b * B + lo - start
                for j, x in enumerate((k, v)):
                    for h in range(H):
                        new = x[r:r + hi - lo, h]
                        if not np.isfinite(new).all():
                            status |= 2
                        s = scale_of(new, self.fmt)
                        if lo:
                            old = np.float64(self.scales[p, h, j])
                            if s > old:
                                self.put(p, h, j, slice(0, lo), self.values(p, h, j, slice(0, lo)) / s)
                            s = max(s, old)
                        with np.errstate(invalid="ignore"):
                            scaled = np.where(np.isnan(new), 0.0, new) / s
                        self.put(p, h, j, slice(lo, hi), scaled)
                        self.scales[p, h, j] = s
                if self.mass is not None:
                    self.mass[p, :, lo:hi] = 0
        return status


def attention(cache, table, lens, cu, q, scale, G, mass_rows=0, decay=1.0):
    """(out, bound of the rounding of out, mass) in 64 bits.  q [rows, Hq, D] float64.

    The bound counts, per element, half a step of bf16 for the output and for
    every probability (2^-8 of it), and 2^-20 for the fp32 arithmetic of scores
    and sums (scores up to 32: 5 units of 2^-24 times 32 times ln 2 for each of a
    probability's numerator and sum)."""
    P, H, _, _, D = cache.data.shape
    out, tol = np.zeros_like(q), np.zeros_like(q)
    mass = None if cache.mass is None else cache.mass.astype(np.float64)
    for i, length in enumerate(lens):
        n = cu[i + 1] - cu[i]
        kv = cache.sequence(table[i], length)
        good = np.array([0 <= int(table[i][t // B]) < P for t in range(length)], dtype=bool)
        w = np.zeros((H, length))
        for r in range(n):
            see = good & (np.arange(length) <= length - n + r)
            if not see.any():
                continue
            for a in range(H * G):
                h = a // G
                s = kv[0, h, see] @ q[cu[i] + r, a] * scale
                p = np.exp(s - s.max())
                p /= p.sum()
                v = kv[1, h, see]
                out[cu[i] + r, a] = p @ v
                tol[cu[i] + r, a] = 2.0 ** -8 * np.abs(p @ v) + (2.0 ** -8 + 2.0 ** -16) * (p @ np.abs(v)) + 1e-30
                if r >= n - mass_rows:
                    w[h, see] += p
        if mass_rows and mass is not None:
            for t in range(length):
                p = int(table[i][t // B])
                if 0 <= p < P:
                    mass[p, :, t % B] = (mass[p, :, t % B] * decay if decay else 0.0) + w[:, t]
    return out, tol, mass


def select(mass, length, budget, sinks, recent):
    """Kept tokens of one head, ascending."""
    if length <= budget:
        return list(range(length))
    fixed = [t for t in range(length) if t < sinks or t >= length - recent]
    key = lambda t: (-math.inf if math.isnan(mass[t]) else mass[t])  # noqa: E731
    rest = sorted((t for t in range(length) if sinks <= t < length - recent), key=lambda t: (math.isnan(mass[t]), -key(t), t))
    return sorted(fixed + rest[:budget - len(fixed)])


def evict(cache, table, lens, dst, budget, sinks, recent):
    """Cuts the cache copy back in place; returns keep [S, H, budget]."""
    P, H, _, _, D = cache.data.shape
    keep = np.full((len(lens), H, budget), -1, dtype=np.int32)
    for i, length in enumerate(lens):
        for h in range(H):
            m = np.array([cache.mass[table[i][t // B], h, t % B] for t in range(length)], dtype=np.float64)
            kept = select(m, length, budget, sinks, recent)
            keep[i, h, :len(kept)] = kept
            kv = cache.sequence(table[i], length)
            for b in range(0, len(kept), B):
                at = kept[b:b + B]
                p = int(dst[i][b // B])
                for j in (0, 1):
                    x = kv[j, h, at]
                    s = scale_of(x, cache.fmt)
                    cache.scales[p, h, j] = s
                    cache.put(p, h, j, slice(0, len(at)), x / s)
                cache.mass[p, h, :len(at)] = m[at]
    return keep


def linear(x, w, bias, act, residual):
    y = x @ w.T
    if bias is not None:
        y = y + bias
    from scipy.special import erf, expit
    if act == "silu":
        y = y * expit(y)
    elif act == "gelu":
        y = 0.5 * y * (1 + erf(y / math.sqrt(2)))
    elif act == "gelu_tanh":
        y = 0.5 * y * (1 + np.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
    return y if residual is None else y + residual
