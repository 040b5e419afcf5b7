"""The operators of include/tst_attention.h from their definitions, in numpy: codes with the roundings to 32 bits that the definition names, attention in
64 bits, with bounds of the roundings that a kernel is allowed."""
import numpy as np

BLOCK = 16
U = 2.0 ** -24
f32 = np.float32


def rotate(x, positions, cos, sin, interleaved):
    """x float32 [T, heads, size]; positions [T]; angles that are not there are NaN."""
    pairs = cos.shape[1]
    ok = (positions >= 0) & (positions < len(cos))
    c, s = (np.where(ok[:, None], t[np.where(ok, positions, 0)], f32("nan"))[:, None] for t in (cos, sin))
    a, b = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if interleaved else (slice(0, pairs), slice(pairs, 2 * pairs))
    y = x.copy()
    with np.errstate(all="ignore"):
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


class Cache:
    """codes int8 [pages, heads, page, size], scale float32 [pages, heads, page / 16], of "k" and "v"."""

    def __init__(self, pages, page, heads, size):
        self.pages, self.page, self.heads, self.size = pages, page, heads, size
        self.codes = {n: np.zeros((pages, heads, page, size), np.int8) for n in "kv"}
        self.scale = {n: np.zeros((pages, heads, page // BLOCK), np.float32) for n in "kv"}

    def page_of(self, table, i, p):
        """None if the cache has no such page."""
        if p < 0 or p // self.page >= table.shape[1]:
            return None
        got = int(table[i, p // self.page])
        return got if 0 <= got < self.pages else None

    def append(self, name, x, table, i, first):
        """x float32 [n, heads, size] at positions first .. of sequence i."""
        n = len(x)
        for b in range(first // BLOCK, (first + n - 1) // BLOCK + 1):
            lo, hi = max(first, b * BLOCK), min(first + n, (b + 1) * BLOCK)
            page = self.page_of(table, i, b * BLOCK)
            if page is None:
                continue
            at, slot = b * BLOCK % self.page, b * BLOCK % self.page // BLOCK
            for h in range(self.heads):
                new, old = x[lo - first:hi - first, h], self.scale[name][page, h, slot]
                there = lo - b * BLOCK
                codes = self.codes[name][page, h, at:at + BLOCK]
                with np.errstate(all="ignore"):
                    a = np.abs(new).max()
                    if not np.isfinite(a) or (there and np.isnan(old)):
                        self.scale[name][page, h, slot] = np.nan
                        codes[there:there + len(new)] = 0
                        continue
                    s = a / f32(127)
                    if there:
                        s = max(s, old)
                        if s > old:
                            codes[:there] = np.rint(codes[:there].astype(np.float32) * (old / s))
                    r = min(f32(1) / s, np.finfo(np.float32).max)
                    codes[there:there + len(new)] = np.clip(np.rint(new * r), -127, 127)
                self.scale[name][page, h, slot] = s

    def values(self, name, table, i, first, last, dtype=np.float32):
        """[last - first, heads, size] of positions first .. last - 1; NaN where there is no page."""
        out = np.full((last - first, self.heads, self.size), np.nan, dtype)
        for p in range(first, last):
            page = self.page_of(table, i, p)
            if page is not None:
                out[p - first] = self.codes[name][page, :, p % self.page].astype(dtype) * self.scale[name][page, :, p % self.page // BLOCK, None].astype(dtype)
        return out


def attention(q, k, v, limit, scale, weight, cut=0.0):
    """One head in 64 bits: q [n, size], k, v [m, size], limit [n]: row i sees keys below limit[i].  -> (Y, bound of |error| before the result is rounded).

    weight: relative rounding of a weight (0 where it has none); cut: that of a query's entry relative to the largest of its row.  A logit is a sum of `size` products in fp32,
    a product by its factor, a subtraction of the largest; an exponential is off by 2^-22 of itself at most; sums of m weights in fp32, in any order.
    A weight that is off by e^d has d twice (above and below the line)."""
    m, size = k.shape
    Y, bound = np.zeros(q.shape), np.zeros(q.shape)
    with np.errstate(all="ignore"):
        z = scale * (q @ k.T)
        dz = abs(scale) * ((size + 8) * U * (np.abs(q) @ np.abs(k).T) + cut * np.abs(q).max(1, keepdims=True, initial=0) * np.abs(k).sum(1)) + 8 * U * np.abs(z)
        for i in range(len(q)):
            n = min(int(limit[i]), m)
            if n <= 0:
                continue
            zi = z[i, :n]
            p = np.exp(zi - zi.max())
            p /= p.sum()
            Y[i] = p @ v[:n]
            d = dz[i, :n].max() + 4 * U * np.abs(zi - zi.max()).max(where=p > 1e-30, initial=0)
            off = 2 * (np.expm1(min(d, 50)) + 2.0 ** -22 + (n + 8) * U) + weight
            bound[i] = off * (p @ np.abs(v[:n])) + n * 2.0 ** -38 * np.abs(v[:n]).max(0)
    return Y, bound
