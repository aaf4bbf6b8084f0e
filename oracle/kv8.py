"""The 8-bit cache in plain numpy, 64 bits, straight from its definition (test
infrastructure; shares no code with the kernels).

An element is value(code) * 2^e with the e4m3 codes of the OCP 8-bit format and
one exponent per (page, KV head, block of positions)."""
from __future__ import annotations

import numpy as np


def _code_values():
    """Value of each of the 256 codes: sign, 4 exponent bits (bias 7), 3 mantissa bits."""
    v = np.zeros(256)
    for c in range(256):
        s, x, m = c >> 7, (c >> 3) & 15, c & 7
        a = (m / 8) * 2.0 ** -6 if x == 0 else (1 + m / 8) * 2.0 ** (x - 7)
        v[c] = np.nan if c & 127 == 127 else (-a if s else a)
    return v


VALUES = _code_values()
_POS = VALUES[:127]                       # ascending, 0 .. 448
_MID = (_POS[:-1] + _POS[1:]) / 2         # exact in binary64


def encode(y):
    """Nearest codes of finite y (|y| saturates at 448), ties to the even code."""
    y = np.asarray(y, np.float64)
    a = np.minimum(np.abs(y), 448.0)
    c = np.searchsorted(_MID, a, side="left")     # first midpoint >= a
    at = np.minimum(c, 125)
    tie = (c < 126) & (a == _MID[at])
    c = c + (tie & (c % 2 == 1))                  # the even one of c and c + 1
    return (c | (np.signbit(y).astype(np.int64) << 7)).astype(np.uint8)


def exponent(amax):
    """The least e >= -126 with amax <= 448 * 2^e."""
    if amax == 0:
        return -126
    m, x = np.frexp(np.float64(amax))             # amax = m 2^x, m in [0.5, 1)
    return max(-126, int(x) - 9 + int(m > 0.875))


def clean(x):
    """What the quantizer takes non-finite inputs for: (x with NaN as +0, finite mask)."""
    x = np.asarray(x, np.float64)
    return np.where(np.isnan(x), 0.0, x), np.isfinite(x)


class Cache:
    """Pools as [NP][Hkv][P][d] codes and [NP][Hkv][P / block] exponent bytes, K and V."""

    def __init__(self, P, hkv, d, block, pages, fill=0):
        self.P, self.hkv, self.d, self.block, self.pages = P, hkv, d, block, pages
        self.codes = [np.full((pages, hkv, P, d), fill, np.uint8) for _ in range(2)]
        self.exps = [np.full((pages, hkv, P // block), fill, np.uint8) for _ in range(2)]

    def append(self, k, v, cu, start, tables):
        """Rows k, v [rows][hkv][d] as 64-bit numbers."""
        tables = np.asarray(tables)
        for b in range(len(start)):
            for i in range(cu[b], cu[b + 1]):
                pos = start[b] + i - cu[b]
                if pos % self.block and i > cu[b] and pos > 0:
                    continue                       # taken with its block's first new row
                n = min(self.block - pos % self.block, cu[b + 1] - i)
                if pos < 0:
                    n = 1
                self._block(k[i:i + n], v[i:i + n], b, pos, tables)

    def _block(self, k, v, b, pos, tables):
        if pos < 0 or pos // self.P >= tables.shape[1]:
            return
        page = tables[b, pos // self.P]
        if not 0 <= page < self.pages:
            return
        slot = pos % self.P
        at, lo = slot // self.block, slot % self.block
        for which, x in ((0, k), (1, v)):
            x, fin = clean(x)
            for h in range(self.hkv):
                a = np.abs(x[:, h])[fin[:, h]]
                e = exponent(a.max() if a.size else 0.0)
                c, ex = self.codes[which][page, h], self.exps[which][page, h]
                if lo:
                    old = int(ex[at]) - 127
                    if old >= e:
                        e = old
                    else:
                        held = slice(slot - lo, slot)
                        c[held] = encode(VALUES[c[held]] * 2.0 ** (old - e))
                ex[at] = e + 127
                with np.errstate(over="ignore", invalid="ignore"):
                    c[slot:slot + len(x)] = encode(x[:, h] * 2.0 ** -e)

    def values(self, which, table, n, h):
        """Positions 0 .. n - 1 of head h: [n][d], and which of them exist."""
        pos = np.arange(n)
        page = np.asarray(table)[pos // self.P]
        ok = (page >= 0) & (page < self.pages)
        page = np.where(ok, page, 0)
        slot = pos % self.P
        e = self.exps[which][page, h, slot // self.block].astype(np.float64) - 127
        x = VALUES[self.codes[which][page, h, slot]] * 2.0 ** e[:, None]
        return np.where(ok[:, None], x, 0.0), ok

    def pool_bytes(self):
        """The four arrays in the library's byte order: k_codes, k_exps, v_codes, v_exps."""
        v = self.codes[1].reshape(self.pages, self.hkv, self.P // 16, 4, 4, self.d // 64, 16, 4)
        v = v.transpose(0, 1, 2, 5, 3, 6, 7, 4)
        return (self.codes[0].reshape(-1), self.exps[0].reshape(-1),
                np.ascontiguousarray(v).reshape(-1), self.exps[1].reshape(-1))


def attend(cache, q, table, total, scale):
    """Rows q [T][hq][d], the last T of `total` positions, over one request:
    out [T][hq][d], lse [T][hq], weights [hkv][total] and, for error bounds, the
    sums p |v| like out, sum |v| like out, and the largest scale * sum |q k|."""
    T, hq, d = q.shape
    g = hq // cache.hkv
    q = np.asarray(q, np.float64)
    out, spread, allv = (np.zeros((T, hq, d)) for _ in range(3))
    lse = np.full((T, hq), -np.inf)
    weights = np.zeros((cache.hkv, total))
    dots = 0.0
    for h in range(cache.hkv):
        k, ok = cache.values(0, table, total, h)
        v, _ = cache.values(1, table, total, h)
        for i in range(T):
            n = total - T + 1 + i
            use = np.nonzero(ok[:max(n, 0)])[0]
            if not use.size:
                continue
            for j in range(h * g, h * g + g):
                z = scale * (k[use] @ q[i, j])
                dots = max(dots, float(np.max(abs(scale) * (np.abs(k[use]) @ np.abs(q[i, j])))))
                top = z.max()
                p = np.exp(z - top)
                l = p.sum()
                p /= l
                lse[i, j] = top + np.log(l)
                out[i, j] = p @ v[use]
                spread[i, j] = p @ np.abs(v[use])
                allv[i, j] = np.abs(v[use]).sum(0) / l
                weights[h, use] += p
    return dict(out=out, lse=lse, weights=weights, spread=spread, allv=allv, dots=dots)


def pick(w, n, keep, recent):
    """Positions that stay of n with weights w, ascending."""
    m, r = min(n, keep), min(recent, n)
    rank = [(-np.inf if np.isnan(x) else -float(x), t) for t, x in enumerate(w[:n - r])]
    # NaN before any number, infinity included
    order = sorted(range(n - r), key=lambda t: (not np.isnan(w[t]), rank[t][0], t))
    return sorted(order[:m - r]) + list(range(n - r, n))


def evict(cache, tables, lens, w, keep, recent, dst):
    """Moves the kept positions into dst's pages (in place in the cache)."""
    B = len(lens)
    kept = np.full((B, cache.hkv, keep), -1, np.int32)
    kept_w = np.zeros((B, cache.hkv, keep), np.float32)
    cap = np.asarray(tables).shape[1] * cache.P
    moved = []
    for b in range(B):
        n = min(max(lens[b], 0), cap)
        for h in range(cache.hkv):
            t = pick(w[b, h], n, keep, recent)
            kept[b, h, :len(t)] = t
            kept_w[b, h, :len(t)] = w[b, h, t]
            moved.append((b, h, t, [cache.values(i, tables[b], n, h)[0][t] if n else None
                                    for i in range(2)]))
    for b, h, t, rows in moved:
        for j in range(0, len(t), cache.block):
            page = dst[b][j // cache.P]
            if not 0 <= page < cache.pages:
                continue
            slot = j % cache.P
            for which in range(2):
                x = rows[which][j:j + cache.block]
                e = exponent(np.abs(x).max())
                cache.exps[which][page, h, slot // cache.block] = e + 127
                cache.codes[which][page, h, slot:slot + len(x)] = encode(x * 2.0 ** -e)
    return kept, kept_w
