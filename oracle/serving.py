"""64-bit forms of shaped sampling, shaped acceptance and the 4-bit K/V cache, from their definitions, in numpy.

TEST INFRASTRUCTURE ONLY: nothing of the product path imports this."""
from __future__ import annotations

import numpy as np

GROUP, UNIT, LIMIT = 32, 16, 2.0 ** 48


# ---- bf16 as float64 values
def bf16(x):
    """Nearest bf16 value (ties to even) of float64 numbers, by way of float32 as the library's conversion has it."""
    b = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    r = ((b + 0x7fff + ((b >> 16) & 1)) >> 16).astype(np.uint32) << 16
    return r.view(np.float32).astype(np.float64)


def bf16_bits(x):
    return (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)


# ---- shaping
def shaped(logits, t=1.0, k=0, p=1.0, mp=0.0):
    """Kept weights of one row in id order, or None where the row has no distribution."""
    x = np.asarray(logits, np.float64)
    if np.isnan(x).any() or (x == np.inf).any() or not np.isfinite(x).any():
        return None
    if not (np.isfinite(t) and t >= 0 and p > 0 and 0 <= mp <= 1):
        return None
    t, p, mp = (float(np.float32(v)) for v in (t, p, mp))
    order = np.argsort(-x, kind="stable")
    top = x[order[0]]
    w = np.zeros_like(x)
    if t == 0:
        w[order[0]] = 1.0
        return w
    with np.errstate(over="ignore"):
        e = np.exp((x[order] - top) / t)
    if k > 0:
        e[k:] = 0.0
    if p < 1:
        run = np.cumsum(e)
        e = np.where(run - e < p * run[-1], e, 0.0)
    w[order] = np.where(e >= mp, e, 0.0)
    return w


def draw(w, u):
    """(first id whose running weight exceeds u times the whole, distance of u to the edges of its share)."""
    run = np.cumsum(w)
    j = int(np.searchsorted(run, float(u) * run[-1], side="right"))
    lo, hi = (run[j - 1] if j else 0.0) / run[-1], run[j] / run[-1]
    return j, min(float(u) - lo if lo > 0 else 1.0, hi - float(u))


def accept(logits, settings, q, drafts, u):
    """(accepted, token, smallest distance of any decision to its border) of one request."""
    k, margin = len(logits) - 1, 1.0
    for i in range(k + 1):
        w = shaped(logits[i], *settings)
        if w is None:
            return i, -1, margin
        P = w / w.sum()
        if i == k:
            break
        x = int(drafts[i])
        if 0 <= x < len(w):
            qx = float(q[i][x])
            ratio = min(P[x] / qx if qx > 0 else (np.inf if P[x] > 0 else 0.0), 1.0)
            if ratio < 1:
                margin = min(margin, abs(float(u[i]) - ratio))
            if qx >= 0 and 0 <= float(u[i]) < ratio:
                continue
        if not (np.asarray(q[i])[P > 0] >= 0).all():
            return i, -1, margin
        rest = np.maximum(P - np.asarray(q[i], np.float64), 0.0, where=P > 0, out=np.zeros_like(P))
        if rest.sum() > 0:
            P = rest
        break
    if not 0 <= float(u[k]) < 1:
        return i, -1, margin
    token, m = draw(P, u[k])
    return i, token, min(margin, m)


# ---- the 4-bit cache
def quantise(x):
    """Codes, scales and zeros of rows [..., columns] in groups of 32."""
    x = np.nan_to_num(np.asarray(x, np.float64), nan=0.0, posinf=LIMIT, neginf=-LIMIT).clip(-LIMIT, LIMIT)
    x = x.reshape(*x.shape[:-1], -1, GROUP)
    zero = bf16(x.min(-1))
    scale = bf16((x.max(-1) - zero) / 15)
    safe = np.where(scale > 0, scale, 1.0)
    codes = np.where(scale[..., None] > 0, np.rint((x - zero[..., None]) / safe[..., None]).clip(0, 15), 0).astype(np.uint8)
    return codes, scale, zero


def values(codes, scale, zero):
    v = codes * scale[..., None] + zero[..., None]
    return v.reshape(*v.shape[:-2], -1)


class Cache:
    """One layer's pool as bytes [pages, heads, units, 20 * head_dim], one nibble at a time."""

    def __init__(self, pool, head_dim, page_size):
        self.pool, self.hd, self.page = pool, head_dim, page_size

    def _unit(self, table_row, head, pos):
        page = int(table_row[pos // self.page]) if pos // self.page < len(table_row) else -1
        if not 0 <= page < self.pool.shape[0]:
            return None
        return self.pool[page, head, pos % self.page // UNIT]

    def _nibbles(self, kv, slot):
        """Byte and shift of every column of a position."""
        c, g = np.arange(self.hd), self.hd // GROUP
        if kv == 0:
            return slot * (self.hd // 2) + (c % 32 // 8 * g + c // 32) * 4 + c % 8 // 2, 4 * (c % 2)
        tile, nib = c // 16, c // 8 % 2 + 2 * (slot // 8) + 4 * (slot % 2)
        lane = c % 8 * 4 + slot % 8 // 2
        return 10 * self.hd + ((tile // 4 * 32 + lane) * 4 + tile % 4) * 4 + nib // 2, 4 * (nib % 2)

    def _scales(self, kv, slot):
        g = np.arange(self.hd // GROUP)
        if kv == 0:
            s = 8 * self.hd + (slot * len(g) + g) * 4
            return s, s + 2
        s = 18 * self.hd + (g * UNIT + slot) * 2
        return s, s + self.hd

    def write(self, table_row, head, pos, kv, row):
        unit = self._unit(table_row, head, pos)
        if unit is None:
            return
        codes, scale, zero = quantise(row)
        at, shift = self._nibbles(kv, pos % UNIT)
        for b, s, c in zip(at, shift, codes.reshape(-1)):
            unit[b] = unit[b] & ~(15 << s) & 255 | int(c) << int(s)
        for where, what in zip(self._scales(kv, pos % UNIT), (scale, zero)):
            bits = bf16_bits(what)
            unit[where], unit[where + 1] = bits & 255, bits >> 8

    def parts(self, table_row, head, pos, kv):
        """(codes, scales, zeros) by column, or None where there is no page."""
        unit = self._unit(table_row, head, pos)
        if unit is None:
            return None
        at, shift = self._nibbles(kv, pos % UNIT)
        codes = (unit[at] >> shift & 15).astype(np.float64)
        s, z = ((unit[w].astype(np.uint32) | unit[w + 1].astype(np.uint32) << 8) << 16 for w in self._scales(kv, pos % UNIT))
        s, z = (np.repeat(v.view(np.float32).astype(np.float64), GROUP) for v in (s, z))
        return codes, s, z

    def attend(self, q, table_row, head, last, scale):
        """Outputs of query rows q [rows, hd] over positions 0..last, and what bounds their rounding: the p-weighted sum of
        scale * |code - 8| + |zero + 8 scale| of the values, and the largest score's sum of magnitudes."""
        ks, vs, size = [], [], []
        mag = np.zeros(len(q))
        for pos in range(last + 1):
            k = self.parts(table_row, head, pos, 0)
            if k is None:
                continue
            v = self.parts(table_row, head, pos, 1)
            ks.append(k[0] * k[1] + k[2])
            vs.append(v[0] * v[1] + v[2])
            size.append(v[1] * abs(v[0] - 8) + abs(v[2] + 8 * v[1]))
            mag = np.maximum(mag, abs(q) @ (15 * abs(k[1]) + abs(k[2])) * scale)
        if not ks:
            return np.zeros_like(q), np.zeros_like(q), mag
        s = q @ np.array(ks).T * scale
        e = np.exp(s - s.max(1, keepdims=True))
        e /= e.sum(1, keepdims=True)
        return e @ np.array(vs), e @ np.array(size), mag
