"""Plain forms of drafted trees' masks, of the bf16 cache's pages and of attention over both, from their definitions.

TEST INFRASTRUCTURE ONLY: nothing of the product path imports this."""
from __future__ import annotations

import numpy as np


# ---- trees
def ancestors(parents, words):
    """(mask uint32 [n, words], depth [n]) of one request's tree, a set per node."""
    n = len(parents)
    mask, depth = np.zeros((n, words), np.uint32), np.full(n, -1, np.int32)
    sets = []
    for i, p in enumerate(parents):
        sets.append((sets[p] if 0 <= p < i else set()) | {i})
        if i < 32 * words:
            depth[i] = len(sets[i]) - 1
            for j in sets[i]:
                mask[i, j // 32] |= np.uint32(1 << j % 32)
    return mask, depth


def bits_of(mask, n):
    """Mask rows as truth values [rows, n]."""
    m = np.asarray(mask).view(np.uint32)
    j = np.arange(n)
    inside = j // 32 < m.shape[1]
    return (m[:, np.minimum(j // 32, m.shape[1] - 1)] >> (j % 32).astype(np.uint32) & 1).astype(bool) & inside


# ---- pages
def block_index(slot, e, hd):
    """Where element (slot, e) lies inside a (page, K or V, head) block: [slot / 8][e / 8][slot % 8][e % 8]."""
    return slot // 8 * 8 * hd + e // 8 * 64 + slot % 8 * 8 + e % 8


class Pool:
    """A pool as 16-bit patterns [layers, pages, 2, heads, page_size * hd]."""

    def __init__(self, bits, hd, page):
        self.bits, self.hd, self.page = bits, hd, page
        self.n_pages = bits.shape[1]

    def where(self, table_row, pos):
        c = pos // self.page
        if pos < 0 or c >= len(table_row) or not 0 <= table_row[c] < self.n_pages:
            return None
        return int(table_row[c]), block_index(pos % self.page, np.arange(self.hd), self.hd)

    def put(self, table_row, pos, layer, kv, rows):
        w = self.where(table_row, pos)
        if w is not None:
            self.bits[layer, w[0], kv][:, w[1]] = rows

    def get(self, table_row, pos, layer, kv):
        w = self.where(table_row, pos)
        return None if w is None else self.bits[layer, w[0], kv][:, w[1]]

    def compact(self, table_row, base, keep):
        """Moves the kept rows (a list of offsets behind base) together; how many count."""
        limit = len(table_row) * self.page - base if base >= 0 else 0
        keep = [j for j in keep if j < limit]
        for to, j in enumerate(keep):
            a, b = self.where(table_row, base + j), self.where(table_row, base + to)
            if a is not None and b is not None and to != j:
                self.bits[:, b[0], :, :, b[1]] = self.bits[:, a[0], :, :, a[1]].copy()
        return len(keep)


def reserve(length, table, refs, page):
    out = []
    n_pages = len(refs)
    for r, n in enumerate(length):
        if not 0 <= n <= table.shape[1] * page:
            out.append(-1)
            continue
        end = -(-int(n) // page)
        need = [c for c in range(end) if not 0 <= table[r, c] < n_pages]
        free = np.flatnonzero(refs == 0)
        if len(need) > len(free):
            out.append(-1)
            continue
        for c, p in zip(need, free):
            table[r, c], refs[p] = p, 1
        out.append(end)
    return out


def fork(src, dst, length, own, table, refs, page, pool=None):
    out, start = [], table.copy()
    slots, n_pages = table.shape[0], len(refs)
    for s, d, n, o in zip(src, dst, length, own):
        if not (0 <= s < slots and 0 <= d < slots and s != d and 0 <= n <= table.shape[1] * page and o >= 0):
            out.append(-1)
            continue
        end = -(-int(n) // page)
        share = min(int(o) // page, end)
        there = [c for c in range(share, end) if 0 <= start[s, c] < n_pages]
        free = np.flatnonzero(refs == 0)
        if len(there) > len(free):
            out.append(-1)
            continue
        table[d] = -1
        for c in range(share):
            if 0 <= start[s, c] < n_pages:
                table[d, c] = start[s, c]
                refs[start[s, c]] += 1
        for c, p in zip(there, free):
            table[d, c], refs[p] = p, 1
            if pool is not None:
                pool.bits[:, p] = pool.bits[:, start[s, c]]
        out.append(end)
    return out


def release(length, table, refs, page):
    for r, n in enumerate(length):
        for c in range(-(-int(n) // page), table.shape[1]) if n >= 0 else ():
            if 0 <= table[r, c] < len(refs):
                refs[table[r, c]] -= 1
                table[r, c] = -1


# ---- attention (torch, 64 bits, on whatever device the inputs are)
def attend(q, k, v, seen, scale):
    """(result, sum of p |v|, largest sum of |q_c k_c| scale of a visible key) of q [rows, heads, hd] over k, v [keys, KV heads, hd]; seen [rows,
    keys].  What is not finite in a row of k or v reaches the rows that see it alone."""
    import torch
    q, k, v = (x.double().transpose(0, 1) for x in (q, k, v))
    G = q.shape[0] // k.shape[0]
    k, v = k.repeat_interleave(G, 0), v.repeat_interleave(G, 0)
    s = (q @ k.transpose(1, 2) * scale).masked_fill(~seen, -float("inf"))
    top = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(torch.isinf(top) & (top < 0), 0.0, top))
    total = e.sum(-1, keepdim=True)
    p = e / torch.where(total == 0, 1.0, total)
    bad = ~torch.isfinite(v)
    fine = torch.where(bad, 0.0, v)
    out = p @ fine
    out = torch.where((seen.double() @ bad.double()) > 0, float("nan"), out)
    size = p @ fine.abs()
    mag = (q.abs() @ torch.nan_to_num(k, 0.0, 0.0, 0.0).abs().transpose(1, 2) * scale).masked_fill(~seen, 0.0).amax(-1, keepdim=True)
    return [x.transpose(0, 1) for x in (out, size, mag)]
