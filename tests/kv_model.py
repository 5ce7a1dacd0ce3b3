"""The 4-bit paged key/value cache in numpy: elements, rows, attention in 64
bits, and the page operations one entry after the other, written from
include/sense.h alone.  Test infrastructure."""
from __future__ import annotations

import math

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
DONE, NO_PAGES, TOO_LONG, REFUSED = 0, 1, 2, 3


def quantise_block(x):
    """(codes [32], scale byte) of 32 values, by search."""
    x = np.asarray(x, np.float64)
    if not np.isfinite(x).all():
        return np.zeros(32, np.uint8), 255
    top = np.abs(x).max()
    e = -127 if top == 0 else max(math.frexp(top)[1] - 1 - 2, -127)
    codes = np.zeros(32, np.uint8)
    for i, v in enumerate(x):
        y = abs(v) * 2.0 ** -e
        gap = np.abs(GRID - min(y, 6.0))
        best = [c for c in range(8) if gap[c] == gap.min()]
        code = best[0] if len(best) == 1 else [c for c in best if c % 2 == 0][0]
        codes[i] = code | (8 if math.copysign(1.0, v) < 0 else 0)
    return codes, e + 127


def quantise_row(x):
    """(bytes [d/2], scales [d/32]) of a row."""
    codes, scales = [], []
    for b in range(len(x) // 32):
        c, s = quantise_block(x[32 * b:32 * b + 32])
        codes.append(c)
        scales.append(s)
    c = np.concatenate(codes)
    return (c[0::2] | c[1::2] << 4).astype(np.uint8), np.array(scales, np.uint8)


def values(codes, scales):
    """Values (float64) of rows [..., d/2] with scales [..., d/32]."""
    c = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (-1,))
    x = GRID[c & 7] * np.where(c & 8, -1.0, 1.0)
    s = np.repeat(scales.astype(np.int64), 32, -1)
    return np.where(s == 255, np.nan, np.ldexp(x, s - 127))


def attention(q, k, v, scale, see):
    """q [m, heads, d], k and v [L, kv_heads, d], see [m, L] bool; float64.
    A row that sees nothing is 0; unseen positions do not count at all."""
    m, heads, d = q.shape
    group = heads // k.shape[1]
    out = np.zeros((m, heads, d))
    for j in range(m):
        at = np.nonzero(see[j])[0]
        if not len(at):
            continue
        kj, vj = k[at], v[at]
        for h in range(heads):
            s = kj[:, h // group] @ q[j, h] * scale
            w = np.exp(s - np.nanmax(s)) if not np.isnan(s).all() else s
            out[j, h] = (w[:, None] * vj[:, h // group]).sum(0) / w.sum()
    return out


class Cache:
    """A cache's arrays and the page operations on them."""

    def __init__(self, layers, pages, page, heads, d, seqs, max_pages):
        self.codes = np.zeros((layers, pages, 2, heads, page, d // 2), np.uint8)
        self.scales = np.zeros((layers, pages, 2, heads, d // 32, page), np.uint8)
        self.table = np.full((seqs, max_pages), -1, np.int32)
        self.lens = np.zeros(seqs, np.int32)
        self.refs = np.zeros(pages, np.int32)
        self.page = page

    @property
    def capacity(self):
        return self.table.shape[1] * self.page

    def pages(self, tokens):
        return -(-tokens // self.page)

    def cell(self, s, p):
        return self.table[s, p // self.page], p % self.page

    def row(self, layer, s, p, which, head):
        page, slot = self.cell(s, p)
        return values(self.codes[layer, page, which, head, slot],
                      self.scales[layer, page, which, head, :, slot])

    def rows(self, layer, s, a, b):
        """[2, b - a, heads, d] values of positions a .. b-1."""
        heads = self.codes.shape[3]
        return np.array([[[self.row(layer, s, p, w, h) for h in range(heads)]
                          for p in range(a, b)] for w in (0, 1)]).reshape(
                              2, b - a, heads, self.codes.shape[5] * 2)

    def write(self, layer, s, p, which, head, x):
        page, slot = self.cell(s, p)
        c, sc = quantise_row(x)
        self.codes[layer, page, which, head, slot] = c
        self.scales[layer, page, which, head, :, slot] = sc

    def release(self, s, tokens):
        for i in range(self.pages(tokens), self.pages(int(self.lens[s]))):
            self.refs[self.table[s, i]] -= 1
            self.table[s, i] = -1
        self.lens[s] = tokens

    def ok(self, s):
        return 0 <= s < len(self.lens)

    def truncate(self, seqs, lens):
        out = []
        for s, n in zip(seqs, lens):
            if not self.ok(s) or n < 0:
                out.append(REFUSED)
                continue
            if n < self.lens[s]:
                self.release(s, n)
            out.append(DONE)
        return out

    def fork(self, src, dst):
        out = []
        held = [self.lens[d] if self.ok(d) else 0 for d in dst]
        for i, (a, b) in enumerate(zip(src, dst)):
            if not self.ok(a) or not self.ok(b) or held[i] > 0 or b in dst[:i] or a in dst:
                out.append(REFUSED)
                continue
            n = self.pages(int(self.lens[a]))
            self.table[b, :n] = self.table[a, :n]
            self.refs[self.table[a, :n]] += 1
            self.lens[b] = self.lens[a]
            out.append(DONE)
        return out

    def reserve(self, seqs, counts):
        out, full = [], False
        free = [int(p) for p in np.nonzero(self.refs <= 0)[0]]    # as before the call
        for i, (s, n) in enumerate(zip(seqs, counts)):
            if not self.ok(s) or n < 0 or s in seqs[:i]:
                out.append(REFUSED)
                continue
            old = int(self.lens[s])
            if old + n > self.capacity:
                out.append(TOO_LONG)
                continue
            last = self.table[s, old // self.page] if n and old % self.page else -1
            copy = last >= 0 and self.refs[last] > 1
            need = self.pages(old + n) - self.pages(old) + copy
            full = full or need > len(free)
            if full:
                out.append(NO_PAGES)
                continue
            if copy:
                new = free.pop(0)
                fill = old % self.page
                self.codes[:, new, :, :, :fill] = self.codes[:, last, :, :, :fill]
                self.scales[:, new, :, :, :, :fill] = self.scales[:, last, :, :, :, :fill]
                self.refs[last] -= 1
                self.refs[new] = 1
                self.table[s, old // self.page] = new
            for p in range(self.pages(old), self.pages(old + n)):
                new = free.pop(0)
                self.refs[new] = 1
                self.table[s, p] = new
            self.lens[s] = old + n
            out.append(DONE)
        return out

    def compact(self, seqs, tails, paths):
        """paths: each entry's picked row, cut to its length."""
        out, cut = [], []
        for i, (s, tail, path) in enumerate(zip(seqs, tails, paths)):
            if not self.ok(s) or s in seqs[:i] or not 0 <= tail <= self.lens[s] or path is None:
                out.append(REFUSED)
                continue
            kept = 0
            while kept < len(path) and path[kept] > (path[kept - 1] if kept else -1) \
                    and path[kept] < tail:
                kept += 1
            base = int(self.lens[s]) - tail
            moves = [(self.cell(s, base + path[j]), self.cell(s, base + j))
                     for j in range(kept) if path[j] != j]
            if any(self.refs[d[0]] > 1 for _, d in moves):
                out.append(REFUSED)
                continue
            for (sp, ss), (dp, ds) in moves:
                self.codes[:, dp, :, :, ds] = self.codes[:, sp, :, :, ss]
                self.scales[:, dp, :, :, :, ds] = self.scales[:, sp, :, :, :, ss]
            cut.append((s, base + kept))
            out.append(DONE)
        for s, n in cut:
            self.release(s, n)
        return out
