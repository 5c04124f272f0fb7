"""Rotary positions, and keys and values in pages of 8 bits, in 64 bits and plain loops: what the GPU tests compare with."""
import math

import torch


def rotate(x, positions, frequencies, interleaved, factor=1.0, inverse=False):
    """x [tokens, heads, dim] in 64 bits."""
    y, pairs = x.clone(), frequencies.numel()
    for i in range(pairs):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
        angle = positions.double() * frequencies[i] * (-1 if inverse else 1)
        c, s = factor * torch.cos(angle)[:, None], factor * torch.sin(angle)[:, None]
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y


def exponent(amax):
    """The smallest E >= -126 with amax <= 448 2^E."""
    e = -126
    while amax > 448 * 2.0 ** e:
        e += 1
    return e


def nearest(t):
    """The nearest number of 1 + 4 + 3 bits, halfway cases to the even one; what is not finite: NaN."""
    t = torch.where(torch.isfinite(t), t, math.nan)
    step = torch.exp2(torch.frexp(t).exponent.double().clamp(min=-5) - 4)
    return torch.round(t / step) * step


def width(dim):
    return -(-dim // 32) * 32


def key_byte(t, c):
    return c // 32 * 1024 + ((c % 32 // 8) * 16 + t % 16) * 16 + t // 16 * 8 + c % 8


def value_byte(t, c):
    return c // 32 * 1024 + ((t % 16 // 4) * 16 + c % 16) * 16 + (c % 32 // 16) * 8 + t // 16 * 4 + t % 4


def places(dim):
    """Byte of (keys or values, token, element) in a block, [2, 32, width]."""
    w = width(dim)
    return torch.tensor([[[f(t, c) for c in range(w)] for t in range(32)] for f in (key_byte, value_byte)])


class Pool:
    """The bookkeeping with lists, and codes (as numbers) and exponents of every block of every page."""

    def __init__(self, layers, num_pages, rows, max_pages, heads, dim, page):
        self.layers, self.num_pages, self.rows, self.max_pages = layers, num_pages, rows, max_pages
        self.heads, self.dim, self.page = heads, dim, page
        self.tables = [[-1] * max_pages for _ in range(rows)]
        self.lengths, self.refs = [0] * rows, [0] * num_pages
        shape = (layers, num_pages, heads, page // 32, 2)
        self.codes = torch.zeros(*shape, 32, width(dim), dtype=torch.float64)
        self.exps = torch.full(shape, -126, dtype=torch.int64)

    def pages(self, n):
        return -(-n // self.page)

    def reserve(self, add):
        free = [p for p in range(self.num_pages) if self.refs[p] == 0]
        start = list(self.refs)
        granted, at = [], 0
        for r, a in enumerate(add):
            a, n = max(a, 0), self.lengths[r]
            had, has = self.pages(n), self.pages(n + a)
            if has > self.max_pages:
                granted.append(0)
                continue
            copy = a > 0 and n % self.page != 0 and start[self.tables[r][had - 1]] > 1
            need = has - had + copy
            if need and at + need > len(free):
                granted.append(0)
                at += need
                continue
            mine = free[at:at + need]
            at += need
            if copy:
                src, dst = self.tables[r][had - 1], mine.pop(0)
                filled = -(-(n % self.page) // 32)
                self.codes[:, dst, :, :filled] = self.codes[:, src, :, :filled]
                self.exps[:, dst, :, :filled] = self.exps[:, src, :, :filled]
                self.refs[src] -= 1
                self.refs[dst] = 1
                self.tables[r][had - 1] = dst
            for j, p in enumerate(mine):
                self.tables[r][had + j], self.refs[p] = p, 1
            self.lengths[r] += a
            granted.append(a)
        return granted

    def recount(self):
        self.refs = [0] * self.num_pages
        for table in self.tables:
            for p in table:
                if p >= 0:
                    self.refs[p] += 1

    def fork(self, parents):
        was = [list(t) for t in self.tables], list(self.lengths)
        for r, p in enumerate(parents):
            if 0 <= p < self.rows:
                self.tables[r], self.lengths[r] = list(was[0][p]), was[1][p]
        self.recount()

    def truncate(self, keep):
        for r, k in enumerate(keep):
            if 0 <= k < self.lengths[r]:
                for j in range(self.pages(k), self.pages(self.lengths[r])):
                    self.tables[r][j] = -1
                self.lengths[r] = k
        self.recount()

    def compact(self):
        used = sum(n > 0 for n in self.refs)
        src = [p for p in range(used, self.num_pages) if self.refs[p] > 0]
        dst = [p for p in range(used) if self.refs[p] == 0]
        to = dict(zip(src, dst))
        for s, d in to.items():
            self.codes[:, d], self.exps[:, d] = self.codes[:, s], self.exps[:, s]
        self.tables = [[to.get(p, p) for p in t] for t in self.tables]
        self.recount()
        return used

    def append(self, layer, k, v, new, granted=None):
        """k, v [tokens, heads, dim]: the rows' newest, one row's after another's."""
        at = 0
        for r, n in enumerate(new):
            x = torch.stack([k[at:at + n], v[at:at + n]]).double()
            at += n
            first = self.lengths[r] - n
            if n == 0 or first < 0 or (granted is not None and granted[r] != n):
                continue
            for b in range(first // 32, -(-self.lengths[r] // 32)):
                page, i = self.tables[r][b * 32 // self.page], b % (self.page // 32)
                if self.refs[page] > 1:
                    continue
                lo, hi = max(first, b * 32), min(self.lengths[r], (b + 1) * 32)
                for h in range(self.heads):
                    for kv in (0, 1):
                        y = x[kv, lo - first:hi - first, h]
                        fine = y[torch.isfinite(y)].abs()
                        kept = lo - b * 32
                        was = int(self.exps[layer, page, h, i, kv]) if kept else -126
                        e = max(was, exponent(float(fine.max()) if fine.numel() else 0.0))
                        block = torch.zeros(32, width(self.dim), dtype=torch.float64)
                        block[:kept] = nearest(self.codes[layer, page, h, i, kv, :kept] * 2.0 ** (was - e))
                        block[kept:hi - b * 32, :self.dim] = nearest(y * 2.0 ** -e)
                        self.codes[layer, page, h, i, kv] = block
                        self.exps[layer, page, h, i, kv] = e

    def values(self, layer, r):
        """A row's keys and values [2, heads, length, dim]."""
        n = self.lengths[r]
        ids = self.tables[r][: self.pages(n)]
        x = self.codes[layer, ids] * torch.exp2(self.exps[layer, ids].double())[..., None, None]   # [pages, heads, blocks, 2, 32, width]
        return x.permute(3, 1, 0, 2, 4, 5).reshape(2, self.heads, -1, width(self.dim))[:, :, :n, :self.dim]

    def attend(self, layer, q, new, group, scale, window=0):
        out, at = torch.zeros(q.shape, dtype=torch.float64), 0
        for r, n in enumerate(new):
            x = q[at:at + n].double()
            if n:
                out[at:at + n] = attend(x, self.values(layer, r), group, scale, window)
            at += n
        return out


def attend(q, kv, group, scale, window=0):
    """q [n, heads * group, dim], kv [2, heads, length, dim]: the last n places' outputs."""
    n, length, out = q.shape[0], kv.shape[2], torch.zeros_like(q)
    for i in range(n):
        place = length - n + i
        lo = max(0, place - window + 1) if window else 0
        if place < 0:
            continue
        for j in range(q.shape[1]):
            k, v = kv[0, j // group, lo:place + 1], kv[1, j // group, lo:place + 1]
            out[i, j] = torch.softmax(scale * (k @ q[i, j]), 0) @ v
    return out
