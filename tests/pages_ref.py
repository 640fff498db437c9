"""A plain model of the paged 8-bit cache in 64 bits (numpy, python lists): what the device's maps, codes and
attention outputs are compared with.  Stored order and rounding follow the text of include/less.h."""
from __future__ import annotations

import math

import numpy as np

TOP = {"int8": 127.0, "e4m3": 448.0}
BLOCK = 16


def places(D, values):
    """[16, D]: byte of (token, dimension) in a tile."""
    at = np.zeros((BLOCK, D), dtype=np.int64)
    for c in range(D // 32):
        for g in range(8):
            for t in range(4):
                base = 16 * (32 * c + 4 * g + t)
                for x in range(16):
                    if values:
                        at[4 * t + x % 4, g * D // 8 + 4 * c + x // 4] = base + x
                    else:
                        j, half = c // (D // 64), c % (D // 64)
                        at[4 * (g // 2) + 2 * j + g % 2, t * D // 4 + 16 * half + x] = base + x
    return at


def code_values(fmt):
    """[256] float64: what a code stands for in units of amax / top."""
    c = np.arange(256)
    if fmt == "int8":
        return np.where(c < 128, c, c - 256).astype(np.float64)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m / 512.0, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    v[(c & 127) == 127] = np.nan
    return np.where(c >= 128, -v, v)


def encode(x, fmt):
    """Nearest code, ties to even."""
    if fmt == "int8":
        return (np.rint(x).astype(np.int64) % 256).astype(np.uint8)
    table = code_values(fmt)[:127]
    mag = np.abs(x)
    up = np.clip(np.searchsorted(table, mag), 0, 126)
    lo = np.maximum(up - 1, 0)
    a, b = mag - table[lo], table[up] - mag
    code = np.where((a < b) | ((a == b) & (lo % 2 == 0)), lo, up)
    return (code + 128 * np.signbit(x)).astype(np.uint8)


class Model:
    def __init__(self, layers, heads, dim, pages, seqs, seq_pages, group, pt, fmt, bf16):
        self.L, self.H, self.D, self.G, self.pt, self.fmt = layers, heads, dim, group, pt, fmt
        self.bf16 = bf16
        self.most = 2.0 ** 100 if bf16 else 65504.0
        self.table = np.full((seqs, seq_pages), -1, np.int64)
        self.lens = np.zeros(seqs, np.int64)
        self.refs = np.zeros(pages, np.int64)
        self.codes = np.zeros((layers, pages, heads, 2, pt * dim), np.uint8)
        self.amax = np.zeros((layers, pages, heads, 2, pt // BLOCK))
        self.at = (places(dim, False), places(dim, True))
        self.val = code_values(fmt)

    # -- maps ---------------------------------------------------------------- #
    def _release(self, s, first, last=None):
        for o in range(first, self.table.shape[1] if last is None else last):
            if self.table[s, o] >= 0:
                self.refs[self.table[s, o]] -= 1
                self.table[s, o] = -1

    def _copy(self, a, b):
        self.codes[:, b], self.amax[:, b] = self.codes[:, a], self.amax[:, a]

    def resize(self, seqs, lens):
        """False if the growth had to be refused."""
        pairs = list({s: (s, w) for s, w in reversed(list(zip(seqs, lens)))}.values())[::-1]
        pairs = sorted(pairs, key=lambda x: list(seqs).index(x[0]))
        for s, w in pairs:
            if w < self.lens[s]:
                self._release(s, -(-w // self.pt))
                self.lens[s] = w
        free = [p for p in range(len(self.refs)) if self.refs[p] == 0]
        plan, shared = [], []
        for s, w in pairs:
            if w > self.lens[s]:
                first = -(-self.lens[s] // self.pt)
                held = self.table[s, self.lens[s] // self.pt] if self.lens[s] % self.pt else None
                if held is not None and held < 0:
                    return False
                if held is not None and self.refs[held] > 1:
                    first -= 1
                    shared.append((s, first, held))
                plan += [(s, o) for o in range(first, -(-w // self.pt))]
        if len(plan) > len(free):
            return False
        for (s, o), page in zip(plan, free):
            self.table[s, o] = page
            self.refs[page] = 1
        for s, o, held in shared:
            self.refs[held] -= 1
            self._copy(held, self.table[s, o])
        for s, w in pairs:
            self.lens[s] = w
        return True

    def fork(self, src, dst):
        free = iter([p for p in range(len(self.refs)) if self.refs[p] == 0])
        for a, b in zip(src, dst):
            whole = self.lens[a] // self.pt
            self.table[b, :whole] = self.table[a, :whole]
            for p in self.table[a, :whole]:
                if p >= 0:
                    self.refs[p] += 1
            if self.lens[a] % self.pt and self.table[a, whole] >= 0:
                self.table[b, whole] = next(free)
                self.refs[self.table[b, whole]] = 1
                self._copy(self.table[a, whole], self.table[b, whole])
            self.lens[b] = self.lens[a]

    def trim(self, seqs, sinks, window):
        for s in seqs:
            for o in range(self.table.shape[1]):
                if o * self.pt >= sinks and (o + 1) * self.pt <= self.lens[s] - window:
                    self._release(s, o, o + 1)

    def compact(self):
        live = int((self.refs > 0).sum())
        src = [p for p in range(live, len(self.refs)) if self.refs[p] > 0]
        dst = [p for p in range(live) if self.refs[p] == 0]
        for a, b in zip(src, dst):
            self._copy(a, b)
            self.refs[b], self.refs[a] = self.refs[a], 0
            self.table[self.table == a] = b

    # -- contents ------------------------------------------------------------ #
    def write(self, seqs, starts, k, v, layer_begin=0):
        """k, v: float64 [rows, layers, heads, D]."""
        done = set()
        for i, s in enumerate(seqs):
            m, n = starts[i + 1] - starts[i], int(self.lens[s])
            if s in done or not m:
                continue
            done.add(s)
            begin = n - m
            for b in range(begin // BLOCK, -(-n // BLOCK)):
                page, inner = self.table[s, b * BLOCK // self.pt], b % (self.pt // BLOCK)
                lo, hi = max(begin, b * BLOCK), min(n, (b + 1) * BLOCK)
                keep = max(0, begin - b * BLOCK)
                for which, x in ((0, k), (1, v)):
                    x = np.nan_to_num(x[starts[i] + lo - begin:starts[i] + hi - begin], nan=0.0, posinf=self.most,
                                      neginf=-self.most)
                    x = np.clip(x, -self.most, self.most)
                    byte = inner * BLOCK * self.D + self.at[which]
                    for lj in range(x.shape[1]):
                        for h in range(self.H):
                            cell = (layer_begin + lj, page, h, which)
                            old = self.amax[cell + (inner,)] if keep else 0.0
                            a = max(old, np.abs(x[:, lj, h]).max())
                            a = 0.0 if a < 2.0 ** -100 else a
                            unit, top = a if a > 0 else 1.0, TOP[self.fmt]
                            tile = np.zeros((BLOCK, self.D), np.uint8)
                            if keep:
                                tile[:keep] = encode(self.val[self.codes[cell][byte[:keep]]] * old / unit, self.fmt)
                            tile[lo - b * BLOCK:hi - b * BLOCK] = encode(x[:, lj, h] * top / unit, self.fmt)
                            self.codes[cell][byte] = tile
                            self.amax[cell + (inner,)] = a

    def rows(self, layer, s, h, which, n):
        j = np.arange(n)
        page, inner = self.table[s, j // self.pt], (j % self.pt) // BLOCK
        byte = (inner * BLOCK * self.D)[:, None] + self.at[which][j % BLOCK]
        x = self.val[self.codes[layer, page[:, None], h, which, byte]]
        x = x * (self.amax[layer, page, h, which, inner] / TOP[self.fmt])[:, None]
        x[page < 0] = 0.0
        return x, page >= 0

    def attention(self, q, seqs, starts, layer_begin=0, window=0, sinks=0, scale=None):
        """(out, bound): float64 [rows, layers, heads * group, D], and how far fp32 arithmetic may be from it.

        The bound: 8 (D / 16) accumulations of a score round to 2^-22 of at most scale * sum |q| |k| each (the tensor
        cores' fp32 sums may truncate), so a probability is off by that much relative, an output by twice that of the
        largest |v|; exponentials and the two sums add less than 2^-19 of it.  An entry of more than 16 rows (tokens x
        query heads of a KV head), and any entry with bf16 output, may have its probabilities rounded to fp16 once: half
        a step is 2^-11 of each p or, below 2^-14 of the row's largest, 2^-25.  With |p' - p| <= 2^-11 p + 2^-25 the sum
        of p' v moves by at most (2^-11 + n 2^-25) max |v| times the sum of p (which is at least the largest p = 1):
        that much of the largest |v| more."""
        scale = self.D ** -0.5 if scale is None else scale
        out, bound = np.zeros(q.shape), np.zeros(q.shape)
        for i, s in enumerate(seqs):
            n, m = int(self.lens[s]), starts[i + 1] - starts[i]
            if not m or not n:
                continue
            j = np.arange(n)
            pos = (n - m + np.arange(m))[:, None]
            see = j <= pos
            if window:
                see &= (j > pos - window) | (j < sinks)
            for lj in range(q.shape[1]):
                for h in range(self.H):
                    k, here = self.rows(layer_begin + lj, s, h, 0, n)
                    v, _ = self.rows(layer_begin + lj, s, h, 1, n)
                    k, v = np.where(here[:, None], k, 0.0), np.where(here[:, None], v, 0.0)
                    for g in range(self.G):
                        qq = q[starts[i]:starts[i + 1], lj, h * self.G + g]
                        ok = see & here
                        z = np.where(ok, qq @ k.T * scale, -np.inf)
                        top = z.max(1, keepdims=True)
                        p = np.exp(z - np.where(np.isfinite(top), top, 0.0))
                        den = p.sum(1, keepdims=True)
                        y = np.divide(p @ v, den, out=np.zeros((m, self.D)), where=den > 0)
                        out[starts[i]:starts[i + 1], lj, h * self.G + g] = y
                        reach = np.where(ok, np.abs(qq) @ np.abs(k).T * scale, 0.0).max(1)
                        most = np.abs(v).max() if v.size else 0.0
                        rel = 2 * (self.D // 16) * reach * 2.0 ** -22 + 2.0 ** -19
                        if m * self.G > 16 or self.bf16:
                            rel = rel + 2.0 ** -11 + n * 2.0 ** -25
                        bound[starts[i]:starts[i + 1], lj, h * self.G + g] = (rel * most)[:, None]
        return out, bound
