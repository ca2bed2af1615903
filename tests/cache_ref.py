"""Plain float64 references of the rotary positions and the paged cache, on the
CPU, written from the definitions in include/dlm.h; they share no code with the
library."""

from __future__ import annotations

import math

import numpy as np
import torch


def half_step(dtype) -> float:
    """Largest relative error of a rounding to dtype."""
    return torch.finfo(dtype).eps / 2


def half_subnormal(dtype) -> float:
    """Largest absolute error of a rounding below dtype's normal range, where values
    lie smallest_normal * eps apart (float16: 2^-24, half of it 2^-25)."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


# ------------------------------------------------------------------ rotary positions

def frequencies(rot, theta=10000.0, scaling=None, factor=1.0, original=0, slow=1.0, fast=32.0):
    """(angle per position of each pair, scale)."""
    if scaling == "ntk":
        theta = theta * factor ** (rot / (rot - 2))
    w = np.array([theta ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=np.float64)
    if scaling == "linear":
        return w / factor, 1.0
    if scaling == "yarn":
        g = np.clip((original * w / (2 * math.pi) - slow) / (fast - slow), 0.0, 1.0)
        return g * w + (1 - g) * w / factor, 0.1 * math.log(factor) + 1.0
    return w, 1.0


def rotate(x, pos, w, scale, interleaved, transpose=False):
    """x [rows, heads, hd] float64, pos [rows] integers."""
    x = x.double()
    n = len(w)
    ang = pos.double()[:, None] * torch.tensor(w)[None, :]
    c, s = scale * ang.cos()[:, None], scale * ang.sin()[:, None]
    if transpose:
        s = -s
    y = x.clone()
    ia = torch.arange(0, 2 * n, 2) if interleaved else torch.arange(n)
    ib = ia + 1 if interleaved else ia + n
    a, b = x[..., ia], x[..., ib]
    y[..., ia] = a * c - b * s
    y[..., ib] = b * c + a * s
    return y


# ------------------------------------------------------------------ attention

def attend(q, k, v, see, scale):
    """q [n, H, hd], k / v [m, KV, hd], see bool [n, m]: (out, sum of p |v|, lse) in float64;
    keys that a row does not see play no part, whatever they hold."""
    n, H, hd = q.shape
    G = H // k.shape[1]
    out, mag = torch.zeros(n, H, hd, dtype=torch.float64), torch.zeros(n, H, hd, dtype=torch.float64)
    lse = torch.full((n, H), -math.inf, dtype=torch.float64)
    q, k, v = q.double(), k.double(), v.double()
    same = bool((see == see[:1]).all()) if n else True
    for h in range(H):
        if same and n:                                  # one mask for all rows
            idx = torch.nonzero(see[0]).view(-1)
            if idx.numel() == 0:
                continue
            z = scale * (q[:, h] @ k[idx, h // G].T)
            m = z.max(-1, keepdim=True).values
            p = torch.exp(z - m)
            s = p.sum(-1, keepdim=True)
            out[:, h], mag[:, h] = (p / s) @ v[idx, h // G], (p / s) @ v[idx, h // G].abs()
            lse[:, h] = (m + torch.log(s)).view(-1)
            continue
        for i in range(n):
            idx = torch.nonzero(see[i]).view(-1)
            if idx.numel() == 0:
                continue
            z = scale * (k[idx, h // G] @ q[i, h])
            m = z.max()
            p = torch.exp(z - m)
            s = p.sum()
            out[i, h], mag[i, h] = (p / s) @ v[idx, h // G], (p / s) @ v[idx, h // G].abs()
            lse[i, h] = m + torch.log(s)
    return out, mag, lse


def pack_mask(see_list, words):
    """int32 [rows, words] from one bool [n, n] per sequence."""
    rows = []
    for see in see_list:
        for line in see:
            w = [0] * words
            for j, s in enumerate(line):
                if s:
                    w[j // 32] |= 1 << (j % 32)
            rows.append([x - (1 << 32) if x >> 31 else x for x in w])
    return torch.tensor(rows, dtype=torch.int32).view(-1, words)


# ------------------------------------------------------------------ pages

class PlainCache:
    """The page operations on Python lists; pool[layer][page] is a dict of places,
    each holding whatever was appended there."""

    def __init__(self, n_pages, page_len, n_seqs, max_pages):
        self.P, self.L, self.B, self.W = n_pages, page_len, n_seqs, max_pages
        self.ref = [0] * n_pages
        self.len = [0] * n_seqs
        self.table = [[-1] * max_pages for _ in range(n_seqs)]
        self.pool = [[None] * page_len for _ in range(n_pages)]

    def _pages(self, n):
        return -(-n // self.L)

    def _release(self, b, first):
        for e in range(first, self.W):
            if self.table[b][e] >= 0:
                self.ref[self.table[b][e]] -= 1
                self.table[b][e] = -1

    def reserve(self, rows):
        held, free = list(self.ref), [p for p in range(self.P) if self.ref[p] == 0]
        ok, used, full = [1] * self.B, 0, False
        for b, n in enumerate(rows):
            if n == 0:
                continue
            first, last = self.len[b] // self.L, self._pages(self.len[b] + n)
            if last > self.W:
                ok[b] = 0
                continue
            want = [e for e in range(first, last) if self.table[b][e] < 0 or held[self.table[b][e]] > 1]
            if want and (full or used + len(want) > len(free)):
                ok[b], full = 0, True
                continue
            for e in want:
                old, new = self.table[b][e], free[used]
                used += 1
                if old >= 0:
                    self.ref[old] -= 1
                    if e == first:
                        fill = self.len[b] % self.L
                        self.pool[new][:fill] = self.pool[old][:fill]
                self.table[b][e], self.ref[new] = new, 1
        return ok

    def append(self, rows, tag):
        for b, n in enumerate(rows):
            for i in range(n):
                t = self.len[b] + i
                if t // self.L < self.W and self.table[b][t // self.L] >= 0:
                    self.pool[self.table[b][t // self.L]][t % self.L] = tag(b, i)

    def commit(self, rows, keep=None):
        ok = [1] * self.B
        for b, n in enumerate(rows):
            if n == 0:
                continue
            a = list(range(n)) if keep is None else keep[b]
            lo, hi = self.len[b] // self.L, self._pages(self.len[b] + n)
            good = all(0 <= x < n for x in a) and all(x < y for x, y in zip(a, a[1:])) and hi <= self.W
            good = good and all(self.table[b][e] >= 0 for e in range(lo, hi))
            if good and a != list(range(len(a))):
                good = all(self.ref[self.table[b][e]] <= 1 for e in range(lo, self._pages(self.len[b] + len(a))))
            ok[b] = int(good)
            if not good:
                continue
            rows_b = [self.pool[self.table[b][(self.len[b] + x) // self.L]][(self.len[b] + x) % self.L] for x in a]
            for i, (x, r) in enumerate(zip(a, rows_b)):
                if x != i:
                    t = self.len[b] + i
                    self.pool[self.table[b][t // self.L]][t % self.L] = r
            self.len[b] += len(a)
            self._release(b, self._pages(self.len[b]))
        return ok

    def fork(self, src, dst):
        ok = []
        for i, (s, d) in enumerate(zip(src, dst)):
            good = 0 <= s < self.B and 0 <= d < self.B and d not in src and dst.count(d) == 1
            ok.append(int(good))
            if good:
                self._release(d, 0)
                for e in range(min(self._pages(self.len[s]), self.W)):
                    self.table[d][e] = self.table[s][e]
                    if self.table[d][e] >= 0:
                        self.ref[self.table[d][e]] += 1
                self.len[d] = self.len[s]
        return ok

    def truncate(self, new_len):
        for b, n in enumerate(new_len):
            if n >= 0:
                self.len[b] = min(self.len[b], n)
                self._release(b, self._pages(self.len[b]))

    def compact(self):
        n = sum(1 for r in self.ref if r)
        move = dict(zip([p for p in range(n, self.P) if self.ref[p]], [p for p in range(n) if not self.ref[p]]))
        for a, b in move.items():
            self.pool[b] = list(self.pool[a])
            self.ref[b], self.ref[a] = self.ref[a], 0
        self.table = [[move.get(p, p) for p in row] for row in self.table]
        return n

    def meta(self):
        return self.ref + self.len + [p for row in self.table for p in row]

    def contents(self, b):
        return [self.pool[self.table[b][t // self.L]][t % self.L] for t in range(self.len[b])]
