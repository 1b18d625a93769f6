"""A paged key-value cache in plain Python and 64-bit numpy: what the library's page
operations, writes and decode attention are compared with."""
from __future__ import annotations

import math

import numpy as np
import torch

D = 128


def round_e4m3(y: np.ndarray) -> np.ndarray:
    """Round to nearest even onto e4m3 (three bits after the leading one, exponents from -6,
    largest 448, at which it saturates); NaN stays."""
    a = np.abs(y)
    with np.errstate(all="ignore"):
        e = np.maximum(np.floor(np.log2(np.where((a > 0) & np.isfinite(a), a, 1.0))), -6.0)
        unit = np.exp2(e - 3)
        q = np.minimum(np.rint(a / unit) * unit, 448.0)
    return np.where(np.isnan(y), np.nan, np.copysign(q, y))


def e4m3_row(x: np.ndarray):
    """(codes' values, e) of one row: the smallest e >= -120 that brings every finite value
    within 448 * 2^e."""
    finite = np.abs(x[np.isfinite(x)])
    top = float(finite.max()) if finite.size else 0.0
    e = -120
    while top > math.ldexp(448.0, e):
        e += 1
    return round_e4m3(x / math.ldexp(1.0, e)), e


def held(x: np.ndarray, bits: int) -> np.ndarray:
    """Rows [..., 128] as the cache holds them."""
    if bits == 16:
        return x
    flat = x.reshape(-1, D)
    return np.stack([c * math.ldexp(1.0, e) for c, e in map(e4m3_row, flat)]).reshape(x.shape)


class Pages:
    """Tables, and for each page the tokens' contents as opaque values."""

    def __init__(self, num_pages, num_slots, max_pages, T):
        self.P, self.T, self.W = num_pages, T, max_pages
        self.length = [0] * num_slots
        self.table = [[] for _ in range(num_slots)]
        self.refs = [0] * num_pages
        self.content = [[None] * T for _ in range(num_pages)]

    def extend(self, slots, add):
        """False (and nothing changed) if there are too few pages or a list is full."""
        plan, need = [], 0
        for s, a in zip(slots, add):
            if s == -1:
                continue
            n = self.length[s]
            if n + a > self.W * self.T:
                return False
            copy = a > 0 and n % self.T != 0 and self.refs[self.table[s][-1]] > 1
            more = -(-(n + a) // self.T) - len(self.table[s])
            plan.append((s, a, copy, more))
            need += more + copy
        free = [p for p in range(self.P) if self.refs[p] == 0][:need]
        if len(free) < need:
            return False
        for s, a, copy, more in plan:
            if copy:
                old, new = self.table[s][-1], free.pop(0)
                k = self.length[s] % self.T
                self.content[new][:k] = self.content[old][:k]
                self.refs[old] -= 1
                self.refs[new] = 1
                self.table[s][-1] = new
            for _ in range(more):
                p = free.pop(0)
                self.refs[p] = 1
                self.table[s].append(p)
            self.length[s] += a
        return True

    def fork(self, parents, children):
        for p, c in zip(parents, children):
            if c == -1:
                continue
            self.length[c] = self.length[p]
            self.table[c] = list(self.table[p])
            for page in self.table[c]:
                self.refs[page] += 1

    def trim(self, slots, keep=None):
        for i, s in enumerate(slots):
            if s == -1:
                continue
            n = 0 if keep is None else keep[i]
            k = -(-n // self.T)
            for page in self.table[s][k:]:
                self.refs[page] -= 1
            self.table[s] = self.table[s][:k]
            self.length[s] = n

    def compact(self):
        live = [p for p in range(self.P) if self.refs[p] > 0]
        holes = [p for p in range(len(live)) if self.refs[p] == 0]
        for p in [p for p in live if p >= len(live)]:
            to = holes.pop(0)
            self.content[to] = list(self.content[p])
            self.refs[to], self.refs[p] = self.refs[p], 0
            for t in self.table:
                t[:] = [to if q == p else q for q in t]

    def set_token(self, slot, pos, value):
        self.content[self.table[slot][pos // self.T]][pos % self.T] = value

    def token(self, slot, pos):
        return self.content[self.table[slot][pos // self.T]][pos % self.T]


def i32(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


def same_tables(cache, ref: Pages):
    """The device's lengths, counts and used entries are the model's."""
    assert cache.seq_len.tolist() == ref.length
    assert cache.page_refs.tolist() == ref.refs
    table = cache.page_table.tolist()
    for s, pages in enumerate(ref.table):
        assert table[s][:len(pages)] == pages, s


def attention(q, k, v, scale=1 / math.sqrt(D)):
    """One row: q [H, D], k, v [n, Hkv, D] in float64 -> out [H, D], and the mean of |v| by the
    softmax's weights, which bounds what rounding the weights does."""
    H, Hkv = q.shape[0], k.shape[1]
    out, size = np.zeros((H, D)), np.zeros((H, D))
    for h in range(H):
        g = h // (H // Hkv)
        with np.errstate(all="ignore"):
            s = k[:, g] @ q[h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            out[h], size[h] = p @ v[:, g], p @ np.abs(v[:, g])
    return out, size
