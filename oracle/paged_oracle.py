"""The paged cache from its definitions, in plain Python and 64 bits: page tables as lists, rotary positions as
complex products, attention head by head."""
from __future__ import annotations

import math

import numpy as np


class Tables:
    """Page tables of heads in order; the free pages are a queue."""

    def __init__(self, heads, page_rows, max_pages, free):
        self.page_rows, self.max_pages = page_rows, max_pages
        self.rows = [0] * heads
        self.pages = [[] for _ in range(heads)]
        self.free = list(free)

    def _pages_of(self, rows):
        return -(-rows // self.page_rows)

    def change(self, add):
        """add[h] more rows for head h, None releases it.  Returns the places of the new rows head by head, or
        None (and changes nothing) where the free pages or a head's table do not suffice."""
        need = 0
        for h, a in enumerate(add):
            if a is None:
                continue
            if a < 0 or self.rows[h] + a > self.max_pages * self.page_rows:
                return None
            need += self._pages_of(self.rows[h] + a) - len(self.pages[h])
        if need > len(self.free):
            return None
        places, back = [], []
        for h, a in enumerate(add):
            if a is None:
                back += self.pages[h]
                self.pages[h], self.rows[h] = [], 0
                places.append([])
                continue
            while len(self.pages[h]) < self._pages_of(self.rows[h] + a):
                self.pages[h].append(self.free.pop(0))
            places.append([self.pages[h][r // self.page_rows] * self.page_rows + r % self.page_rows
                           for r in range(self.rows[h], self.rows[h] + a)])
            self.rows[h] += a
        self.free += back
        return places


def rotate(x, positions, freqs, interleaved=False, backward=False, scale=1.0):
    """x [tokens, heads, d]: the leading 2 * len(freqs) elements turned, the rest as it is."""
    x = np.asarray(x, dtype=np.float64)
    half = len(freqs)
    angle = np.asarray(positions, dtype=np.float64)[:, None] * np.asarray(freqs, dtype=np.float64)[None, :]
    turn = scale * np.exp((-1j if backward else 1j) * angle)[:, None, :]
    out = x.copy()
    first = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    second = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    z = (x[..., first] + 1j * x[..., second]) * turn
    out[..., first], out[..., second] = z.real, z.imag
    return out


def attend(q, k, v, scale=None, softcap=0.0):
    """q [group, d] over k, v [rows, d]: out [group, d], the log of the sum of exponentials [group]."""
    group, d = q.shape
    if len(k) == 0:
        return np.zeros((group, d)), np.full(group, -np.inf)
    x = (q @ k.T) * (1.0 / math.sqrt(d) if not scale else scale)
    if softcap:
        x = softcap * np.tanh(x / softcap)
    top = x.max(axis=1, keepdims=True)
    e = np.exp(x - top)
    total = e.sum(axis=1, keepdims=True)
    return (e / total) @ v, np.log(total[:, 0]) + top[:, 0]
