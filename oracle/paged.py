"""Plain definitions of the paged cache's operators: attention of new rows over pages (sliding window, sinks), rotary
rules, and the bookkeeping of pages.  Test infrastructure: numpy fp64, one row at a time, never imported by the
product path."""
from __future__ import annotations

import math
from typing import List, Optional, Sequence

import numpy as np


def sees(p: int, window: int, sinks: int) -> np.ndarray:
    """Positions that a row at position p attends to."""
    j = np.arange(p + 1)
    return j if window == 0 else j[(j > p - window) | (j < sinks)]


def attention(q, K, V, table, length: int, n_new: int, window: int, sinks: int, rows: Optional[Sequence[int]] = None):
    """q [n_new, H_q, d_h], K and V [n_pages, page, H_kv, d_h], one sequence's table row; fp64.  Returns the output and the
    same sum over |V| (the scale of a rounding of the probabilities), of the new rows `rows` only where given (the
    others stay zero).  A page that is none reads as zeros."""
    n_pages, page, h_kv, d_h = K.shape
    g = q.shape[1] // h_kv
    out, mag = np.zeros((n_new,) + q.shape[1:]), np.zeros((n_new,) + q.shape[1:])
    for i in range(n_new) if rows is None else rows:
        p = length - n_new + i
        j = sees(p, window, sinks)
        if p < 0 or j.size == 0:
            continue
        pages = np.asarray(table)[j // page]
        there = (pages >= 0) & (pages < n_pages)
        k, v = np.zeros((j.size, h_kv, d_h)), np.zeros((j.size, h_kv, d_h))
        k[there], v[there] = K[pages[there], (j % page)[there]], V[pages[there], (j % page)[there]]
        for h in range(h_kv):
            z = q[i, h * g:(h + 1) * g] @ k[:, h].T / math.sqrt(d_h)
            w = np.exp(z - z.max(axis=1, keepdims=True))
            w /= w.sum(axis=1, keepdims=True)
            out[i, h * g:(h + 1) * g], mag[i, h * g:(h + 1) * g] = w @ v[:, h], w @ np.abs(v[:, h])
    return out, mag


def frequencies(base, rot, scaling="plain", factor=1.0, orig_len=0, low=1.0, high=4.0) -> np.ndarray:
    out = []
    lo = hi = 0
    if scaling == "index":
        def index_of(turns):                             # the pair that makes so many turns within orig_len
            return rot / 2 * math.log(orig_len / (2 * math.pi * turns)) / math.log(base)
        lo, hi = max(math.floor(index_of(high)), 0), min(math.ceil(index_of(low)), rot - 1)
    for j in range(rot // 2):
        w = base ** (-2 * j / rot)
        if scaling == "plain":
            share = 1.0
        elif scaling == "linear":
            share = 0.0
        elif scaling == "turns":
            share = (orig_len / (2 * math.pi / w) - low) / (high - low)
        else:
            share = 1 - (j - lo) / max(hi - lo, 0.001)
        share = min(max(share, 0.0), 1.0)
        out.append(w / factor * (1 - share) + w * share)
    return np.array(out)


def turn(x, pos, freq, interleaved: bool, mscale: float = 1.0) -> np.ndarray:
    """x [rows, heads, d_h] fp64, pos [rows]: pairs as complex numbers times exp(i pos freq)."""
    y, half = np.array(x, dtype=np.float64), len(freq)
    wave = mscale * np.exp(1j * np.asarray(pos, dtype=np.float64)[:, None, None] * freq)
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    z = (y[..., a] + 1j * y[..., b]) * wave
    y[..., a], y[..., b] = z.real, z.imag
    return y


class Pages:
    """The bookkeeping, one sequence and one page at a time; `copies` lists (from, to, tokens) of the last call."""

    def __init__(self, n_pages: int, page: int, n_seqs: int, max_pages: int):
        self.page, self.max_pages = page, max_pages
        self.refs: List[int] = [0] * n_pages
        self.table: List[List[int]] = [[-1] * max_pages for _ in range(n_seqs)]
        self.len: List[int] = [0] * n_seqs
        self.copies: List[tuple] = []

    def held(self, s: int) -> List[int]:
        return self.table[s][:-(-self.len[s] // self.page)]

    def _refuse(self, seqs) -> bool:
        return len(set(seqs)) != len(seqs) or any(not 0 <= s < len(self.len) for s in seqs)

    def grow(self, seqs: Sequence[int], more: Sequence[int]) -> Optional[str]:
        self.copies = []
        if self._refuse(seqs) or any(c < 0 for c in more):
            return "index"
        if any(self.len[s] + c > self.max_pages * self.page for s, c in zip(seqs, more)):
            return "length"
        shared = {s: bool(c and self.len[s] % self.page and self.refs[self.held(s)[-1]] > 1) for s, c in zip(seqs, more)}
        free = [p for p, k in enumerate(self.refs) if k == 0]
        need = sum(-(-(self.len[s] + c) // self.page) - len(self.held(s)) + shared[s] for s, c in zip(seqs, more))
        if need > len(free):
            return "pages"
        for s, c in zip(seqs, more):
            used = len(self.held(s))
            if shared[s]:
                old, new = self.table[s][used - 1], free.pop(0)
                self.copies.append((old, new, self.len[s] % self.page))
                self.refs[old] -= 1
                self.refs[new] = 1
                self.table[s][used - 1] = new
            self.len[s] += c
            for i in range(used, -(-self.len[s] // self.page)):
                self.table[s][i] = free.pop(0)
                self.refs[self.table[s][i]] = 1
        return None

    def fork(self, src: Sequence[int], dst: Sequence[int]) -> Optional[str]:
        if self._refuse(dst) or any(not 0 <= s < len(self.len) for s in src) or any(self.len[d] for d in dst):
            return "index"
        held = [(list(self.held(s)), self.len[s]) for s in src]
        for d, (pages, n) in zip(dst, held):
            self.table[d][:len(pages)], self.len[d] = pages, n
            for p in pages:
                self.refs[p] += 1
        return None

    def free(self, seqs: Sequence[int]) -> Optional[str]:
        if self._refuse(seqs):
            return "index"
        for s in seqs:
            for i, p in enumerate(self.held(s)):
                self.refs[p] -= 1
                self.table[s][i] = -1
            self.len[s] = 0
        return None

    def compact(self) -> None:
        used = [p for p, k in enumerate(self.refs) if k]
        n = len(used)
        move = dict(zip([p for p in used if p >= n], [p for p, k in enumerate(self.refs) if not k and p < n]))
        self.copies = [(p, to, self.page) for p, to in move.items()]
        for p, to in move.items():
            self.refs[to], self.refs[p] = self.refs[p], 0
        for s in range(len(self.len)):
            for i, p in enumerate(self.held(s)):
                self.table[s][i] = move.get(p, p)
