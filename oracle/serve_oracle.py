"""Plain CPU statement of the 8-bit serving operators: linear layers quantized token by token, the paged cache, its attention.

Codes and scales are the fp32 values Eq. 1 defines (two IEEE divisions, one product before the rounding); everything behind
them is in 64 bits.  Pages and sequences are plain Python integers.
"""
from __future__ import annotations

import numpy as np


def scales(absmax, qmax=127.0):
    a = np.asarray(absmax, np.float32)
    with np.errstate(divide="ignore", over="ignore"):
        return (np.where(a == 0, np.float32(1), a / np.float32(qmax)).astype(np.float32),
                np.where(a == 0, np.float32(1), np.float32(qmax) / a).astype(np.float32))


def codes(x, inv, qmax=127.0):
    """Codes of finite or other x: NaN and Inf give 0, a zero always 0."""
    x = np.asarray(x, np.float32)
    ok = np.isfinite(x) & (x != 0)
    with np.errstate(invalid="ignore", over="ignore"):
        p = (np.where(ok, x, np.float32(0)) * inv).astype(np.float32)
    p = np.where(ok, p, np.float32(0))
    return np.clip(np.rint(p), -qmax, qmax).astype(np.int8)


def finite_max(x, axis):
    x = np.abs(np.asarray(x, np.float32))
    return np.max(np.where(np.isfinite(x), x, np.float32(0)), axis=axis, initial=np.float32(0)).astype(np.float32)


def quantize_tokens(x, bits=8):
    qmax = float(2 ** (bits - 1) - 1)
    s, inv = scales(finite_max(x, 1), qmax)
    return codes(x, inv[:, None], qmax), s


def linear(qx, sx, qw, sw, bias=None, act="none"):
    y = qx.astype(np.float64) @ qw.astype(np.float64).T * sx.astype(np.float64)[:, None] * sw.astype(np.float64)[None, :]
    if bias is not None:
        y = y + bias.astype(np.float64)
    if act == "relu":
        y = np.maximum(y, 0)
    elif act == "gelu":
        y = 0.5 * y * (1 + np.tanh(np.sqrt(2 / np.pi) * (y + 0.044715 * y ** 3)))
    return y


class Pool:
    """Sequences and their pages.  A call that cannot be carried out whole returns False and changes nothing."""

    def __init__(self, n_pages, page, max_seqs, max_pages):
        self.n_pages, self.page, self.max_seqs, self.max_pages = n_pages, page, max_seqs, max_pages
        self.table = [[] for _ in range(max_seqs)]
        self.lens = [0] * max_seqs
        self.refs = [0] * n_pages

    def pages_for(self, tokens):
        return -(-tokens // self.page)

    def free_pages(self):
        return [p for p, r in enumerate(self.refs) if r == 0]

    def extend(self, seqs, rows):
        real = [s for s in seqs if s >= 0]
        if len(set(real)) != len(real) or any(s >= self.max_seqs for s in real):
            return False
        want = [(s, r, self.pages_for(self.lens[s] + r) - len(self.table[s])) for s, r in zip(seqs, rows) if s >= 0]
        free = self.free_pages()
        if any(self.pages_for(self.lens[s] + r) > self.max_pages for s, r, _ in want) or sum(w for _, _, w in want) > len(free):
            return False
        for s, r, w in want:
            for _ in range(w):
                p = free.pop(0)
                self.refs[p] = 1
                self.table[s].append(p)
            self.lens[s] += r
        return True

    def free(self, seqs):
        for s in seqs:
            if s < 0:
                continue
            for p in self.table[s]:
                self.refs[p] -= 1
            self.table[s] = []
            self.lens[s] = 0

    def fork(self, parents, children):
        """(src, dst), or None where the call is refused."""
        pairs = [(f, p, c) for f, (p, c) in enumerate(zip(parents, children)) if c >= 0]
        kids = [c for _, _, c in pairs]
        if len(set(kids)) != len(kids) or any(c >= self.max_seqs or not 0 <= p < self.max_seqs for _, p, c in pairs):
            return None
        if any(self.lens[c] for c in kids):
            return None
        parts = [f for f, p, _ in pairs if self.lens[p] % self.page]
        free = self.free_pages()
        if len(parts) > len(free):
            return None
        src, dst = [-1] * len(parents), [-1] * len(parents)
        was = [(list(self.table[p]) if p >= 0 else [], self.lens[p] if p >= 0 else 0) for p in parents]
        for f, p, c in pairs:
            row, length = was[f]
            full = length // self.page
            for page in row[:full]:
                self.refs[page] += 1
            self.table[c] = row[:full]
            if length % self.page:
                src[f], dst[f] = row[full], free.pop(0)
                self.refs[dst[f]] = 1
                self.table[c].append(dst[f])
            self.lens[c] = length
        return src, dst

    def compact(self):
        live = [p for p, r in enumerate(self.refs) if r > 0]
        where = {p: p for p in live if p < len(live)}
        holes = [p for p in range(len(live)) if self.refs[p] == 0]
        where.update(zip([p for p in live if p >= len(live)], holes))
        refs = [0] * self.n_pages
        for p in live:
            refs[where[p]] = self.refs[p]
        self.refs = refs
        self.table = [[where[p] for p in row] for row in self.table]
        return [where.get(p, -1) for p in range(self.n_pages)]

    def table_array(self):
        t = np.full((self.max_seqs, self.max_pages), -1, np.int32)
        for s, row in enumerate(self.table):
            t[s, :len(row)] = row
        return t


class Cache:
    """One layer's codes and maxima."""

    def __init__(self, pool, heads, dim):
        self.pool, self.heads, self.dim = pool, heads, dim
        self.codes = [np.zeros((pool.n_pages, heads, pool.page, dim), np.int8) for _ in range(2)]
        self.absmax = [np.zeros((pool.n_pages, heads), np.float32) for _ in range(2)]

    def append(self, k, v, seqs, starts):
        page = self.pool.page
        for z, x in enumerate((k, v)):
            for i, s in enumerate(seqs):
                rows = x[starts[i]:starts[i + 1]]
                if s < 0 or not len(rows):
                    continue
                first = self.pool.lens[s] - len(rows)
                for j in range(first // page, self.pool.pages_for(self.pool.lens[s])):
                    lo, hi = max(first, j * page), min(first + len(rows), (j + 1) * page)
                    number = self.pool.table[s][j]
                    new = rows[lo - first:hi - first].transpose(1, 0, 2)
                    for h in range(self.heads):
                        held = self.absmax[z][number, h] if lo > j * page else np.float32(0)
                        now = max(held, finite_max(new[h], None))
                        if lo > j * page and now > held > 0:
                            old = self.codes[z][number, h, :lo - j * page]
                            old[:] = np.rint((old.astype(np.float32) * (held / now).astype(np.float32)).astype(np.float32)).astype(np.int8)
                        self.codes[z][number, h, lo - j * page:hi - j * page] = codes(new[h], scales(now)[1])
                        self.absmax[z][number, h] = now

    def copy_pages(self, src, dst):
        for p, d in zip(range(len(dst)) if src is None else src, dst):
            if p >= 0 and d >= 0 and p != d:
                for z in range(2):
                    self.codes[z][d] = self.codes[z][p]
                    self.absmax[z][d] = self.absmax[z][p]

    def values(self, s):
        """Keys and values of sequence s: [len, heads, dim] each, 64 bits."""
        row = self.pool.table[s]
        out = []
        for z in range(2):
            x = self.codes[z][row].astype(np.float64) * scales(self.absmax[z][row])[0].astype(np.float64)[:, :, None, None]
            out.append(x.transpose(0, 2, 1, 3).reshape(-1, self.heads, self.dim)[:self.pool.lens[s]])
        return out


def seen(rows, length, causal, window):
    """[rows, length]: whether row r (the token length - rows + r) sees token t."""
    pos = length - rows + np.arange(rows)[:, None]
    t = np.arange(length)[None, :]
    if not causal:
        return np.broadcast_to(pos >= 0, (rows, length)).copy()
    return (t <= pos) & ((t > pos - window) if window else True) & (pos >= 0)


def attention(q, k, v, sm_scale, causal=True, window=0):
    """q [rows, q_heads, dim], k and v [len, heads, dim]: (out, per-element size of what is summed, largest |q||k| sum)."""
    rows, q_heads, dim = q.shape
    length, heads, _ = k.shape
    q = q.astype(np.float64)
    out, weight, spread = np.zeros(q.shape), np.zeros(q.shape), np.zeros((rows, q_heads))
    if length == 0:
        return out, weight, spread
    mask = seen(rows, length, causal, window)
    for h in range(q_heads):
        kh, vh = k[:, h // (q_heads // heads)], v[:, h // (q_heads // heads)]
        s = np.where(mask, q[:, h] @ kh.T * sm_scale, -np.inf)
        some = mask.any(1)
        top = np.where(some, s.max(1), 0)
        p = np.where(mask, np.exp(s - top[:, None]), 0)
        total = np.where(some, p.sum(1), 1)
        out[:, h] = p @ vh / total[:, None]
        weight[:, h] = p @ np.abs(vh) / total[:, None]
        spread[:, h] = np.where(mask, np.abs(q[:, h]) @ np.abs(kh).T * sm_scale, 0).max(1)
    return out, weight, spread
