"""What the decode operators are to compute, in numpy and 64 bits, written from their definitions:
4-bit weights, attention over a paged cache, and the care of its pages."""

import numpy as np

U24 = 2.0 ** -24


def ceil(a, b):
    return -(-a // b)


# ---- 4-bit weights ----

def bf16(a):
    """Rounded to the nearest bf16, ties to even."""
    u = np.ascontiguousarray(a, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7fff + (u >> 16 & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)


def q4_quantize(w, mask, group):
    """Codes [rows][cols] and scales [groups][rows] of fp32 weights."""
    w = np.asarray(w, np.float32) * (1 if mask is None else (mask != 0))
    rows, cols = w.shape
    n = np.full((rows, cols), 8, np.int64)
    scales = np.zeros((ceil(cols, group), rows), np.float32)
    for g in range(ceil(cols, group)):
        block = w[:, g * group:(g + 1) * group].astype(np.float32)
        s = bf16(np.abs(block).max(1) * (np.float32(1) / np.float32(7)))
        scales[g] = s
        with np.errstate(all="ignore"):
            q = np.clip(np.rint((block / s[:, None]).astype(np.float32)), -7, 7)
        n[:, g * group:(g + 1) * group] = np.where(s[:, None] == 0, 0, q) + 8
    return n, scales


def q4_bytes(n):
    """Codes as they lie in memory."""
    rows, cols = n.shape
    out = np.zeros((rows, ceil(ceil(cols, 2), 16) * 16), np.uint8)
    even, odd = n[:, 0::2], n[:, 1::2]
    out[:, :even.shape[1]] |= even.astype(np.uint8)
    out[:, :odd.shape[1]] |= (odd << 4).astype(np.uint8)
    return out


def q4_scales(scales):
    """Scales as they lie in memory (as fp32 values)."""
    out = np.zeros((scales.shape[0], ceil(scales.shape[1], 16) * 16), np.float32)
    out[:, :scales.shape[1]] = scales
    return out


def q4_weights(n, scales, group):
    g = np.arange(n.shape[1]) // group
    return scales.astype(np.float64)[g].T * (n - 8)


# ---- attention ----

def attention(q, keys, values, pages, page_size, length, window, scale):
    """One query head: (y, lse, sum of p |v|, root of the sum of (p v)^2, largest sum of |q k| times
    scale), from [page][slot][dim] keys and values of its key head."""
    first = max(0, length - window) if window else 0
    at = [(pages[t // page_size], t % page_size) for t in range(first, min(length, len(pages) * page_size))]
    at = [(p, s) for p, s in at if 0 <= p < keys.shape[0]]
    if not at:
        return np.zeros(q.shape), -np.inf, np.zeros(q.shape), np.zeros(q.shape), 0.0
    p, s = np.array(at).T
    k, v = keys[p, s].astype(np.float64), values[p, s].astype(np.float64)
    score = k @ q.astype(np.float64) * scale
    top = score.max()
    e = np.exp(score - top)
    w = e / e.sum()
    return w @ v, top + np.log(e.sum()), w @ np.abs(v), np.sqrt((w * w) @ (v * v)), float((np.abs(k) @ np.abs(q)).max() * abs(scale))


# ---- pages ----

class Pages:
    """Tables, lengths, counts, and what every slot holds (a token's number, 0: never written)."""

    def __init__(self, seqs, width, pages, page_size):
        self.table = np.full((seqs, width), -1, np.int64)
        self.lens, self.refs = np.zeros(seqs, np.int64), np.zeros(pages, np.int64)
        self.data = np.zeros((pages, page_size), np.int64)
        self.page = page_size

    def in_rows(self, r):
        return 0 <= r < len(self.lens)

    def drop(self, row):
        for e in row:
            if e >= 0:
                self.refs[e] -= 1

    def fork(self, parents, children):
        pairs = [(p, c) for p, c in zip(parents, children) if self.in_rows(p) and self.in_rows(c)]
        rows = [(self.table[p].copy(), self.lens[p]) for p, _ in pairs]
        for row, _ in rows:
            for e in row:
                if e >= 0:
                    self.refs[e] += 1
        for (_, c), (row, n) in zip(pairs, rows):
            self.drop(self.table[c])
            self.table[c], self.lens[c] = row, n

    def release(self, rows):
        for r in rows:
            if self.in_rows(r):
                self.drop(self.table[r])
                self.table[r], self.lens[r] = -1, 0

    def extend(self, rows, counts):
        refs = self.refs.copy()
        free = [i for i in range(len(refs)) if refs[i] == 0]
        plan, used = [], 0
        for r, c in zip(rows, counts):
            if not self.in_rows(r) or c <= 0:
                plan.append(None)
                continue
            n = int(self.lens[r])
            entries = list(range(ceil(n, self.page), ceil(n + c, self.page)))
            if entries and entries[-1] >= self.table.shape[1]:
                return [-1] * len(rows)
            if n % self.page:
                e = self.table[r, n // self.page]
                if e < 0 or refs[e] > 1:
                    entries = [n // self.page] + entries
            plan.append(entries)
            used += len(entries)
        if used > len(free):
            return [-1] * len(rows)
        pos, before, it = [], self.data.copy(), iter(free)
        for r, c, entries in zip(rows, counts, plan):
            pos.append(int(self.lens[r]) if self.in_rows(r) else -1)
            for e in entries or []:
                new, old = next(it), self.table[r, e]
                if e == self.lens[r] // self.page and self.lens[r] % self.page and old >= 0:
                    m = self.lens[r] % self.page
                    self.data[new, :m] = before[old, :m]
                    self.refs[old] -= 1
                self.table[r, e], self.refs[new] = new, 1
            if entries is not None:
                self.lens[r] += c
        return pos

    def compact(self):
        used = int((self.refs > 0).sum())
        src = [i for i in range(used, len(self.refs)) if self.refs[i] > 0]
        dst = [i for i in range(used) if self.refs[i] == 0]
        to = dict(zip(src, dst))
        for a, b in to.items():
            self.data[b] = self.data[a]
            self.refs[a], self.refs[b] = 0, self.refs[a]
        self.table = np.array([[to.get(e, e) for e in row] for row in self.table.tolist()], np.int64).reshape(self.table.shape)
        return used, len(src)

    def write(self, row, pos, value):
        if self.in_rows(row) and pos >= 0 and pos // self.page < self.table.shape[1]:
            e = self.table[row, pos // self.page]
            if e >= 0:
                self.data[e, pos % self.page] = value
