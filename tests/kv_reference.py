"""Plain 64-bit attention over a paged cache, and the page book with Python
lists: what the GPU tests of the key-value cache compare with."""
import numpy as np


def attention(q, k, v, table, length, first, scale, window, n_sinks):
    """q [rows, heads, dim] at positions first, first + 1, ...; k and v
    [pages, kv_heads, page_rows, dim], all float64.  Returns the output and
    bounds' ingredients: the weighted mean of |v| and the largest sum of
    |q_d k_d| scale over the visible tokens of each row and head."""
    rows, heads, dim = q.shape
    n_pages, kv_heads, pr, _ = k.shape
    group = heads // kv_heads
    out = np.zeros_like(q)
    mean_abs = np.zeros_like(q)
    reach = np.zeros((rows, heads, 1))
    for r in range(rows):
        p = first + r
        if p < 0:
            continue
        j = np.arange(0, min(p + 1, length))
        if window:
            j = j[(j > p - window) | (j < n_sinks)]
        page = np.asarray(table, dtype=np.int64)[j // pr]
        ok = (page >= 0) & (page < n_pages)
        j, page = j[ok], page[ok]
        if not len(j):
            continue
        for h in range(heads):
            kk, vv = k[page, h // group, j % pr], v[page, h // group, j % pr]
            s = kk @ q[r, h] * scale
            w = np.exp(s - s.max())
            out[r, h] = w @ vv / w.sum()
            mean_abs[r, h] = w @ np.abs(vv) / w.sum()
            reach[r, h] = (np.abs(kk) @ np.abs(q[r, h])).max() * scale
    return out, mean_abs, reach


def allowance(out, mean_abs, reach, dim, n_tokens, bf16):
    """How far a correct kernel may be from `out`: the output's rounding, half
    a unit in the last place; each weight rounded once to the storage type in
    numerator and denominator (2 u of the weighted mean of |v|; for binary16 also
    2^-24 per token where weights are subnormal); a float32 score off by
    (dim + 8) 2^-24 of its terms, and its exponential by 2^-20, which moves
    weights by that much, numerator and denominator again; float32 sums over
    the tokens."""
    u = 2.0 ** -9 if bf16 else 2.0 ** -12
    weight = u + (dim + 8) * 2.0 ** -24 * reach + 2.0 ** -20 + n_tokens * 2.0 ** -24
    sub = 0.0 if bf16 else n_tokens * 2.0 ** -23 * np.maximum(1.0, mean_abs)
    tiny = 2.0 ** -133 if bf16 else 2.0 ** -25
    return u * np.abs(out) * (1 + 2 * u) + 2 * weight * mean_abs * (1 + 4 * u) + sub + tiny


class Book:
    """The page book by its definition."""

    def __init__(self, tables, lens, n_pages, page_rows):
        self.t = [list(map(int, r)) for r in tables]
        self.lens = [int(v) for v in lens]
        self.pr, self.n_pages = page_rows, n_pages
        self.refs = [0] * n_pages
        for s in range(len(self.lens)):
            for p in self.pages(s):
                self.refs[p] += 1

    def held(self, s):
        return -(-max(0, self.lens[s]) // self.pr)

    def pages(self, s):
        return [p for p in self.t[s][:self.held(s)] if 0 <= p < self.n_pages]

    def free_pages(self):
        return [p for p in range(self.n_pages) if self.refs[p] == 0]

    def grow(self, add):
        free, wanted, taken, stayed, room = self.free_pages(), 0, 0, 0, len(self.t[0]) * self.pr
        for s in range(len(self.lens)):
            to = self.lens[s] + max(0, int(add[s]))
            if to > room:
                stayed += 1
                continue
            need = -(-to // self.pr) - self.held(s)
            wanted += need
            if need and wanted > len(free):
                stayed += 1
                continue
            at = self.held(s)
            for i in range(need):
                p = free[taken + i]
                self.t[s][at + i] = p
                self.refs[p] = 1
            taken += need
            self.lens[s] = to
        return [taken, stayed]

    def free(self, seqs):
        for s in seqs:
            for p in self.pages(s):
                self.refs[p] -= 1
            self.lens[s] = 0
            self.t[s] = [-1] * len(self.t[s])

    def fork(self, parents, children):
        """Returns info and the (src, dst, rows) copied."""
        self.free(children)
        free, taken, empty, copies = self.free_pages(), 0, 0, []
        for a, c in zip(parents, children):
            full, tail = divmod(self.lens[a], self.pr)
            src = self.t[a][full] if tail else -1
            row = [-1] * len(self.t[c])
            if 0 <= src < self.n_pages:
                if taken == len(free):
                    empty += 1
                    continue
                row[full] = free[taken]
                self.refs[free[taken]] = 1
                copies.append((src, free[taken], tail))
                taken += 1
            for e in range(full):
                if 0 <= self.t[a][e] < self.n_pages:
                    row[e] = self.t[a][e]
                    self.refs[row[e]] += 1
            self.t[c], self.lens[c] = row, self.lens[a]
        return [taken, empty], copies

    def trim(self, window, n_sinks):
        for s in range(len(self.lens)):
            for e in range(self.held(s)):
                if (e + 1) * self.pr - 1 <= self.lens[s] - window and e * self.pr >= n_sinks:
                    if 0 <= self.t[s][e] < self.n_pages:
                        self.refs[self.t[s][e]] -= 1
                    self.t[s][e] = -1

    def compact(self):
        """Returns info and the (src, dst) moved; the book has the new ids."""
        live = [p for p in range(self.n_pages) if self.refs[p]]
        n = len(live)
        src = [p for p in live if p >= n]
        dst = [p for p in range(n) if not self.refs[p]]
        to = {p: p for p in live}
        to.update(zip(src, dst))
        for s in range(len(self.lens)):
            h = self.held(s)
            self.t[s] = [to.get(p, -1) if e < h else -1 for e, p in enumerate(self.t[s])]
        refs = [0] * self.n_pages
        for p in live:
            refs[to[p]] = self.refs[p]
        self.refs = refs
        return [n, len(src)], list(zip(src, dst))
