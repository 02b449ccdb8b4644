"""CPU oracle of the paged key/value cache and of what works on it: the book-keeping (room, forks, ends, accepted paths,
moves to the front), the norm and rotation of queries and keys, and attention of the last tokens of every sequence over
pages.  TEST INFRASTRUCTURE: plain Python and numpy in fp64, one sequence and one head at a time, from the statements of
include/dsla.h; shares nothing with the product.
"""
import numpy as np

FULL, ENTRY = 2, 4


class Cache:
    """table [n_seqs][max_pages], lens, refs and a list of pools [n_pages][H_kv][page][d] (any dtype, moved as they are)."""

    def __init__(self, n_pages, page, n_seqs, max_pages, pools=()):
        self.n_pages, self.page, self.n_seqs, self.max_pages = n_pages, page, n_seqs, max_pages
        self.table = np.full((n_seqs, max_pages), -1, np.int32)
        self.lens = np.zeros(n_seqs, np.int32)
        self.refs = np.zeros(n_pages, np.int32)
        self.pools = list(pools)
        self.status = 0

    def pages(self, tokens):
        return -(-tokens // self.page)

    def valid(self, s, t):
        p = int(self.table[s, t // self.page])
        return p if 0 <= p < self.n_pages else None

    def entries(self, cu, row, total):
        """(tokens' first number, how many, row) of every entry, or None where they are out of range."""
        out = []
        for b in range(len(row)):
            a, e = (b, b + 1) if cu is None else (int(cu[b]), int(cu[b + 1]))
            out.append((a, e - a, int(row[b])) if 0 <= a <= e <= total and 0 <= row[b] < self.n_seqs else None)
        return out

    def extend(self, cu, row, total):
        free = [p for p in range(self.n_pages) if self.refs[p] == 0]
        start, used, short, seen, copies = np.full(len(row), -1, np.int32), 0, False, set(), []
        for b, e in enumerate(self.entries(cu, row, total)):
            if e is None or e[2] in seen or not 0 <= self.lens[e[2]] <= self.max_pages * self.page:
                self.status |= ENTRY
                continue
            _, n, s = e
            seen.add(s)
            at = int(self.lens[s])
            if at + n > self.max_pages * self.page:
                self.status |= FULL
                continue
            first, last = self.pages(at), None
            if at % self.page and n:
                last = self.valid(s, at - 1)
                if last is None:
                    self.status |= ENTRY
                    continue
                # (whether it is shared is judged before the call changes anything)
                last = last if self.refs[last] + sum(c[0] == last for c in copies) > 1 else None
                first -= last is not None
            need = self.pages(at + n) - first
            if need and (short or used + need > len(free)):
                short = True
                self.status |= FULL
                continue
            if last is not None:
                self.refs[last] -= 1
                copies.append((last, free[used], at % self.page))
            for c in range(first, first + need):
                self.table[s, c] = free[used]
                self.refs[free[used]] = 1
                used += 1
            self.lens[s] = at + n
            start[b] = at
        for src, dst, rows in copies:
            for p in self.pools:
                p[dst, :, :rows] = p[src, :, :rows]
        return start

    def cut(self, s, keep):
        for c in range(self.pages(keep), self.pages(int(self.lens[s]))):
            p = int(self.table[s, c])
            if 0 <= p < self.n_pages:
                self.refs[p] -= 1
            else:
                self.status |= ENTRY
            self.table[s, c] = -1
        self.lens[s] = keep

    def truncate(self, new_lens):
        for s in range(self.n_seqs):
            if 0 <= new_lens[s] < self.lens[s]:
                if self.lens[s] > self.max_pages * self.page:
                    self.status |= ENTRY
                else:
                    self.cut(s, int(new_lens[s]))

    def fork(self, parent):
        for s in range(self.n_seqs):
            f = int(parent[s])
            if f < 0:
                continue
            if f >= self.n_seqs or parent[f] >= 0 or self.lens[s] != 0 or not 0 <= self.lens[f] <= self.max_pages * self.page:
                self.status |= ENTRY
                continue
            n = self.pages(int(self.lens[f]))
            self.table[s, :n] = self.table[f, :n]
            for p in self.table[f, :n]:
                if 0 <= p < self.n_pages:
                    self.refs[p] += 1
                else:
                    self.status |= ENTRY
            self.lens[s] = self.lens[f]

    def accept(self, cu, row, total, start, path, n_accepted):
        todo, entries = [], self.entries(cu, row, total)
        takes_part = [e is not None and start[b] >= 0 for b, e in enumerate(entries)]
        for b, e in enumerate(entries):
            k = int(n_accepted[b])
            if k < 0 or (e is not None and start[b] < 0):
                continue
            if e is None or e[2] in [int(r) for r, part in zip(row[:b], takes_part) if part] or k > e[1] or self.lens[e[2]] != start[b] + e[1]:
                self.status |= ENTRY
                continue
            a, n, s = e
            way, at = [int(x) for x in path[a:a + k]], int(start[b])
            if any(not 0 <= x < n for x in way) or any(x >= y for x, y in zip(way, way[1:])):
                self.status |= ENTRY
                continue
            pairs = [(self.valid(s, at + x), (at + x) % self.page, self.valid(s, at + i), (at + i) % self.page) for i, x in enumerate(way) if x != i]
            if any(p is None or q is None or self.refs[q] != 1 for p, _, q, _ in pairs):
                self.status |= ENTRY
                continue
            todo.append((s, at + k, pairs))
        for s, keep, pairs in todo:
            for pool in self.pools:
                rows = [pool[p, :, i].copy() for p, i, _, _ in pairs]
                for (_, _, q, j), x in zip(pairs, rows):
                    pool[q, :, j] = x
            self.cut(s, keep)

    def compact(self):
        live = [p for p in range(self.n_pages) if self.refs[p] > 0]
        L = len(live)
        to = dict(zip([p for p in live if p >= L], [p for p in range(L) if self.refs[p] <= 0]))
        for src, dst in to.items():
            for p in self.pools:
                p[dst] = p[src]
            self.refs[dst], self.refs[src] = self.refs[src], 0
        for s in range(self.n_seqs):
            for c in range(self.pages(int(self.lens[s]))):
                self.table[s, c] = to.get(int(self.table[s, c]), self.table[s, c])
        return L


def rotate(x, weight, eps, position, inv_freq, interleaved):
    """x [M, heads, d]: normalised by the root mean square where there is a weight, then rotated.  Returns the result and, for every
    element, the sum of the absolute values of the (normalised) features that it is made of."""
    y = np.asarray(x, np.float64)
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + float(np.float32(eps))) * np.asarray(weight, np.float64)
    out, size = y.copy(), np.abs(y)
    for i, f in enumerate(np.asarray(inv_freq, np.float64)):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + len(inv_freq))
        c, s = np.cos(np.asarray(position, np.float64) * f)[:, None], np.sin(np.asarray(position, np.float64) * f)[:, None]
        out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., a] * s + y[..., b] * c
        size[..., a] = size[..., b] = np.abs(y[..., a]) + np.abs(y[..., b])
    return out, size


def attention(cache, k_pages, v_pages, cu, row, start, q, scale, tree=None):
    """q [total, H, d], pools fp64 [n_pages, H_kv, page, d].  Returns o, the weighted mean of |v| for every element, and for every query
    and head the largest sum |q||k| scale over the keys that it sees; rows of entries that take no part are NaN."""
    total, H, d = q.shape
    o, size, reach = (np.full(s, np.nan) for s in ((total, H, d), (total, H, d), (total, H)))
    H_kv, page = k_pages.shape[1], cache.page
    for b, e in enumerate(cache.entries(cu, row, total)):
        if e is None or start[b] < 0:
            continue
        a, n, s = e
        at = int(start[b])
        where = [(t, cache.valid(s, t)) for t in range(at + n)]
        where = [(t, p) for t, p in where if p is not None]
        t, p = np.array([x for x, _ in where], int), np.array([x for _, x in where], int)
        for j in range(n):
            mask = (1 << (j + 1)) - 1 if tree is None else int(tree[a + j]) & (2 ** 64 - 1)
            seen = np.array([x < at or mask >> (x - at) & 1 for x in t.tolist()], bool)
            for h in range(H):
                g = h // (H // H_kv)
                keys, values = k_pages[p[seen], g, t[seen] % page], v_pages[p[seen], g, t[seen] % page]
                if not seen.any():
                    o[a + j, h] = size[a + j, h] = reach[a + j, h] = 0
                    continue
                with np.errstate(all="ignore"):
                    score = scale * (keys @ q[a + j, h])
                    w = np.exp(score - score.max())
                    o[a + j, h] = w @ values / w.sum()
                    size[a + j, h] = w @ np.abs(values) / w.sum()
                    reach[a + j, h] = abs(scale) * (np.abs(keys) @ np.abs(q[a + j, h])).max()
    return o, size, reach
