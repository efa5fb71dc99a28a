"""The operators on a paged key/value cache, spelled out: plain numpy in float64, loops over tokens and heads, page
tables as Python lists.  Test infrastructure; shares no code with the HIP path."""
import numpy as np


class Refused(Exception):
    """What the operators report through their status word: "room" (free pages) or "argument"."""


class Cache:
    """table: one list of pages per sequence; k, v: [layers, n_pages, page_tokens, kv_heads, head_dim] of any dtype."""

    def __init__(self, k, v, n_seqs, max_pages):
        self.k, self.v = k, v
        self.page = k.shape[2]
        self.max_pages = max_pages
        self.table = [[] for _ in range(n_seqs)]
        self.length = [0] * n_seqs
        self.refs = [0] * k.shape[1]

    def table_array(self):
        out = np.full((len(self.table), self.max_pages), -1, dtype=np.int32)
        for s, pages in enumerate(self.table):
            out[s, :len(pages)] = pages
        return out

    def pages_for(self, n):
        return (n + self.page - 1) // self.page

    def place(self, s, pos):
        return self.table[s][pos // self.page], pos % self.page

    def _take(self, count):
        free = [p for p, n in enumerate(self.refs) if n == 0][:count]
        if len(free) < count:
            raise Refused("room")
        return free

    def _apply(self, plans, free, copies):
        """plans: {sequence: (new list of pages, None for one to take)}; copies: (s, old place, position)."""
        old = {s: list(self.table[s]) for s in plans}
        shared = list(self.refs)
        for s, pages in sorted(plans.items()):
            self.table[s] = [free.pop(0) if p is None else p for p in pages]
        for s in plans:
            for p in set(self.table[s]) - set(old[s]):
                self.refs[p] = 1
            for p in set(old[s]) - set(self.table[s]):
                self.refs[p] -= 1
        assert not free and all(shared[p] > 0 or self.refs[p] <= 1 for p in range(len(shared)))
        data = [(pool[:, a, b].copy()) for s, (a, b), _ in copies for pool in (self.k, self.v)]
        for s, _, pos in copies:
            a, b = self.place(s, pos)
            for pool in (self.k, self.v):
                pool[:, a, b] = data.pop(0)

    def reserve(self, extra):
        plans, copies, need = {}, [], 0
        for s, n in enumerate(extra):
            if n < 0:
                continue
            pages, length = list(self.table[s]), self.length[s]
            if length > len(pages) * self.page or self.pages_for(length + n) > self.max_pages:
                raise Refused("argument")
            for i in range(length // self.page, min(self.pages_for(length + n), len(pages)) if n > 0 else 0):
                if self.refs[pages[i]] > 1:
                    copies += [(s, self.place(s, pos), pos) for pos in range(i * self.page, length)]
                    pages[i] = None
            pages += [None] * (self.pages_for(length + n) - len(pages))
            plans[s] = pages
            need += pages.count(None)
        self._apply(plans, self._take(need), copies)

    def fork(self, src, dst):
        if len(set(dst)) < len(dst) or set(src) & set(dst) or not all(0 <= i < len(self.table) for i in [*src, *dst]):
            raise Refused("argument")
        if any(self.length[s] > len(self.table[s]) * self.page for s in src):
            raise Refused("argument")
        for s, d in zip(src, dst):
            for p in self.table[d]:
                self.refs[p] -= 1
            self.table[d] = self.table[s][:self.pages_for(self.length[s])]
            self.length[d] = self.length[s]
            for p in self.table[d]:
                self.refs[p] += 1

    def compact(self, keep, n_keep, start=None):
        plans, copies, need, lengths = {}, [], 0, {}
        for s, n in enumerate(n_keep):
            if n < 0:
                continue
            first = self.length[s] if start is None else start[s]
            if n > (0 if keep is None else len(keep[s])) or not 0 <= first <= self.length[s] or self.length[s] > len(self.table[s]) * self.page:
                raise Refused("argument")
            mine = [int(x) for x in keep[s][:n]] if n else []
            if any(b <= a for a, b in zip([-1] + mine, mine)) or (mine and first + mine[-1] >= len(self.table[s]) * self.page):
                raise Refused("argument")
            pages = self.table[s][:self.pages_for(first + n)]
            moved = [i for i in range(n) if mine[i] != i]
            if moved:
                begin = first + moved[0]
                for i in range(begin // self.page, len(pages)):
                    if self.refs[pages[i]] > 1:
                        pages[i] = None
                if pages[begin // self.page] is None:
                    begin = begin // self.page * self.page
                copies += [(s, self.place(s, pos if pos < first else first + mine[pos - first]), pos) for pos in range(begin, first + n)]
            plans[s], lengths[s] = pages, first + n
            need += pages.count(None)
        self._apply(plans, self._take(need), copies)
        for s, n in lengths.items():
            self.length[s] = n


def norm_rope(x, gain, gain_offset, eps, position, rope_dim, base, interleaved):
    """x [tokens, heads, d] -> normed (gain not None) and rotated, float64."""
    x = x.astype(np.float64)
    if gain is not None:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * (gain_offset + gain.astype(np.float64))
    out = x.copy()
    for i in range(rope_dim // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rope_dim // 2)
        t = np.asarray(position, dtype=np.float64)[:, None] * float(base) ** (-2.0 * i / rope_dim)
        out[..., a] = x[..., a] * np.cos(t) - x[..., b] * np.sin(t)
        out[..., b] = x[..., a] * np.sin(t) + x[..., b] * np.cos(t)
    return out


def attention(q, k, v, seen, scale):
    """q [n, heads, d], k / v [positions, kv_heads, d], seen [n, positions] -> [n, heads, d]; a row that sees nothing is 0.
    Only what a row sees is looked at."""
    n, heads, d = q.shape
    group = heads // k.shape[1]
    out = np.zeros((n, heads, d))
    for i in range(n):
        at = np.flatnonzero(seen[i])
        if at.size == 0:
            continue
        for h in range(heads):
            kk, vv = k[at, h // group].astype(np.float64), v[at, h // group].astype(np.float64)
            s = scale * (kk @ q[i, h].astype(np.float64))
            w = np.exp(s - s.max())
            out[i, h] = (w @ vv) / w.sum()
    return out
