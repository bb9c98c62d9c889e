"""What the calls on a paged cache do, restated in plain Python on host arrays, one entry after the other, from the description
in mate.h (no code shared with the library)."""
import numpy as np

TEXT = 0x7FFFFFFF


class CacheModel:
    def __init__(self, pages, page_size, seqs, width, rng=None):
        self.ps, self.pages, self.width = page_size, pages, width
        self.table = np.full((seqs, width), -1, np.int32)
        self.lens, self.prefix = np.zeros(seqs, np.int32), np.zeros(seqs, np.int32)
        self.refs = np.zeros(pages, np.int32)
        # a slot's content is known by a number: what was written there last
        self.slots = np.zeros((pages, page_size), np.int64)

    def n_pages(self, n):
        return -(-n // self.ps)

    def free_pages(self):
        return [p for p in range(self.pages) if self.refs[p] <= 0]

    def extend(self, seqs, counts):
        """Returns granted; what does not fit stops everyone behind it who needs pages."""
        granted, seen, free, stopped = [], set(), self.free_pages(), False
        for s, n in zip(seqs, counts):
            ok = 0 <= s < len(self.lens) and n >= 0 and s not in seen
            if ok and self.lens[s] + n > self.width * self.ps:
                ok = False
            elif ok:
                seen.add(s)
            need = self.n_pages(self.lens[s] + n) - self.n_pages(self.lens[s]) if ok else 0
            if ok and need > 0 and (stopped or need > len(free)):
                ok, stopped = False, True
            if ok:
                first = self.n_pages(self.lens[s])
                for i in range(need):
                    self.table[s, first + i] = free[0]
                    self.refs[free.pop(0)] = 1
                self.lens[s] += n
            granted.append(n if ok else 0)
        return granted

    def place(self, s, at):
        return self.table[s, at // self.ps], at % self.ps

    def append(self, seqs, counts, marks):
        for i, (s, n) in enumerate(zip(seqs, counts)):
            for j in range(n):
                page, slot = self.place(s, self.lens[s] - n + j)
                self.slots[page, slot] = marks[i][j]

    def fork(self, parents, children):
        before, free = (self.lens.copy(), self.table.copy(), self.prefix.copy(), self.slots.copy()), self.free_pages()
        lens, table, prefix, slots = before
        seen = set()
        for p, c in zip(parents, children):
            if not (0 <= p < len(lens) and 0 <= c < len(lens)) or lens[c] != 0 or c in seen:
                continue
            seen.add(c)
            full, fill = divmod(int(lens[p]), self.ps)
            if fill and not free:
                continue
            self.table[c, :full] = table[p, :full]
            for q in table[p, :full]:
                self.refs[q] += 1
            if fill:
                to = free.pop(0)
                self.refs[to] = 1
                self.table[c, full] = to
                self.slots[to, :fill] = slots[table[p, full], :fill]
            self.lens[c], self.prefix[c] = lens[p], prefix[p]

    def free(self, seqs):
        for s in seqs:
            if not 0 <= s < len(self.lens) or self.lens[s] == 0:
                continue
            for q in self.table[s, :self.n_pages(self.lens[s])]:
                self.refs[q] -= 1
            self.table[s], self.lens[s] = -1, 0

    def compact(self):
        live = int((self.refs > 0).sum())
        holes = [p for p in range(live) if self.refs[p] <= 0]
        movers = [p for p in range(live, self.pages) if self.refs[p] > 0]
        to = {a: b for a, b in zip(movers, holes)}
        for a, b in to.items():
            self.slots[b], self.refs[b], self.refs[a] = self.slots[a], self.refs[a], 0
        for s in range(len(self.lens)):
            for i in range(self.n_pages(self.lens[s])):
                self.table[s, i] = to.get(int(self.table[s, i]), self.table[s, i])
        return live


def attention(q, k, v, row, col, q_row, q_col, prefix, view, scale):
    """One new token and one head in 64 bits: q [d], k, v [n, d], ids of the n cached tokens.  Returns (O, LSE)."""
    n = len(k)
    at = np.arange(n)
    always = (at < prefix) | (q_row == TEXT)
    by_row = (row >= 0) & (always | (row == TEXT) | (row == q_row))
    by_col = (col >= 0) & (always | (col == TEXT) | (col == q_col))
    keep = {0: by_row, 1: by_col, 2: by_row | by_col}[view]
    if q_row < 0:
        keep = np.zeros(n, bool)
    if not keep.any():
        return np.zeros(v.shape[1]), -np.inf
    x = scale * (k[keep].astype(np.float64) @ q.astype(np.float64))
    top = x.max()
    w = np.exp(x - top)
    return w @ v[keep].astype(np.float64) / w.sum(), top + np.log(w.sum())


def turn(x, positions, freqs, interleaved, mscale=1.0, backward=False):
    """Rotary positions in 64 bits, pair by pair: x [..., N, d], positions [..., N]."""
    y = np.array(x, np.float64)
    half = len(freqs)
    for i, f in enumerate(freqs):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        t = np.asarray(positions, np.float64) * f * (-1 if backward else 1)
        u, w = y[..., a].copy(), y[..., b].copy()
        y[..., a] = mscale * (u * np.cos(t) - w * np.sin(t))
        y[..., b] = mscale * (u * np.sin(t) + w * np.cos(t))
    return y
