"""Paged key-value caches in plain sequential Python / NumPy float64.

Pages: one sequence after the other, one page at a time, from the rules of include/saki_kv.h.
Rotary positions and attention: token by token from their definitions.
"""
import numpy as np

OK, NO_PAGES, TOO_LONG, BAD = 0, 1, 2, 3


class Table:
    """pages [n_seq, max_pages], length, held [n_seq], refs [n_pages]; a page is free iff refs is 0."""

    def __init__(self, n_seq, max_pages, n_pages, page_size):
        self.pages = np.full((n_seq, max_pages), -1, dtype=np.int64)
        self.length = np.zeros(n_seq, dtype=np.int64)
        self.held = np.zeros(n_seq, dtype=np.int64)
        self.refs = np.zeros(n_pages, dtype=np.int64)
        self.page_size = page_size

    def copy(self):
        t = Table(0, 1, 1, self.page_size)
        t.pages, t.length, t.held, t.refs = (x.copy() for x in (self.pages, self.length, self.held, self.refs))
        return t

    def _sound(self, b):
        return 0 <= self.held[b] <= self.pages.shape[1] and 0 <= self.length[b] <= self.held[b] * self.page_size

    def reserve(self, n_new):
        """Returns (status, copies): copies are (source page, new page, slots)."""
        P, (n_seq, width) = self.page_size, self.pages.shape
        status, plan, writers = [OK] * n_seq, {}, {}
        for b in range(n_seq):
            n, L, H = int(n_new[b]), int(self.length[b]), int(self.held[b])
            if n < 0 or not self._sound(b):
                status[b] = BAD
                continue
            if n == 0:
                continue
            need = -(-(L + n) // P)
            if need > width:
                status[b] = TOO_LONG
                continue
            page = None
            if L % P:
                page = int(self.pages[b, L // P])
                if not 0 <= page < self.refs.size:
                    status[b] = BAD
                    continue
                if self.refs[page] > 1:
                    writers.setdefault(page, []).append(b)
                else:
                    page = None
            plan[b] = (page, max(0, need - H))
        for page, seqs in writers.items():
            if len(seqs) == self.refs[page]:
                plan[seqs[-1]] = (None, plan[seqs[-1]][1])
        total = sum((page is not None) + fresh for page, fresh in plan.values())
        free = [int(p) for p in np.nonzero(self.refs == 0)[0]]
        if total > len(free):
            for b in plan:
                status[b] = NO_PAGES
            return status, []
        copies = []
        for b in sorted(plan):
            page, fresh = plan[b]
            if page is not None:
                to = free.pop(0)
                copies.append((page, to, int(self.length[b]) % P))
                self.pages[b, self.length[b] // P] = to
                self.refs[to] = 1
                self.refs[page] -= 1
            for _ in range(fresh):
                to = free.pop(0)
                self.pages[b, self.held[b]] = to
                self.held[b] += 1
                self.refs[to] = 1
        return status, copies

    def commit(self, delta, done=None):
        P, status = self.page_size, []
        for b in range(self.pages.shape[0]):
            to = 0 if done is not None and done[b] else int(self.length[b]) + (0 if delta is None else int(delta[b]))
            if not self._damaged(b) and 0 <= to <= self.held[b] * P:
                keep = -(-to // P)
                for i in range(keep, int(self.held[b])):
                    self.refs[self.pages[b, i]] -= 1
                    self.pages[b, i] = -1
                self.length[b], self.held[b] = to, keep
                status.append(OK)
            else:
                status.append(BAD)
        return status

    def _damaged(self, b):
        return self.length[b] < 0 or not 0 <= self.held[b] <= self.pages.shape[1]

    def fork(self, src, dst):
        status = []
        for i, (s, d) in enumerate(zip(src, dst)):
            n_seq = self.pages.shape[0]
            if not (0 <= s < n_seq and 0 <= d < n_seq) or d in list(src) or d in list(dst)[:i] or \
                    self.length[d] or self.held[d] or not self._sound(s):
                status.append(BAD)
                continue
            n = -(-int(self.length[s]) // self.page_size)
            self.pages[d, :n] = self.pages[s, :n]
            for p in self.pages[s, :n]:
                self.refs[p] += 1
            self.length[d], self.held[d] = self.length[s], n
            status.append(OK)
        return status

    def compact(self):
        """Returns (live pages, moves): moves are (source, destination)."""
        n = int((self.refs > 0).sum())
        holes = [p for p in range(n) if self.refs[p] == 0]
        moving = [p for p in range(n, self.refs.size) if self.refs[p] > 0]
        moves = list(zip(moving, holes))
        for s, d in moves:
            self.refs[d], self.refs[s] = self.refs[s], 0
            self.pages[self.pages == s] = d
        return n, moves


def rope(x, position, freq, rotary_dim, interleaved, amplitude):
    """One head's vector [dim] at a position (freq in turns per position)."""
    y = np.array(x, dtype=np.float64)
    for i in range(rotary_dim // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary_dim // 2)
        turn = float(position) * float(freq[i])
        angle = 2 * np.pi * (turn - np.floor(turn))
        c, s = amplitude * np.cos(angle), amplitude * np.sin(angle)
        y[a], y[b] = x[a] * c - x[b] * s, x[b] * c + x[a] * s
    return y


def attention(q, k, v, positions, scale, window=0, sinks=0):
    """q [n, heads, d] at `positions`, k and v [length, kv_heads, d] -> out [n, heads, d], lse [n, heads], in 64
    bits.  Hidden tokens are left out of the sums, whatever they hold; a token with no score above -infinity
    gets 0 and -infinity."""
    n, heads, d = q.shape
    group = heads // k.shape[1]
    out, lse = np.zeros((n, heads, d)), np.full((n, heads), -np.inf)
    j = np.arange(k.shape[0])
    for i in range(n):
        seen = j <= positions[i]
        if window > 0:
            seen &= (j > positions[i] - window) | (j < sinks)
        for h in range(heads):
            kk, vv = k[seen, h // group].astype(np.float64), v[seen, h // group].astype(np.float64)
            with np.errstate(invalid="ignore", over="ignore"):
                s = scale * (kk @ q[i, h].astype(np.float64))
                if s.size == 0 or (s == -np.inf).all():
                    continue
                top = s.max()
                w = np.exp(s - top)
                out[i, h] = (w[:, None] * vv).sum(0) / w.sum()
                lse[i, h] = top + np.log(w.sum())
    return out, lse
