"""Plain references of the paged cache: the pages as Python lists, attention in 64 bits a sequence at a time."""
import math

import numpy as np


class Pages:
    """The cache's metadata and, as one number per token and layer, its contents."""

    def __init__(self, n_pages, page, max_seqs, max_pages):
        self.P, self.max_pages = page, max_pages
        self.rows = [[] for _ in range(max_seqs)]
        self.length = [0] * max_seqs
        self.ref = [0] * n_pages
        self.data = np.zeros((n_pages, page), np.int64)
        self.refused = 0  # most negative code

    def _code(self, c):
        self.refused = min(self.refused, c)

    def _named(self, seqs):
        return {s for s in seqs if list(seqs).count(s) > 1}

    def _ok(self, s, twice):
        return 0 <= s < len(self.rows) and s not in twice

    def extend(self, seqs, cu, n_new):
        twice, todo, need = self._named(seqs), [], 0
        if any(not 0 <= a <= b <= n_new for a, b in zip(cu, cu[1:])):  # as a whole
            self._code(-1)
            return [-1] * n_new
        for i, s in enumerate(seqs):
            a, b = cu[i], cu[i + 1]
            if not self._ok(s, twice) or not 0 <= a <= b <= n_new or self.length[s] + b - a > self.max_pages * self.P:
                self._code(-1)
                continue
            L, new = self.length[s], b - a
            cow = int(new > 0 and L % self.P != 0 and self.ref[self.rows[s][-1]] > 1)
            k = -(-(L + new) // self.P) - len(self.rows[s]) + cow
            todo.append((i, s, a, new, cow, k))
            need += k
        slots = [-1] * n_new
        free = [p for p, r in enumerate(self.ref) if r == 0]
        if need > len(free):
            self._code(-6)
            return slots
        olds = [(s, self.rows[s][-1]) for _, s, _, _, cow, _ in todo if cow]
        for i, s, a, new, cow, k in todo:
            got, free = free[:k], free[k:]
            if cow:
                old = self.rows[s].pop()
                self.ref[old] -= 1
                self.data[got[0]] = self.data[old]
            self.rows[s] += got
            for p in got:
                self.ref[p] = 1
            for t in range(new):
                pos = self.length[s] + t
                slots[a + t] = self.rows[s][pos // self.P] * self.P + pos % self.P
            self.length[s] += new
        assert len(olds) == sum(t[4] for t in todo)
        return slots

    def write(self, slots, values):
        for x, v in zip(slots, values):
            if 0 <= x < self.data.size:
                self.data[x // self.P, x % self.P] = v

    def free(self, seqs, keep=None):
        twice = self._named(seqs)
        for i, s in enumerate(seqs):
            want = 0 if keep is None else keep[i]
            if not self._ok(s, twice) or want < 0:
                self._code(-1)
                continue
            left = min(want, self.length[s])
            for p in self.rows[s][-(-left // self.P):]:
                self.ref[p] -= 1
            self.rows[s] = self.rows[s][: -(-left // self.P)]
            self.length[s] = left

    def fork(self, src, dst, tokens=None):
        twice = self._named(dst)
        for i, (s, d) in enumerate(zip(src, dst)):
            ok = self._ok(d, twice) and 0 <= s < len(self.rows) and s not in dst and self.length[d] == 0
            n = (self.length[s] if tokens is None else tokens[i]) if ok else 0
            if not ok or not 0 <= n <= self.length[s]:
                self._code(-1)
                continue
            self.rows[d] = self.rows[s][: -(-n // self.P)]
            for p in self.rows[d]:
                self.ref[p] += 1
            self.length[d] = n

    def copy(self, src, dst):
        twice, todo, need = self._named(dst), [], 0
        for s, d in zip(src, dst):
            if not self._ok(d, twice) or not 0 <= s < len(self.rows) or s in dst or self.length[d] != 0:
                self._code(-1)
                continue
            todo.append((s, d))
            need += len(self.rows[s])
        free = [p for p, r in enumerate(self.ref) if r == 0]
        if need > len(free):
            self._code(-6)
            return
        for s, d in todo:
            k = len(self.rows[s])
            got, free = free[:k], free[k:]
            self.data[got] = self.data[self.rows[s]]
            for p in got:
                self.ref[p] = 1
            self.rows[d], self.length[d] = got, self.length[s]

    def compact(self):
        used = [p for p, r in enumerate(self.ref) if r > 0]
        n = len(used)
        holes = [p for p in range(n) if self.ref[p] == 0]
        to = [p if r > 0 else -1 for p, r in enumerate(self.ref)]
        for a, b in zip([p for p in used if p >= n], holes):
            to[a] = b
            self.data[b], self.ref[b], self.ref[a] = self.data[a], self.ref[a], 0
        self.rows = [[to[p] for p in row] for row in self.rows]
        return to

    def table(self):
        t = np.full((len(self.rows), self.max_pages), -1, np.int32)
        for i, row in enumerate(self.rows):
            t[i, : len(row)] = row
        return t


def attention(q, k, v, scale):
    """Queries [t, Hq, D] that are the last t of the tokens of keys and values [H, n, D]; all float64 arrays.  Returns
    the result, log of the sum of exponentials, and sum_j p_j |v_j| (the scale of what rounding p does)."""
    t, hq, D = q.shape
    H, n, _ = k.shape
    out, lse, mag = np.zeros((t, hq, D)), np.full((t, hq), -math.inf), np.zeros((t, hq, D))
    for i in range(t):
        see = n - t + i + 1
        if see <= 0:
            continue
        for h in range(hq):
            kh, vh = k[h // (hq // H), :see], v[h // (hq // H), :see]
            s = kh @ q[i, h] * scale
            top = s.max()
            w = np.exp(s - top)
            z = w.sum()
            out[i, h], mag[i, h], lse[i, h] = w @ vh / z, w @ np.abs(vh) / z, top + math.log(z)
    return out, lse, mag
