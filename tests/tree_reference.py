"""Plain definitions, in 64 bits and on lists, of the calls on trees and paged caches: what their tests compare with."""
import math

import numpy as np


def ancestors(parents):
    """Per node: the set of itself and its ancestors, empty for a node out of use."""
    out = []
    for i, p in enumerate(parents):
        out.append({i} if p == -1 else (out[p] | {i} if 0 <= p < i and out[p] else set()))
    return out


def visible(parents, length, window, prefix):
    """[n, length + n] truth values: which cached positions and nodes a node sees."""
    above = ancestors(parents)
    n = len(parents)
    see = np.zeros((n, length + n), dtype=bool)
    depth = [len(a) - 1 for a in above]
    for i in range(n):
        if not above[i]:
            continue
        for s in range(length):
            see[i, s] = window == 0 or s < prefix or length + depth[i] - s < window
        for j in above[i]:
            see[i, length + j] = window == 0 or depth[i] - depth[j] < window
    return see


def attention(q, k, v, see, scale, unit):
    """q [n, H, dh], k and v [Hkv, keys, dh] float64: out, lse and bounds on the errors of a kernel that keeps scores, softmax and
    sums in float32 and rounds p and the output to a type whose rounding is off by at most `unit`, relatively."""
    n, H, dh = q.shape
    G = H // k.shape[0]
    out, lse = np.zeros((n, H, dh)), np.full((n, H), -np.inf)
    tol_out, tol_lse = np.zeros((n, H, dh)), np.zeros((n, H))
    for h in range(H):
        for i in range(n):
            at = np.nonzero(see[i])[0]
            if len(at) == 0:
                continue
            kk, vv = k[h // G][at], v[h // G][at]
            z = scale * (kk @ q[i, h])
            m = z.max()
            e = np.exp(z - m)
            p = e / e.sum()
            out[i, h], lse[i, h] = p @ vv, m + math.log(e.sum())
            # a score: dh products summed in float32, the scale, the exponent's reduction; a sum of len(at) terms
            score = (dh + 4) * 2.0 ** -24 * scale * (np.abs(kk) @ np.abs(q[i, h])).max() + 4 * 2.0 ** -24 * np.abs(z).max() + 2.0 ** -21
            sums = (len(at) + 8) * 2.0 ** -24
            tol_out[i, h] = (unit + 2 * (score + sums)) * (p @ np.abs(vv)) + unit * np.abs(out[i, h]) * (1 + unit) + 1e-7
            tol_lse[i, h] = score + sums + 4 * 2.0 ** -24 * abs(lse[i, h])
    return out, lse, tol_out, tol_lse


def accept(tokens, parents, predicted):
    """The path and the token behind it."""
    if not parents or parents[0] != -1:
        return [], -1
    path = [0]
    while True:
        cur = path[-1]
        child = [j for j in range(cur + 1, len(parents)) if parents[j] == cur and tokens[j] == predicted[cur]]
        if not child:
            return path, predicted[cur]
        path.append(child[0])


class Pages:
    """A pool on lists.  data[(layer, kv)] is [pages, heads, slots, dim]; of the errors the lowest code stays in `status`."""

    OK, INVALID, STATE, CAPACITY = 0, -1, -2, -3

    def __init__(self, n_pages, page, max_seqs, max_pages, data):
        self.n_pages, self.page, self.max_seqs, self.max_pages, self.data = n_pages, page, max_seqs, max_pages, data
        self.tables, self.lens, self.status = [[] for _ in range(max_seqs)], [0] * max_seqs, 0

    def fail(self, code):
        self.status = min(self.status, code)

    def refs(self):
        r = [0] * self.n_pages
        for t in self.tables:
            for p in t:
                r[p] += 1
        return r

    def table(self):
        return [t + [-1] * (self.max_pages - len(t)) for t in self.tables]

    def _ids(self, seqs):
        seen = set()
        for e, s in enumerate(seqs):
            if s < 0:
                continue
            if s >= self.max_seqs or s in seen:
                self.fail(self.INVALID)
                continue
            seen.add(s)
            yield e, s

    def fork(self, src, dst):
        taken = []
        for e, (s, d) in enumerate(zip(src, dst)):
            if s < 0 or d < 0:
                continue
            others = [b for a, b in zip(src, dst) if a >= 0]
            if s >= self.max_seqs or d >= self.max_seqs or s in others or d in [b for a, b in zip(src[:e], dst[:e]) if a >= 0]:
                self.fail(self.INVALID)
                continue
            taken.append((s, d))
        for s, d in taken:
            self.tables[d] = self.tables[s][:-(-self.lens[s] // self.page)]
            self.lens[d] = self.lens[s]

    def truncate(self, seqs, lens):
        for e, s in self._ids(seqs):
            self.lens[s] = min(self.lens[s], max(lens[e], 0))
            del self.tables[s][-(-self.lens[s] // self.page):]

    def reserve(self, seqs, grow):
        for e, s in self._ids(seqs):
            if grow[e] <= 0:
                continue
            n, t, refs = self.lens[s], self.tables[s], self.refs()
            need = -(-(n + grow[e]) // self.page)
            copy = n % self.page != 0 and refs[t[n // self.page]] > 1
            free = [p for p in range(self.n_pages) if refs[p] == 0]
            want = max(0, need - len(t)) + copy
            if need > self.max_pages or want > len(free):
                self.fail(self.CAPACITY)
                continue
            if copy:
                new, old = free.pop(0), t[n // self.page]
                for x in self.data.values():
                    x[new][:, :n % self.page] = x[old][:, :n % self.page]
                t[n // self.page] = new
            while len(t) < need:
                t.append(free.pop(0))

    def append(self, seqs, row_off, rows, path=None, n_acc=None, max_rows=None):
        """rows[(layer, kv)] [rows, heads, dim]"""
        for e, s in self._ids(seqs):
            own = row_off[e + 1] - row_off[e]
            take = list(range(own)) if path is None else list(path[e][:max(n_acc[e], 0)])
            if (max_rows is not None and len(take) > max_rows) or (path is not None and n_acc[e] > len(path[e])) or any(r < 0 or r >= own for r in take):
                self.fail(self.INVALID)
                continue
            n, t, refs = self.lens[s], self.tables[s], self.refs()
            pages = range(n // self.page, -(-(n + len(take)) // self.page)) if take else []
            if any(j >= len(t) or refs[t[j]] != 1 for j in pages):
                self.fail(self.STATE)
                continue
            for j, r in enumerate(take):
                at = n + j
                for key, x in self.data.items():
                    x[t[at // self.page]][:, at % self.page] = rows[key][row_off[e] + r]
            self.lens[s] += len(take)

    def compact(self):
        refs = self.refs()
        used = [p for p in range(self.n_pages) if refs[p] > 0]
        holes = [p for p in range(len(used)) if refs[p] == 0]
        goes = dict(zip([p for p in used if p >= len(used)], holes))
        for old, new in goes.items():
            for x in self.data.values():
                x[new] = x[old]
        self.tables = [[goes.get(p, p) for p in t] for t in self.tables]
        return len(used)
