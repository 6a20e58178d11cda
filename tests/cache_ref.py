"""Plain forms of the paged cache's operations and of attention, for the tests:
numpy, one row and one token at a time, float64."""
import numpy as np


class Cache:
    """A pool as keys and values [layer][page][kv head][slot][dh] (the pool's layout is undone here)."""

    def __init__(self, pool):
        pool = np.asarray(pool)
        self.L, self.n, _, self.hkv, self.P, self.dh = pool.shape
        self.k = pool[:, :, 0].copy()
        v = pool[:, :, 1].reshape(self.L, self.n, self.hkv, self.P // 16, self.dh, 16)
        self.v = v.transpose(0, 1, 2, 3, 5, 4).reshape(self.k.shape).copy()

    def pool(self):
        v = self.v.reshape(self.L, self.n, self.hkv, self.P // 16, 16, self.dh).transpose(0, 1, 2, 3, 5, 4)
        return np.stack([self.k, v.reshape(self.k.shape)], axis=2)

    def there(self, page):
        return 0 <= page < self.n

    def fork(self, table, lens, parent, new):
        """(table, lens, info); copies pages."""
        rows_in, width = table.shape
        parent = np.arange(rows_in) if parent is None else parent
        rows, cap = len(parent), width * self.P
        new = np.zeros(rows, np.int64) if new is None else new
        out = np.full((rows, width), -1, np.int32)
        length = np.zeros(rows, np.int32)
        shares, writers, todo = set(), {}, []
        for r in range(rows):
            p = int(parent[r])
            have = min(max(int(lens[p]), 0), cap) if 0 <= p < rows_in else 0
            length[r] = min(max(have + int(new[r]), 0), cap)
            kept = min(have, int(length[r]))
            old = -(-kept // self.P)
            whole = kept // self.P if length[r] > kept else old
            entry = [int(table[p, c]) if self.there(int(table[p, c])) else -1 for c in range(old)]
            shares |= {e for e in entry[:whole] if e >= 0}
            if old > whole and entry[whole] >= 0:
                writers.setdefault(entry[whole], r)
            todo.append((entry, whole, old, -(-int(length[r]) // self.P)))
        live = shares | set(writers)
        free = [p for p in range(self.n) if p not in live]
        total, copies = 0, []
        for r, (entry, whole, old, pages) in enumerate(todo):
            take = []
            if old > whole and entry[whole] >= 0 and (entry[whole] in shares or writers[entry[whole]] != r):
                take.append((whole, entry[whole]))
            take += [(c, -1) for c in range(old, pages)]
            for c, e in enumerate(entry):
                out[r, c] = e
            for c, source in take:
                out[r, c] = free[total] if total < len(free) else -1
                if source >= 0:
                    copies.append((source, int(out[r, c])))
                total += 1
        if total <= len(free):
            for a, b in copies:
                self.k[:, b], self.v[:, b] = self.k[:, a], self.v[:, a]
        return out, length, np.array([max(len(free) - total, 0), max(total - len(free), 0)], np.int32)

    def compact(self, table, lens):
        rows, width = table.shape
        used = [[c for c in range(min(-(-max(int(lens[r]), 0) // self.P), width)) if self.there(int(table[r, c]))]
                for r in range(rows)]
        live = sorted({int(table[r, c]) for r in range(rows) for c in used[r]})
        holes = [p for p in range(len(live)) if p not in set(live)]
        high = [p for p in live if p >= len(live)]
        to = {p: p for p in live}
        for a, b in zip(high, holes):
            to[a] = b
            self.k[:, b], self.v[:, b] = self.k[:, a], self.v[:, a]
        out = np.full((rows, width), -1, np.int32)
        for r in range(rows):
            for c in used[r]:
                out[r, c] = to[int(table[r, c])]
        return out, np.array([len(live), len(high)], np.int32)

    def write(self, layer, table, lens, k, v, start):
        for r in range(len(lens)):
            a, b = int(start[r]), int(start[r + 1])
            length = min(max(int(lens[r]), 0), table.shape[1] * self.P)
            for i in range(a, b):
                t = length - (b - a) + (i - a)
                if t >= 0 and self.there(int(table[r, t // self.P])):
                    self.k[layer, table[r, t // self.P], :, t % self.P] = k[i].reshape(self.hkv, self.dh)
                    self.v[layer, table[r, t // self.P], :, t % self.P] = v[i].reshape(self.hkv, self.dh)

    def row(self, layer, table_row, length):
        """Keys and values [length][kv head][dh] of a row, and which of them are there."""
        t = np.arange(length)
        page = np.asarray(table_row)[t // self.P].astype(np.int64)
        ok = (page >= 0) & (page < self.n)
        page = np.where(ok, page, 0)
        return self.k[layer][page, :, t % self.P], self.v[layer][page, :, t % self.P], ok


def attend(q, k, v, seen, c_qk, c_pv):
    """q [n][h][dh] over k, v [S][kv head][dh]; seen bool [n][S]: float64 [n][h][dh], 0 where nothing is seen, and how far
    a computed value may be from it, [n][h][1] (see tolerance)."""
    n, h, dh = q.shape
    k, v = (np.repeat(np.asarray(a, np.float64), h // a.shape[1], axis=1) for a in (k, v))
    out, tol = np.zeros((n, h, dh)), np.zeros((n, h, 1))
    for i in range(n):
        at = np.flatnonzero(seen[i])
        if len(at) == 0:
            continue
        s = np.einsum("hd,shd->hs", q[i].astype(np.float64), k[at]) * float(c_qk)
        p = np.exp(s - s.max(axis=1, keepdims=True))
        total = p.sum(axis=1, keepdims=True)
        out[i] = np.einsum("hs,shd->hd", p / total, v[at]) * float(c_pv)
        tol[i] = tolerance(len(at) / total, c_pv)
    return out, tol


def paged(cache, layer, table, lens, q, start, h, c_qk, c_pv, causal=True):
    """Attention of a ragged chunk over a cache, as attend, [n][h * dh] both."""
    out, tol = np.full((q.shape[0], h, cache.dh), np.nan), np.zeros((q.shape[0], h, cache.dh))
    cap = table.shape[1] * cache.P
    for r in range(len(lens)):
        a, b = int(start[r]), int(start[r + 1])
        length = min(max(int(lens[r]), 0), cap)
        k, v, ok = cache.row(layer, table[r], length)
        last = length - (b - a) + np.arange(b - a) if causal else np.full(b - a, length - 1)
        seen = (np.arange(length)[None, :] <= last[:, None]) & ok[None, :]
        out[a:b], tol[a:b] = attend(q[a:b].reshape(b - a, h, cache.dh), k, v, seen, c_qk, c_pv)
    return out.reshape(q.shape[0], -1), tol.reshape(q.shape[0], -1)


def tolerance(share, c_pv):
    """How far an attention output may be from float64; share: keys over the sum of the weights, the largest one being 1.
    A weight is a fixed-point number of unit 1 / 0x7F7F7F of the largest weight so far, which is at most the largest: half
    a unit for each key, times |v| <= 128 in the numerator and as much again through the denominator, over the sum.  The
    exponential: its argument rounds by 2^-24 of at most 24 (smaller weights vanish), times ln 2, plus 2^-23 for the
    exponential itself and 2^-24 for c_qk: 1.2e-6 of each weight, in the numerator and the denominator; the sums, the
    joins and the division in fp32 are 8 roundings more."""
    return abs(c_pv) * 128.0 * (share / 0x7F7F7F + 2.4e-6 + 8 * 2.0 ** -24)


def check_codes(got, ref, tol):
    """int8 codes equal to the rounded float64 values, except where these are within tol of a rounding border."""
    want = np.clip(np.rint(ref), -127, 127)
    near = np.abs(ref - np.floor(ref) - 0.5) <= tol
    assert np.array_equal(got[~near], want[~near])
    assert np.all(np.abs(got - want) <= 1)
    assert near.mean() <= 0.5  # (a share of 2 tol is expected; the other codes are held exactly)
