"""Plain fp64 / integer implementations of the 8-bit paged cache and of its pages'
bookkeeping, one request and one page at a time, for the tests."""
import numpy as np


def e4m3_values():
    """The value of each of the 256 codes."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[c] = np.nan if c & 127 == 127 else (-x if c & 128 else x)
    return v


VALUES = e4m3_values()


def e4m3_round(x):
    """The nearest e4m3 value, ties to even, at most 448; NaN for what is not finite."""
    x = np.asarray(x, np.float64)
    ok = np.isfinite(x)
    a = np.where(ok, np.abs(x), 0.0)
    step = 2.0 ** (np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
    return np.where(ok, np.copysign(np.minimum(np.round(a / step) * step, 448.0), x), np.nan)


def pow2_scale(amax):
    """The smallest power of two s with amax <= 448 s, exponent in [-100, 120]; 0 for 0."""
    if not amax > 0:
        return 0.0
    k = -160
    while 448 * 2.0 ** k < amax:
        k += 1
    return 2.0 ** min(max(k, -100), 120)


def pow2_ceil(s):
    s = abs(float(s))
    if not (0 < s < np.inf):
        return 0.0
    return 2.0 ** min(max(int(np.ceil(np.log2(s))), -100), 120)


def append_block(old_codes, s_old, new):
    """One block of one head: values of its earlier tokens [n_old, D] and their scale, new rows [n, D] ->
    (values of all tokens' codes, scale)."""
    fine = np.abs(new[np.isfinite(new)])
    s_old = float(s_old) if len(old_codes) else 0.0
    s = max(pow2_scale(fine.max() if fine.size else 0.0), pow2_ceil(s_old)) or 1.0
    if len(old_codes) and s_old != s:
        old_codes = e4m3_round(old_codes * (s_old / s))
    return np.concatenate([old_codes, e4m3_round(new / s)]), s


def attention(q, k, v, kv, ql, group, scale):
    """q [ql, Hq, D], k [Hkv, kv, D], v [Hkv, kv, Dv] -> out [ql, Hq, Dv], lse [ql, Hq]."""
    out, lse = np.zeros((ql, q.shape[1], v.shape[2])), np.zeros((ql, q.shape[1]))
    for h in range(q.shape[1]):
        for t in range(ql):
            n = kv - ql + t + 1
            z = scale * (k[h // group, :n] @ q[t, h])
            m = z.max()
            p = np.exp(z - m)
            out[t, h] = (p / p.sum()) @ v[h // group, :n]
            lse[t, h] = m + np.log(p.sum())
    return out, lse


class Pages:
    """Block tables, lengths, holders' counts and page contents, changed in place."""

    def __init__(self, table, kv_len, page, num_pages, contents):
        self.table, self.kv, self.page, self.n = table.copy(), kv_len.copy(), page, num_pages
        self.contents = [c.copy() for c in contents]  # [num_pages, ...]
        self.ref = np.zeros(num_pages, np.int32)
        for r in range(len(self.kv)):
            for i in range(self.held(r)):
                self.ref[self.table[r, i]] += 1

    def held(self, r, tokens=None):
        t = self.kv[r] if tokens is None else tokens
        return -(-int(t) // self.page)

    def fork(self, parent, child, length=None):
        before, seen = self.kv.copy(), set()
        R = len(self.kv)
        for i, (p, c) in enumerate(zip(parent, child)):
            first = c not in seen
            seen.add(c)
            if not (0 <= p < R and 0 <= c < R) or p == c or before[c] != 0 or not first:
                continue
            t = before[p] if length is None else min(before[p], max(length[i], 0))
            for j in range(self.held(None, t)):
                self.table[c, j] = self.table[p, j]
                self.ref[self.table[c, j]] += 1
            self.kv[c] = t

    def reserve(self, q_len):
        R, most = len(self.kv), self.table.shape[1] * self.page
        ok = [0 <= self.kv[r] and q_len[r] >= 0 and self.kv[r] + q_len[r] <= most for r in range(R)]
        partial = {}  # request -> its shared, partly filled page
        for r in range(R):
            if ok[r] and q_len[r] > 0 and self.kv[r] % self.page:
                pg = self.table[r, self.kv[r] // self.page]
                if self.ref[pg] > 1:
                    partial[r] = pg
        growers = {}
        for r, pg in partial.items():
            growers.setdefault(pg, []).append(r)
        keeps = {g[-1] for pg, g in growers.items() if len(g) == self.ref[pg]}
        free = [p for p in range(self.n) if self.ref[p] == 0]
        step, wanted, taken = np.zeros(R, np.int32), 0, 0
        drops = []
        for r in range(R):
            if not ok[r]:
                continue
            copy = r in partial and r not in keeps
            need = self.held(None, self.kv[r] + q_len[r]) - self.held(r) + copy
            wanted += need
            if not (wanted <= len(free) or (need == 0 and r not in keeps)):
                continue
            col = self.held(r) - copy
            for i in range(need):
                pg = free[taken]
                taken += 1
                if copy and i == 0:
                    for c in self.contents:
                        c[pg] = c[partial[r]]
                    drops.append(partial[r])
                self.table[r, col + i] = pg
                self.ref[pg] = 1
            step[r] = self.kv[r] + q_len[r]
        for pg in drops:
            self.ref[pg] -= 1
        return step

    def _drop(self, r, now, keep):
        for i in range(self.held(None, keep), self.held(None, now)):
            self.ref[self.table[r, i]] -= 1
        self.kv[r] = keep

    def commit(self, step, q_len, accepted=None):
        for r in range(len(self.kv)):
            if step[r] > 0:
                kept = q_len[r] if accepted is None else min(max(accepted[r] + 1, 0), q_len[r])
                self._drop(r, step[r], step[r] - q_len[r] + kept)

    def trim(self, new_len):
        for r in range(len(self.kv)):
            self._drop(r, self.kv[r], min(self.kv[r], max(new_len[r], 0)))

    def compact(self):
        used = int((self.ref > 0).sum())
        to = {s: d for s, d in zip([p for p in range(used, self.n) if self.ref[p] > 0],
                                   [p for p in range(used) if self.ref[p] == 0])}
        for s, d in to.items():
            self.ref[d], self.ref[s] = self.ref[s], 0
            for c in self.contents:
                c[d] = c[s]
        for r in range(len(self.kv)):
            for i in range(self.held(r)):
                self.table[r, i] = to.get(self.table[r, i], self.table[r, i])
        return used
