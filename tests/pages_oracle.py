"""The paged cache of include/lessdec.h written out in numpy and float64: what the GPU tests compare with.  Plain loops over slots,
pages and tokens; nothing here is taken from the kernels."""
import numpy as np

BLOCK = 16


def code_values():
    """What the 256 e4m3 codes stand for: sign, four bits of exponent with bias 7, three of mantissa; 0x7f and 0xff are NaN."""
    v = np.zeros(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        x = (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        v[c] = np.nan if c & 127 == 127 else -x if c & 128 else x
    return v


VALUES = code_values()
_POSITIVE = VALUES[:127]
_HALVES = (_POSITIVE[1:] + _POSITIVE[:-1]) / 2


def nearest(x, e):
    """The value of the code nearest to x / 2^e, ties to the even code, times 2^e; NaN where x is not finite."""
    y = np.minimum(np.abs(np.where(np.isfinite(x), x, 0)) * 2.0 ** -e, 448.0)
    below = np.searchsorted(_HALVES, y, side="left")           # y on a half: the code below
    tie = (below < len(_HALVES)) & (y == _HALVES[np.minimum(below, len(_HALVES) - 1)]) & (below % 2 == 1)
    r = _POSITIVE[below + tie] * np.where(np.signbit(x), -1.0, 1.0) * 2.0 ** e
    return np.where(np.isfinite(x), r, np.nan)


def exponent(x):
    top = np.max(np.abs(x[np.isfinite(x)]), initial=0.0)
    e = -40
    while top > 448.0 * 2.0 ** e and e < 40:
        e += 1
    return e


class Cache:
    def __init__(self, slots, pages, page, table_len, heads, dim, layers=1, group=1, sinks=0, window=0, scale=None):
        self.slots, self.pages, self.page, self.wide, self.heads, self.dim = slots, pages, page, table_len, heads, dim
        self.layers, self.group, self.sinks, self.window = layers, group, sinks, window
        self.scale = dim ** -0.5 if scale is None else scale
        self.table = np.full((slots, table_len), -1)
        self.length, self.refs = np.zeros(slots, int), np.zeros(pages, int)
        self.kv = np.zeros((2, layers, pages, heads, page, dim))
        self.exps = np.zeros((2, layers, pages, heads, page // BLOCK), int)

    # -- bookkeeping
    def reserve(self, n_new):
        granted, plan, stopped = np.zeros(self.slots, int), [], False
        wants = [n > 0 and self.length[s] + n <= self.wide * self.page for s, n in enumerate(n_new)]
        for s in range(self.slots):
            if wants[s] and self.window:
                for i in range(self.wide):
                    tokens = np.arange(i * self.page, (i + 1) * self.page)
                    if self.table[s, i] >= 0 and np.all((tokens <= self.length[s] - self.window) & (tokens >= self.sinks)):
                        self.refs[self.table[s, i]] -= 1
                        self.table[s, i] = -1
        for s in range(self.slots):
            if not wants[s] or stopped:
                continue
            n, part = self.length[s] + n_new[s], self.length[s] // self.page
            entries = list(range(-(-self.length[s] // self.page), -(-n // self.page)))
            old = self.table[s, part] if self.length[s] % self.page else -1
            if old >= 0 and self.refs[old] > 1:
                entries = [part] + entries
            free = np.flatnonzero(self.refs == 0)
            if len(entries) > len(free):
                stopped = True
                continue
            for i, p in zip(entries, free):
                if i == part and old >= 0:
                    self.refs[old] -= 1
                    plan.append((old, p))
                self.table[s, i] = p
                self.refs[p] = 1
            granted[s], self.length[s] = n_new[s], n
        return granted, plan

    def select(self, source):
        table, length = self.table.copy(), self.length.copy()
        for s, f in enumerate(source):
            if f == -1:
                self.table[s], self.length[s] = -1, 0
            elif 0 <= f < self.slots:
                self.table[s], self.length[s] = table[f], length[f]
        self.refs[:] = 0
        np.add.at(self.refs, self.table[self.table >= 0], 1)

    def compact(self):
        used = int((self.refs > 0).sum())
        plan = list(zip([p for p in range(used, self.pages) if self.refs[p]], [p for p in range(used) if not self.refs[p]]))
        for a, b in plan:
            self.table[self.table == a] = b
            self.refs[b], self.refs[a] = self.refs[a], 0
        return plan

    def copy(self, plan):
        for a, b in plan:
            self.kv[:, :, b], self.exps[:, :, b] = self.kv[:, :, a], self.exps[:, :, a]

    # -- tokens
    def place(self, s, j):
        """(page, token in it) of a slot's token, or None."""
        p = self.table[s, j // self.page]
        return (p, j % self.page) if 0 <= p < self.pages else None

    def append(self, layer, k, v, start):
        for s in range(self.slots):
            count = start[s + 1] - start[s]
            begin = self.length[s] - count
            for j0 in range(max(0, begin) // BLOCK * BLOCK, self.length[s] if count else 0, BLOCK):
                here = self.place(s, j0)
                if here is None:
                    continue
                p, t0 = here
                new = np.arange(max(j0, begin), min(j0 + BLOCK, self.length[s]))
                off = max(0, begin - j0)
                for which, rows in ((0, k), (1, v)):
                    for h in range(self.heads):
                        x = rows[start[s] + new - begin, h].astype(np.float64)
                        e, block = exponent(x), self.kv[which, layer, p, h, t0:t0 + BLOCK]
                        if off:
                            e = max(e, self.exps[which, layer, p, h, t0 // BLOCK])
                            block[:off] = nearest(block[:off], e)
                        block[new - j0] = nearest(x, e)
                        self.exps[which, layer, p, h, t0 // BLOCK] = e

    def tokens(self, layer, s):
        """[2, heads, length, dim], zeros where the slot has no page, and which tokens are there."""
        n = self.length[s]
        x, there = np.zeros((2, self.heads, n, self.dim)), np.zeros(n, bool)
        for j in range(n):
            here = self.place(s, j)
            if here is not None:
                x[:, :, j], there[j] = self.kv[:, layer, here[0], :, here[1]], True
        return x, there

    def read(self, layer, slots, first, count, most):
        out = np.zeros((2, len(slots), self.heads, count, self.dim))
        for i, s in enumerate(slots):
            if not 0 <= s < self.slots:
                continue
            x, _ = self.tokens(layer, s)
            at = first if first >= 0 else self.length[s] + first
            for n in range(count):
                if 0 <= at + n < self.length[s]:
                    out[:, i, :, n] = x[:, :, at + n]
        return np.where(np.isnan(out), out, np.clip(out, -most, most))

    def attend(self, layer, q, start, half_step):
        """out and lse in float64, and how far a result may be off: half a step of the output's type on out; on every weight p_j, of
        which out = sum p_j v_j, half a step of fp16 (2^-11), fp32 sums of D products in a score, on numerator and denominator
        alike, fp32 sums over the tokens and a little for the exponentials; and 2^-25 of fp16's smallest steps beside a largest
        weight of 2^6 or more."""
        rows = q.shape[0]
        out, lse = np.zeros((rows, self.heads * self.group, self.dim)), np.full((rows, self.heads * self.group), -np.inf)
        tol, lse_tol = np.zeros_like(out), np.zeros_like(lse)
        for s in range(self.slots):
            count = start[s + 1] - start[s]
            if count == 0:
                continue
            x, there = self.tokens(layer, s)
            j = np.arange(self.length[s])
            block_e = np.zeros((self.heads, self.length[s]))
            for t in j[there]:
                p, at = self.place(s, t)
                block_e[:, t] = self.exps[1, layer, p, :, at // BLOCK]
            for i in range(count):
                p = self.length[s] - count + i
                seen = there & (j <= p)
                if self.window:
                    seen &= (j > p - self.window) | (j < self.sinks)
                if not seen.any():
                    continue
                for hq in range(self.heads * self.group):
                    h = hq // self.group
                    row = q[start[s] + i, hq].astype(np.float64)
                    k, v = x[0, h, seen], x[1, h, seen]
                    with np.errstate(all="ignore"):
                        score = k @ row * self.scale
                        top = score.max() if not np.isnan(score).any() else np.nan
                        if top == -np.inf:
                            continue
                        w = np.exp(score - top)
                        total = w.sum()
                        w /= total
                        y = (w[:, None] * v).sum(0)
                        size = np.abs(k) @ np.abs(row) * self.scale
                        u = 2.0 ** -24
                        delta = (self.dim + 8) * u * size.max()
                        spread = (w[:, None] * np.abs(v)).sum(0)
                        smallest = 448 * np.max(w * 2.0 ** block_e[h, seen]) * len(w) * 2.0 ** -31
                        r = start[s] + i
                        out[r, hq], lse[r, hq] = y, top + np.log(total)
                        tol[r, hq] = half_step * np.abs(y) + spread * (2.0 ** -11 + 2 * delta + (2 * len(w) + 64) * u) + smallest
                        lse_tol[r, hq] = delta + (len(w) + 64) * u + 8 * u * np.abs(lse[r, hq])
        return out, lse, tol, lse_tol
