"""Plain numpy forms of the operators around a drafting round: the paged cache
(sequence by sequence, page by page), causal attention over it, verification
from given probabilities, forks of sequences, rows held in 8 or 4 bits, and log
probabilities of given tokens. fp64 throughout."""
from __future__ import annotations

import numpy as np

OK, ERANGE, EPAGES = 0, -1, -2


class Cache:
    """K and V rows in natural order, [layers][n_pages][hkv][page][d] fp64."""

    def __init__(self, layers, hkv, d, page, n_pages, batch, max_pages):
        self.page, self.n_pages, self.batch, self.max_pages = page, n_pages, batch, max_pages
        self.K = np.zeros((layers, n_pages, hkv, page, d))
        self.V = np.zeros((layers, n_pages, hkv, page, d))
        self.table = [[] for _ in range(batch)]
        self.rows, self.open, self.refs = [0] * batch, [0] * batch, [0] * n_pages
        self.flags = set()

    def _need(self, b, n):
        """Pages that n more rows of sequence b take, and the shared page that is
        copied first (or None)."""
        if n == 0:
            return 0, None
        have = len(self.table[b])
        total = -(-(self.rows[b] + n) // self.page)
        if self.rows[b] % self.page and self.refs[self.table[b][-1]] > 1:
            return total - have + 1, self.table[b][-1]
        return total - have, None

    def reserve(self, n_new, max_new):
        free = [p for p in range(self.n_pages) if self.refs[p] == 0]
        plans = []
        for b in range(self.batch):
            n = int(n_new[b])
            if not 0 <= n <= max_new:
                self.flags.add(ERANGE)
                n = 0
            elif self.rows[b] + n > self.max_pages * self.page:
                self.flags.add(EPAGES)
                n = 0
            plans.append((n,) + self._need(b, n))
        wanted = 0
        for b, (n, need, shared) in enumerate(plans):
            at, wanted = wanted, wanted + need
            self.open[b] = 0
            if need > 0 and wanted > len(free):
                self.flags.add(EPAGES)
                continue
            got = free[at:at + need]
            for p in got:
                self.refs[p] = 1
            if shared is not None:
                self.refs[shared] -= 1
                self.K[:, got[0]] = self.K[:, shared]
                self.V[:, got[0]] = self.V[:, shared]
                self.table[b].pop()
            self.table[b] += got
            self.rows[b] += n
            self.open[b] = n

    def write(self, K, V, layer=0):
        """K, V [batch][max_new][layers][hkv][d]."""
        nl = K.shape[2]
        for b in range(self.batch):
            for r in range(min(self.open[b], K.shape[1])):
                pos = self.rows[b] - self.open[b] + r
                p, o = self.table[b][pos // self.page], pos % self.page
                self.K[layer:layer + nl, p, :, o] = K[b, r]
                self.V[layer:layer + nl, p, :, o] = V[b, r]

    def keep(self, kept):
        for b in range(self.batch):
            k = int(kept[b])
            if not 0 <= k <= self.open[b]:
                self.flags.add(ERANGE)
                continue
            self.rows[b] -= self.open[b] - k
            self.open[b] = k
            while len(self.table[b]) > -(-self.rows[b] // self.page):
                self.refs[self.table[b].pop()] -= 1

    def fork(self, src):
        src = [int(x) for x in src]
        for b, a in enumerate(src):
            if a == b:
                continue
            if not -1 <= a < self.batch or (a >= 0 and src[a] != a):
                self.flags.add(ERANGE)
                continue
            for p in self.table[b]:
                self.refs[p] -= 1
            self.table[b] = list(self.table[a]) if a >= 0 else []
            for p in self.table[b]:
                self.refs[p] += 1
            self.rows[b], self.open[b] = (self.rows[a], 0) if a >= 0 else (0, 0)
            if a >= 0:
                self.open[a] = 0

    def compact(self):
        n = sum(r > 0 for r in self.refs)
        holes = [p for p in range(n) if self.refs[p] == 0]
        moved = [p for p in range(n, self.n_pages) if self.refs[p] > 0]
        for a, p in zip(moved, holes):
            self.K[:, p], self.V[:, p] = self.K[:, a], self.V[:, a]
            self.refs[p], self.refs[a] = self.refs[a], 0
            for t in self.table:
                t[:] = [p if x == a else x for x in t]

    def tables(self):
        t = np.full((self.batch, self.max_pages), -1, np.int32)
        for b, ids in enumerate(self.table):
            t[b, :len(ids)] = ids
        return t

    def sequence(self, layer, b):
        """K and V rows [rows][hkv][d] of a sequence."""
        ids, n = self.table[b], self.rows[b]
        flat = lambda X: X[layer, ids].transpose(0, 2, 1, 3).reshape(  # noqa: E731
            -1, X.shape[2], X.shape[4])[:n]
        return flat(self.K), flat(self.V)


def attend(q, K, V, scale):
    """q [m][hq][d], the queries of the last m of K's and V's rows [n][hkv][d] ->
    o [m][hq][d] and lse [m][hq]; keys a row does not see are left out before
    anything is computed with them."""
    m, hq, d = q.shape
    n, hkv = K.shape[:2]
    o, lse = np.zeros((m, hq, d)), np.full((m, hq), -np.inf)
    with np.errstate(all="ignore"):
        for i in range(m):
            seen = max(0, n - m + i + 1)
            for h in range(hq):
                g = h // (hq // hkv)
                s = scale * (K[:seen, g] @ q[i, h])
                if not len(s) or np.all(s == -np.inf):
                    continue
                top = np.nanmax(s) if not np.all(np.isnan(s)) else np.nan
                e = np.exp(s - top)
                o[i, h] = (e[:, None] * V[:seen, g]).sum(0) / e.sum()
                lse[i, h] = top + np.log(e.sum())
    return o, lse


def verify_probs(P, Q, y, n, u):
    """Eq. 1-2 from probabilities [B + 1][V], [B][V] (or None) and uniforms
    [B + 1] of one sequence: (accepted, token)."""
    P = np.asarray(P, np.float64)
    Q = None if Q is None else np.asarray(Q, np.float64)
    u = np.asarray(u, np.float64)
    B, V = P.shape[0] - 1, P.shape[1]
    n = B if n is None else min(max(int(n), 0), B)
    r = 0
    while r < n:
        t = int(y[r])
        if not 0 <= t < V or not u[r] * (1.0 if Q is None else Q[r, t]) < P[r, t]:
            break
        r += 1

    def positive(w):
        w = np.where(np.isfinite(w), w, 0.0)
        return np.maximum(w, 0.0)
    w = positive(P[r])
    if r < n:
        with np.errstate(invalid="ignore"):
            q = Q[r] if Q is not None else (np.arange(V) == int(y[r])).astype(np.float64)
            left = positive(P[r] - q)
        w = left if left.any() else w
    some = np.flatnonzero(w)
    if not len(some):
        return r, 0
    c = np.cumsum(w)
    over = np.flatnonzero((w > 0) & (c > u[B] * c[-1]))
    return r, int(over[0] if len(over) else some[-1])


# Rows in codes: the magnitudes of a code, the limit of a block's largest one in units of
# its scale, the lowest exponent, the largest magnitude that is coded as it is.
def _e4m3(code):
    e, m = code >> 3, code & 7
    return m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)


MX = {4: ([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], 7.0, -125, 1.5 * 2.0 ** 127),
      8: ([_e4m3(c) for c in range(127)], 464.0, -117, 1.875 * 2.0 ** 127)}


def mx_values(x, bits):
    """What rows [..., d] are held as: 32 dimensions share the smallest scale 2^e that
    their largest magnitude is within the limit of; each is the nearest code, the one of
    even number where two are as near."""
    grid, limit, lowest, top = MX[bits]
    grid = np.array(grid)
    x = np.asarray(x, np.float64)
    blocks = x.reshape(-1, 32)
    bad = ~np.isfinite(blocks).all(1, keepdims=True)
    blocks = np.clip(np.where(bad, 0.0, blocks), -top, top)
    scales = 2.0 ** np.arange(lowest, 128)
    most = np.abs(blocks).max(1, keepdims=True)
    scale = scales[np.searchsorted(limit * scales, most)]         # the first that holds it
    y = np.abs(blocks) / scale
    hi = np.minimum(np.searchsorted(grid, y), len(grid) - 1)      # the codes around
    lo = np.maximum(hi - 1, 0)
    up, down = np.abs(grid[hi] - y), np.abs(y - grid[lo])
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    out = np.where(bad, np.nan, np.copysign(grid[code] * scale, blocks))
    return out.reshape(x.shape)


class CodedCache(Cache):
    """A cache that holds its rows in 8 or 4 bits."""

    def __init__(self, bits, *sizes):
        super().__init__(*sizes)
        self.bits = bits

    def write(self, K, V, layer=0):
        super().write(mx_values(K, self.bits), mx_values(V, self.bits), layer)


def logprobs(z, y, temperature, top):
    """One row of logits: (log p(y), entropy, rank of y, the first `top` tokens, their log p)."""
    z = np.asarray(z, np.float64)
    V = len(z)
    ahead = lambda v: (np.isnan(z[v]), -z[v] if not np.isnan(z[v]) else 0.0, v)  # noqa: E731
    order = sorted(range(V), key=ahead)[:top] if V <= 4096 else list(
        np.lexsort((np.arange(V), -np.where(np.isnan(z), -np.inf, z), np.isnan(z)))[:top])
    given = 0 <= y < V
    rank = V
    if given:
        numbers = ~np.isnan(z)
        first = np.arange(V) < y
        rank = int((z > z[y]).sum() + ((z == z[y]) & first).sum()) if numbers[y] else \
            int(numbers.sum() + (~numbers & first).sum())
    if np.isnan(z).any() or np.isposinf(z).any():
        return np.nan, np.nan, rank, order, np.full(top, np.nan)
    if np.all(np.isneginf(z)):
        return -np.inf, 0.0, rank, order, np.full(top, -np.inf)
    x = (z - z.max()) / temperature
    p = np.exp(x)
    # the entries at the maximum are 1 each: their number is kept apart from the others' sum
    ls = np.log1p((x == 0).sum() - 1 + p[x != 0].sum())
    some = p > 0
    entropy = ls - (p[some] * x[some]).sum() / p.sum()
    return (x[y] - ls if given else -np.inf), entropy, rank, order, x[order] - ls
