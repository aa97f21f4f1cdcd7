"""Plain models that the tests of the answering operators compare with: a key-value cache's
bookkeeping in Python integers, and attention and token log probabilities in 64 bits."""
import numpy as np


class CacheModel:
    """The bookkeeping of copes_kv_cache, one list of pages per slot."""

    def __init__(self, n_pages, page_size, n_slots, width):
        self.n_pages, self.ps, self.width = n_pages, page_size, width
        self.pages = [[] for _ in range(n_slots)]
        self.length = [0] * n_slots
        self.refs = [0] * n_pages
        self.copies = []  # (from, to) pairs of the last call, whole pages

    def _free(self):
        return [p for p in range(self.n_pages) if self.refs[p] == 0]

    def _take(self, count):
        free = self._free()
        if len(free) < count:
            return None
        for p in free[:count]:
            self.refs[p] = 1
        return free[:count]

    def _slot(self, s):
        return 0 <= s < len(self.length)

    def grow(self, slots, add):
        """0, or the error bit of a call that changes nothing."""
        if len(set(slots)) < len(slots) or not all(map(self._slot, slots)) or min(add, default=0) < 0:
            return 32
        if any(self.length[s] + a > self.width * self.ps for s, a in zip(slots, add)):
            return 32
        need = [-(-(self.length[s] + a) // self.ps) - len(self.pages[s]) for s, a in zip(slots, add)]
        new = self._take(sum(need))
        if new is None:
            return 64
        for s, a, k in zip(slots, add, need):
            self.pages[s] += [new.pop(0) for _ in range(k)]
            self.length[s] += a
        return 0

    def fork(self, parents, children):
        self.copies = []
        both = list(parents) + list(children)
        if len(set(children)) < len(children) or not all(map(self._slot, both)) or set(parents) & set(children):
            return 32
        if any(self.length[c] for c in children):
            return 32
        partly = [self.length[p] % self.ps != 0 for p in parents]
        new = self._take(sum(partly))
        if new is None:
            return 64
        for p, c, copied in zip(parents, children, partly):
            shared = self.pages[p][:self.length[p] // self.ps]
            for x in shared:
                self.refs[x] += 1
            self.pages[c], self.length[c] = list(shared), self.length[p]
            if copied:
                self.pages[c].append(new.pop(0))
                self.copies.append((self.pages[p][-1], self.pages[c][-1]))
        return 0

    def free(self, slots):
        bad = 0
        for s in slots:
            if not self._slot(s):
                bad = 32
                continue
            for p in self.pages[s]:
                self.refs[p] -= 1
            self.pages[s], self.length[s] = [], 0
        return bad

    def compact(self):
        used = [p for p in range(self.n_pages) if self.refs[p]]
        n = len(used)
        moves = dict(zip([p for p in used if p >= n], [p for p in range(n) if not self.refs[p]]))
        for a, b in moves.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.pages = [[moves.get(p, p) for p in row] for row in self.pages]
        self.copies = list(moves.items())
        return n, len(moves)

    def table(self):
        out = np.full((len(self.length), self.width), -1, np.int32)
        for s, row in enumerate(self.pages):
            out[s, :len(row)] = row
        return out


def attention(q, keys, values, scale):
    """One row: q [heads, d], keys and values [tokens, kv heads, d], in float64.  Returns out,
    lse, and sum p |v| and the largest sum |scale q k| per head (for error bounds)."""
    heads, d = q.shape
    kv = keys.shape[1]
    out, lse = np.zeros((heads, d)), np.full(heads, -np.inf)
    mass, size = np.zeros((heads, d)), np.zeros(heads)
    if len(keys) == 0:
        return out, lse, mass, size
    for h in range(heads):
        g = h // (heads // kv)
        s = keys[:, g] @ q[h] * scale
        e = np.exp(s - s.max())
        out[h] = e @ values[:, g] / e.sum()
        mass[h] = e @ np.abs(values[:, g]) / e.sum()
        lse[h] = s.max() + np.log(e.sum())
        size[h] = (np.abs(keys[:, g]) @ np.abs(q[h])).max() * abs(scale)
    return out, lse, mass, size


def token_logprobs(x, target, top, scale):
    """One row in float64: logprob, entropy, ids, their logprobs, and lse."""
    order = np.lexsort((np.arange(len(x)), np.where(np.isnan(x), -np.inf, -x), ~np.isnan(x)))
    ids = order[:top]
    if np.isnan(x).any() or np.isposinf(x).any():
        lp = 0.0 if target < 0 else np.nan
        return lp, np.nan, ids, np.full(top, np.nan), np.nan
    if np.isneginf(x).all():
        lp = np.nan if target >= len(x) else 0.0 if target < 0 else -np.inf
        return lp, 0.0, ids, np.full(top, -np.inf), -np.inf
    y = (x - x.max()) * scale
    e = np.exp(y)
    log_sum = np.log(e.sum())
    p = e / e.sum()
    with np.errstate(invalid="ignore"):
        entropy = log_sum - np.where(p > 0, p * y, 0.0).sum()
    lp = np.nan if target >= len(x) else 0.0 if target < 0 else y[target] - log_sum
    return lp, entropy, ids, y[ids] - log_sum, x.max() * scale + log_sum
