"""Plain fp64 numpy of the sampling operators: a paged cache kept page by page, attention of drafted trees over it, draft
verification as a distribution that is made 1 again after every rejection.  Shares no code with the HIP path."""
import numpy as np


class Book:
    """A paged cache's bookkeeping and pools, an entry of a call after the other."""

    def __init__(self, table, length, held, refs, page_size, k=None, v=None):
        self.table = np.array(table, dtype=np.int64)
        self.len, self.held, self.refs = (np.array(x, dtype=np.int64) for x in (length, held, refs))
        self.ps = page_size
        self.pools = [np.array(p) for p in (k, v) if p is not None]  # [layers, pages, hkv, ps, d]

    def sound(self, s):
        return 0 <= self.held[s] <= self.table.shape[1] and 0 <= self.len[s] <= self.held[s] * self.ps

    def _free_pages(self):
        return [p for p in range(len(self.refs)) if self.refs[p] <= 0]

    def _entries(self, slots):
        """(index, slot, it counts) of the entries that name anything."""
        seen = set()
        for i, s in enumerate(slots):
            if s < 0:
                continue
            fine = s < len(self.len) and s not in seen
            seen.add(s)
            yield i, s, fine

    def reserve(self, slots, add):
        want, bad = [], 0
        for i, s, fine in self._entries(slots):
            pages = -(-(self.len[s] + add[i]) // self.ps) if fine else 0
            if not fine or add[i] < 0 or not self.sound(s) or pages > self.table.shape[1]:
                bad += 1
            else:
                want.append((s, max(0, pages - self.held[s])))
        free, need = self._free_pages(), sum(n for _, n in want)
        if need > len(free):
            return [need - len(free), bad]
        for s, n in want:
            for _ in range(n):
                self.table[s, self.held[s]] = p = free.pop(0)
                self.refs[p] = 1
                self.held[s] += 1
        return [0, bad]

    def fork(self, src, dst):
        todo, bad, taken = [], 0, set()
        old_len, old_held = self.len.copy(), self.held.copy()
        for a, b in zip(src, dst):
            if a < 0 and b < 0:
                continue
            fine = 0 <= a < len(old_len) and 0 <= b < len(old_len) and a != b and b not in taken
            if 0 <= b < len(old_len):
                taken.add(b)
            fine = fine and old_held[b] == 0 and old_len[b] == 0 and self.sound(a)
            if fine and old_len[a] % self.ps:
                fine = 0 <= self.table[a, old_len[a] // self.ps] < len(self.refs)
            if fine:
                todo.append((a, b))
            else:
                bad += 1
        free = self._free_pages()
        need = sum(old_len[a] % self.ps > 0 for a, _ in todo)
        if need > len(free):
            return [int(need - len(free)), bad]
        for a, b in todo:
            whole, rest = divmod(int(old_len[a]), self.ps)
            for c in range(whole):
                self.table[b, c] = p = self.table[a, c]
                if 0 <= p < len(self.refs):
                    self.refs[p] += 1
            if rest:
                self.table[b, whole] = p = free.pop(0)
                self.refs[p] = 1
                for pool in self.pools:
                    pool[:, p, :, :rest] = pool[:, self.table[a, whole], :, :rest]
            self.len[b], self.held[b] = old_len[a], whole + (rest > 0)
        return [0, bad]

    def free(self, slots):
        for s in slots:
            if 0 <= s < len(self.len):
                for c in range(min(self.held[s], self.table.shape[1])):
                    if 0 <= self.table[s, c] < len(self.refs):
                        self.refs[self.table[s, c]] -= 1
                self.len[s] = self.held[s] = 0

    def compact(self):
        live = int((self.refs > 0).sum())
        movers = [p for p in range(live, len(self.refs)) if self.refs[p] > 0]
        for p, hole in zip(movers, [p for p in range(live) if self.refs[p] <= 0]):
            for pool in self.pools:
                pool[:, hole] = pool[:, p]
            self.refs[hole], self.refs[p] = self.refs[p], 0
            for s in range(len(self.len)):
                row = self.table[s, :self.held[s]]
                row[row == p] = hole
        return live

    def shared(self, slots, group):
        out = []
        for g in range(0, len(slots), group):
            m = [s for s in slots[g:g + group] if s >= 0]
            n = 0
            if len(m) > 1 and all(s < len(self.len) and self.sound(s) for s in m):
                most = min(int(self.len[s]) // self.ps for s in m)
                while n < most and len({int(self.table[s, n]) for s in m}) == 1:
                    n += 1
            out.append(n)
        return out

    def place(self, s, t):
        return int(self.table[s, t // self.ps]), t % self.ps

    def append(self, layer, slot, j, k, v):
        """A token's (rotated) keys and values at place len + j, if it has a page."""
        t = int(self.len[slot]) + j
        if self.sound(slot) and t < self.held[slot] * self.ps:
            p, r = self.place(slot, t)
            if 0 <= p < len(self.refs):
                self.pools[0][layer, p, :, r], self.pools[1][layer, p, :, r] = k, v

    def accept(self, slots, count, path=None, max_new=1 << 30):
        bad = 0
        for i, s, fine in self._entries(slots):
            m = int(count[i])
            if m == 0:  # (also the entry by which a slot counts that is named again)
                continue
            fine = fine and 0 < m <= max_new and self.sound(s)
            nodes = [int(x) for x in path[i][:m]] if fine and path is not None else list(range(m))
            fine = fine and all(b > a for a, b in zip([-1] + nodes, nodes)) and max(nodes) < max_new
            if not fine or self.len[s] + nodes[-1] >= self.held[s] * self.ps:
                bad += 1
                continue
            for j, at in enumerate(nodes):
                (a, x), (b, y) = self.place(s, int(self.len[s]) + at), self.place(s, int(self.len[s]) + j)
                for pool in self.pools:
                    pool[:, b, :, y] = pool[:, a, :, x].copy()
            self.len[s] += m
        return [0, bad]


def depths(parents):
    out = []
    for i, p in enumerate(parents):
        out.append(out[p] + 1 if 0 <= p < i else 0)
    return out


def rotate(x, pos, base):
    """The half-split rotary embedding of rows x [..., d] at one position."""
    d = x.shape[-1]
    a = pos * base ** (-2.0 * np.arange(d // 2) / d)
    lo, hi = x[..., :d // 2], x[..., d // 2:]
    return np.concatenate([lo * np.cos(a) - hi * np.sin(a), hi * np.cos(a) + lo * np.sin(a)], axis=-1)


def tree_attn(book, layer, slots, q, parents=None, count=None, scale=None):
    """(o, lse, sum of |terms| of o, greatest sum of |terms| of a row's scores) of nodes q [n, N, hq, d]; parents [n][N],
    None: chains."""
    n, N, hq, d = q.shape
    K, V = (p[layer] for p in book.pools)
    hkv = K.shape[1]
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    o, lse, size = np.zeros((n, N, hq, d)), np.zeros((hq, n * N)), np.zeros((n, N, hq, d))
    score = np.zeros((n, N, hq))
    for i, s in enumerate(slots):
        c = N if count is None else max(0, min(int(count[i]), N))
        if s < 0 or c == 0:
            continue
        if s >= len(book.len) or not book.sound(s) or book.len[s] + c > book.held[s] * book.ps:
            o[i, :c], lse[:, i * N:i * N + c] = np.nan, np.nan
            continue
        L = int(book.len[s])
        at = [book.place(s, t) for t in range(L + c)]
        page, row = np.array([a for a, _ in at]), np.array([b for _, b in at])
        for g in range(hkv):
            k, v = K[page, g, row], V[page, g, row]
            for a in range(c):
                path, b, ok = [], a, True
                while b >= 0:
                    path.append(b)
                    up = b - 1 if parents is None else int(parents[i][b])
                    ok = ok and -1 <= up < b
                    b = up if ok else -1
                see = np.array(list(range(L)) + [L + b for b in path])
                for h in range(g * hq // hkv, (g + 1) * hq // hkv):
                    x = scale * (k[see] @ q[i, a, h])
                    m = x.max()
                    e = np.exp(x - m)
                    o[i, a, h] = e @ v[see] / e.sum() if ok else np.nan
                    size[i, a, h] = e @ np.abs(v[see]) / e.sum()
                    lse[h, i * N + a] = m + np.log(e.sum()) if ok else np.nan
                    score[i, a, h] = scale * (np.abs(k[see]) @ np.abs(q[i, a, h])).max()
    return o, lse, size, score


def _softmax(x, lowest, T=1.0):
    """Probabilities of a row of logits at temperature T, masked entries and those below 2^-999 of the largest 0; None if it
    cannot be used."""
    x = np.where(x <= lowest, -np.inf, x)
    if np.isnan(x).any() or (x == np.inf).any() or not (x > -np.inf).any():
        return None
    e = np.exp((x - x.max()) / T)
    e[e <= 2.0 ** -999] = 0.0
    return e / e.sum()


def verify(target, tokens, u, draft=None, parents=None, count=None, temperature=None, max_children=1, lowest=-3.0e38):
    """(count, tokens, path, logp) of pp_verify_draft.  The residual is a distribution r of its own: a child y follows if
    u < r(y) / q(y), else r = max(r - q, 0) made 1 again (given drafts: u < r(y), else r without y)."""
    n, N, V = target.shape
    out_n, out_t, out_p, out_l = np.zeros(n, int), np.full((n, N), -1), np.full((n, N), -1), np.zeros((n, N))
    for i in range(n):
        c = N if count is None else max(0, min(int(count[i]), N))
        if c == 0:
            continue
        T = 1.0 if temperature is None else float(temperature[i])
        greedy = not T > 0
        at, m = 0, 0
        out_p[i, 0] = 0
        with np.errstate(invalid="ignore", over="ignore"):
            while True:
                row = target[i, at].astype(np.float64)
                p = _softmax(row, lowest, 1.0 if greedy else T)
                r = None if p is None else p.copy()
                q = None
                if p is not None and greedy:
                    r = np.zeros(V)
                    r[int(np.argmax(np.where(np.isnan(row) | (row <= lowest), -np.inf, row)))] = 1.0
                usable = p is not None
                if usable and draft is not None and not greedy:
                    q = _softmax(draft[i, at].astype(np.float64), lowest, T)
                    usable = q is not None
                step, tried = None, 0
                for j in range(1, c):
                    up = j - 1 if parents is None else int(parents[i][j])
                    if up != at or up >= j or not usable or tried >= max_children:
                        continue
                    tried += 1
                    y = int(tokens[i, j])
                    known = 0 <= y < V
                    if known and (u[i, j] * q[y] < r[y] if q is not None else u[i, j] < r[y]):
                        step = (j, y)
                        break
                    if q is not None:
                        r = np.maximum(r - q, 0)
                    elif known:
                        r[y] = 0
                    if r.sum() > 0:
                        r = r / r.sum()
                if step is None:
                    break
                out_t[i, m], out_l[i, m] = step[1], np.log(p[step[1]])
                at, m = step[0], m + 1
                out_p[i, m] = at
        if p is None:
            out_l[i, m] = np.nan
        else:
            if not r.sum() > 0:
                r = p
            past = np.cumsum(r) > float(u[i, 0]) * r.sum()
            y = int(np.argmax(past)) if past.any() else int(np.nonzero(r)[0][-1])
            out_t[i, m], out_l[i, m] = y, np.log(p[y])
        out_n[i] = m + 1
    return out_n, out_t, out_p, out_l
