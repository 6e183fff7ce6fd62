"""Plain float64 model of the paged 4-bit cache, for the tests: Python lists and numpy, written from the interface's text."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def block_exponent(block):
    """The smallest e in [-100, 125] with max |x| < 7 * 2^e, by search."""
    top = np.abs(block).max()
    for e in range(-100, 126):
        if top < 7.0 * 2.0 ** e:
            return e
    return 125


def nearest_code(y):
    """Magnitude code of y >= 0: the nearest level, ties to the even code, 6 above."""
    gap = np.abs(LEVELS - min(y, 6.0))
    best = np.nonzero(gap == gap.min())[0]
    return int(best[0]) if len(best) == 1 else int(best[best % 2 == 0][0])


def quantise(rows):
    """rows [..., d] (float64) -> codes [..., d] (0 .. 15) and scale bytes [..., d / 32]."""
    rows = np.asarray(rows, dtype=np.float64)
    flat = rows.reshape(-1, rows.shape[-1] // 32, 32)
    codes = np.zeros(flat.shape, dtype=np.uint8)
    bytes_ = np.zeros(flat.shape[:2], dtype=np.uint8)
    for i in range(flat.shape[0]):
        for j in range(flat.shape[1]):
            x = flat[i, j]
            if not np.isfinite(x).all():
                bytes_[i, j] = 255
                continue
            e = block_exponent(x)
            bytes_[i, j] = e + 127
            codes[i, j] = [nearest_code(abs(v) / 2.0 ** e) | (8 if np.signbit(v) else 0) for v in x]
    return codes.reshape(rows.shape), bytes_.reshape(rows.shape[:-1] + (-1,))


def values(codes, bytes_):
    """The numbers that codes and scale bytes stand for (float64, NaN for byte 255)."""
    mag = LEVELS[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    scale = np.where(bytes_ == 255, np.nan, 2.0 ** (bytes_.astype(np.float64) - 127))
    return mag * np.repeat(scale, 32, axis=-1)


def fast_values(rows):
    """values(quantise(rows)) without the loops."""
    x = np.asarray(rows, dtype=np.float64)
    b = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    finite = np.isfinite(b).all(-1, keepdims=True)
    b = np.where(finite, b, 0.0)
    top = np.abs(b).max(-1, keepdims=True)
    m, e = np.frexp(np.where(top > 0, top, 1.0))
    scale = 2.0 ** np.where(top > 0, np.clip(e - 3 + (m >= 0.875), -100, 125), -100)
    y = np.abs(b) / scale
    q = np.zeros_like(y)
    for lo, hi, even_low in zip(LEVELS[:-1], LEVELS[1:], (True, False) * 4):
        mid = (lo + hi) / 2
        q = np.where((y > mid) | ((y == mid) & (not even_low)), hi, q)
    return np.where(finite, np.copysign(q, b) * scale, np.nan).reshape(x.shape)


class Pool:
    """Decodes a pool's bytes (numpy uint8) into values, by page."""

    def __init__(self, shape, raw):
        s = shape
        self.s, pr, d = s, shape.page_rows, shape.head_dim
        self.rec = np.asarray(raw).reshape(s.layers, s.n_pages, s.n_kv_heads, pr * 2 * (d // 2 + d // 32))

    def rows(self, layer, page, first_part):
        """[n_kv][page_rows][d] of one page: the keys (first_part) or the values."""
        s, pr, d = self.s, self.s.page_rows, self.s.head_dim
        half = pr * (d // 2 + d // 32)
        r = self.rec[layer, page, :, : half] if first_part else self.rec[layer, page, :, half:]
        packed = r[:, : pr * (d // 2)].reshape(-1, pr, d // 2)
        codes = np.stack((packed & 15, packed >> 4), -1).reshape(-1, pr, d)
        return values(codes, r[:, pr * (d // 2):].reshape(-1, pr, d // 32))

    def sequence(self, layer, pages, n, first_part):
        """[n_kv][n][d] of a sequence whose rows lie in `pages`."""
        s = self.s
        if n == 0:
            return np.zeros((s.n_kv_heads, 0, s.head_dim))
        return np.concatenate([self.rows(layer, p, first_part) for p in pages], axis=1)[:, :n]


def attend(q, k, v, bias=None):
    """q [hq][d], k, v [hkv][n][d] (float64): outputs [hq][d], probabilities [hq][n], the largest sum |q k| / sqrt(d), and
    sum a |v| [hq][d]."""
    hq, d = q.shape
    n = k.shape[1]
    if n == 0:
        return np.zeros((hq, d)), np.zeros((hq, 0)), 0.0, np.zeros((hq, d))
    kk, vv = np.repeat(k, hq // k.shape[0], axis=0), np.repeat(v, hq // v.shape[0], axis=0)
    z = np.einsum("hd,hnd->hn", q, kk) / np.sqrt(d)
    if bias is not None:
        z = z + bias
    e = np.exp(z - z.max(-1, keepdims=True))
    a = e / e.sum(-1, keepdims=True)
    size = np.einsum("hd,hnd->hn", np.abs(q), np.abs(kk)).max() / np.sqrt(d)
    return np.einsum("hn,hnd->hd", a, vv), a, size, np.einsum("hn,hnd->hd", a, np.abs(vv))


class Pages:
    """Tables, lengths, counts, utilities and positions as Python values; `page` ids follow the interface's rules."""

    def __init__(self, batch, n_pages, max_pages, page_rows):
        self.pr, self.max_pages, self.n_pages = page_rows, max_pages, n_pages
        self.table = [[] for _ in range(batch)]
        self.len = [0] * batch
        self.refs = [0] * n_pages
        self.u = [dict() for _ in range(batch)]      # slot row -> value ever written
        self.pos = [dict() for _ in range(batch)]
        self.data = {}                                # (page, row) -> token of whatever was stored there

    def _pages(self, n):
        return -(-n // self.pr)

    def _grant(self, need):
        free = [p for p in range(self.n_pages) if self.refs[p] == 0]
        out, used = [], 0
        for n in need:
            used += n
            out.append(free[used - n: used] if n == 0 or used <= len(free) else None)
        return out

    def reserve(self, add, new_pos, prior):
        """prior(list of utilities) -> the new rows' utility.  Returns the rows granted."""
        need, copies = [], []
        for b, n in enumerate(add):
            ok = n >= 0 and self.len[b] + n <= self.max_pages * self.pr
            copy = ok and n > 0 and self.len[b] % self.pr and self.refs[self.table[b][-1]] > 1
            need.append(self._pages(self.len[b] + n) - self._pages(self.len[b]) + bool(copy) if ok and n > 0 else 0)
            copies.append(bool(copy) if ok and n > 0 else None)
        granted = []
        for b, got in enumerate(self._grant(need)):
            if got is None or copies[b] is None:
                granted.append(0)
                continue
            got = list(got)
            if copies[b]:
                old, new = self.table[b][-1], got.pop(0)
                for r in range(self.len[b] % self.pr):
                    self.data[new, r] = self.data.get((old, r))
                self.table[b][-1] = new
                self.refs[old] -= 1
                self.refs[new] = 1
            for p in got:
                self.table[b].append(p)
                self.refs[p] = 1
            old = [self.u[b][i] for i in range(self.len[b])]
            for i in range(add[b]):
                self.u[b][self.len[b] + i] = prior(old)
                self.pos[b][self.len[b] + i] = new_pos[b] + i
            self.len[b] += add[b]
            granted.append(add[b])
        return granted

    def place(self, b, i):
        return self.table[b][i // self.pr], i % self.pr

    def store(self, b, i, token):
        self.data[self.place(b, i)] = token

    def tokens(self, b):
        return [self.data.get(self.place(b, i)) for i in range(self.len[b])]

    def fork(self, src, dst):
        done = set()
        before = list(self.len)
        for i, (s, d) in enumerate(zip(src, dst)):
            if not (0 <= s < len(self.len) and 0 <= d < len(self.len)) or s in dst or d in done or before[d]:
                if 0 <= d < len(self.len):
                    done.add(d)
                continue
            done.add(d)
            self.table[d], self.len[d] = list(self.table[s]), self.len[s]
            for p in self.table[s]:
                self.refs[p] += 1
            for i in range(self.len[s]):
                self.u[d][i], self.pos[d][i] = self.u[s][i], self.pos[s][i]

    def free(self, slots):
        for b in set(slots):
            if 0 <= b < len(self.len):
                for p in self.table[b]:
                    self.refs[p] -= 1
                self.table[b], self.len[b] = [], 0

    def best(self, b, budget):
        order = sorted(range(self.len[b]), key=lambda i: (-self.u[b][i], self.pos[b][i]))
        kept = set(order[:budget])
        return [i in kept for i in range(self.len[b])]

    def compact(self, keep):
        """keep: per slot a list of truth values over its rows."""
        plans, need = [], []
        for b, m in enumerate(keep):
            k = sum(map(bool, m))
            holes = [i for i in range(k) if not m[i]]
            moves = dict(zip(holes, [i for i in range(k, len(m)) if m[i]]))
            pages = sorted({i // self.pr for i in holes if self.refs[self.table[b][i // self.pr]] > 1})
            plans.append((k, moves, pages))
            need.append(len(pages))
        grants = self._grant(need)
        new_data, refs = dict(self.data), list(self.refs)
        for b, ((k, moves, pages), got) in enumerate(zip(plans, grants)):
            if got is None:
                continue
            table = list(self.table[b])
            for j, p in zip(pages, got):
                table[j] = p
                refs[p] = 1
                refs[self.table[b][j]] -= 1
                for i in range(j * self.pr, min(k, (j + 1) * self.pr)):
                    new_data[p, i % self.pr] = self.data.get(self.place(b, i))
            for dst, src in moves.items():
                new_data[table[dst // self.pr], dst % self.pr] = self.data.get(self.place(b, src))
            u, pos = dict(self.u[b]), dict(self.pos[b])
            for dst, src in moves.items():
                u[dst], pos[dst] = self.u[b][src], self.pos[b][src]
            for j in range(self._pages(k), len(table)):
                refs[table[j]] -= 1
            self.table[b], self.u[b], self.pos[b], self.len[b] = table[: self._pages(k)], u, pos, k
        self.data, self.refs = new_data, refs
