"""The 4-bit key/value cache, stated plainly in numpy: float64, one token and head at a time where that is clearest, and a book
of pages kept as Python lists.  Test infrastructure only; shares no code with the library."""
import numpy as np


def rotate(x, positions, inv_freq, rope):
    """x [rows, heads, dim] float32 -> float32: channel pairs turned by position * inv_freq (rope 0: not, 1: halves, 2: neighbours)."""
    if rope == 0:
        return x.astype(np.float32)
    half = x.shape[-1] // 2
    angle = np.asarray(positions, np.float64)[:, None] * np.asarray(inv_freq, np.float64)
    c = np.cos(angle).astype(np.float32).astype(np.float64)[:, None]
    s = np.sin(angle).astype(np.float32).astype(np.float64)[:, None]
    i, j = (slice(0, half), slice(half, None)) if rope == 1 else (slice(0, None, 2), slice(1, None, 2))
    a, b = x[..., i].astype(np.float64), x[..., j].astype(np.float64)
    y = np.empty(x.shape, np.float32)
    y[..., i] = (a * c - b * s).astype(np.float32)
    y[..., j] = (b * c + a * s).astype(np.float32)
    return y


def quantize(x):
    """x [..., dim] float32 -> codes uint8, alpha float32, beta int32: Eq. (2) at 4 bits, alpha = (max - min) * fl32(1/15), products
    with 1 / alpha exact in float64 and rounded to the nearest integer, ties to even."""
    x = np.asarray(x, np.float32)
    low, high = x.min(-1), x.max(-1)
    alpha = (high - low) * (np.float32(1) / np.float32(15))
    alpha = np.where(alpha < np.float32(2.0 ** -126), np.float32(1), alpha).astype(np.float32)
    inv = (np.float32(1) / alpha).astype(np.float64)
    beta = np.clip(-np.rint(low.astype(np.float64) * inv), -2147483647.0, 2147483647.0)
    codes = np.clip(np.rint(x.astype(np.float64) * inv[..., None]) + beta[..., None], 0, 15)
    return codes.astype(np.uint8), alpha, beta.astype(np.int32)


class Pages:
    """One layer's pages, [n_pages, page bytes] uint8, taken apart byte by byte of the documented layout."""

    def __init__(self, raw, heads, dim, page):
        self.raw, self.heads, self.dim, self.page = raw, heads, dim, page

    def _at(self, page, head, place, value):
        base = head * self.page * (self.dim + 16)
        code = base + (value * self.page + place) * (self.dim // 2)
        par = base + self.page * self.dim + 8 * value * self.page + 4 * place
        return page, code, par

    def put(self, page, head, place, value, codes, alpha, beta):
        p, code, par = self._at(page, head, place, value)
        self.raw[p, code:code + self.dim // 2] = codes[0::2] | (codes[1::2] << 4)
        self.raw[p, par:par + 4] = np.frombuffer(np.float32(alpha).tobytes(), np.uint8)
        self.raw[p, par + 4 * self.page:par + 4 * self.page + 4] = np.frombuffer(np.int32(beta).tobytes(), np.uint8)

    def get(self, page, head, place, value):
        """The float64 values of a token's key or value, and (alpha, beta)."""
        p, code, par = self._at(page, head, place, value)
        b = self.raw[p, code:code + self.dim // 2]
        codes = np.empty(self.dim, np.float64)
        codes[0::2], codes[1::2] = b & 15, b >> 4
        alpha = np.frombuffer(self.raw[p, par:par + 4].tobytes(), np.float32)[0]
        beta = np.frombuffer(self.raw[p, par + 4 * self.page:par + 4 * self.page + 4].tobytes(), np.int32)[0]
        return np.float64(alpha) * (codes - np.float64(beta)), float(alpha), int(beta)


def rows_of(rows, row_start, slot, length):
    """(row, line, position) of every row that belongs to a sequence."""
    out = []
    n_seqs = len(row_start) - 1 if row_start is not None else len(slot) if slot is not None else len(length)
    for i in range(n_seqs):
        r0, r1 = (row_start[i], row_start[i + 1]) if row_start is not None else (i, i + 1)
        line = slot[i] if slot is not None else i
        for r in range(r0, r1):
            out.append((int(r), int(line), int(length[line]) - int(r1) + int(r) if 0 <= line < len(length) else -1))
    return out


def page_at(table, n_pages, page, line, position):
    if not 0 <= line < table.shape[0] or position < 0 or position // page >= table.shape[1]:
        return -1
    p = int(table[line, position // page])
    return p if 0 <= p < n_pages else -1


def append(pages, table, tokens, k, v):
    """k, v [rows, heads, dim] float32 (keys already rotated) into the pages of `tokens` (as rows_of gives them)."""
    for value, x in ((0, k), (1, v)):
        codes, alpha, beta = quantize(x)
        for r, line, pos in tokens:
            p = page_at(table, pages.raw.shape[0], pages.page, line, pos)
            if p >= 0:
                for h in range(pages.heads):
                    pages.put(p, h, pos % pages.page, value, codes[r, h], alpha[r, h], beta[r, h])


def attention(q, pages, table, tokens, length, scale, window=0, out=None, close=False):
    """q [rows, q_heads, dim] float32 -> (out, bound on sum w |v|, bound on the scores' fp32 error, bound on the sums' fp32 error),
    float64 of q's shape; rows of no token keep what `out` has.  2^-24 is half a step of fp32.  The bounds allow a rounding per addend in any
    order; close: as many as sums on the matrix cores make, 32 addends to a rounding, split over four waves."""
    heads, dim = pages.heads, pages.dim
    group = q.shape[1] // heads
    out = np.zeros(q.shape) if out is None else out.astype(np.float64)
    absv, err_s, err_o = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape)
    cached = {}

    def lines(line, h, upto):
        if (line, h) not in cached:
            ks, vs, al, be, where = [], [], [], [], []
            for t in range(upto):
                p = page_at(table, pages.raw.shape[0], pages.page, line, t)
                if p >= 0:
                    kk, ka, kb = pages.get(p, h, t % pages.page, 0)
                    vv, va, vb = pages.get(p, h, t % pages.page, 1)
                    ks.append(kk), vs.append(vv), al.append((ka, va)), be.append((kb, vb)), where.append(t)
            cached[line, h] = [np.array(x, np.float64).reshape(len(where), *s) for x, s in ((ks, (dim,)), (vs, (dim,)), (al, (2,)), (be, (2,)))] + [np.array(where, np.int64)]
        return cached[line, h]

    for r, line, pos in tokens:
        out[r] = 0.0
        if not 0 <= line < table.shape[0] or pos < 0:
            continue
        for h in range(heads):
            ks, vs, al, be, where = lines(line, h, min(int(length[line]), table.shape[1] * pages.page))
            seen = (where <= pos) & ((where > pos - window) if window else True)
            if not seen.any():
                continue
            k, v, a, b = ks[seen], vs[seen], np.abs(al[seen]), np.abs(be[seen])
            for j in range(group):
                x = q[r, h * group + j].astype(np.float64)
                s = scale * (k @ x)
                w = np.exp(s - s.max())
                w /= w.sum()
                o = h * group + j
                out[r, o] = w @ v
                absv[r, o] = w @ np.abs(v)
                # sums of dim products (16 + code) q, (16 + beta) sum q, and a few roundings of the score itself
                if close:  # an operation per 32 channels, off by 2 * 2^-24 of its magnitudes (1.7 measured); the queries' sum: dim / 8
                    # additions and three across lanes
                    sums = abs(scale) * a[:, 0] * (2 * 31.0 * (dim // 32 + 1) + (16.0 + b[:, 0]) * (dim // 8 + 5)) * np.abs(x).sum()
                    adds = 4 * (seen.sum() // 128 + 1) + 16  # two operations a step of 32 tokens for each part of the weights, waves and parts joined
                else:
                    sums = abs(scale) * a[:, 0] * (47.0 + b[:, 0]) * np.abs(x).sum() * (dim + 8)
                    adds = seen.sum() + 32
                err_s[r, o] = 2.0 ** -24 * (sums.max() + 8 * np.abs(s).max() + 16)
                err_o[r, o] = 2.0 ** -24 * adds * (w * a[:, 1] * ((47.0 if close else 32.0) + b[:, 1])).sum()
    return out, absv, err_s, err_o


def attention_bound(want, absv, err_s, err_o, q_half, out_half):
    """How far an output may be off: its own rounding (half a step `out_half`), that of each weight to the queries' type (`q_half`)
    above and below the line, and what `attention` says of the scores' and the sums' fp32 errors."""
    return (out_half * (np.abs(want) + q_half * absv) + q_half * (absv + np.abs(want))) * (1 + 2.0 ** -7) + 2.0 * np.expm1(err_s) * absv + 2.0 * err_o + 1e-30


class Book:
    """Lines as Python lists of pages."""

    def __init__(self, n_lines, per_line, n_pages, page):
        self.lines, self.length = [[] for _ in range(n_lines)], [0] * n_lines
        self.per_line, self.n_pages, self.page = per_line, n_pages, page

    def refs(self):
        n = [0] * self.n_pages
        for line in self.lines:
            for p in line:
                n[p] += 1
        return n

    def _fresh(self):
        n = self.refs()
        return next((p for p in range(self.n_pages) if n[p] == 0), None)

    def reserve(self, line, count):
        """False where pages run out or the line is too short (the book is then spoilt)."""
        self.length[line] += count
        while len(self.lines[line]) * self.page < self.length[line]:
            p = self._fresh()
            if p is None or len(self.lines[line]) == self.per_line:
                return False
            self.lines[line].append(p)
        return True

    def fork(self, parent, child):
        """(source, destination) of a copy, None for none, False where pages run out."""
        whole = self.length[parent] // self.page
        self.lines[child], self.length[child] = list(self.lines[parent][:whole]), self.length[parent]
        if self.length[parent] % self.page == 0:
            return None
        p = self._fresh()
        if p is None:
            return False
        self.lines[child].append(p)
        return self.lines[parent][whole], p

    def free(self, line):
        self.lines[line], self.length[line] = [], 0

    def compact(self):
        n = self.refs()
        used = sum(x > 0 for x in n)
        src = [p for p in range(used, self.n_pages) if n[p]]
        dst = [p for p in range(used) if not n[p]]
        to = dict(zip(src, dst))
        self.lines = [[to.get(p, p) for p in line] for line in self.lines]
        return src, dst

    def table(self):
        t = np.full((len(self.lines), self.per_line), -1, np.int32)
        for i, line in enumerate(self.lines):
            t[i, :len(line)] = line
        return t
