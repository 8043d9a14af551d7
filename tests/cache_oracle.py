"""The 8-bit paged K/V cache in plain 64-bit form, from the definitions in include/crisp.h: codes,
scales and the order of a tile's bytes, appending, attention, and the pages' bookkeeping with
Python lists.  Test infrastructure only."""
import numpy as np

D = 128
E4M3, INT8 = 0, 1
MAX = {E4M3: 448.0, INT8: 127.0}
E_MIN = -64


def e4m3_values():
    """The 256 values of e4m3: sign, 4 exponent bits of bias 7, 3 mantissa bits, no infinity."""
    out = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        out[c] = np.nan if c & 127 == 127 else (-v if c & 128 else v)
    return out


_E4M3 = e4m3_values()


def round_codes(x, fmt):
    """The nearest value that a code has, ties to even; NaN 0, beyond MAX the largest."""
    x = np.clip(np.where(np.isnan(x), 0.0, x), -MAX[fmt], MAX[fmt])
    if fmt == INT8:
        return np.rint(x)
    _, e = np.frexp(np.maximum(np.abs(x), 2.0 ** -6))  # 2^(e - 1) <= |x| < 2^e
    step = np.ldexp(1.0, e - 4)
    return np.rint(x / step) * step


def scale_exponent(x, fmt):
    """The smallest e >= E_MIN with |x| <= MAX 2^e for the finite values x."""
    x = np.abs(x[np.isfinite(x)])
    top = x.max() if x.size else 0.0
    e = E_MIN
    while top > MAX[fmt] * 2.0 ** e:
        e += 1
    return e


def tile_index():
    """Byte of (token t, element e) in a tile of K and of V."""
    t, e = np.arange(64)[:, None], np.arange(D)[None, :]
    k = ((t // 4 % 4 * 2 + e // 16 % 2) * 64 + e // 32 * 16 + t // 16 * 4 + t % 4) * 16 + e % 16
    v = (e // 16 * 64 + t // 16 * 16 + e % 16) * 16 + t % 16
    return k, v


def decode(pages, fmt):
    """uint8 [n_pages, H, B / 64, 2, 8192] -> code values [n_pages, H, 2, B, 128]."""
    n, h, tiles = pages.shape[:3]
    val = _E4M3[pages] if fmt == E4M3 else pages.view(np.int8).astype(np.float64)
    k, v = tile_index()
    out = np.empty((n, h, 2, tiles * 64, D))
    for tl in range(tiles):
        out[:, :, 0, tl * 64:(tl + 1) * 64] = val[:, :, tl, 0][:, :, k]
        out[:, :, 1, tl * 64:(tl + 1) * 64] = val[:, :, tl, 1][:, :, v]
    return out


def encode(codes, fmt):
    """Code values [n_pages, H, 2, B, 128] -> uint8 pages (-0 and 0 are both 0)."""
    n, h, _, B, _ = codes.shape
    if fmt == E4M3:
        order = np.argsort(_E4M3[:127])
        at = order[np.searchsorted(_E4M3[:127][order], np.abs(codes))]
        byte = (at | np.where(codes < 0, 128, 0)).astype(np.uint8)
    else:
        byte = codes.astype(np.int8).view(np.uint8)
    pages = np.zeros((n, h, B // 64, 2, 8192), dtype=np.uint8)
    k, v = tile_index()
    for tl in range(B // 64):
        pages[:, :, tl, 0, k] = byte[:, :, 0, tl * 64:(tl + 1) * 64]
        pages[:, :, tl, 1, v] = byte[:, :, 1, tl * 64:(tl + 1) * 64]
    return pages


class Cache:
    """codes [n_pages, H, 2, B, 128] and exponents [n_pages, H, 2]; written marks what an append has put there."""

    def __init__(self, n_pages, heads, block, fmt):
        self.codes = np.zeros((n_pages, heads, 2, block, D))
        self.exp = np.zeros((n_pages, heads, 2), dtype=np.int64)
        self.written = np.zeros((n_pages, block), dtype=bool)
        self.block, self.fmt = block, fmt

    def append(self, table, seq_len, row_ptr, k, v):
        n_pages, heads = self.codes.shape[:2]
        for s in range(len(seq_len)):
            groups = {}
            for r in range(row_ptr[s], row_ptr[s + 1]):
                pos = seq_len[s] + r - row_ptr[s]
                slot = pos // self.block
                if slot < table.shape[1] and 0 <= table[s, slot] < n_pages:
                    groups.setdefault(int(table[s, slot]), []).append((pos % self.block, r))
            for page, rows in groups.items():
                at, src = [a for a, _ in rows], [r for _, r in rows]
                for h in range(heads):
                    for x, t in ((0, k), (1, v)):
                        e = scale_exponent(t[h, src], self.fmt)
                        if at[0] > 0:
                            old = self.exp[page, h, x]
                            if e > old:
                                self.codes[page, h, x] = round_codes(self.codes[page, h, x] * 2.0 ** float(old - e), self.fmt)
                            e = max(e, old)
                        self.exp[page, h, x] = e
                        self.codes[page, h, x, at] = round_codes(t[h, src] * 2.0 ** float(-e), self.fmt)
                self.written[page, at] = True

    def values(self, table_row, n, x):
        """[H, n, 128] of tensor x, and which of the n positions have a page."""
        n_pages, heads = self.codes.shape[:2]
        out, ok = np.zeros((heads, n, D)), np.zeros(n, dtype=bool)
        for j in range(n):
            slot = j // self.block
            if slot < len(table_row) and 0 <= table_row[slot] < n_pages:
                p = table_row[slot]
                out[:, j] = self.codes[p, :, x, j % self.block] * np.ldexp(1.0, self.exp[p, :, x])[:, None]
                ok[j] = True
        return out, ok

    def attention(self, table, seq_len, row_ptr, q, scale):
        """(o, tolerance), both [H_q, n_rows, 128]; rows outside row_ptr are NaN.

        The tolerance counts what a kernel with bf16 operands, 32-bit sums and a bf16 result may be off by:
        the result's rounding 2^-8 |o|; the probabilities' rounding, 2^-8 of sum p |v|; the scores' 32-bit
        sums of 128 products, each partial sum off by 2^-24, with the product by the scale and the
        exponential's argument (a few 2^-24 of its size): dS; and the 32-bit sums over the keys and
        their rescalings, at most (keys / 16 + 64) roundings of 2^-24."""
        hq, n_rows = q.shape[:2]
        heads = self.codes.shape[1]
        G = hq // heads
        o, tol = np.full((hq, n_rows, D), np.nan), np.full((hq, n_rows, D), np.nan)
        for s in range(len(seq_len)):
            r0, r1 = row_ptr[s], row_ptr[s + 1]
            n = seq_len[s] + r1 - r0
            if r1 <= r0:
                continue
            k, ok = self.values(table[s], n, 0)
            v, _ = self.values(table[s], n, 1)
            for h in range(hq):
                x = q[h, r0:r1] @ k[h // G].T * scale
                size = np.abs(q[h, r0:r1]) @ np.abs(k[h // G]).T * scale
                see = ok[None, :] & (np.arange(n)[None, :] <= (seq_len[s] + np.arange(r1 - r0))[:, None])
                x = np.where(see, x, -np.inf)
                top = np.max(x, axis=1, keepdims=True, initial=-np.inf)
                p = np.exp(x - np.where(np.isfinite(top), top, 0.0))
                l = p.sum(1, keepdims=True)
                p = np.divide(p, l, out=np.zeros_like(p), where=l > 0)
                o[h, r0:r1] = p @ v[h // G]
                ds = np.where(see, size * 140 * 2.0 ** -24 + 8 * np.abs(np.where(see, x - np.where(np.isfinite(top), top, 0), 0)) * 2.0 ** -24, 0.0)
                rel = 2.0 ** -8 + 2 * ds.max(1, initial=0.0, keepdims=True) + (n / 16 + 64) * 2.0 ** -24 + 2.0 ** -20
                tol[h, r0:r1] = 2.0 ** -8 * np.abs(o[h, r0:r1]) + rel * (p @ np.abs(v[h // G])) + 1e-30
        return o, tol


class Pool:
    """Uses of each page, table and lengths, with Python lists."""

    def __init__(self, n_pages, block, table, seq_len):
        self.uses, self.block = [0] * n_pages, block
        self.table, self.seq_len = [list(map(int, r)) for r in table], [int(x) for x in seq_len]

    def free_pages(self):
        return [p for p, u in enumerate(self.uses) if u == 0]

    def reserve(self, counts):
        free, asked, granted = self.free_pages(), 0, []
        taken = 0
        for s, c in enumerate(counts):
            row, n = self.table[s], self.seq_len[s]
            last = -(-(n + max(c, 0)) // self.block)
            if c <= 0 or last > len(row):
                granted.append(0)
                continue
            if any(0 <= row[j] < len(self.uses) and self.uses[row[j]] > 1 for j in range(n // self.block, last)):
                granted.append(0)
                continue
            lack = [j for j in range(n // self.block, last) if row[j] < 0]
            asked += len(lack)
            if lack and asked > len(free):
                granted.append(0)
                continue
            for j in lack:
                row[j] = free[taken]
                self.uses[row[j]] = 1
                taken += 1
            granted.append(c)
        return granted

    def fork(self, src, dst):
        n_seqs, free, copies = len(self.table), self.free_pages(), []
        lens, rows = list(self.seq_len), [list(r) for r in self.table]
        claimed, rank = set(), 0
        for s, d in zip(src, dst):
            ok = 0 <= s < n_seqs and 0 <= d < n_seqs and s != d and lens[d] == 0 and (not rows[d] or rows[d][0] < 0)
            if not ok or d in claimed:
                copies.append((-2, -2))
                continue
            claimed.add(d)
            n, full = lens[s], lens[s] // self.block
            pair = (-1, -1)
            if n % self.block:
                if not 0 <= rows[s][full] < len(self.uses):
                    copies.append((-2, -2))
                    continue
                rank += 1
                if rank > len(free):
                    copies.append((-2, -2))
                    continue
                pair = (rows[s][full], free[rank - 1])
                self.uses[pair[1]] = 1
            self.table[d] = rows[s][:full] + ([pair[1]] if n % self.block else [])
            self.table[d] += [-1] * (len(rows[s]) - len(self.table[d]))
            for p in rows[s][:full]:
                if 0 <= p < len(self.uses):
                    self.uses[p] += 1
            self.seq_len[d] = n
            copies.append(pair)
        return copies

    def free(self, ids):
        for s in ids:
            if 0 <= s < len(self.table):
                for p in self.table[s]:
                    if 0 <= p < len(self.uses) and self.uses[p] > 0:
                        self.uses[p] -= 1
                self.table[s] = [-1] * len(self.table[s])
                self.seq_len[s] = 0

    def compact(self):
        used = [p for p, u in enumerate(self.uses) if u > 0]
        n = len(used)
        holes, movers = [p for p in range(n) if self.uses[p] == 0], [p for p in used if p >= n]
        home = dict(zip(movers, holes))
        for p, q in home.items():
            self.uses[q], self.uses[p] = self.uses[p], 0
        self.table = [[home.get(p, p) for p in r] for r in self.table]
        return list(zip(movers, holes))

    def words(self):
        """The pool tensor's contents."""
        n = len(self.uses)
        bits = np.zeros(-(-n // 32) * 32, dtype=np.int64)
        bits[:n] = np.array(self.uses) > 0
        words = (bits.reshape(-1, 32) << np.arange(32)).sum(1).astype(np.uint32).view(np.int32)
        return np.concatenate([np.array(self.uses, dtype=np.int32), words])
