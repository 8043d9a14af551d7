"""Rotary positions, attention over packed prompts and eviction from the K/V cache in plain 64-bit form, from the definitions in
include/crisp.h.  Test infrastructure only."""
import math

import numpy as np

from tests import cache_oracle as O

D = 128
HALF, INTERLEAVED = 0, 1
PLAIN, LINEAR, BASE, BANDS, RAMP = 0, 1, 2, 3, 4


def frequencies(dim, base, rule=PLAIN, factor=1.0, original=0.0, low=0.0, high=0.0):
    """Angle a token of each pair, and the gain."""
    f = np.array([(base * factor ** (dim / (dim - 2)) if rule == BASE else base) ** (-2.0 * i / dim) for i in range(dim // 2)])
    gain = 1.0
    if rule == LINEAR:
        f = f / factor
    elif rule == BANDS:
        for i, x in enumerate(f):
            share = (original * x / (2 * math.pi) - low) / (high - low)
            share = min(max(share, 0.0), 1.0)
            f[i] = x * share + x / factor * (1 - share)
    elif rule == RAMP:
        pair = [dim * math.log(original / (2 * math.pi * n)) / (2 * math.log(base)) for n in (high, low)]
        a, b = max(math.floor(pair[0]), 0), min(math.ceil(pair[1]), dim - 1)
        for i, x in enumerate(f):
            share = 1.0 - min(max((i - a) / max(b - a, 0.001), 0.0), 1.0)
            f[i] = x * share + x / factor * (1 - share)
        gain = 0.1 * math.log(factor) + 1.0
    return f, gain


def rope(x, start, ptr, f, gain, dim, layout):
    """(y, tolerance) [heads, n_rows, 128]; rows outside ptr are NaN.

    The tolerance: the result's rounding, 2^-8 |y|; the angle, whose turns are off by 2^-52 of themselves (their product and the
    frequency) and by 2^-26 as a 32-bit fraction of at most 1/2; sine and cosine, the gain and the two products' sum, 12 roundings of 2^-24;
    both times the size of the pair."""
    y, tol = np.full(x.shape, np.nan), np.full(x.shape, np.nan)
    one = np.array([i for i in range(dim // 2)]) if layout == HALF else np.arange(0, dim, 2)
    two = one + (dim // 2 if layout == HALF else 1)
    for s in range(len(start)):
        for r in range(ptr[s], ptr[s + 1]):
            p = int(start[s]) + r - int(ptr[s])
            turns = np.longdouble(p) * (f.astype(np.longdouble) / (2 * np.longdouble(np.pi)))
            a = (2 * np.pi * (turns - np.rint(turns))).astype(np.float64)
            x1, x2 = x[:, r, one], x[:, r, two]
            y[:, r] = x[:, r]
            y[:, r, one] = gain * (x1 * np.cos(a) - x2 * np.sin(a))
            y[:, r, two] = gain * (x2 * np.cos(a) + x1 * np.sin(a))
            off = 2 * np.pi * (np.abs(turns).astype(np.float64) * 2.0 ** -52 + 2.0 ** -26) + 12 * 2.0 ** -24
            tol[:, r] = 0.0
            size = gain * (np.abs(x1) + np.abs(x2)) * off
            tol[:, r, one] = 2.0 ** -8 * np.abs(y[:, r, one]) + size
            tol[:, r, two] = 2.0 ** -8 * np.abs(y[:, r, two]) + size
    return y, tol


def packed_attention(q, k, v, ptr, scale):
    """(o, tolerance) [H_q, n_rows, 128]; rows outside ptr are NaN.

    The tolerance is the cache attention's (tests/cache_oracle.py): the result's rounding 2^-8 |o|, the probabilities' 2^-8 of
    sum p |v| in the products and of |o| in their sum, the scores' 32-bit sums and arguments dS, and the sums over the keys."""
    hq, n_rows = q.shape[:2]
    G = hq // k.shape[0]
    o, tol = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    for s in range(len(ptr) - 1):
        a, b = ptr[s], ptr[s + 1]
        if b <= a:
            continue
        n = b - a
        see = np.tril(np.ones((n, n), dtype=bool))
        for h in range(hq):
            kk, vv, qq = k[h // G, a:b], v[h // G, a:b], q[h, a:b]
            x = np.where(see, qq @ kk.T * scale, -np.inf)
            size = np.abs(qq) @ np.abs(kk).T * scale
            top = x.max(1, keepdims=True)
            p = np.exp(x - top)
            p /= p.sum(1, keepdims=True)
            o[h, a:b] = p @ vv
            ds = np.where(see, size * 140 * 2.0 ** -24 + 8 * np.abs(np.where(see, x - top, 0.0)) * 2.0 ** -24, 0.0)
            rel = 2.0 ** -8 + 2 * ds.max(1, keepdims=True) + (n / 16 + 64) * 2.0 ** -24 + 2.0 ** -20
            tol[h, a:b] = 2 * 2.0 ** -8 * np.abs(o[h, a:b]) + rel * (p @ np.abs(vv)) + 1e-30
    return o, tol


def cache_weights(cache, table, seq_len, ptr, q, scale, weights, held):
    """(out, tolerance) [n_seqs, H_kv, width] of an O.Cache; positions that are not written are NaN.

    The tolerance of a weight, the sum of the pairs' p: of each p twice its score's error dS (its own and the normaliser's), the normaliser's sum
    over the keys in 32 bits ((keys / 16 + 64) 2^-24), its logarithm (of size up to 128 + |x|: dS has that), exponentials 2^-21;
    and the sum over the pairs with the old weight, a rounding each."""
    hq = q.shape[0]
    heads = cache.codes.shape[1]
    G = hq // heads
    out, tol = np.full(weights.shape, np.nan), np.full(weights.shape, np.nan)
    width = weights.shape[2]
    for s in range(len(seq_len)):
        r0, r1 = ptr[s], ptr[s + 1]
        n = seq_len[s] + r1 - r0
        k, ok = cache.values(table[s], n, 0)
        w, t = np.zeros((heads, n)), np.zeros((heads, n))
        for h in range(hq):
            if r1 == r0:
                break
            x = q[h, r0:r1] @ k[h // G].T * scale
            size = np.abs(q[h, r0:r1]) @ np.abs(k[h // G]).T * scale
            see = ok[None, :] & (np.arange(n)[None, :] <= (seq_len[s] + np.arange(r1 - r0))[:, None])
            x = np.where(see, x, -np.inf)
            top = np.max(x, axis=1, keepdims=True, initial=-np.inf)
            top = np.where(np.isfinite(top), top, 0.0)
            p = np.exp(x - top)
            l = p.sum(1, keepdims=True)
            p = np.divide(p, l, out=np.zeros_like(p), where=l > 0)
            ds = np.where(see, size * 140 * 2.0 ** -24 + 8 * (np.abs(np.where(see, x - top, 0)) + np.abs(top) + 20) * 2.0 ** -24, 0.0)
            w[h // G] += p.sum(0)
            t[h // G] += (p * (2 * ds.max(1, initial=0.0, keepdims=True) + (n / 16 + 64) * 2.0 ** -24 + 2.0 ** -21)).sum(0)
        m = min(n, width)
        old = np.where(np.arange(m) < held[s], weights[s, :, :m], 0.0)
        out[s, :, :m] = old + w[:, :m]
        tol[s, :, :m] = t[:, :m] + ((r1 - r0) * G + 2) * 2.0 ** -24 * (np.abs(old) + w[:, :m]) + 1e-30
    return out, tol


def cache_keep(weights, held, seq_len, keep, cap, sink, recent):
    """kept, count and the weights that move (NaN elsewhere)."""
    n_seqs, heads, width = weights.shape
    kept = np.full((n_seqs, heads, cap), -1, dtype=np.int32)
    count = np.zeros(n_seqs, dtype=np.int32)
    new = np.full(weights.shape, np.nan, dtype=np.float32)
    moved = np.zeros(weights.shape, dtype=bool)
    for s in range(n_seqs):
        n, m = int(seq_len[s]), int(keep[s])
        if not (n <= width and 0 < m < n and m <= cap):
            continue
        count[s] = m
        last = min(recent, m)
        first = min(sink, m - last)
        for h in range(heads):
            w = np.where(np.arange(n) < held[s], weights[s, h, :n], np.float32(0.0))
            rank = sorted(range(first, n - last), key=lambda j: (1 if np.isnan(w[j]) else 0, -w[j] if not np.isnan(w[j]) else 0.0, j))
            at = sorted(list(range(first)) + rank[:m - first - last] + list(range(n - last, n)))
            kept[s, h, :m] = at
            new[s, h, :m] = w[at]
            moved[s, h, :m] = True
    return kept, count, new, moved


def cache_gather(cache, table, kept, count, new_table):
    """The pages of new_table in an O.Cache written."""
    n_pages, heads = cache.codes.shape[:2]
    B = cache.block
    codes, exps = cache.codes.copy(), cache.exp.copy()
    for s in range(len(count)):
        for b in range(-(-int(min(count[s], kept.shape[2])) // B)):
            to = new_table[s, b] if b < new_table.shape[1] else -1
            if not 0 <= to < n_pages:
                continue
            cache.written[to] = True
            for h in range(heads):
                for x in (0, 1):
                    rows = np.zeros((B, D))
                    for i in range(min(B, int(min(count[s], kept.shape[2])) - b * B)):
                        j = int(kept[s, h, b * B + i])
                        page = table[s, j // B] if 0 <= j < table.shape[1] * B else -1
                        if 0 <= page < n_pages:
                            rows[i] = np.nan_to_num(codes[page, h, x, j % B], nan=0.0) * 2.0 ** float(exps[page, h, x])
                    e = O.scale_exponent(rows, cache.fmt)
                    cache.codes[to, h, x] = O.round_codes(rows * 2.0 ** float(-e), cache.fmt)
                    cache.exp[to, h, x] = e
