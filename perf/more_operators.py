"""Operators beside the sparse prefill and the 8-bit paged K/V cache: what they compute in plain
form, the calls that a program makes of them, and the cases that their speed is measured on.

Operators (`op`):
  rope      rotary positions on q and k, from the projection's output into the layout that the
            attention takes: steps, prompts, part of a head, five rules for the frequencies
  packed    causal attention over whole prompts of different lengths, packed behind one another
  weights   the attention weight that each cached token gets from new rows, summed over the rows and
            the query heads of its KV head, added to what it has: what eviction goes by
  keep      which tokens of each sequence and KV head stay: the first few, the last ones and those of
            the largest weight; and these tokens' weights
  gather    the tokens that stay moved to pages of their own, quantised anew

A page's bytes per KV head come in tiles of 64 tokens, K then V, in the order of `_place`.
"""
import math
import random

import torch

own = False

D = 128
MAX = {"e4m3": 448.0, "int8": 127.0}
E_MIN = -64
HEADS = [(32, 8), (28, 4), (8, 2), (7, 1), (4, 1), (2, 2)]
SCALINGS = ["plain", "linear", "base", "bands", "ramp"]


def _rope(name, seqs, lo, hi, far, hq, hkv, dim=128, layout="half", scaling="plain", mix=1):
    return dict(name=name, op="rope", seqs=seqs, lo=lo, hi=hi, far=far, hq=hq, hkv=hkv, dim=dim, layout=layout, scaling=scaling, mix=mix)


def _packed(name, seqs, lo, hi, hq, hkv, fused=True, mix=1):
    return dict(name=name, op="packed", seqs=seqs, lo=lo, hi=hi, hq=hq, hkv=hkv, fused=fused, mix=mix)


def _weights(name, seqs, lo, hi, rows, hq, hkv, fmt="e4m3", block=64, add=True, mix=1):
    return dict(name=name, op="weights", seqs=seqs, lo=lo, hi=hi, rows=rows, hq=hq, hkv=hkv, fmt=fmt, block=block, add=add, mix=mix)


def _keep(name, seqs, lo, hi, keep, hkv, mix=1):
    return dict(name=name, op="keep", seqs=seqs, lo=lo, hi=hi, keep=keep, sink=4, recent=min(64, keep // 4), hkv=hkv, mix=mix)


def _gather(name, seqs, lo, hi, keep, hkv, fmt="e4m3", block=64, mix=1):
    return dict(name=name, op="gather", seqs=seqs, lo=lo, hi=hi, keep=keep, hkv=hkv, fmt=fmt, block=block, mix=mix)


def listed():
    return [
        # one step of a batch: a row a sequence, latency only
        _rope("rope-step", 64, 1, 1, 100000, 32, 8),
        # a long prompt's q and k
        _rope("rope-prompt-32k", 1, 32768, 32768, 0, 32, 8, scaling="bands", mix=2),
        # chunks of several prompts, half of each head rotated, neighbouring elements in pairs, far positions
        _rope("rope-ragged-far", 24, 1, 700, 1000000, 28, 4, dim=64, layout="interleaved", scaling="ramp", mix=3),
        # a dozen short prompts that arrived together
        _packed("packed-short", 12, 1, 90, 32, 8, mix=4),
        # a batch of prompts of all lengths, 7 query heads a KV head
        _packed("packed-ragged-2k", 16, 40, 2500, 28, 4, fused=False, mix=5),
        # three documents
        _packed("packed-12k", 3, 5000, 12000, 32, 8, mix=6),
        # a decoding step's weights added to those so far
        _weights("weights-step-8k", 48, 300, 8191, 1, 32, 8, mix=7),
        # a long prompt seen by its last 32 rows
        _weights("weights-window-128k", 1, 131000, 131000, 32, 28, 4, fmt="int8", block=128, add=False, mix=8),
        # a batch held to 1024 tokens a sequence
        _keep("keep-batch-4k", 32, 700, 4100, 1024, 8, mix=9),
        # a long document's tokens cut to a sixth
        _keep("keep-100k", 1, 100003, 100003, 16384, 4, mix=10),
        # the same two moved
        _gather("gather-batch-4k", 32, 700, 4100, 1024, 8, mix=11),
        _gather("gather-100k", 1, 100003, 100003, 16384, 4, fmt="int8", block=128, mix=12),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    """One more case: lengths and counts on log scales, every head layout, block, format and rule."""
    op = rng.choice(["rope"] * 3 + ["packed"] * 3 + ["weights"] * 3 + ["keep"] * 2 + ["gather"] * 2)
    hq, hkv = rng.choice(HEADS)
    fmt, block, mix = rng.choice(["e4m3", "int8"]), rng.choice([64, 128]), rng.randrange(1 << 20)
    if op == "rope":
        seqs = _log(rng, 1, 256)
        hi = rng.choice([1, _log(rng, 1, max(1, 32768 // seqs))])
        return dict(op=op, seqs=seqs, lo=_log(rng, 1, hi), hi=hi, far=rng.choice([0, 30000, 1000000]), hq=hq, hkv=hkv, dim=rng.choice([32, 64, 96, 128]),
                    layout=rng.choice(["half", "interleaved"]), scaling=rng.choice(SCALINGS), mix=mix)
    if op == "packed":
        seqs = _log(rng, 1, 64)
        hi = _log(rng, 2, int(12000 / math.sqrt(max(seqs, 2) / 2)))
        return dict(op=op, seqs=seqs, lo=_log(rng, 1, hi), hi=hi, hq=hq, hkv=hkv, fused=rng.random() < 0.5, mix=mix)
    if op == "weights":
        kind = rng.choice(["step", "step", "draft", "window"])
        seqs = _log(rng, 1, 4 if kind == "window" else 64)
        rows = {"step": 1, "draft": rng.randint(2, 9), "window": _log(rng, 16, 64)}[kind]
        hi = _log(rng, 64, min(131072, max(1024, (2000000 if kind != "window" else 300000) // (seqs * max(rows, hkv)))))
        return dict(op=op, seqs=seqs, lo=_log(rng, 1, hi), hi=hi, rows=rows, hq=hq, hkv=hkv, fmt=fmt, block=block, add=rng.random() < 0.5, mix=mix)
    seqs = _log(rng, 1, 48)
    hi = _log(rng, 64, min(100000, max(1024, 1000000 // (seqs * hkv))))
    case = dict(op=op, seqs=seqs, lo=_log(rng, 1, hi), hi=hi, keep=max(1, int(hi * rng.uniform(0.05, 0.8))), hkv=hkv, mix=mix)
    if op == "keep":
        return dict(case, sink=rng.choice([0, 1, 4, 16]), recent=_log(rng, 1, 256))
    return dict(case, fmt=fmt, block=block)


# What a case fixes by itself: lengths, rows of the call, frequencies


def _lens(case):
    r = random.Random(case["mix"])
    return [r.randint(case["lo"], case["hi"]) for _ in range(case["seqs"])]


def _counts(case):
    """Rows of a weights case's sequences."""
    r, rows = random.Random(case["mix"] + 1), case["rows"]
    return [rows if rows == 1 or case["seqs"] == 1 else r.randint(max(1, rows // 6), rows) for _ in range(case["seqs"])]


def _ptr(counts):
    return [sum(counts[:i]) for i in range(len(counts) + 1)]


def _kept_of(case, n):
    """How many of a sequence's n tokens are chosen: keep of them, or none where it has no more than that."""
    return case["keep"] if n > case["keep"] else 0


# A long context's rules: base 10000 (or 500000), 8 times as long as the 8192 tokens it stems from
BASE, FACTOR, ORIGINAL, LOW, HIGH, FAST, SLOW = 500000.0, 8.0, 8192.0, 1.0, 4.0, 32.0, 1.0


def _frequencies(case):
    """Angle a token of each pair of elements (64 bits), and the gain of all rotated elements."""
    dim, rule = case["dim"], case["scaling"]
    i = torch.arange(dim // 2, dtype=torch.float64)
    base = BASE * FACTOR ** (dim / (dim - 2)) if rule == "base" else BASE
    f = base ** (-2.0 * i / dim)
    if rule == "linear":
        f = f / FACTOR
    if rule == "bands":  # by the turns that a pair makes in the original length: few, many, between
        x = ((ORIGINAL * f / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0, 1)
        f = f * (x + (1 - x) / FACTOR)
    if rule == "ramp":  # along the pairs, between those that make `fast` and `slow` turns in the original length
        at = [dim * math.log(ORIGINAL / (2 * math.pi * n)) / (2 * math.log(BASE)) for n in (FAST, SLOW)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), dim - 1)
        x = 1 - ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        f = f * (x + (1 - x) / FACTOR)
    return f, (0.1 * math.log(FACTOR) + 1.0 if rule == "ramp" else 1.0)


# Rotary positions


def _rows_of(st, n_rows):
    """Sequence of each row, and the row's place in it."""
    ptr = st["row_ptr"].long()
    r = torch.arange(n_rows, device=ptr.device)
    seq = torch.searchsorted(ptr, r, right=True) - 1
    return seq, r - ptr[seq]


def _plain_rope(st):
    case = st["case"]
    dim = case["dim"]
    seq, i = _rows_of(st, st["q"].shape[1])
    a = (st["start"].long()[seq] + i).double()[:, None] * st["angle"]
    cos, sin = (torch.cos(a) * st["gain"]).float(), (torch.sin(a) * st["gain"]).float()

    def turn(x):
        x = x.float()
        y = x.clone()
        if case["layout"] == "half":
            x1, x2 = x[..., :dim // 2], x[..., dim // 2:dim]
            y[..., :dim // 2], y[..., dim // 2:dim] = x1 * cos - x2 * sin, x2 * cos + x1 * sin
        else:
            x1, x2 = x[..., 0:dim:2], x[..., 1:dim:2]
            y[..., 0:dim:2], y[..., 1:dim:2] = x1 * cos - x2 * sin, x2 * cos + x1 * sin
        return y.to(torch.bfloat16)

    return turn(st["q"]), turn(st["k"])


def _exact_rope(case, st):
    first = 0
    out = [torch.empty(x.shape, dtype=torch.float64, device="cuda") for x in (st["q"], st["k"])]
    f, gain = _frequencies(case)
    half = case["dim"] // 2
    for start, n in zip(st["start"].tolist(), _lens(case)):
        at = torch.arange(start, start + n, dtype=torch.float64, device="cuda")
        turn = torch.polar(torch.full((n, half), gain, dtype=torch.float64, device="cuda"), torch.outer(at, f.cuda()))
        for x, y in zip((st["q"], st["k"]), out):
            x, y = x[:, first:first + n].double(), y[:, first:first + n]
            y[..., case["dim"]:] = x[..., case["dim"]:]
            pairs = x[..., :case["dim"]].unflatten(-1, (2, half) if case["layout"] == "half" else (half, 2))
            pairs = pairs.transpose(-1, -2) if case["layout"] == "half" else pairs
            z = torch.view_as_real(torch.complex(pairs[..., 0], pairs[..., 1]) * turn)
            y[..., :case["dim"]] = (z.transpose(-1, -2) if case["layout"] == "half" else z).flatten(-2)
        first += n
    return tuple(out)


# Attention over packed prompts


def _plain_packed(st):
    case, q, k, v = st["case"], st["q"], st["k"], st["v"]
    hkv, G = case["hkv"], case["hq"] // case["hkv"]
    o = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
    first = 0
    for n in st["lens"]:  # a sequence's scores are as much as is formed at once
        at = slice(first, first + n)
        qs = q[:, at].float().reshape(hkv, G * n, D)
        s = torch.bmm(qs, k[:, at].float().transpose(1, 2).contiguous()).view(hkv, G, n, n).mul_(1.0 / math.sqrt(D))
        s.masked_fill_(torch.ones(n, n, dtype=torch.bool, device=q.device).triu_(1), -math.inf)
        p = s.sub_(s.amax(-1, keepdim=True)).exp_()
        p = p.div_(p.sum(-1, keepdim=True))
        o[:, at] = torch.bmm(p.view(hkv, G * n, n), v[:, at].float().contiguous()).view(case["hq"], n, D).to(torch.bfloat16)
        first += n
    return o


def _exact_packed(case, st):
    G, first = case["hq"] // case["hkv"], 0
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    for n in _lens(case):
        at = slice(first, first + n)
        after = torch.ones(n, n, dtype=torch.bool, device="cuda").triu_(1)
        for h in range(case["hq"]):
            k, v = st["k"][h // G, at].double(), st["v"][h // G, at].double()
            s = (st["q"][h, at].double() @ k.T / math.sqrt(D)).masked_fill_(after, -math.inf)
            out[h, at] = torch.softmax(s, -1) @ v
        first += n
    return out


# The cache


def _codes_to_f32(x, fmt):
    return x.view(torch.float8_e4m3fn if fmt == "e4m3" else torch.int8).float()


def _f32_to_codes(x, fmt):
    return (x.to(torch.float8_e4m3fn) if fmt == "e4m3" else torch.round(x).to(torch.int8)).view(torch.uint8)


def _exponent(amax, fmt):
    """The smallest e >= E_MIN with amax <= MAX 2^e."""
    m, x = torch.frexp(amax)
    top_m, top_x = math.frexp(MAX[fmt])
    return torch.where(amax > 0, x - top_x + (m > top_m), E_MIN).clamp(min=E_MIN)


def _two_to(e):
    return ((e.int() + 127) << 23).view(torch.float32)


def _place(token, d, which):
    """Byte of a token's element d within one head's part of a page: K (0) or V (1)."""
    t = token % 64
    k_at = (((t // 4 % 4 * 2 + d // 16 % 2) * 4 + d // 32) * 16 + t // 16 * 4 + t % 4) * 16 + d % 16
    v_at = ((d // 16 * 4 + t // 16) * 16 + d % 16) * 16 + t % 16
    return token // 64 * (2 * 64 * D) + which * (64 * D) + (v_at if which else k_at)


def _held(pages, case):
    """The pages' codes as the values that they stand for, under the scales that come with them."""
    return pages.view(torch.float8_e4m3fn if case["fmt"] == "e4m3" else torch.int8)


def _plain_weights(st):
    case, q, fmt, B = st["case"], st["q"], st["case"]["fmt"], st["case"]["block"]
    pages, scales, table, ptr, seq_len = st["pages"], st["scales"], st["table"], st["row_ptr"].long(), st["seq_len"].long()
    S, hkv, G = table.shape[0], case["hkv"], case["hq"] // case["hkv"]
    L, nmax, n_rows, dev = st["max_len"], st["max_rows"], q.shape[1], q.device
    pos, d = torch.arange(L, device=dev), torch.arange(D, device=dev)
    page = table[:, pos // B].long().clamp(min=0)                              # [S, L]
    byte = _place((pos % B)[:, None], d, 0)                                    # [L, D]
    size = pages[0, 0].numel()
    at = ((page[:, None] * hkv + torch.arange(hkv, device=dev)[:, None]) * size)[..., None] + byte
    k = _codes_to_f32(pages.view(-1)[at], fmt) * scales[page].permute(0, 2, 1, 3)[..., :1]
    k = k.reshape(S * hkv, L, D)
    i = torch.arange(nmax, device=dev)
    rows = (ptr[:-1, None] + i).clamp(max=n_rows - 1)
    qp = q[:, rows].float().reshape(hkv, G, S, nmax, D).permute(2, 0, 1, 3, 4).reshape(S * hkv, G * nmax, D)
    s = torch.bmm(qp, k.transpose(1, 2).contiguous()).view(S, hkv, G, nmax, L) * (1.0 / math.sqrt(D))
    see = pos <= (seq_len[:, None] + i)[:, :, None]
    s = s.masked_fill_(~see[:, None, None], -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    there = (i < (ptr[1:] - ptr[:-1])[:, None]).to(p.dtype)                    # rows that the sequence has
    w = (p * there[:, None, None, :, None]).sum((2, 3))
    w = w + torch.where(pos < st["held"][:, None, None], st["weights"][:, :, :L], 0.0)
    seen = pos < (seq_len + ptr[1:] - ptr[:-1])[:, None, None]
    st["out"][:, :, :L] = torch.where(seen, w, st["out"][:, :, :L])
    return st["out"]


def _exact_weights(case, st):
    lens, counts = _lens(case), _counts(case)
    B, G = case["block"], case["hq"] // case["hkv"]
    d, first = torch.arange(D, device="cuda"), 0
    out = st["out"].double()
    for s, (n, c) in enumerate(zip(lens, counts)):
        pos = torch.arange(n + c, device="cuda")
        page = st["table"][s, pos // B].long()
        hidden = pos[None, :] > (n + torch.arange(c, device="cuda"))[:, None]
        for h in range(case["hkv"]):
            byte = st["pages"][:, h].reshape(st["pages"].shape[0], -1)[page[:, None], _place((pos % B)[:, None], d, 0)]
            k = _value(byte, case["fmt"]) * st["scales"][page, h, 0].double()[:, None]
            old = st["weights"][s, h, :n + c].double()
            out[s, h, :n + c] = torch.where(pos < st["held"][s], old, 0.0)
            for g in range(h * G, (h + 1) * G):
                x = (st["q"][g, first:first + c].double() @ k.T / math.sqrt(D)).masked_fill_(hidden, -math.inf)
                out[s, h, :n + c] += torch.softmax(x, -1).sum(0)
        first += c
    return out


def _plain_keep(st):
    case, w, seq_len, keep = st["case"], st["weights"], st["seq_len"].long()[:, None, None], st["keep"].long()[:, None, None]
    pos = torch.arange(w.shape[2], device=w.device)
    count = torch.where(keep < seq_len, keep, 0)
    recent = count.clamp(max=case["recent"])
    sink = (count - recent).clamp(max=case["sink"])
    sure = (pos < sink) | (pos >= seq_len - recent)
    score = torch.where(sure, math.inf, w).masked_fill(pos >= seq_len, -1.0)
    order = torch.argsort(score, dim=-1, descending=True, stable=True)
    chosen = torch.zeros_like(w, dtype=torch.bool).scatter_(2, order, (pos < count).expand_as(order).contiguous())
    cap = case["keep"]
    kept = torch.sort(torch.where(chosen, pos, w.shape[2]), dim=-1)[0][..., :cap]
    there = torch.arange(cap, device=w.device) < count
    new = torch.where(there, w.gather(2, kept.clamp(max=w.shape[2] - 1)), st["new"][..., :cap])
    st["new"][..., :cap] = new
    return torch.where(there, kept, -1).int(), count[:, 0, 0].int(), st["new"]


def _exact_keep(case, st):
    """Only the weights that move are numbers with a fraction."""
    new = st["new"].double().cpu()
    w = st["weights"].double().cpu()
    for s, n in enumerate(_lens(case)):
        m = _kept_of(case, n)
        recent = min(case["recent"], m)
        sink = min(case["sink"], m - recent)
        for h in range(case["hkv"] if m else 0):
            x = w[s, h, :n].tolist()
            best = sorted(range(sink, n - recent), key=lambda j: (-x[j], j))[:m - recent - sink]
            at = list(range(sink)) + sorted(best) + list(range(n - recent, n))
            new[s, h, :m] = w[s, h, at]
    return None, None, new.cuda()


def _plain_gather(st):
    case, fmt, B, hkv = st["case"], st["case"]["fmt"], st["case"]["block"], st["case"]["hkv"]
    pages, scales, kept, dev = st["pages"], st["scales"], st["kept"].long(), st["pages"].device
    cap, d, head = kept.shape[2], torch.arange(D, device=dev), torch.arange(hkv, device=dev)[:, None]
    size, seq = pages[0, 0].numel(), torch.arange(kept.shape[0], device=dev)[:, None, None]
    there = torch.arange(cap, device=dev) < st["count"][:, None, None]
    at = kept.clamp(min=0)
    page = st["table"][seq, at // B].long().clamp(min=0)                       # [S, hkv, cap]
    i = torch.arange(cap, device=dev)
    slots = -(-cap // B)
    to = st["new_table"][:, :slots].long()                                     # [S, slots]
    flat, blank = pages.view(-1), torch.zeros(1, device=dev)
    for x in (0, 1):  # K and V have scales of their own
        byte = ((page * hkv + head) * size)[..., None] + _place((at % B)[..., None], d, x)
        value = _codes_to_f32(flat[byte], fmt) * scales[page, head, x][..., None]
        value = torch.where(there[..., None], value, blank)
        value = torch.nn.functional.pad(value, (0, 0, 0, slots * B - cap)).view(*kept.shape[:2], slots, B, D)
        e = _exponent(value.abs().amax((3, 4)), fmt)                           # [S, hkv, slots]
        codes = _f32_to_codes(value * _two_to(-e)[..., None, None], fmt)
        used = (torch.arange(slots, device=dev) * B < st["count"][:, None]) & (to >= 0)
        n = torch.nonzero(used)
        dst = to[n[:, 0], n[:, 1]]                                             # pages written
        where = ((dst[:, None] * hkv + head[:, 0]) * size)[..., None, None] + _place(torch.arange(B, device=dev)[:, None], d, x)
        flat[where] = codes.permute(0, 2, 1, 3, 4)[n[:, 0], n[:, 1]]
        scales[dst, :, x] = _two_to(e).permute(0, 2, 1)[n[:, 0], n[:, 1]]
    return _held(pages, case), scales


def _power(e):
    """2^e in 64 bits from a table of the host's exact powers, |e| <= 200."""
    return torch.tensor([2.0 ** i for i in range(-200, 201)], dtype=torch.float64, device=e.device)[e.long() + 200]


def _value(byte, fmt):
    """The value of a code, an e4m3 one by its fields: 1 sign, 4 exponent (bias 7), 3 mantissa bits."""
    if fmt == "int8":
        return byte.view(torch.int8).double()
    byte = byte.long()
    exp, man = (byte >> 3) & 15, (byte & 7).double()
    size = torch.where(exp > 0, (1 + man / 8) * _power(exp - 7), man / 8 * 2.0 ** -6)
    return torch.where(byte >= 128, -size, size)


def _rounded(x, fmt):
    """The nearest value of a format, ties to even; |x| <= MAX."""
    if fmt == "int8":
        return torch.round(x)
    step = _power(torch.frexp(x.abs().clamp(min=2.0 ** -6))[1] - 4)
    return torch.round(x / step) * step


def _exact_gather(case, st):
    B, fmt = case["block"], case["fmt"]
    pages, scales = _value(st["pages"], fmt), st["scales"].double()
    src, d = pages.clone().view(*pages.shape[:2], -1), torch.arange(D, device="cuda")
    flat, was = pages.view(*pages.shape[:2], -1), scales.clone()
    for s, n in enumerate(_lens(case)):
        for b in range(-(-_kept_of(case, n) // B)):
            to = int(st["new_table"][s, b])
            for h in range(case["hkv"]):
                at = st["kept"][s, h, b * B:min(_kept_of(case, n), (b + 1) * B)].long()
                of = st["table"][s, at // B].long()
                for x in (0, 1):
                    v = src[of[:, None], h, _place((at % B)[:, None], d, x)] * was[of, h, x][:, None]
                    e = E_MIN + (v.abs().amax() > MAX[fmt] * _power(torch.arange(E_MIN, 128, device="cuda"))).sum()
                    flat[to, h][_place(torch.arange(B, device="cuda")[:, None], d, x)] = 0.0
                    flat[to, h][_place(torch.arange(at.numel(), device="cuda")[:, None], d, x)] = _rounded(v * _power(-e), fmt)
                    scales[to, h, x] = _power(e)
    return (pages if fmt == "e4m3" else None), scales


# The inputs


def _normal(gen, heads, n, gain):
    """bf16 rows: normal, a few elements of a head larger throughout, as keys have them."""
    x = torch.randn(heads, n, D, generator=gen, device="cuda")
    big = 1.0 + gain * (torch.rand(heads, 1, D, generator=gen, device="cuda") > 0.97)
    return (x * big).to(torch.bfloat16)


def _projection(gen, n, hq, hkv, fused):
    """q, k and v of n rows: views of one product's output [n, heads, 128], or a tensor each."""
    parts = [_normal(gen, hq, n, 0.0), _normal(gen, hkv, n, 3.0), _normal(gen, hkv, n, 0.0)]
    if not fused:
        return parts
    return torch.cat([x.transpose(0, 1) for x in parts], 1).contiguous().transpose(0, 1).split([hq, hkv, hkv])


def _table(gen, lens, block, spare=0):
    """Pages at random places for sequences of these lengths, -1 behind them; and the places left over."""
    need = [-(-n // block) for n in lens]
    width, total = max(max(need), 1), sum(need)
    place = torch.randperm(total + spare, generator=gen, device="cuda", dtype=torch.int32)
    start = torch.tensor(_ptr(need), device="cuda")[:-1]
    slot = torch.arange(width, device="cuda")
    at = (start[:, None] + slot).clamp(max=max(total - 1, 0))
    return torch.where(slot < torch.tensor(need, device="cuda")[:, None], place[at], -1).contiguous(), place[total:]


def _fill(gen, n_pages, hkv, fmt, block):
    """Every page full of codes as quantised rows have them: normal, the largest of a page near the top, scales that differ."""
    shape = (n_pages, hkv, block // 64, 2, 64 * D)
    pages = torch.empty(shape, dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // (hkv * block * D))
    for p in range(0, n_pages, step):
        x = torch.randn(min(step, n_pages - p), *shape[1:], generator=gen, device="cuda").mul_(MAX[fmt] / 5.5)
        pages[p:p + step] = _f32_to_codes(x.clamp_(-MAX[fmt], MAX[fmt]), fmt)
    # the codes' deviation times the scale: about one
    top = round(math.log2(5.5 / MAX[fmt]))
    return pages, _two_to(torch.randint(top - 1, top + 1, (n_pages, hkv, 2), generator=gen, device="cuda"))


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _scores(gen, seqs, hkv, width):
    """Accumulated weights: spread over some powers of ten, the first tokens' far above the rest, some equal, some 0."""
    w = torch.exp(2.0 * torch.randn(seqs, hkv, width, generator=gen, device="cuda") - 6.0)
    w[..., :4] += 3.0
    w = torch.where(torch.rand(w.shape, generator=gen, device="cuda") < 0.05, torch.round(w * 1000.0) / 1000.0, w)
    return w.contiguous()


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    op, hkv, lens = case["op"], case["hkv"], _lens(case)
    st = dict(case=case)
    if op in ("rope", "packed"):
        st["row_ptr"] = _ints(_ptr(lens))
        st["q"], st["k"], st["v"] = _projection(gen, sum(lens), case["hq"], hkv, case.get("fused", True))
        if op == "packed":
            st["lens"] = lens
            return st
        r = random.Random(case["mix"] + 2)
        st["start"] = _ints([r.randint(0, case["far"]) for _ in lens])
        f, st["gain"] = _frequencies(case)
        st["angle"] = f.cuda()
        if own:
            from paper_2609_01925_amd import crisp as C
            layout = {"half": C.ROPE_HALF, "interleaved": C.ROPE_INTERLEAVED}[case["layout"]]
            rule = {"plain": C.ROPE_PLAIN, "linear": C.ROPE_LINEAR, "base": C.ROPE_BASE, "bands": C.ROPE_BANDS, "ramp": C.ROPE_RAMP}[case["scaling"]]
            band = {"bands": (LOW, HIGH), "ramp": (SLOW, FAST)}.get(case["scaling"], (0.0, 0.0))
            st["rope"] = C.make_rope(case["dim"], layout, BASE, rule, FACTOR, ORIGINAL, *band)
        return st
    st["seq_len"] = _ints(lens)
    if op == "keep":
        width = -(-max(lens) // 64) * 64
        st["weights"] = _scores(gen, len(lens), hkv, width)
        st["new"] = torch.zeros_like(st["weights"])
        st["held"], st["keep"] = st["seq_len"].clone(), _ints([case["keep"]] * len(lens))
        return st
    block, fmt = case["block"], case["fmt"]
    if op == "weights":
        counts = _counts(case)
        st["table"], left = _table(gen, [a + b for a, b in zip(lens, counts)], block, spare=3)
        st["row_ptr"] = _ints(_ptr(counts))
        st["max_len"], st["max_rows"] = max(a + b for a, b in zip(lens, counts)), max(counts)
        st["weights"] = _scores(gen, len(lens), hkv, st["table"].shape[1] * block)
        st["out"] = torch.zeros_like(st["weights"])
        st["held"] = st["seq_len"].clone() if case["add"] else torch.zeros_like(st["seq_len"])
        st["q"] = _normal(gen, case["hq"], sum(counts), 0.0)
    else:
        m = [_kept_of(case, n) for n in lens]
        slots = -(-case["keep"] // block)
        st["table"], left = _table(gen, lens, block, spare=len(lens) * slots + 3)
        st["new_table"] = left[:len(lens) * slots].view(len(lens), slots).contiguous()
        st["count"] = _ints(m)
        st["kept"] = torch.full((len(lens), hkv, case["keep"]), -1, dtype=torch.int32, device="cuda")
        for s, (n, c) in enumerate(zip(lens, m)):
            if c:
                best = torch.rand(hkv, n, generator=gen, device="cuda").topk(c, dim=-1)[1]
                st["kept"][s] = best.sort(-1)[0].int()
    n_pages = int((st["table"] >= 0).sum()) + left.numel()
    st["pages"], st["scales"] = _fill(gen, n_pages, hkv, fmt, block)
    if own:
        from paper_2609_01925_amd import crisp as C
        st["cache"] = C.Cache(st["pages"], st["scales"], C.CACHE_E4M3 if fmt == "e4m3" else C.CACHE_INT8)
        if op == "weights":
            st["ws"] = C.cache_weights_workspace(st["cache"], case["hq"], len(lens), st["q"].shape[1])
    return st


def run(st):
    case = st["case"]
    op = case["op"]
    if not own:
        return {"rope": _plain_rope, "packed": _plain_packed, "weights": _plain_weights, "keep": _plain_keep, "gather": _plain_gather}[op](st)
    from paper_2609_01925_amd import crisp as C
    if op == "rope":
        return C.crisp_rope(st["rope"], st["start"], st["row_ptr"], st["q"], st["k"])
    if op == "packed":
        return C.crisp_packed_attn(st["row_ptr"], st["q"], st["k"], st["v"])
    if op == "weights":
        return C.crisp_cache_weights(st["cache"], st["table"], st["seq_len"], st["row_ptr"], st["q"], st["weights"], st["held"], out=st["out"], ws=st["ws"])
    if op == "keep":
        kept, count = C.crisp_cache_keep(st["weights"], st["held"], st["seq_len"], st["keep"], case["keep"], case["sink"], case["recent"], new_weights=st["new"])
        return kept, count, st["new"]
    C.crisp_cache_gather(st["cache"], st["table"], st["kept"], st["count"], st["new_table"])
    return _held(st["pages"], case), st["scales"]


def work(case):
    op, hkv, lens = case["op"], case["hkv"], _lens(case)
    rows = sum(lens)
    if op == "rope":
        return {"bytes": 4.0 * D * (case["hq"] + hkv) * rows, "flops": 3.0 * case["dim"] * (case["hq"] + hkv) * rows}
    if op == "packed":
        return {"bytes": 4.0 * D * (case["hq"] + hkv) * rows, "flops": 4.0 * D * case["hq"] * sum(n * (n + 1) // 2 for n in lens)}
    if op == "weights":
        counts = _counts(case)
        keys = sum(a + b for a, b in zip(lens, counts))
        seen = sum(b * a + b * (b + 1) // 2 for a, b in zip(lens, counts))
        return {"bytes": (D + 4.0) * hkv * keys + (4.0 * hkv * rows if case["add"] else 0.0) + 2.0 * D * case["hq"] * sum(counts), "flops": 2.0 * D * case["hq"] * seen}
    m = sum(_kept_of(case, n) for n in lens)
    if op == "keep":
        return {"bytes": 4.0 * hkv * (sum(n for n in lens if _kept_of(case, n)) + 2 * m), "flops": 0.0}
    return {"bytes": hkv * m * (4.0 * D + 4.0), "flops": 0.0}


# The definitions in 64 bits


def exact(case, seed):
    st = prepare(case, seed)
    return {"rope": _exact_rope, "packed": _exact_packed, "weights": _exact_weights, "keep": _exact_keep, "gather": _exact_gather}[case["op"]](case, st)
