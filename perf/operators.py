"""The operators of the 8-bit paged K/V cache: what they compute in plain form, the calls that a
program makes of them, and the cases that their speed is measured on.

A cache holds one layer's K and V in pages of `block` tokens for all KV heads: 8-bit codes (e4m3
or int8) with one power-of-two scale per page, KV head and tensor.  A table lists each sequence's
pages.  Operators (`op`):
  attn      attention of new rows over the cached keys: a decode step (one row a sequence), a
            few drafted rows, or a chunk of a prompt over a long history
  append    K and V rows quantised into the pages behind what a sequence already holds
  fork      sequences dropped and forked anew from others, as a beam step does: shared pages are
            counted, a partial last page is copied
  compact   the pages in use moved to the front of the cache
  turnover  finished sequences freed, and pages reserved for the ones that take their slots

A page's bytes per KV head come in tiles of 64 tokens, K then V, in the order in which the
attention's matrix instructions take them (`_k_order` and `_v_order`).
"""
import math
import random

import torch

own = False

D = 128
MAX = {"e4m3": 448.0, "int8": 127.0}
E_MIN = -64
HEADS = [(32, 8), (28, 4), (16, 4), (8, 2), (7, 1), (4, 1), (2, 2)]


def _attn(name, seqs, lo, hi, rows, hq, hkv, fmt="e4m3", block=64, mix=1):
    return dict(name=name, op="attn", seqs=seqs, lo=lo, hi=hi, rows=rows, hq=hq, hkv=hkv, fmt=fmt, block=block, mix=mix)


def _append(name, seqs, lo, hi, rows, hkv, fmt="e4m3", block=64, mix=1):
    return dict(name=name, op="append", seqs=seqs, lo=lo, hi=hi, rows=rows, hkv=hkv, fmt=fmt, block=block, mix=mix)


def listed():
    return [
        # one chat turn being decoded: latency only
        _attn("attn-one-1k", 1, 999, 999, 1, 32, 8),
        # a server's decode step, sequences of very different lengths
        _attn("attn-batch-8k", 48, 300, 8191, 1, 32, 8, mix=2),
        # one long document decoded, 7 query heads a KV head, 128-token pages
        _attn("attn-long-128k", 1, 131071, 131071, 1, 28, 4, fmt="int8", block=128),
        # drafted tokens checked, one to six a sequence
        _attn("attn-draft-3k", 24, 700, 3200, 6, 32, 8, fmt="int8", mix=3),
        # chunks of three prompts over long histories
        _attn("attn-chunk-20k", 3, 15000, 23000, 450, 28, 4, block=128, mix=4),
        # the step's K and V into the cache
        _append("append-step", 64, 100, 8000, 1, 8, mix=5),
        # a long prompt's K and V
        _append("append-prompt-32k", 1, 0, 0, 32768, 8, fmt="int8", block=128),
        # chunks of different lengths, pages half full
        _append("append-ragged", 24, 0, 5000, 700, 4, mix=6),
        # a beam step of 8 requests of 4 beams each
        dict(name="fork-beams", op="fork", parents=8, width=3, lo=1500, hi=4200, hkv=8, fmt="int8", block=64, mix=7),
        # one prompt of 30k tokens sampled 16 times
        dict(name="fork-samples-30k", op="fork", parents=1, width=16, lo=30011, hi=30011, hkv=4, fmt="int8", block=128, mix=8),
        # a cache of 4096 pages, 60 % in use everywhere, gathered at its front
        dict(name="compact-4096", op="compact", pages=4096, used=60, hkv=8, fmt="int8", block=64, mix=9),
        # a batch's finished sequences replaced by new prompts
        dict(name="turnover-256", op="turnover", seqs=256, pages=32768, part=25, lo=200, hi=6000, block=64, mix=10),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    """One more case: lengths and counts on log scales, every head layout, block and format."""
    op = rng.choice(["attn"] * 5 + ["append"] * 3 + ["fork", "fork", "compact", "turnover"])
    hq, hkv = rng.choice(HEADS)
    fmt, block, mix = rng.choice(["e4m3", "int8"]), rng.choice([64, 128]), rng.randrange(1 << 20)
    if op in ("attn", "append"):
        kind = rng.choice(["step", "step", "draft", "chunk"])
        seqs = _log(rng, 1, 4 if kind == "chunk" else 64)
        rows = {"step": 1, "draft": rng.randint(2, 9), "chunk": _log(rng, 40, 450)}[kind]
        hi = _log(rng, 64, min(98304, max(1024, 400000 // (seqs * hkv))))
        lo = _log(rng, 1, hi)
        if kind == "chunk":
            hi = min(hi, 20000 if hq * seqs <= 84 else 6000)
            lo = min(lo, hi)
        case = dict(op=op, seqs=seqs, lo=lo, hi=hi, rows=rows, hq=hq, hkv=hkv, fmt=fmt, block=block, mix=mix)
        if op == "append":
            del case["hq"]
        return case
    if op == "fork":
        lo = _log(rng, 64, 8000)
        return dict(op=op, parents=rng.randint(1, 8), width=rng.randint(1, 6), lo=lo, hi=lo + _log(rng, 1, 2000), hkv=hkv, fmt="int8", block=block, mix=mix)
    if op == "compact":
        return dict(op=op, pages=_log(rng, 64, 3000), used=rng.randint(20, 90), hkv=hkv, fmt="int8", block=block, mix=mix)
    return dict(op=op, seqs=_log(rng, 2, 512), pages=32768, part=rng.randint(5, 60), lo=_log(rng, 64, 400), hi=_log(rng, 500, 4000), block=block, mix=mix)


# What a case fixes by itself: lengths before the call, and rows of the call


def _lens(case):
    r = random.Random(case["mix"])
    n = case["parents"] if case["op"] == "fork" else case["seqs"]
    lens = [r.randint(case["lo"], case["hi"]) for _ in range(n)]
    rows = case.get("rows", 0)
    counts = [rows if rows <= 1 or n == 1 else r.randint(max(1, rows // 6), rows) for _ in range(n)]
    return lens, counts


def _used(case):
    """Which pages of a compact case are in use."""
    r = random.Random(case["mix"])
    return [r.random() * 100 < case["used"] for _ in range(case["pages"])]


def _gone(case):
    """The sequences of a turnover case that end, and the lengths of those that take their slots."""
    r = random.Random(case["mix"] + 1)
    ids = sorted(r.sample(range(case["seqs"]), max(1, case["seqs"] * case["part"] // 100)))
    return ids, [r.randint(case["lo"], case["hi"]) for _ in ids]


# The cache in plain form


def _k_order(x):
    """K codes of tiles [..., 8192] as [..., 64 tokens, 128]: byte (t, half, g, hi, lo, b) is token
    16 hi + 4 t + lo, element 32 g + 16 half + b."""
    lead = x.shape[:-1]
    n = len(lead)
    x = x.reshape(*lead, 4, 2, 4, 4, 4, 16)
    return x.permute(*range(n), n + 3, n, n + 4, n + 2, n + 1, n + 5).reshape(*lead, 64, D)


def _k_bytes(x):
    lead = x.shape[:-2]
    n = len(lead)
    x = x.reshape(*lead, 4, 4, 4, 4, 2, 16)
    return x.permute(*range(n), n + 1, n + 4, n + 3, n, n + 2, n + 5).reshape(*lead, 64 * D)


def _v_order(x):
    """V codes of tiles [..., 8192] as [..., 64 tokens, 128]: byte (dt, g, r, b) is token 16 g + b, element 16 dt + r."""
    lead = x.shape[:-1]
    n = len(lead)
    x = x.reshape(*lead, 8, 4, 16, 16)
    return x.permute(*range(n), n + 1, n + 3, n, n + 2).reshape(*lead, 64, D)


def _v_bytes(x):
    lead = x.shape[:-2]
    n = len(lead)
    x = x.reshape(*lead, 4, 16, 8, 16)
    return x.permute(*range(n), n + 2, n, n + 3, n + 1).reshape(*lead, 64 * D)


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
    return ((e.int() + 127) << 23).view(torch.float32)  # pow() on the GPU is not held to exact powers


def _plain_attn(st):
    case, q, fmt, B = st["case"], st["q"], st["case"]["fmt"], st["case"]["block"]
    pages, scales, table, row_ptr, seq_len = st["pages"], st["scales"], st["table"], st["row_ptr"].long(), st["seq_len"].long()
    S, hkv, G = table.shape[0], case["hkv"], case["hq"] // case["hkv"]
    L, nmax, n_rows = st["max_len"], st["max_rows"], q.shape[1]
    mp = -(-L // B)
    at = table[:, :mp].long().clamp(min=0)
    tiles = pages[at].transpose(1, 2)  # [S, hkv, mp, B/64, 2, 8192]
    sc = scales[at].transpose(1, 2)    # [S, hkv, mp, 2]
    k = _codes_to_f32(_k_order(tiles[..., 0, :]), fmt).reshape(S, hkv, mp, B * D) * sc[..., :1]
    v = _codes_to_f32(_v_order(tiles[..., 1, :]), fmt).reshape(S, hkv, mp, B * D) * sc[..., 1:]
    k, v = k.reshape(S * hkv, mp * B, D)[:, :L], v.reshape(S * hkv, mp * B, D)[:, :L]
    i = torch.arange(nmax, device=q.device)
    rows = (row_ptr[:-1, None] + i).clamp(max=n_rows - 1)
    qp = q[:, rows].float().reshape(hkv, G, S, nmax, D).permute(2, 0, 1, 3, 4).reshape(S * hkv, G * nmax, D)
    s = torch.bmm(qp, k.transpose(1, 2).contiguous()).view(S, hkv, G, nmax, L) * (1.0 / math.sqrt(D))
    see = torch.arange(L, device=q.device) <= (seq_len[:, None] + i)[:, :, None]
    s = s.masked_fill_(~see[:, None, None], -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    o = torch.bmm(p.view(S * hkv, G * nmax, L), v).view(S, hkv, G, nmax, D)
    r = torch.arange(n_rows, device=q.device)
    seq = torch.searchsorted(row_ptr, r, right=True) - 1
    return o[seq, :, :, r - row_ptr[seq]].reshape(n_rows, case["hq"], D).transpose(0, 1).to(torch.bfloat16)


def _plain_append(st):
    case, fmt, B, hkv = st["case"], st["case"]["fmt"], st["case"]["block"], st["case"]["hkv"]
    pages, scales, table, row_ptr, seq_len = st["pages"], st["scales"], st["table"], st["row_ptr"].long(), st["seq_len"].long()
    n_rows, n_pages = st["k"].shape[1], pages.shape[0]
    r = torch.arange(n_rows, device=pages.device)
    seq = torch.searchsorted(row_ptr, r, right=True) - 1
    pos = seq_len[seq] + r - row_ptr[seq]
    page, slot = table[seq, pos // B].long(), pos % B
    x = torch.stack((st["k"], st["v"])).float()  # [2, hkv, n_rows, D]
    amax = torch.zeros(n_pages, 2, hkv, device=x.device).index_reduce_(0, page, x.abs().amax(-1).permute(2, 0, 1), "amax")
    e = _exponent(amax, fmt).transpose(1, 2)  # [n_pages, hkv, 2]
    # a sequence's page that is partly full: its scale never shrinks, its codes are rounded again under the new one
    part = torch.nonzero((seq_len % B > 0) & (row_ptr[1:] > row_ptr[:-1]))[:, 0]
    p0 = table[part, seq_len[part] // B].long()
    e_old = (torch.frexp(scales[p0])[1] - 1).to(e.dtype)
    e[p0] = torch.maximum(e[p0], e_old)
    codes = _codes_to_f32(pages[p0], fmt) * _two_to(e_old - e[p0]).view(-1, hkv, 1, 2, 1)
    pages[p0] = _f32_to_codes(codes, fmt)
    scales[page] = _two_to(e[page])
    new = _f32_to_codes(x * _two_to(-e[page]).permute(2, 1, 0).unsqueeze(-1), fmt)  # [2, hkv, n_rows, D]
    t, d = (slot % 64)[:, None], torch.arange(D, device=x.device)
    k_at = (((t // 4 % 4 * 2 + d // 16 % 2) * 4 + d // 32) * 16 + t // 16 * 4 + t % 4) * 16 + d % 16
    v_at = ((d // 16 * 4 + t // 16) * 16 + d % 16) * 16 + t % 16
    base = (page * hkv)[None, :, None] + torch.arange(hkv, device=x.device)[:, None, None]
    base = ((base * (B // 64) + (slot // 64)[None, :, None]) * 2) * (64 * D)
    flat = pages.view(-1)
    flat[(base + k_at).reshape(-1)] = new[0].reshape(-1)
    flat[(base + 64 * D + v_at).reshape(-1)] = new[1].reshape(-1)
    return pages, scales


# The pages' bookkeeping in plain form: pool = uses of each page, then one bit a page that is in use


def _pool_of(ref):
    n = ref.numel()
    bits = torch.zeros(-(-n // 32) * 32, dtype=torch.int64, device=ref.device)
    bits[:n] = ref > 0
    words = (bits.view(-1, 32) << torch.arange(32, device=ref.device)).sum(1)
    return torch.cat((ref.int(), words.to(torch.int32)))


def _plain_free(ref, table, seq_len, ids):
    rows = table[ids]
    ref.index_add_(0, rows.clamp(min=0).flatten(), -(rows >= 0).flatten().to(ref.dtype))
    table[ids] = -1
    seq_len[ids] = 0


def _free_pages(ref):
    return torch.argsort((ref > 0).int(), stable=True)


def _plain_turnover(st):
    n, B = st["case"]["pages"], st["case"]["block"]
    pool, table, seq_len, count = st["pool"], st["table"], st["seq_len"], st["counts"].long()
    ref = pool[:n].clone()
    _plain_free(ref, table, seq_len, st["ids"].long())
    slot = torch.arange(table.shape[1], device=table.device)
    lens = seq_len.long()
    last = -(-(lens + count) // B)
    fits = (count > 0) & (last <= table.shape[1])
    lack = (slot >= (lens // B)[:, None]) & (slot < last[:, None]) & (table < 0) & fits[:, None]
    need = lack.sum(1)
    granted = fits & (need.cumsum(0) <= (ref == 0).sum())
    take = lack & granted[:, None]
    rank = take.flatten().long().cumsum(0).view(take.shape) - 1
    got = _free_pages(ref)[rank.clamp(min=0)]
    table.copy_(torch.where(take, got.int(), table))
    ref.index_add_(0, got.flatten(), take.flatten().to(ref.dtype))
    pool.copy_(_pool_of(ref))
    return table, seq_len, pool, torch.where(granted, count, 0).int()


def _plain_fork(st):
    n, B = st["pages"].shape[0], st["case"]["block"]
    pool, table, seq_len, src, dst = st["pool"], st["table"], st["seq_len"], st["src"].long(), st["dst"].long()
    pages, scales = st["pages"], st["scales"]
    ref = pool[:n].clone()
    _plain_free(ref, table, seq_len, dst)
    lens = seq_len[src].long()
    slot = torch.arange(table.shape[1], device=table.device)
    share = slot < (lens // B)[:, None]
    rows = table[src]
    ref.index_add_(0, rows.clamp(min=0).flatten().long(), share.flatten().to(ref.dtype))
    part = lens % B > 0
    fresh = _free_pages(ref)[part.long().cumsum(0).sub(1).clamp(min=0)].int()
    tail = part[:, None] & (slot == (lens // B)[:, None])
    old = rows.gather(1, (lens // B).clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    table[dst] = torch.where(share, rows, torch.where(tail, fresh[:, None], -1))
    seq_len[dst] = lens.int()
    ref.index_add_(0, fresh.long(), part.to(ref.dtype))
    copies = torch.where(part[:, None], torch.stack((old, fresh), 1), -1)
    of, to = copies[part].long().unbind(1)
    pages[to], scales[to] = pages[of], scales[of]
    pool.copy_(_pool_of(ref))
    return table, seq_len, pool, copies, _held(pages, st["case"]), scales


def _plain_compact(st):
    n, pages, scales = st["case"]["pages"], st["pages"], st["scales"]
    ref, table = st["pool"][:n].clone(), st["table"].clone()
    in_use = ref > 0
    page = torch.arange(n, device=ref.device)
    front = page < in_use.sum()
    holes, movers = torch.nonzero(front & ~in_use)[:, 0], torch.nonzero(~front & in_use)[:, 0]
    home = page.clone()
    home[movers] = holes
    table = torch.where(table >= 0, home[table.clamp(min=0).long()].int(), table)
    ref[holes] = ref[movers]
    ref[movers] = 0
    pages[holes], scales[holes] = pages[movers], scales[movers]
    moves = torch.full((max(1, n // 2), 2), -1, dtype=torch.int32, device=ref.device)
    moves[:holes.numel()] = torch.stack((movers, holes), 1).int()
    count = torch.full((1,), holes.numel(), dtype=torch.int32, device=ref.device)
    return table, _pool_of(ref), moves, count, _held(pages, st["case"]), scales


def _held(pages, case):
    """The pages' codes as the values that they stand for, under the scales that come with them."""
    return pages.view(torch.float8_e4m3fn if case["fmt"] == "e4m3" else torch.int8)


# The inputs


def _rows(gen, heads, n, gain):
    """bf16 rows: normal, a few elements of a head larger throughout, as keys have them."""
    x = torch.randn(heads, n, D, generator=gen, device="cuda")
    big = 1.0 + gain * (torch.rand(heads, 1, D, generator=gen, device="cuda") > 0.97)
    return (x * big).to(torch.bfloat16)


def _table(gen, lens, block, spare=0):
    """Pages at random places for sequences of these lengths; -1 behind them."""
    need = [-(-n // block) for n in lens]
    width = max(max(need), 1)
    total = sum(need)
    place = torch.randperm(total + spare, generator=gen, device="cuda", dtype=torch.int32)
    start = torch.tensor([0] + need, device="cuda").cumsum(0)[:-1]
    slot = torch.arange(width, device="cuda")
    at = (start[:, None] + slot).clamp(max=max(total - 1, 0))
    return torch.where(slot < torch.tensor(need, device="cuda")[:, None], place[at], -1).contiguous(), total + spare


def _fill(gen, n_pages, hkv, fmt, block):
    """Every page full of quantised rows."""
    tiles = block // 64
    pages = torch.empty(n_pages, hkv, tiles, 2, 64 * D, dtype=torch.uint8, device="cuda")
    scales = torch.empty(n_pages, hkv, 2, device="cuda")
    step = max(1, (1 << 25) // (hkv * block * D))
    for p in range(0, n_pages, step):
        m = min(step, n_pages - p)
        for x in (0, 1):
            rows = _rows(gen, hkv, m * block, 3.0 if x == 0 else 0.0).float().view(hkv, m, block, D).transpose(0, 1)
            e = _exponent(rows.abs().amax((2, 3)), fmt)
            codes = _f32_to_codes(rows * _two_to(-e)[..., None, None], fmt).view(m, hkv, tiles, 64, D)
            pages[p:p + m, :, :, x] = _k_bytes(codes) if x == 0 else _v_bytes(codes)
            scales[p:p + m, :, x] = _two_to(e)
    return pages, scales


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    op, block = case["op"], case["block"]
    st = dict(case=case)
    if op in ("attn", "append"):
        lens, counts = _lens(case)
        st["table"], n_pages = _table(gen, [a + b for a, b in zip(lens, counts)], block, spare=3)
        st["pages"], st["scales"] = _fill(gen, n_pages, case["hkv"], case["fmt"], block)
        st["seq_len"] = _ints(lens)
        st["row_ptr"] = _ints([sum(counts[:i]) for i in range(len(counts) + 1)])
        st["max_len"], st["max_rows"] = max(a + b for a, b in zip(lens, counts)), max(counts)
        if op == "attn":
            st["q"] = _rows(gen, case["hq"], sum(counts), 0.0)
        else:
            st["k"], st["v"] = _rows(gen, case["hkv"], sum(counts), 3.0), _rows(gen, case["hkv"], sum(counts), 0.0)
    elif op == "fork":
        lens, _ = _lens(case)
        n = len(lens)
        kids = n * case["width"]
        table, n_pages = _table(gen, lens, block, spare=kids + 5)
        st["table"] = torch.cat((table, torch.full((kids, table.shape[1]), -1, dtype=torch.int32, device="cuda")))
        st["seq_len"] = _ints(lens + [0] * kids)
        st["src"] = _ints([i % n for i in range(kids)])
        st["dst"] = _ints([n + i for i in range(kids)])
        st["pages"], st["scales"] = _fill(gen, n_pages, case["hkv"], case["fmt"], block)
        ref = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
        ref[table[table >= 0].long()] = 1
        st["pool"] = _pool_of(ref)
    elif op == "compact":
        ref = _ints([int(u) for u in _used(case)])
        at = torch.nonzero(ref)[:, 0].int()
        at = at[torch.randperm(at.numel(), generator=gen, device="cuda")]
        seqs = 16
        table = torch.full((seqs * -(-max(1, at.numel()) // seqs),), -1, dtype=torch.int32, device="cuda")
        table[:at.numel()] = at
        st["table"] = table.view(seqs, -1).contiguous()
        ref[at[::3].long()] += 1  # pages that a second table would hold too
        st["pool"] = _pool_of(ref)
        st["pages"], st["scales"] = _fill(gen, case["pages"], case["hkv"], case["fmt"], block)
    else:
        lens, _ = _lens(case)
        ids, new = _gone(case)
        wide = -(-case["hi"] // block)
        table, n_pages = _table(gen, lens, block, spare=max(0, case["pages"] - sum(-(-n // block) for n in lens)))
        st["table"] = torch.full((len(lens), wide), -1, dtype=torch.int32, device="cuda")
        st["table"][:, :table.shape[1]] = table
        ref = torch.zeros(case["pages"], dtype=torch.int32, device="cuda")
        ref[table[table >= 0].long()] = 1
        st["pool"] = _pool_of(ref)
        st["seq_len"] = _ints(lens)
        st["ids"] = _ints(ids)
        counts = [0] * len(lens)
        for i, n in zip(ids, new):
            counts[i] = n
        st["counts"] = _ints(counts)
    if own:
        from paper_2609_01925_amd import crisp as C
        if "pages" in st:
            st["cache"] = C.Cache(st["pages"], st["scales"], C.CACHE_E4M3 if case["fmt"] == "e4m3" else C.CACHE_INT8)
        if op == "attn":
            st["ws"] = C.cache_workspace(st["cache"], case["hq"], st["table"].shape[0], st["q"].shape[1])
    return st


def run(st):
    op = st["case"]["op"]
    if not own:
        plain = {"attn": _plain_attn, "fork": _plain_fork, "compact": _plain_compact, "turnover": _plain_turnover}
        if op in plain:
            return plain[op](st)
        pages, scales = _plain_append(st)
        return _held(pages, st["case"]), scales
    from paper_2609_01925_amd import crisp as C
    table, block = st["table"], st["case"]["block"]
    if op == "attn":
        return C.crisp_cache_attn(st["cache"], table, st["seq_len"], st["row_ptr"], st["q"], ws=st["ws"])
    if op == "append":
        C.crisp_cache_append(st["cache"], table, st["seq_len"], st["row_ptr"], st["k"], st["v"])
        return _held(st["pages"], st["case"]), st["scales"]
    if op == "fork":
        C.crisp_pool_free(st["pool"], table, st["seq_len"], st["dst"])
        copies = C.crisp_pool_fork(st["pool"], block, table, st["seq_len"], st["src"], st["dst"])
        C.crisp_cache_copy(st["cache"], copies)
        return table, st["seq_len"], st["pool"], copies, _held(st["pages"], st["case"]), st["scales"]
    if op == "compact":
        pool, table = st["pool"].clone(), table.clone()
        moves, count = C.crisp_pool_compact(pool, table)
        C.crisp_cache_copy(st["cache"], moves, count)
        return table, pool, moves, count, _held(st["pages"], st["case"]), st["scales"]
    C.crisp_pool_free(st["pool"], table, st["seq_len"], st["ids"])
    granted = C.crisp_pool_reserve(st["pool"], block, table, st["seq_len"], st["counts"])
    return table, st["seq_len"], st["pool"], granted


def work(case):
    op, block = case["op"], case["block"]
    if op in ("attn", "append"):
        lens, counts = _lens(case)
        rows = sum(counts)
        if op == "attn":
            keys = sum(a + b for a, b in zip(lens, counts))
            seen = sum(b * a + b * (b + 1) // 2 for a, b in zip(lens, counts))
            return {"bytes": 2.0 * D * case["hkv"] * keys + 4.0 * D * case["hq"] * rows, "flops": 4.0 * D * case["hq"] * seen}
        return {"bytes": 6.0 * D * case["hkv"] * rows, "flops": 4.0 * D * case["hkv"] * rows}
    page = 2.0 * D * block * case.get("hkv", 0)
    if op == "fork":
        lens, _ = _lens(case)
        kids = sum(case["width"] for n in lens if n % block)
        slots = case["width"] * sum(-(-n // block) for n in lens)
        return {"bytes": 2 * page * kids + 16.0 * slots, "flops": 0.0}
    if op == "compact":
        used = _used(case)
        moved = sum(not u for u in used[:sum(used)])
        return {"bytes": 2 * page * moved + 8.0 * sum(used) + case["pages"] / 4, "flops": 0.0}
    ids, new = _gone(case)
    lens, _ = _lens(case)
    slots = sum(-(-n // block) for n in new) + sum(-(-lens[i] // block) for i in ids)
    return {"bytes": 16.0 * slots + case["pages"] / 4, "flops": 0.0}


# The definitions in 64 bits


def _power(e):
    """2^e in 64 bits from a table of the host's exact powers, |e| <= 200."""
    return torch.tensor([2.0 ** i for i in range(-200, 201)], dtype=torch.float64, device=e.device)[e.long() + 200]


def _e4m3_value(byte):
    """The value of an e4m3 code by its fields: 1 sign, 4 exponent (bias 7), 3 mantissa bits."""
    byte = byte.long()
    exp, man = (byte >> 3) & 15, (byte & 7).double()
    size = torch.where(exp > 0, (1 + man / 8) * _power(exp - 7), man / 8 * 2.0 ** -6)
    return torch.where(byte >= 128, -size, size)


def _round_e4m3(x):
    """The nearest e4m3 value, ties to even; |x| <= 448."""
    step = _power(torch.frexp(x.abs().clamp(min=2.0 ** -6))[1] - 4)
    return torch.round(x / step) * step


def _value(byte, fmt):
    return _e4m3_value(byte) if fmt == "e4m3" else byte.view(torch.int8).double()


def _place(token, d, which, block):
    """Byte of a token's element d within one head's part of a page."""
    t = token % 64
    if which == 0:
        at = (t // 4 % 4) * 2048 + (d // 16 % 2) * 1024 + (d // 32) * 256 + (t // 16) * 64 + (t % 4) * 16 + d % 16
    else:
        at = (d // 16) * 1024 + (t // 16) * 256 + (d % 16) * 16 + t % 16
    return token // 64 * 16384 + which * 8192 + at


def _exact_attn(case, st):
    lens, counts = _lens(case)
    B, G = case["block"], case["hq"] // case["hkv"]
    d = torch.arange(D, device="cuda")
    out, first = torch.empty(case["hq"], sum(counts), D, dtype=torch.float64, device="cuda"), 0
    for s, (n, c) in enumerate(zip(lens, counts)):
        pos = torch.arange(n + c, device="cuda")
        page = st["table"][s, pos // B].long()
        for h in range(case["hkv"]):
            flat = st["pages"][:, h].reshape(st["pages"].shape[0], -1)
            kv = []
            for x in (0, 1):
                byte = flat[page[:, None], _place((pos % B)[:, None], d, x, B)]
                kv.append(_value(byte, case["fmt"]) * st["scales"][page, h, x].double()[:, None])
            q = st["q"][h * G:(h + 1) * G, first:first + c].double()
            logits = (q.reshape(-1, D) @ kv[0].T / math.sqrt(D)).view(G, c, -1)
            hidden = pos[None, :] > (n + torch.arange(c, device="cuda"))[:, None]
            p = torch.softmax(logits.masked_fill(hidden, -math.inf), -1)
            out[h * G:(h + 1) * G, first:first + c] = (p.view(G * c, -1) @ kv[1]).view(G, c, D)
        first += c
    return out


def _exact_append(case, st):
    lens, counts = _lens(case)
    B, fmt, top = case["block"], case["fmt"], MAX[case["fmt"]]
    pages, scales = _value(st["pages"], fmt), st["scales"].double()
    n_pages, hkv = pages.shape[:2]
    flat = pages.view(n_pages, hkv, -1)
    d, first = torch.arange(D, device="cuda"), 0
    rounded = _round_e4m3 if fmt == "e4m3" else torch.round
    for s, (n, c) in enumerate(zip(lens, counts)):
        where = st["table"][s].tolist()
        for b in range(n // B, (n + c - 1) // B + 1):
            a, z = max(n, b * B), min(n + c, (b + 1) * B)
            for x, rows in ((0, st["k"]), (1, st["v"])):
                new = rows[:, first + a - n:first + z - n].double()
                size = new.abs().amax((1, 2))
                powers = _power(torch.arange(E_MIN, 128, device="cuda"))
                e = E_MIN + (size[:, None] > top * powers).sum(1)
                if a > b * B:
                    before = torch.frexp(scales[where[b], :, x])[1] - 1
                    e = torch.maximum(e, before)
                    at = _place(torch.arange(B, device="cuda")[:, None], d, x, B).flatten()
                    flat[where[b]][:, at] = rounded(flat[where[b]][:, at] * _power(before - e)[:, None])
                at = _place(torch.arange(a - b * B, z - b * B, device="cuda")[:, None], d, x, B).flatten()
                flat[where[b]][:, at] = rounded(new * _power(-e)[:, None, None]).flatten(1)
                scales[where[b], :, x] = _power(e)
        first += c
    return (pages if fmt == "e4m3" else None), scales


def exact(case, seed):
    if case["op"] == "turnover":
        return None
    st = prepare(case, seed)
    if case["op"] == "attn":
        return _exact_attn(case, st)
    if case["op"] == "append":
        return _exact_append(case, st)
    scales = st["scales"].double()
    if case["op"] == "fork":
        lens, _ = _lens(case)
        free = [p for p, r in enumerate(st["pool"][:scales.shape[0]].tolist()) if r == 0]
        for s in st["src"].tolist():
            if lens[s] % case["block"]:
                scales[free.pop(0)] = scales[st["table"][s, lens[s] // case["block"]].item()]
        return None, None, None, None, None, scales
    used = _used(case)
    total = sum(used)
    holes = [p for p in range(total) if not used[p]]
    movers = [p for p in range(total, len(used)) if used[p]]
    moved = scales.clone()
    for of, to in zip(movers, holes):
        moved[to] = scales[of]
    return None, None, None, None, None, moved
