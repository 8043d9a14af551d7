"""The 8-bit paged K/V cache through the public binding: appends and scales bit for bit and attention
within counted roundings of the 64-bit oracle (tests/cache_oracle.py), page bookkeeping equal to it;
lengths from none to several pages, ragged batches, holes, strides, streams and graphs."""
import math
import sys

import numpy as np
import pytest
import torch

from tests import cache_oracle as O
from tests.helpers import to_f64

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
FORMATS = [O.E4M3, O.INT8]


def _crisp():
    from paper_2609_01925_amd import crisp as C
    return C


def _say(msg):
    print(f"[gpu-case] {msg}", flush=True)
    sys.stdout.flush()


def _ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device=DEV)


def _rand(heads, n, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(heads, n, 128, generator=g) * scale).to(torch.bfloat16)


def _ptr(counts):
    return np.concatenate([[0], np.cumsum(counts)])


def _table(lens, block, rng, extra=2, width=None):
    """Pages at random places, and the number of pages."""
    need = [-(-n // block) for n in lens]
    width = max(need + [1]) if width is None else width
    place = rng.permutation(sum(need) + extra)
    t = np.full((len(lens), width), -1, dtype=np.int32)
    for s, n in enumerate(need):
        t[s, :n], place = place[:n], place[n:]
    return t, sum(need) + extra


def _new(C, n_pages, heads, block, fmt, junk=True):
    """A cache on both sides; the device's holds arbitrary bytes (NaN codes and scales among them)."""
    c = C.make_cache(n_pages, heads, block, fmt, device=DEV)
    c.pages.fill_(0x7f if junk else 0)
    c.scales.fill_(math.nan if junk else 1.0)
    return c, O.Cache(n_pages, heads, block, fmt)


def _check_written(c, oracle):
    """Codes of written tokens and scales of written pages, bit for bit."""
    got = O.decode(c.pages.cpu().numpy(), c.fmt)
    p, t = np.nonzero(oracle.written)
    np.testing.assert_array_equal(got[p, :, :, t], oracle.codes[p, :, :, t])
    pages = oracle.written.any(1)
    np.testing.assert_array_equal(c.scales.cpu().numpy()[pages], np.ldexp(1.0, oracle.exp[pages]))


def _append(C, c, oracle, table, lens, counts, k, v):
    ptr = _ptr(counts)
    C.crisp_cache_append(c, _ints(table), _ints(lens), _ints(ptr), k.to(DEV), v.to(DEV))
    oracle.append(table, lens, ptr, to_f64(k), to_f64(v))


def _check_attn(C, c, oracle, table, lens, counts, q, scale=0.0):
    ptr = _ptr(counts)
    o = C.crisp_cache_attn(c, _ints(table), _ints(lens), _ints(ptr), q.to(DEV), softmax_scale=scale)
    want, tol = oracle.attention(table, lens, ptr, to_f64(q), scale or 1 / math.sqrt(128))
    got = to_f64(o)
    live = ~np.isnan(want)
    assert np.isfinite(got[live]).all()
    worst = np.max(np.abs(got - want)[live] / tol[live], initial=0.0)
    assert worst <= 1.0, f"{worst:.3f} of the tolerance"
    return o


# ------------------------------------------------------------------ appending


@pytest.mark.parametrize("rows_a_call", [512, 4])
@pytest.mark.parametrize("fmt", FORMATS)
def test_every_bf16_value(fmt, rows_a_call):
    """All 65536 bit patterns, 128 neighbours in magnitude a row, so that a page's values lie within
    a few octaves: rounding, subnormal codes, zeros, infinities and NaN."""
    C = _crisp()
    _say(f"append every bf16 value fmt={fmt} rows a call={rows_a_call}")
    bits = np.arange(1 << 15).reshape(-1, 64)
    bits = np.concatenate([bits, bits | 0x8000], 1).astype(np.uint16)  # [512, 128]
    x = torch.from_numpy(bits.view(np.int16)).view(torch.bfloat16)[None]
    table = np.arange(8, dtype=np.int32)[None]
    for rows in (x, x[:, torch.randperm(512, generator=torch.Generator().manual_seed(1))]):
        c, oracle = _new(C, 8, 1, 64, fmt)
        for i in range(0, 512, rows_a_call):
            _append(C, c, oracle, table, [i], [rows_a_call], rows[:, i:i + rows_a_call], -rows[:, i:i + rows_a_call])
        _check_written(c, oracle)


@pytest.mark.parametrize("block", [64, 128])
@pytest.mark.parametrize("fmt", FORMATS)
def test_append_ragged_in_steps(fmt, block):
    """Several appends of ragged batches, of no rows to several pages, sizes growing and shrinking so
    that scales grow inside pages: codes behind older tokens are rounded again."""
    C = _crisp()
    _say(f"append in steps fmt={fmt} block={block}")
    rng = np.random.default_rng(7 + fmt)
    steps = [[1, 0, 63, 64, 65, 200], [1, 1, 1, 1, 1, 1], [0, 129, 1, 0, 31, 3], [1, 1, 1, 64, 1, 130]]
    total = np.sum(steps, 0)
    table, n_pages = _table(total, block, rng)
    c, oracle = _new(C, n_pages, 3, block, fmt)
    lens = np.zeros(6, dtype=np.int64)
    for i, counts in enumerate(steps):
        k, v = _rand(3, sum(counts), 10 * i, 3.0 ** i), _rand(3, sum(counts), 10 * i + 1, 1.7 ** -i)
        _append(C, c, oracle, table, lens, counts, k, v)
        lens += counts
        _check_written(c, oracle)


@pytest.mark.parametrize("n_seqs,long", [(20, 41), (64, 129), (70, 141), (520, 700)])
@pytest.mark.parametrize("fmt,block", [(O.E4M3, 128), (O.INT8, 64)])
def test_append_short_and_long_together(fmt, block, n_seqs, long):
    """A batch of single rows with one chunk among them, some without a row, some in a page's last place, a few of
    two to five rows: the pages written by a wave and by a workgroup in one call, up to 64 sequences and past them."""
    C = _crisp()
    _say(f"append short and long fmt={fmt} block={block} sequences={n_seqs} long={long}")
    rng = np.random.default_rng(n_seqs + fmt)
    counts = rng.choice([0, 1, 1, 1, 1, 2, 5], n_seqs)
    counts[n_seqs // 3], counts[n_seqs // 3 + 1] = long, 4
    first = rng.integers(1, block + 1, n_seqs)
    first[::7] = block - 1
    table, n_pages = _table(first + counts, block, rng)
    c, oracle = _new(C, n_pages, 2, block, fmt)
    _append(C, c, oracle, table, 0 * first, first, _rand(2, first.sum(), 1), _rand(2, first.sum(), 2))
    _append(C, c, oracle, table, first, counts, _rand(2, counts.sum(), 3, 1.6), _rand(2, counts.sum(), 4, 0.5))
    _check_written(c, oracle)


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_token_by_token_with_growing_values(fmt):
    """A page filled one token at a time, each larger than all before; then past it."""
    C = _crisp()
    _say(f"append token by token fmt={fmt}")
    c, oracle = _new(C, 3, 2, 64, fmt)
    table = np.array([[2, 0]], dtype=np.int32)
    for t in range(70):
        k, v = _rand(2, 1, t, 1.2 ** t), _rand(2, 1, 100 + t, 2.0 ** (t % 5))
        _append(C, c, oracle, table, [t], [1], k, v)
        if t % 9 == 0 or t > 62:
            _check_written(c, oracle)


@pytest.mark.parametrize("rows_a_call", [768, 3])
@pytest.mark.parametrize("fmt", FORMATS)
def test_append_extreme_values(fmt, rows_a_call):
    """Zeros, the smallest and largest bf16, values under the smallest scale, infinities and NaN (which move no scale)."""
    C = _crisp()
    _say(f"append extremes fmt={fmt}")
    top = torch.finfo(torch.bfloat16).max
    rows = torch.zeros(1, 12 * 64, 128)
    rows[0, 64] = top
    rows[0, 128] = 1e-38
    rows[0, 192:256] = torch.randn(64, 128) * 2.0 ** -66
    rows[0, 256:320] = torch.randn(64, 128)
    rows[0, 260, ::3] = math.inf
    rows[0, 261, ::5] = -math.inf
    rows[0, 262, ::2] = math.nan
    rows[0, 320:384] = math.nan
    rows[0, 384:448] = math.inf
    rows[0, 448:512] = 448.0
    rows[0, 512:576] = 127.0
    rows[0, 576:640] = 127.5
    rows[0, 640:704] = 450.0
    rows[0, 704:] = torch.randn(64, 128) * 2.0 ** 100
    rows = rows.to(torch.bfloat16)
    c, oracle = _new(C, 12, 1, 64, fmt)
    table = np.arange(12, dtype=np.int32)[::-1][None].copy()
    for i in range(0, 768, rows_a_call):
        _append(C, c, oracle, table, [i], [rows_a_call], rows[:, i:i + rows_a_call], rows[:, i:i + rows_a_call])
    _check_written(c, oracle)


@pytest.mark.parametrize("n_seqs", [65, 130, 5000])
def test_append_with_rows_before_the_first_sequence(n_seqs):
    """More sequences than one look holds, and rows that lie before all of them: those are stored nowhere."""
    C = _crisp()
    _say(f"append n_seqs={n_seqs}, rows before the first")
    counts = [1 + s % 2 for s in range(n_seqs)]
    n = sum(counts)
    k, v = _rand(2, n + 40, n_seqs), _rand(2, n + 40, n_seqs + 1)
    table = _ints(np.arange(n_seqs)[:, None])
    sides = []
    for lead in (0, 37):
        c, _ = _new(C, n_seqs + 1, 2, 64, O.E4M3, junk=False)
        C.crisp_cache_append(c, table, _ints([3] * n_seqs), _ints(_ptr(counts) + lead), k[:, 37 - lead:].contiguous().to(DEV),
                             v[:, 37 - lead:].contiguous().to(DEV))
        sides.append(c)
    assert torch.equal(sides[0].pages, sides[1].pages) and torch.equal(sides[0].scales, sides[1].scales)
    assert (sides[0].pages[:n_seqs].flatten(1) != 0).any(1).all() and (sides[0].pages[n_seqs] == 0).all()


def test_append_leaves_the_rest():
    """Other pages, other tokens of the page, and rows of no page stay as they were; positions past the
    table and in holes are dropped."""
    C = _crisp()
    _say("append leaves the rest")
    table = np.array([[1, -1, 4], [9999, 3, -7]], dtype=np.int32)
    c, oracle = _new(C, 6, 2, 64, O.E4M3, junk=False)
    before = c.pages.clone()
    counts = [250, 140]  # past three slots; rows 390.. belong to nobody
    k, v = _rand(2, 400, 1), _rand(2, 400, 2)
    k[:, 390:] = math.nan
    _append(C, c, oracle, table, [10, 0], counts, k, v)
    _check_written(c, oracle)
    for p in (0, 2, 5):
        assert torch.equal(c.pages[p], before[p]) and (c.scales[p] == 1).all()
    got = O.decode(c.pages.cpu().numpy(), O.E4M3)
    assert (got[1, :, :, :10] == 0).all() and (got[3, :, :, 76:] == 0).all()


@pytest.mark.parametrize("layout", ["rows_first", "packed_qkv", "one_row", "shared_head"])
def test_strides(layout):
    """K, V, Q and the output as a model's projections leave them: [n_rows, heads, 128], slices of one
    packed tensor, a broadcast head."""
    C = _crisp()
    _say(f"strides {layout}")
    rng = np.random.default_rng(3)
    lens, counts = np.array([70, 3]), [5, 9] if layout != "one_row" else [1, 0]
    n = sum(counts)
    table, n_pages = _table(lens + counts, 64, rng)
    c, oracle = _new(C, n_pages, 2, 64, O.INT8)
    _append(C, c, oracle, table, [0, 0], lens, _rand(2, 73, 4), _rand(2, 73, 5))
    packed = torch.randn(n, 8, 128, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16).to(DEV)
    if layout == "shared_head":
        k = packed[:, 4:5].transpose(0, 1).expand(2, n, 128)
        q, v = packed[:, :4].transpose(0, 1), packed[:, 6:8].transpose(0, 1)
    else:
        q, k, v = (packed[:, a:b].transpose(0, 1) for a, b in ((0, 4), (4, 6), (6, 8)))
    assert layout == "one_row" or not k.is_contiguous()
    ptr = _ptr(counts)
    C.crisp_cache_append(c, _ints(table), _ints(lens), _ints(ptr), k, v)
    oracle.append(table, lens, ptr, to_f64(k), to_f64(v))
    _check_written(c, oracle)
    out = torch.zeros(n, 6, 128, dtype=torch.bfloat16, device=DEV)
    view = out[:, 1:5].transpose(0, 1)
    C.crisp_cache_attn(c, _ints(table), _ints(lens), _ints(ptr), q, out=view)
    want, tol = oracle.attention(table, lens, ptr, to_f64(q), 1 / math.sqrt(128))
    assert (np.abs(to_f64(view) - want) <= tol).all()
    assert (out[:, 0] == 0).all() and (out[:, 5] == 0).all()


# ------------------------------------------------------------------ attention


@pytest.mark.parametrize("hq,hkv", [(4, 4), (8, 2), (7, 1), (14, 2), (40, 2)])
@pytest.mark.parametrize("fmt,block", [(O.E4M3, 64), (O.INT8, 128)])
def test_one_row_each(fmt, block, hq, hkv):
    """Decoding a ragged batch: lengths of one token to several pages, at and beside tile and page ends."""
    C = _crisp()
    _say(f"one row each fmt={fmt} block={block} heads={hq}/{hkv}")
    rng = np.random.default_rng(hq)
    lens = np.array([0, 1, 62, 63, 64, 127, 128, 129, 300, 511, 700])
    table, n_pages = _table(lens + 1, block, rng)
    c, oracle = _new(C, n_pages, hkv, block, fmt)
    _append(C, c, oracle, table, 0 * lens, lens, _rand(hkv, lens.sum(), 1, 2.0), _rand(hkv, lens.sum(), 2))
    ones = [1] * len(lens)
    _append(C, c, oracle, table, lens, ones, _rand(hkv, len(lens), 3, 2.0), _rand(hkv, len(lens), 4))
    _check_attn(C, c, oracle, table, lens, ones, _rand(hq, len(lens), 5, 1.5))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("counts", [[3, 0, 1, 8, 5], [17, 130, 1, 0, 64], [0, 0, 200, 0, 0]])
def test_rows_of_different_counts(fmt, counts):
    """Drafted tokens and chunks: every row sees the positions up to its own, sequences without rows are passed over."""
    C = _crisp()
    _say(f"rows of different counts fmt={fmt} {counts}")
    rng = np.random.default_rng(11)
    lens = np.array([40, 64, 0, 150, 333])
    table, n_pages = _table(lens + counts, 64, rng)
    c, oracle = _new(C, n_pages, 2, 64, fmt)
    _append(C, c, oracle, table, 0 * lens, lens, _rand(2, lens.sum(), 1), _rand(2, lens.sum(), 2))
    _append(C, c, oracle, table, lens, counts, _rand(2, sum(counts), 3), _rand(2, sum(counts), 4))
    _check_attn(C, c, oracle, table, lens, counts, _rand(6, sum(counts), 5))


@pytest.mark.parametrize("hq,hkv", [(4, 2), (7, 1), (3, 3)])
def test_long_chunks_with_and_without_history(hq, hkv):
    """Chunks whose last rows see several times what the first ones do, beside one with a long history: odd and even
    numbers of row groups, cut between workgroups and whole."""
    C = _crisp()
    _say(f"long chunks heads={hq}/{hkv}")
    rng = np.random.default_rng(hq)
    lens, counts = np.array([0, 5, 900, 64, 0]), np.array([1100, 0, 140, 333, 260])
    table, n_pages = _table(lens + counts, 128, rng)
    c, oracle = _new(C, n_pages, hkv, 128, O.E4M3)
    _append(C, c, oracle, table, 0 * lens, lens, _rand(hkv, lens.sum(), 1), _rand(hkv, lens.sum(), 2))
    _append(C, c, oracle, table, lens, counts, _rand(hkv, counts.sum(), 3), _rand(hkv, counts.sum(), 4))
    _check_attn(C, c, oracle, table, lens, counts, _rand(hq, counts.sum(), 5))


@pytest.mark.parametrize("fmt,rows,hq", [(O.E4M3, 1, 4), (O.INT8, 1, 1), (O.E4M3, 33, 4)])
def test_long_sequence_is_split(fmt, rows, hq):
    """One sequence of 20000 tokens cut over many workgroups, one KV head, beside a short one."""
    C = _crisp()
    _say(f"long sequence fmt={fmt} rows={rows}")
    rng = np.random.default_rng(5)
    lens, counts = np.array([20000, 37]), [rows, 1]
    table, n_pages = _table(lens + counts, 64, rng)
    c, oracle = _new(C, n_pages, 1, 64, fmt)
    _append(C, c, oracle, table, 0 * lens, lens, _rand(1, lens.sum(), 1), _rand(1, lens.sum(), 2))
    _append(C, c, oracle, table, lens, counts, _rand(1, sum(counts), 3), _rand(1, sum(counts), 4))
    a = _check_attn(C, c, oracle, table, lens, counts, _rand(hq, sum(counts), 5, 3.0))
    b = _check_attn(C, c, oracle, table, lens, counts, _rand(hq, sum(counts), 5, 3.0))
    assert torch.equal(a, b)


def test_many_sequences():
    """More sequences than a workgroup has threads, most of them short, some without rows."""
    C = _crisp()
    _say("many sequences")
    rng = np.random.default_rng(6)
    lens, counts = rng.integers(0, 150, 700), rng.integers(0, 3, 700)
    table, n_pages = _table(lens + counts, 64, rng)
    c, oracle = _new(C, n_pages, 1, 64, O.E4M3)
    _append(C, c, oracle, table, 0 * lens, lens, _rand(1, lens.sum(), 1), _rand(1, lens.sum(), 2))
    _append(C, c, oracle, table, lens, counts, _rand(1, counts.sum(), 3), _rand(1, counts.sum(), 4))
    _check_written(c, oracle)
    _check_attn(C, c, oracle, table, lens, counts, _rand(2, counts.sum(), 5))


@pytest.mark.parametrize("n_seqs", [5000, 70000])
def test_very_many_sequences(n_seqs):
    """Sequences of one token each, every ninth without a row: the result of a row that sees one token is its v, here
    whole numbers that the codes hold exactly."""
    C = _crisp()
    _say(f"very many sequences n={n_seqs}")
    c = C.make_cache(n_seqs, 1, 64, O.E4M3, DEV)
    counts = np.ones(n_seqs, dtype=np.int64)
    counts[::9] = 0
    n = int(counts.sum())
    g = torch.Generator().manual_seed(n_seqs)
    k = torch.randn(1, n, 128, generator=g).to(torch.bfloat16).to(DEV)
    v = torch.randint(-16, 17, (1, n, 128), generator=g).to(torch.bfloat16).to(DEV)
    table = torch.randperm(n_seqs, generator=g).to(torch.int32)[:, None].to(DEV)
    lens, ptr = torch.zeros(n_seqs, dtype=torch.int32, device=DEV), _ints(_ptr(counts))
    C.crisp_cache_append(c, table, lens, ptr, k, v)
    o = C.crisp_cache_attn(c, table, lens, ptr, k.expand(2, n, 128))
    assert torch.equal(o, v.expand(2, n, 128))


def test_peaked_scores_and_scales_far_apart():
    """Scores from far below to far above, pages whose scales are 2^40 apart, a given softmax scale."""
    C = _crisp()
    _say("peaked scores")
    rng = np.random.default_rng(8)
    lens, counts = np.array([0, 0]), [500, 64]
    table, n_pages = _table(counts, 64, rng)
    c, oracle = _new(C, n_pages, 2, 64, O.E4M3)
    k, v = _rand(2, 564, 1), _rand(2, 564, 2)
    k[:, 100:164] *= 2.0 ** -20
    v[:, 200:300] *= 2.0 ** 20
    v[:, 300:420] *= 2.0 ** -20
    k[:, 420:430] *= 16
    _append(C, c, oracle, table, lens, counts, k, v)
    q = _rand(4, 564, 3, 4.0)
    q[:, 5] = 0
    _check_attn(C, c, oracle, table, lens, counts, q, scale=0.5)
    _check_attn(C, c, oracle, table, lens, counts, q)


@pytest.mark.parametrize("rows", [1, 70])
def test_scales_that_vanish(rows):
    """A softmax_scale whose products are 0 in 32 bits: every token that a row sees has the same weight, the others none."""
    C = _crisp()
    _say(f"vanishing scale rows={rows}")
    table, n_pages = _table([30 + rows], 64, np.random.default_rng(3))
    c, oracle = _new(C, n_pages, 1, 64, O.E4M3)
    _append(C, c, oracle, table, [0], [30 + rows], _rand(1, 30 + rows, 1, 1e-18), _rand(1, 30 + rows, 2))
    _check_attn(C, c, oracle, table, [30], [rows], _rand(2, rows, 3), scale=1e-42)


def test_holes_and_rows_that_see_nothing():
    """Pages that are missing hold no keys, at the front, inside and behind; a row with none gets 0."""
    C = _crisp()
    _say("holes")
    rng = np.random.default_rng(9)
    lens, counts = np.array([400, 260, 90, 500]), [1, 40, 2, 1]
    table, n_pages = _table(lens + counts, 64, rng)
    c, oracle = _new(C, n_pages, 2, 64, O.INT8)
    _append(C, c, oracle, table, 0 * lens, lens, _rand(2, lens.sum(), 1), _rand(2, lens.sum(), 2))
    _append(C, c, oracle, table, lens, counts, _rand(2, sum(counts), 3), _rand(2, sum(counts), 4))
    table[0, [0, 3]] = -1, n_pages + 3
    table[1, 4] = 1 << 30
    table[2] = -5
    o = _check_attn(C, c, oracle, table, lens, counts, _rand(4, sum(counts), 5))
    assert (o[:, 41:43] == 0).all()
    short = table[:, :3].copy()  # a table that ends before the lengths do
    _check_attn(C, c, oracle, short, lens, counts, _rand(4, sum(counts), 6))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows", [1, 9, 60])
def test_queries_that_are_not_finite(rows, fmt):
    """A NaN or an infinity in a query makes its row NaN, by the formula, and no other; a row that sees nothing stays 0."""
    C = _crisp()
    _say(f"queries that are not finite rows={rows} fmt={fmt}")
    rng = np.random.default_rng(rows)
    lens, counts = np.array([400, 0, 100]), np.array([rows] * 3)
    table, n_pages = _table(lens + counts, 64, rng)
    table[1] = -1  # sees nothing
    c, oracle = _new(C, n_pages, 2, 64, fmt)
    _append(C, c, oracle, table, 0 * lens, lens, _rand(2, lens.sum(), 1), _rand(2, lens.sum(), 2))
    _append(C, c, oracle, table, lens, counts, _rand(2, counts.sum(), 3), _rand(2, counts.sum(), 4))
    q = _rand(10, counts.sum(), 5)
    bad = np.zeros((10, counts.sum()), dtype=bool)
    for h, r, value in ((0, 0, math.nan), (3, 0, math.inf), (9, rows - 1, -math.inf), (4, 2 * rows, math.nan), (4, rows, math.nan)):
        q[h, r, 7 * h % 128] = value
        bad[h, r] = r // rows != 1
    o = to_f64(C.crisp_cache_attn(c, _ints(table), _ints(lens), _ints(_ptr(counts)), q.to(DEV)))
    q[torch.from_numpy(bad)] = 0
    q[4, rows] = 0
    want, tol = oracle.attention(table, lens, _ptr(counts), to_f64(q), 1 / math.sqrt(128))
    assert np.isnan(o[bad]).all()
    assert (np.abs(o - want)[~bad] <= tol[~bad]).all()
    assert (o[:, rows:2 * rows] == 0).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows", [1, 20, 90])
def test_queries_with_outliers(rows, fmt):
    """A few elements of every query are 1000 times the others and meet keys that are 0 there, so that the scores come from
    the small ones; one head is of subnormal size; then large queries against keys that are small."""
    C = _crisp()
    _say(f"queries with outliers rows={rows} fmt={fmt}")
    table, n_pages = _table([500 + rows], 64, np.random.default_rng(rows))
    c, oracle = _new(C, n_pages, 1, 64, fmt)
    k = _rand(1, 500 + rows, 1)
    k[:, :, [3, 64, 127]] = 0
    _append(C, c, oracle, table, [0], [500 + rows], k, _rand(1, 500 + rows, 2))
    q = _rand(4, rows, 3)
    q[:, :, [3, 64, 127]] *= 1000
    q[1] *= 1e-38
    q[2, :, 5] = 0
    _check_attn(C, c, oracle, table, [500], [rows], q)
    c, oracle = _new(C, n_pages, 1, 64, fmt)
    _append(C, c, oracle, table, [0], [500 + rows], _rand(1, 500 + rows, 4, 2.0 ** -60), _rand(1, 500 + rows, 5))
    _check_attn(C, c, oracle, table, [500], [rows], _rand(4, rows, 6, 2.0 ** 62))


def test_padded_rows_are_left():
    """Rows behind the last sequence's keep what the output held; NaN in them and in dropped rows reaches nothing."""
    C = _crisp()
    _say("padded rows")
    rng = np.random.default_rng(10)
    lens, counts = np.array([100, 7]), [2, 3]
    table, n_pages = _table(lens + counts, 64, rng)
    c, oracle = _new(C, n_pages, 2, 64, O.E4M3)
    _append(C, c, oracle, table, 0 * lens, lens, _rand(2, 107, 1), _rand(2, 107, 2))
    k, v, q = _rand(2, 9, 3), _rand(2, 9, 4), _rand(4, 9, 5)
    for x in (k, v, q):
        x[:, 5:] = math.nan
    _append(C, c, oracle, table, lens, counts, k, v)
    out = torch.full((4, 9, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    C.crisp_cache_attn(c, _ints(table), _ints(lens), _ints(_ptr(counts)), q.to(DEV), out=out)
    want, tol = oracle.attention(table, lens, _ptr(counts), to_f64(q), 1 / math.sqrt(128))
    assert (np.abs(to_f64(out[:, :5]) - want[:, :5]) <= tol[:, :5]).all()
    assert (out[:, 5:] == 7).all()


def test_malformed_offsets_stay_inside():
    """Offsets that fall, pass the rows or begin below 0, negative lengths are cut to the rows and the table.  Row 0
    sees written tokens only and has their result; the others also see tokens that were never appended (NaN
    codes here), so nothing is known of them."""
    C = _crisp()
    _say("malformed offsets")
    rng = np.random.default_rng(12)
    lens = np.array([64, 64, 64, 64])
    table, n_pages = _table(lens + 20, 64, rng)
    c, oracle = _new(C, n_pages, 1, 64, O.E4M3)
    _append(C, c, oracle, table, 0 * lens, lens, _rand(1, 256, 1), _rand(1, 256, 2))
    q = _rand(2, 10, 3)
    out = torch.full((2, 10, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    C.crisp_cache_attn(c, _ints(table), _ints([63, -5, 63, 10 ** 9]), _ints([-3, 2, 1, 1, 99]), q.to(DEV), out=out)
    ref = np.array([0, 2, 2, 2, 10])  # sequence 1 falls: none; sequence 3: rows 1 .. 10, written after or before 0's
    want, tol = oracle.attention(table, np.array([63, 0, 63, 127]), ref, to_f64(q), 1 / math.sqrt(128))
    assert (np.abs(to_f64(out[:, :1]) - want[:, :1]) <= tol[:, :1]).all()


def test_offsets_past_32_bits():
    """A cache of 6 GB: pages past 2^31 and 2^32 bytes, appended to, attended to (by one row and by many) and copied."""
    C = _crisp()
    _say("offsets past 32 bits")
    n_pages = 200_000
    c = C.make_cache(n_pages, 2, 64, O.E4M3, DEV)
    assert c.pages.numel() > 6 << 30
    rows = 330
    at = np.array([n_pages - 1, 140_000, 65_536, 131_072, 7, n_pages - 2])
    oracle = O.Cache(6, 2, 64, O.E4M3)
    local, table = np.arange(6, dtype=np.int32)[None], at.astype(np.int32)[None]
    k, v, q = _rand(2, rows, 1), _rand(2, rows, 2), _rand(4, rows, 3)
    ptr = _ptr([rows])
    C.crisp_cache_append(c, _ints(table), _ints([0]), _ints(ptr), k.to(DEV), v.to(DEV))
    oracle.append(local, [0], ptr, to_f64(k), to_f64(v))
    for n in (rows, 1):
        o = C.crisp_cache_attn(c, _ints(table), _ints([rows - n]), _ints([0, n]), q[:, :n].to(DEV))
        want, tol = oracle.attention(local, [rows - n], [0, n], to_f64(q[:, :n]), 1 / math.sqrt(128))
        assert (np.abs(to_f64(o) - want) <= tol).all()
    moved = np.array([3, 150_000, 199_000, 5, 70_000, 196_000])
    C.crisp_cache_copy(c, _ints(np.stack([at, moved], 1)))
    for a, b in zip(at, moved):
        assert torch.equal(c.pages[a], c.pages[b]) and torch.equal(c.scales[a], c.scales[b])


# ------------------------------------------------------------------ the two together


def test_steps_on_streams_and_in_a_graph():
    """Append and attention of a decoding step captured once and replayed with lengths that grow on the
    device, beside an eager step of another batch on a side stream, equal to the eager steps bit for bit."""
    C = _crisp()
    _say("steps in a graph")
    rng = np.random.default_rng(13)
    lens, steps = np.array([60, 128, 5]), 6
    table, n_pages = _table(lens + steps, 64, rng)
    t, ptr = _ints(table), _ints([0, 1, 2, 3])
    k0, v0 = _rand(2, lens.sum(), 1), _rand(2, lens.sum(), 2)
    rows = [[_rand(h, 3, 10 * i + j).to(DEV) for j, h in enumerate((2, 2, 8))] for i in range(steps)]

    def fresh():
        c, oracle = _new(C, n_pages, 2, 64, O.E4M3, junk=False)
        _append(C, c, oracle, table, 0 * lens, lens, k0, v0)
        return c, _ints(lens)

    c, n = fresh()
    want = []
    for k, v, q in rows:
        C.crisp_cache_append(c, t, n, ptr, k, v)
        want.append(C.crisp_cache_attn(c, t, n, ptr, q))
        n += 1
    torch.cuda.synchronize()
    pages = c.pages.clone()

    c, n = fresh()
    ws = C.cache_workspace(c, 8, 3, 3)
    k, v, q = (x.clone() for x in rows[0])
    o = torch.empty(8, 3, 128, dtype=torch.bfloat16, device=DEV)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        C.crisp_cache_append(c, t, n, ptr, k, v)
        C.crisp_cache_attn(c, t, n, ptr, q, ws=ws, out=o)
    torch.cuda.synchronize()
    c2, n2 = fresh()
    c.pages.copy_(c2.pages)
    c.scales.copy_(c2.scales)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        C.crisp_cache_append(c, t, n, ptr, k, v)
        C.crisp_cache_attn(c, t, n, ptr, q, ws=ws, out=o)
    for i in range(steps):
        for x, y in zip((k, v, q), rows[i]):
            x.copy_(y)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):  # unrelated work beside the replay
            C.crisp_cache_attn(c2, t, n2, ptr, rows[0][2])
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want[i]), f"step {i}"
        n += 1
    assert torch.equal(c.pages, pages)


# ------------------------------------------------------------------ pages


def _pool_state(C, n_pages, block, n_seqs, width):
    pool = C.crisp_pool_init(n_pages, DEV)
    table = torch.full((n_seqs, width), -1, dtype=torch.int32, device=DEV)
    seq_len = torch.zeros(n_seqs, dtype=torch.int32, device=DEV)
    return pool, table, seq_len, O.Pool(n_pages, block, table.cpu().numpy(), [0] * n_seqs)


def _same_pool(pool, table, seq_len, oracle, where):
    np.testing.assert_array_equal(table.cpu().numpy(), np.array(oracle.table, dtype=np.int32), err_msg=where)
    np.testing.assert_array_equal(seq_len.cpu().numpy(), oracle.seq_len, err_msg=where)
    np.testing.assert_array_equal(pool.cpu().numpy(), oracle.words(), err_msg=where)


@pytest.mark.parametrize("n_pages", [1, 31, 32, 33, 500, 5000])
def test_pool_operations_in_random_order(n_pages):
    """Reservations (some refused), lengths that grow, forks (good and refused ones), frees (ids out of range
    and repeated) and compactions, against lists after every call."""
    C = _crisp()
    _say(f"pool operations n_pages={n_pages}")
    rng = np.random.default_rng(n_pages)
    block, n_seqs, width = 64, 20, max(2, n_pages // 12)
    pool, table, seq_len, oracle = _pool_state(C, n_pages, block, n_seqs, width)
    for step in range(40):
        what = rng.integers(4)
        if what <= 1:
            counts = rng.integers(-2, 2 + block * width // 3, n_seqs) * (rng.random(n_seqs) < 0.4)
            got = C.crisp_pool_reserve(pool, block, table, seq_len, _ints(counts))
            want = oracle.reserve([int(x) for x in counts])
            assert got.tolist() == want, step
            seq_len += got
            oracle.seq_len = [a + b for a, b in zip(oracle.seq_len, want)]
        elif what == 2:
            n = int(rng.integers(1, 9))
            src, dst = rng.integers(-1, n_seqs + 1, n), rng.integers(-1, n_seqs + 1, n)
            empty = [s for s in range(n_seqs) if oracle.seq_len[s] == 0]
            if empty:
                dst[: n // 2 + 1] = rng.choice(empty, n // 2 + 1)
            got = C.crisp_pool_fork(pool, block, table, seq_len, _ints(src), _ints(dst))
            assert [tuple(x) for x in got.tolist()] == oracle.fork(src.tolist(), dst.tolist()), step
        else:
            ids = rng.integers(-2, n_seqs + 2, int(rng.integers(1, 6)))
            C.crisp_pool_free(pool, table, seq_len, _ints(ids))
            oracle.free(ids.tolist())
        _same_pool(pool, table, seq_len, oracle, f"step {step} op {what}")
        if step % 7 == 3:  # tokens taken back, perhaps into pages that a fork shares
            back = rng.integers(0, 100, n_seqs) * (rng.random(n_seqs) < 0.3)
            seq_len -= torch.minimum(_ints(back), seq_len)
            oracle.seq_len = [max(0, a - int(b)) for a, b in zip(oracle.seq_len, back)]
        if step % 5 == 4:
            moves, count = C.crisp_pool_compact(pool, table)
            want = oracle.compact()
            assert count.item() == len(want) and moves[: len(want)].tolist() == [list(x) for x in want]
            assert (moves[len(want):] == -1).all()
            _same_pool(pool, table, seq_len, oracle, f"step {step} compact")


def test_shared_page_is_not_reserved_again():
    """A sequence whose tokens are taken back into a page that its fork shares gets no rows there; a fork of it does."""
    C = _crisp()
    _say("shared page")
    pool, table, seq_len, oracle = _pool_state(C, 10, 64, 4, 4)
    counts = [128, 0, 0, 0]
    assert C.crisp_pool_reserve(pool, 64, table, seq_len, _ints(counts)).tolist() == oracle.reserve(counts) == counts
    seq_len[0] = oracle.seq_len[0] = 128
    assert C.crisp_pool_fork(pool, 64, table, seq_len, _ints([0]), _ints([1])).tolist() == [[-1, -1]]
    oracle.fork([0], [1])
    seq_len[0] = oracle.seq_len[0] = 125
    assert C.crisp_pool_reserve(pool, 64, table, seq_len, _ints([1, 1, 0, 0])).tolist() == oracle.reserve([1, 1, 0, 0]) == [0, 1, 0, 0]
    assert C.crisp_pool_fork(pool, 64, table, seq_len, _ints([0]), _ints([2])).tolist() == [list(x) for x in oracle.fork([0], [2])]
    assert C.crisp_pool_reserve(pool, 64, table, seq_len, _ints([0, 0, 3, 0])).tolist() == oracle.reserve([0, 0, 3, 0]) == [0, 0, 3, 0]
    _same_pool(pool, table, seq_len, oracle, "shared")


def test_pool_large_reservation_and_many_sequences():
    """More pages in one call than are collected at a time, and the largest number of sequences."""
    C = _crisp()
    _say("pool large")
    n_seqs = 4096
    pool, table, seq_len, oracle = _pool_state(C, 20000, 128, n_seqs, 40)
    rng = np.random.default_rng(2)
    for step in range(3):
        counts = rng.integers(0, 700, n_seqs)
        assert C.crisp_pool_reserve(pool, 128, table, seq_len, _ints(counts)).tolist() == oracle.reserve(counts.tolist())
        _same_pool(pool, table, seq_len, oracle, f"reserve {step}")
        seq_len += torch.where(table[:, 0] >= 0, 130, 0).int()
        oracle.seq_len = [n + (130 if r[0] >= 0 else 0) for n, r in zip(oracle.seq_len, oracle.table)]
        ids = rng.integers(0, n_seqs, 1500)
        C.crisp_pool_free(pool, table, seq_len, _ints(ids))
        oracle.free(ids.tolist())
        _same_pool(pool, table, seq_len, oracle, f"free {step}")
    src, dst = rng.integers(0, n_seqs, 4096), rng.integers(0, n_seqs, 4096)
    got = C.crisp_pool_fork(pool, 128, table, seq_len, _ints(src), _ints(dst))
    assert [tuple(x) for x in got.tolist()] == oracle.fork(src.tolist(), dst.tolist())
    _same_pool(pool, table, seq_len, oracle, "fork")


@pytest.mark.parametrize("fmt,block,heads", [(O.E4M3, 64, 3), (O.INT8, 128, 1)])
def test_copy_pages(fmt, block, heads):
    """Codes and scales of the first `count` pairs; pages out of range and copies onto themselves move nothing."""
    C = _crisp()
    _say(f"copy pages block={block}")
    c = C.make_cache(40, heads, block, fmt, DEV)
    c.pages.copy_(torch.randint(0, 256, c.pages.shape, dtype=torch.uint8))
    c.scales.copy_(torch.randn(c.scales.shape))
    pages, scales = c.pages.clone(), c.scales.clone()
    pairs = [(3, 0), (3, 7), (39, 8), (-1, 9), (5, -1), (40, 10), (6, 40), (11, 11), (20, 30), (21, 31)]
    C.crisp_cache_copy(c, _ints(pairs), _ints([9]))
    for a, b in pairs[:9]:
        if 0 <= a < 40 and 0 <= b < 40:
            pages[b], scales[b] = pages[a], scales[a]
    assert torch.equal(c.pages, pages) and torch.equal(c.scales, scales)
    for count in (0, -3):
        C.crisp_cache_copy(c, _ints(pairs), _ints([count]))
    assert torch.equal(c.pages, pages)
    C.crisp_cache_copy(c, _ints(pairs[9:]))
    pages[31], scales[31] = pages[21], scales[21]
    assert torch.equal(c.pages, pages) and torch.equal(c.scales, scales)
