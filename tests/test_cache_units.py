"""Attention over the 8-bit cache by each way of dividing it: units of 128 rows (both formats, whole and cut, the first and last
row groups in pairs), units of one sequence cut in step, and units of more than 64 sequences that are cut.  Which one a
call takes follows from its workspace's size, which every test asserts."""
import math

import numpy as np
import pytest
import torch

from tests import cache_oracle as O
from tests.helpers import to_f64
from tests.test_cache import DEV, FORMATS, _append, _crisp, _ints, _new, _ptr, _rand, _say, _table

pytestmark = pytest.mark.gpu

MOST = 512  # workgroups of a call whose units are cut


def _slots(rows):
    """Bytes of workspace of MOST shares of units of so many rows: a record of 24 bytes a share and two partial results."""
    return MOST * 24 + MOST * 2 * rows * 130 * 4


def _takes(C, c, hq, n_seqs, width, n_rows, unit):
    got = C.crisp_cache_attn_workspace_size(c, hq, n_seqs, width, n_rows)
    assert got == _slots(128) if unit == 128 else got <= _slots(32), got


def _wide(table, width):
    out = np.full((len(table), max(width, table.shape[1])), -1, dtype=np.int32)
    out[:, :table.shape[1]] = table
    return out


def _split_tol(fmt, oracle, table, lens, ptr, q, scale):
    """Units of 128 rows on e4m3: an element of q below 2^-14 of its row's largest is off by up to 2^-22 of that, so a score by
    scale 2^-22 max|q| (sum of |k| over such elements), and the result by twice that of max|v|."""
    tol = np.zeros(q.shape[:2] + (1,))
    if fmt != O.E4M3:
        return tol
    G = q.shape[0] // oracle.codes.shape[1]
    for s in range(len(lens)):
        r0, r1 = ptr[s], ptr[s + 1]
        if r1 == r0:
            continue
        n = lens[s] + r1 - r0
        k, v = (np.abs(oracle.values(table[s], n, x)[0]) for x in (0, 1))
        for h in range(q.shape[0]):
            x = np.abs(q[h, r0:r1])
            top = x.max(-1, keepdims=True)
            small = (x < top * 2.0 ** -14) @ k[h // G].T
            tol[h, r0:r1] = 2 * scale * 2.0 ** -22 * top * small.max(-1, keepdims=True) * v[h // G].max()
    return tol


def _check(C, c, oracle, table, lens, counts, q, unit, scale=0.0, live=None):
    """The call's result against the oracle's, twice with equal bits."""
    ptr = _ptr(counts)
    _takes(C, c, q.shape[0], len(lens), table.shape[1], q.shape[1], unit)
    ws = C.cache_workspace(c, q.shape[0], len(lens), q.shape[1], table.shape[1])
    call = lambda: C.crisp_cache_attn(c, _ints(table), _ints(lens), _ints(ptr), q.to(DEV), softmax_scale=scale, ws=ws)
    o = call()
    ws.fill_(0xff)  # NaN in every partial result
    assert torch.equal(o, call())
    x, f = to_f64(q), scale or 1 / math.sqrt(128)
    want, tol = oracle.attention(table, lens, ptr, x, f)
    if unit == 128:
        tol = tol + _split_tol(c.fmt, oracle, table, lens, ptr, x, f)
    got, live = to_f64(o), ~np.isnan(want)
    assert np.isfinite(got[live]).all()
    worst = np.max(np.abs(got - want)[live] / tol[live], initial=0.0)
    assert worst <= 1.0, f"{worst:.3f} of the tolerance"
    return o


def _filled(C, fmt, block, hkv, lens, counts, width, seed=0, k_scale=1.0):
    """A cache that holds lens tokens and counts rows of each sequence, its oracle and the wide table."""
    table, n_pages = _table(lens + counts, block, np.random.default_rng(seed))
    table = _wide(table, width)
    c, oracle = _new(C, n_pages, hkv, block, fmt)
    if lens.sum():
        _append(C, c, oracle, table, 0 * lens, lens, _rand(hkv, lens.sum(), seed + 1, k_scale), _rand(hkv, lens.sum(), seed + 2))
    _append(C, c, oracle, table, lens, counts, _rand(hkv, counts.sum(), seed + 3, k_scale), _rand(hkv, counts.sum(), seed + 4))
    return c, oracle, table


@pytest.mark.parametrize("hq,hkv,lens,counts,width", [
    (4, 2, [0], [1100], 700),                              # an even number of row groups, over no history
    (7, 1, [0], [1000], 700),                              # an odd number, 7 heads a KV head
    (4, 2, [1500], [1000], 700),                           # many keys before the first row
    (2, 2, [700], [97], 6200),                             # a wave without a row, one row group
    (3, 3, [0, 5, 900, 64, 0], [1100, 0, 140, 333, 260], 700),
    (4, 2, [257, 0, 64, 1], [130, 257, 64, 300], 700)])
@pytest.mark.parametrize("fmt,block", [(O.E4M3, 64), (O.E4M3, 128), (O.INT8, 64), (O.INT8, 128)])
def test_units_of_128_rows(fmt, block, hq, hkv, lens, counts, width):
    """Chunks in units of 128 rows, each grain of a unit a share of its own, joined in units of 128."""
    C = _crisp()
    _say(f"units of 128 rows fmt={fmt} block={block} heads={hq}/{hkv} lens={lens} counts={counts}")
    lens, counts = np.array(lens), np.array(counts)
    c, oracle, table = _filled(C, fmt, block, hkv, lens, counts, width * 64 // block)
    _check(C, c, oracle, table, lens, counts, _rand(hq, counts.sum(), 5, 1.5), 128)


@pytest.mark.parametrize("fmt", FORMATS)
def test_units_of_128_rows_whole_and_cut(fmt):
    """More grains than shares: units of up to five grains, some whole inside a share, some cut, some ending with one."""
    C = _crisp()
    _say(f"units of 128 rows whole and cut fmt={fmt}")
    lens, counts = np.array([0, 100]), np.array([1200, 31])
    c, oracle, table = _filled(C, fmt, 64, 3, lens, counts, 64)
    _check(C, c, oracle, table, lens, counts, _rand(48, counts.sum(), 5, 1.5), 128)


@pytest.mark.parametrize("fmt", FORMATS)
def test_units_of_128_rows_of_many_sequences(fmt):
    """More than 64 sequences, so that shares are found by the workgroup; some without rows."""
    C = _crisp()
    _say(f"units of 128 rows of many sequences fmt={fmt}")
    rng = np.random.default_rng(4)
    lens, counts = rng.integers(0, 500, 90), rng.integers(40, 120, 90)
    counts[::8] = 0
    c, oracle, table = _filled(C, fmt, 64, 1, lens, counts, 200)
    _check(C, c, oracle, table, lens, counts, _rand(2, counts.sum(), 5, 1.5), 128)


@pytest.mark.parametrize("fmt", FORMATS)
def test_units_of_128_rows_with_holes(fmt):
    """Pages that are missing at the front, inside and behind; whole grains without a page; rows that see none get 0."""
    C = _crisp()
    _say(f"units of 128 rows with holes fmt={fmt}")
    lens, counts = np.array([900, 0, 130]), np.array([200, 400, 90])
    c, oracle, table = _filled(C, fmt, 64, 2, lens, counts, 900)
    table[0, [0, 2, 3, 4, 5, 6, 7, 15]] = -1, 9999, -7, -1, -1, -1, 1 << 30, -1
    table[1, :2] = -1
    table[2, :4] = -1
    o = _check(C, c, oracle, table, lens, counts, _rand(4, counts.sum(), 5), 128)
    assert (o[:, 200:328] == 0).all() and (o[:, 328:600] != 0).any() and (o[:, 600:] == 0).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_units_of_128_rows_and_outliers(fmt):
    """A few elements of every query 1000 times the others that meet keys which are 0 there; a head of subnormal size; large queries
    against small keys; scales of pages 2^40 apart."""
    C = _crisp()
    _say(f"units of 128 rows and outliers fmt={fmt}")
    rows, lens, counts = 120, np.array([500]), np.array([120])
    table = _wide(_table([620], 64, np.random.default_rng(1))[0], 3200)
    c, oracle = _new(C, 12, 1, 64, fmt)
    k, v = _rand(1, 620, 1), _rand(1, 620, 2)
    k[:, :, [3, 64, 127]] = 0
    v[:, 64:128] *= 2.0 ** 20
    v[:, 200:330] *= 2.0 ** -20
    _append(C, c, oracle, table, [0], [620], k, v)
    q = _rand(4, rows, 3)
    q[:, :, [3, 64, 127]] *= 1000
    q[1] *= 1e-38
    q[2, :, 5] = 0
    q[3, 7] = 0
    _check(C, c, oracle, table, lens, counts, q, 128)
    c, oracle = _new(C, 12, 1, 64, fmt)
    _append(C, c, oracle, table, [0], [620], _rand(1, 620, 4, 2.0 ** -60), _rand(1, 620, 5))
    _check(C, c, oracle, table, lens, counts, _rand(4, rows, 6, 2.0 ** 62), 128)
    _check(C, c, oracle, table, lens, counts, _rand(4, rows, 7), 128, scale=1e-42)


@pytest.mark.parametrize("rows,width,unit", [(3, 30, 32), (60, 30, 32), (120, 3200, 128)])
@pytest.mark.parametrize("fmt", FORMATS)
def test_small_codes(fmt, rows, width, unit):
    """Elements of K and V 2^12 and 2^15 times the others, where every query is 0: scores and results come from the smallest codes
    (subnormal ones of e4m3)."""
    C = _crisp()
    _say(f"small codes fmt={fmt} rows={rows}")
    lens, counts = np.array([500]), np.array([rows])
    table = _wide(_table(lens + counts, 64, np.random.default_rng(1))[0], width)
    c, oracle = _new(C, 12, 1, 64, fmt)
    big = 2.0 ** (12 if fmt == O.E4M3 else 5)
    k, v = _rand(1, 500 + rows, 1), _rand(1, 500 + rows, 2)
    k[:, :, :5] *= big
    k[:, 100:300, 5:9] *= 8 * big
    v[:, :, 77] *= 8 * big
    _append(C, c, oracle, table, [0], [500 + rows], k, v)
    q = _rand(4, rows, 3, 2.0)
    q[:, :, :9] = 0
    _check(C, c, oracle, table, lens, counts, q, unit)


@pytest.mark.parametrize("fmt", FORMATS)
def test_units_of_128_rows_that_are_not_finite(fmt):
    """A NaN or an infinity makes its row NaN and no other, in the first, a middle and the last row group."""
    C = _crisp()
    _say(f"units of 128 rows that are not finite fmt={fmt}")
    lens, counts = np.array([400, 70]), np.array([300, 100])
    c, oracle, table = _filled(C, fmt, 64, 2, lens, counts, 900)
    _takes(C, c, 4, 2, table.shape[1], 400, 128)
    q = _rand(4, 400, 5)
    bad = np.zeros((4, 400), dtype=bool)
    for h, r, value in ((0, 0, math.nan), (1, 0, math.inf), (3, 150, -math.inf), (2, 299, math.nan), (1, 300, math.nan), (0, 399, math.inf)):
        q[h, r, (7 * h + r) % 128] = value
        bad[h, r] = True
    o = to_f64(C.crisp_cache_attn(c, _ints(table), _ints(lens), _ints(_ptr(counts)), q.to(DEV)))
    q[torch.from_numpy(bad)] = 0
    want, tol = oracle.attention(table, lens, _ptr(counts), to_f64(q), 1 / math.sqrt(128))
    assert np.isnan(o[bad]).all()
    assert (np.abs(o - want)[~bad] <= tol[~bad]).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_units_of_128_rows_past_32_bits(fmt):
    """Pages past 2^31 and 2^32 bytes, and a padded batch whose other rows stay as they were."""
    C = _crisp()
    _say(f"units of 128 rows past 32 bits fmt={fmt}")
    n_pages, rows = 200_000, 330
    c = C.make_cache(n_pages, 2, 64, fmt, DEV)
    at = np.array([n_pages - 1, 140_000, 65_536, 131_072, 7, n_pages - 2])
    oracle = O.Cache(6, 2, 64, fmt)
    local, table = np.arange(6, dtype=np.int32)[None], _wide(at.astype(np.int32)[None], 1200)
    k, v, q = _rand(2, rows, 1), _rand(2, rows, 2), _rand(4, rows + 20, 3)
    q[:, rows:] = math.nan
    C.crisp_cache_append(c, _ints(table), _ints([0]), _ints([0, rows]), k.to(DEV), v.to(DEV))
    oracle.append(local, [0], [0, rows], to_f64(k), to_f64(v))
    _takes(C, c, 4, 1, 1200, rows + 20, 128)
    out = torch.full((4, rows + 20, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    C.crisp_cache_attn(c, _ints(table), _ints([0]), _ints([0, rows]), q.to(DEV), out=out)
    want, tol = oracle.attention(local, [0], [0, rows], to_f64(q[:, :rows]), 1 / math.sqrt(128))
    assert (np.abs(to_f64(out[:, :rows]) - want) <= tol).all()
    assert (out[:, rows:] == 7).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_units_of_128_rows_in_a_graph(fmt):
    """Captured with strided rows (packed q, k, v; the output beside them), replayed with other lengths and counts, eager work between."""
    C = _crisp()
    _say(f"units of 128 rows in a graph fmt={fmt}")
    total = np.array([1100, 600])
    table, n_pages = _table(total, 64, np.random.default_rng(3))
    table = _ints(_wide(table, 900))
    c, other = (_new(C, n_pages, 2, 64, fmt, junk=False)[0] for _ in range(2))
    n = 500
    packed = torch.zeros(n, 8, 128, dtype=torch.bfloat16, device=DEV)
    q, k, v = (packed[:, a:b].transpose(0, 1) for a, b in ((0, 4), (4, 6), (6, 8)))
    out = torch.zeros(n, 4, 128, dtype=torch.bfloat16, device=DEV)
    lens, ptr = _ints([0, 0]), _ints([0, 0, 0])
    _takes(C, c, 4, 2, 900, n, 128)
    ws = C.cache_workspace(c, 4, 2, n, 900)

    def step(c, o):
        C.crisp_cache_append(c, table, lens, ptr, k, v)
        C.crisp_cache_attn(c, table, lens, ptr, q, ws=ws, out=o.transpose(0, 1))

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(c, out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(c, out)
    held = np.zeros(2, dtype=np.int64)
    for i, counts in enumerate(([400, 100], [1, 250], [300, 0], [0, 200], [390, 1])):
        packed.copy_(torch.randn(n, 8, 128, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16))
        lens.copy_(_ints(held))
        ptr.copy_(_ints(_ptr(counts)))
        want = torch.zeros_like(out)
        step(other, want)
        torch.cuda.synchronize()
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        held += counts


# rows of 2 heads a KV head: 7 groups of 32 rows; 3, 4 and 6 KV heads give 24, 18 and 12 shares a unit
@pytest.mark.parametrize("hkv", [3, 4, 6])
@pytest.mark.parametrize("fmt", FORMATS)
def test_row_groups_of_one_sequence_in_step(fmt, hkv):
    """One sequence whose units are each cut into the same number of shares, which divides its 24 grains or not; then of 17."""
    C = _crisp()
    _say(f"row groups in step fmt={fmt} KV heads={hkv}")
    for n, block in ((6000, 64), (4200, 128)):
        lens, counts = np.array([n]), np.array([100])
        c, oracle, table = _filled(C, fmt, block, hkv, lens, counts, 0)
        _check(C, c, oracle, table, lens, counts, _rand(2 * hkv, 100, 5, 1.5), 32)


@pytest.mark.parametrize("rows", ["one", "some"])
@pytest.mark.parametrize("n_seqs", [65, 130, 300])
def test_cut_units_of_many_sequences(n_seqs, rows):
    """More than 64 sequences of none to 1500 tokens in a table whose units are cut: one row each, or up to 20 and some without."""
    C = _crisp()
    _say(f"cut units of many sequences n={n_seqs} rows={rows}")
    rng = np.random.default_rng(n_seqs)
    lens = rng.integers(0, 1500, n_seqs)
    lens[[3, 40]] = 0, 1500
    counts = np.ones(n_seqs, dtype=np.int64) if rows == "one" else rng.integers(0, 21, n_seqs)
    fmt = FORMATS[n_seqs % 2]
    c, oracle, table = _filled(C, fmt, 64, 2, lens, counts, 30)
    _check(C, c, oracle, table, lens, counts, _rand(4, counts.sum(), 5, 1.5), 32)
