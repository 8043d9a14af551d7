"""Eviction from the K/V cache by accumulated attention weight through the public binding, against the 64-bit oracle
(tests/packed_oracle.py): weights within counted roundings, the choice and the gathered pages bit for bit; lengths from one token to
many tiles, ragged batches, holes, budgets from one token to all but one, ties, values that are not finite, graphs."""
import math
import sys

import numpy as np
import pytest
import torch

from tests import cache_oracle as O
from tests import packed_oracle as R
from tests.helpers import to_f64
from tests.test_cache import _append, _check_written, _new, _ptr, _rand, _table

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


def _floats(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(DEV)


def _filled(C, lens, heads, block, fmt, seed, spread=None, extra=2, width=None):
    """A cache on both sides that holds `lens` tokens of each sequence; spread: powers of two that rows differ by."""
    rng = np.random.default_rng(seed)
    table, n_pages = _table(lens, block, rng, extra=extra, width=width)
    c, oracle = _new(C, n_pages, heads, block, fmt)
    n = sum(lens)
    k, v = _rand(heads, n, seed), _rand(heads, n, seed + 1)
    if spread:
        by = torch.from_numpy(2.0 ** rng.integers(-spread, spread + 1, n)).float()[None, :, None]
        k, v = (k.float() * by).to(torch.bfloat16), (v.float() * by).to(torch.bfloat16)
    _append(C, c, oracle, table, [0] * len(lens), lens, k, v)
    return c, oracle, table, n_pages


# ------------------------------------------------------------------ weights


def _check_weights(C, c, oracle, table, lens, counts, hq, held=None, width=None, scale=0.0, seed=0, gain=1.0):
    """lens: tokens before the rows (their K is in the cache as well)."""
    ptr = _ptr(counts)
    heads = oracle.codes.shape[1]
    width = table.shape[1] * oracle.block if width is None else width
    rng = np.random.default_rng(seed)
    w = rng.random((len(lens), heads, width)).astype(np.float32)
    held = [0] * len(lens) if held is None else held
    for s, h in enumerate(held):  # what does not count may be anything
        w[s, :, max(h, 0):] = math.nan
    q = _rand(hq, int(ptr[-1]) + 3, seed + 5, gain)
    out = torch.full(w.shape, 7.0, dtype=torch.float32, device=DEV)
    got = C.crisp_cache_weights(c, _ints(table), _ints(lens), _ints(ptr), q.to(DEV), _floats(w), _ints(held), scale, out)
    assert got is out
    want, tol = R.cache_weights(oracle, table, lens, ptr, to_f64(q), scale or 1 / math.sqrt(128), w.astype(np.float64), held)
    y = to_f64(out)
    live = ~np.isnan(want)
    assert np.isfinite(y[live]).all() and (y[~live] == 7.0).all()
    worst = np.max(np.abs(y - want)[live] / tol[live], initial=0.0)
    assert worst <= 1.0, f"{worst:.3f} of the tolerance"
    inplace = _floats(w)
    C.crisp_cache_weights(c, _ints(table), _ints(lens), _ints(ptr), q.to(DEV), inplace, _ints(held), scale)
    assert torch.equal(inplace[torch.from_numpy(live).to(DEV)], out[torch.from_numpy(live).to(DEV)])
    return out


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n", [0, 1, 15, 63, 64, 65, 127, 128, 200, 255, 256, 257, 1000])
def test_weights_of_a_step(n, fmt):
    C = _crisp()
    _say(f"weights n={n} fmt={fmt}")
    c, oracle, table, _ = _filled(C, [n + 1], 2, 64, fmt, n)
    _check_weights(C, c, oracle, table, [n], [1], 8, held=[n], seed=n)


@pytest.mark.parametrize("hq,heads", [(1, 1), (2, 2), (3, 1), (7, 1), (16, 1), (17, 1), (40, 2), (8, 8)])
def test_weights_head_layouts(hq, heads):
    C = _crisp()
    _say(f"weights heads={hq},{heads}")
    c, oracle, table, _ = _filled(C, [131, 40], heads, 64, O.E4M3, hq)
    _check_weights(C, c, oracle, table, [128, 33], [3, 7], hq, held=[100, 33], seed=hq)


@pytest.mark.parametrize("rows", [2, 9, 16, 33, 128, 129, 260])
@pytest.mark.parametrize("block", [64, 128])
def test_weights_of_many_rows(rows, block):
    """More pairs of row and head than one pass holds; rows that end inside tiles."""
    C = _crisp()
    _say(f"weights rows={rows} block={block}")
    lens = [70, 0, 301]
    counts = [rows, 1, max(1, rows // 3)]
    c, oracle, table, _ = _filled(C, [a + b for a, b in zip(lens, counts)], 2, block, O.INT8, rows)
    _check_weights(C, c, oracle, table, lens, counts, 6, held=[70, 0, 5], seed=rows)


@pytest.mark.parametrize("slots", [2, 40])
def test_weights_of_whole_prompts(slots):
    """All rows of prompts of some thousands, dozens of passes of 256 pairs; alone, and among slots that hold nothing."""
    C = _crisp()
    _say(f"weights of whole prompts, {slots} slots")
    counts = [2100, 1333] + [0] * (slots - 2)
    c, oracle, table, _ = _filled(C, counts, 1, 64, O.E4M3, 12)
    _check_weights(C, c, oracle, table, [0] * slots, counts, 4, held=[0] * slots, seed=12)


def test_weights_of_a_ragged_batch():
    """Sequences without rows, without tokens, more than a wave looks over; nothing held, some held, more held than there is."""
    C = _crisp()
    _say("weights ragged batch")
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 400, 70).tolist()
    counts = rng.integers(0, 4, 70).tolist()
    c, oracle, table, _ = _filled(C, [a + b for a, b in zip(lens, counts)], 1, 64, O.E4M3, 3)
    _check_weights(C, c, oracle, table, lens, counts, 4, held=[int(rng.integers(-5, 500)) for _ in lens], seed=3)


@pytest.mark.parametrize("width", [1, 63, 64, 100, 129, 400])
def test_weights_narrow_and_wide_buffers(width):
    """Positions past the width are dropped (they still count in the softmax); a width past the table's reach is served too."""
    C = _crisp()
    _say(f"weights width={width}")
    c, oracle, table, _ = _filled(C, [200, 131], 2, 64, O.E4M3, width)
    _check_weights(C, c, oracle, table, [198, 130], [2, 1], 4, held=[50, 130], width=width, seed=width)


def test_weights_of_a_long_history_in_chunks():
    C = _crisp()
    _say("weights 20000 tokens")
    c, oracle, table, _ = _filled(C, [20003], 1, 128, O.E4M3, 7)
    _check_weights(C, c, oracle, table, [20000], [3], 7, held=[19990], seed=7)


def test_weights_many_rows_keep_few_chunks():
    """So many pairs that the statistics of the chunks would pass the workspace's bound."""
    C = _crisp()
    _say("weights 9000 rows")
    c, oracle, table, _ = _filled(C, [700], 1, 64, O.INT8, 8)
    heads, n = 300, 699
    ptr = [0, 1]
    q = _rand(heads, 9000, 3)
    w, held = torch.zeros(1, 1, 704, device=DEV), _ints([0])
    got = C.crisp_cache_weights(c, _ints(table), _ints([n]), _ints(ptr), q.to(DEV), w, held)
    want, tol = R.cache_weights(oracle, table, [n], ptr, to_f64(q[:, :1]), 1 / math.sqrt(128), np.zeros((1, 1, 704)), [0])
    live = ~np.isnan(want)
    assert (np.abs(to_f64(got) - want)[live] <= tol[live]).all()


def test_weights_holes_and_bad_pages():
    """Positions without a page take no weight, and their places say so."""
    C = _crisp()
    _say("weights holes")
    c, oracle, table, n_pages = _filled(C, [400, 130], 2, 64, O.E4M3, 4)
    table[0, 1], table[0, 4], table[1, 0] = -1, n_pages + 7, -1
    _check_weights(C, c, oracle, table, [398, 129], [2, 1], 4, held=[300, 129], seed=4)
    table[1] = -1
    _check_weights(C, c, oracle, table, [398, 129], [2, 1], 4, held=[300, 129], seed=4)


@pytest.mark.parametrize("hq", [0, 4])
def test_weights_without_rows(hq):
    """No row in the whole call: what is held goes to out, the positions behind it become 0."""
    C = _crisp()
    _say(f"weights without rows hq={hq}")
    c, oracle, table, _ = _filled(C, [200, 131], 2, 64, O.E4M3, 1)
    _check_weights(C, c, oracle, table, [198, 130], [0, 0], 4, held=[50, 130], seed=1)
    w, out = torch.rand(2, 2, 256, device=DEV), torch.full((2, 2, 256), 7.0, device=DEV)
    rows = torch.zeros(hq, 0 if hq else 3, 128, dtype=torch.bfloat16, device=DEV)
    C.crisp_cache_weights(c, _ints(table), _ints([198, 130]), _ints([0, 0, 0]), rows, w, _ints([50, 200]), out=out)
    want = torch.full_like(out, 7.0)
    want[0, :, :198], want[0, :, :50], want[1, :, :130] = 0.0, w[0, :, :50], w[1, :, :130]
    assert torch.equal(out, want)


def test_weights_of_forks():
    """Sequences that share all their pages: more tiles together than the cache has, so that some sequences' scores wait and others' do not."""
    C = _crisp()
    _say("weights of forks")
    c, oracle, table, _ = _filled(C, [300], 2, 64, O.E4M3, 6)
    _check_weights(C, c, oracle, np.repeat(table, 9, 0), [299] * 9, [1] * 9, 8, held=[299, 0, 5] * 3, seed=6)
    _check_weights(C, c, oracle, np.repeat(table, 9, 0), [298, 1, 250, 64, 299, 0, 127, 298, 60], [1, 2, 0, 1, 1, 1, 1, 2, 1], 8,
                   held=[0] * 9, seed=7)


def test_weights_of_many_sequences():
    """More of them than scores are kept for."""
    C = _crisp()
    _say("weights of 1030 sequences")
    rng = np.random.default_rng(8)
    lens, counts = rng.integers(0, 140, 1030).tolist(), rng.integers(0, 3, 1030).tolist()
    c, oracle, table, _ = _filled(C, [a + b for a, b in zip(lens, counts)], 1, 64, O.INT8, 8)
    _check_weights(C, c, oracle, table, lens, counts, 3, held=lens, seed=8)


def test_weights_of_a_few_rows_beside_many():
    """Few rows a sequence on average, one sequence with many; and the other way round."""
    C = _crisp()
    _say("weights of mixed rows")
    for counts, seed in (([1] * 30 + [90] + [1] * 9, 1), ([100, 1, 0, 140], 2)):
        lens = [70 + 13 * (s % 7) for s in range(len(counts))]
        c, oracle, table, _ = _filled(C, [a + b for a, b in zip(lens, counts)], 2, 64, O.E4M3, seed)
        _check_weights(C, c, oracle, table, lens, counts, 8, held=lens, seed=seed)


@pytest.mark.parametrize("n_seqs,rows", [(3, 40), (70, 9), (70, 1), (3, 2)])
def test_weights_with_rows_before_the_first_sequence(n_seqs, rows):
    """Rows that lie before all sequences, or behind them, weigh nothing."""
    C = _crisp()
    _say(f"weights n_seqs={n_seqs} rows={rows}, rows before the first")
    c, oracle, table, _ = _filled(C, [100] * n_seqs, 1, 64, O.E4M3, n_seqs)
    ends = _ptr([rows] * n_seqs)
    q = _rand(4, int(ends[-1]) + 60, 1)
    args = (c, _ints(table), _ints([100 - rows] * n_seqs))
    w, held = torch.rand(n_seqs, 1, 128, device=DEV), _ints([7] * n_seqs)
    got = [C.crisp_cache_weights(*args, _ints(ends + lead), q[:, 37 - lead:].contiguous().to(DEV), w, held, out=torch.zeros_like(w))
           for lead in (0, 37)]
    assert torch.equal(*got) and got[0].isfinite().all()


def test_weights_values_out_of_range_stay_within_the_buffers():
    """Lengths, offsets of rows and what is held are brought into range; offsets that do not ascend change nothing elsewhere."""
    C = _crisp()
    _say("weights out of range")
    c, oracle, table, _ = _filled(C, [250, 190, 60], 2, 64, O.E4M3, 9)
    t = _ints(table)
    for hq, n in ((4, 6), (8, 100)):
        q = _rand(hq, n, 1).to(DEV)
        w = torch.rand(3, 2, 256, device=DEV)
        big = torch.full((3, 3, 2, 256), 7.0, device=DEV)
        out = big[1]

        def run(lens, ends, held):
            big.fill_(7.0)
            C.crisp_cache_weights(c, t, _ints(lens), _ints(ends), q, w, _ints(held), out=out)
            assert (big[0] == 7.0).all() and (big[2] == 7.0).all()
            return out.clone()

        lowest, highest = -(1 << 31), (1 << 31) - 1
        for first in (1 << 30, 200):  # (rows of the first and the last see places that nothing was stored in: NaN here)
            got = run([first, -7, 40], [lowest, 2, 4, highest], [highest, lowest, 5])
            want = run([min(first, 256), 0, 40], [0, 2, 4, n], [256, 0, 5])
            assert torch.equal(torch.nan_to_num(got, nan=-1.0), torch.nan_to_num(want, nan=-1.0))
            assert first > 256 or not got[:2].isnan().any()
        run([100, 100, 40], [5, 1, 6, 3], [1, 2, 3])
        run([100, 100, 40], [highest, lowest, highest, 0], [1, 2, 3])


def test_weights_and_moves_without_a_table():
    """A table of no pages: nothing is seen, what is held stays, kept positions are zeros."""
    C = _crisp()
    _say("weights and gather, table without pages")
    c, _ = _new(C, 3, 2, 64, O.E4M3)
    empty = torch.empty(2, 0, dtype=torch.int32, device=DEV)
    for rows in (1, 9):
        w = torch.rand(2, 2, 100, device=DEV)
        got = C.crisp_cache_weights(c, empty, _ints([70, 3]), _ints([0, rows, 2 * rows]), _rand(4, 2 * rows, 1).to(DEV), w, _ints([60, 100]),
                                    out=torch.full_like(w, 7.0))
        # no position is in the table's range: lengths are brought into it, only the rows' own positions are left
        want = torch.full_like(w, 7.0)
        want[0, :, :rows], want[1, :, :rows] = w[0, :, :rows], w[1, :, :rows]
        assert torch.equal(got, want)
    kept = torch.zeros(2, 2, 5, dtype=torch.int32, device=DEV)
    C.crisp_cache_gather(c, empty, kept, _ints([5, 0]), _ints([[1], [2]]))
    assert (c.pages[1] == 0).all() and (c.pages[2] == 0x7f).all() and (c.scales[1] == 2.0 ** -64).all()


@pytest.mark.parametrize("gain,scale", [(30.0, 0.0), (1e-3, 0.0), (1.0, 3.0), (1.0, 1e-30)])
def test_weights_sharp_and_flat_scores(gain, scale):
    C = _crisp()
    _say(f"weights gain={gain} scale={scale}")
    c, oracle, table, _ = _filled(C, [520], 2, 64, O.E4M3, 6, spread=3)
    _check_weights(C, c, oracle, table, [510], [10], 4, scale=scale, seed=6, gain=gain)


def test_weights_not_finite():
    """A row that is not finite makes the sums of what it sees NaN: its own KV head's and sequence's, up to its position."""
    C = _crisp()
    _say("weights not finite")
    c, oracle, table, _ = _filled(C, [150, 90], 2, 64, O.E4M3, 9)
    lens, counts = [140, 88], [10, 2]
    for bad in (math.nan, math.inf):
        q = _rand(4, 12, 1)
        w, held = torch.zeros(2, 2, 192, device=DEV), _ints([0, 0])
        clean = C.crisp_cache_weights(c, _ints(table), _ints(lens), _ints(_ptr(counts)), q.to(DEV), w, held, out=torch.zeros_like(w))
        q[1, 4, 9] = bad
        got = C.crisp_cache_weights(c, _ints(table), _ints(lens), _ints(_ptr(counts)), q.to(DEV), w, held, out=torch.zeros_like(w))
        assert torch.isnan(got[0, 0, :145]).all()
        got[0, 0, :145], clean[0, 0, :145] = 0, 0
        assert torch.equal(got, clean)


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("counts", [[2, 1, 1], [9, 1, 4], [12, 10, 12], [40, 3, 33]])
def test_weights_of_rows_whose_scores_are_all_minus_infinity(counts, sign):
    """A row of q that is not finite makes the sums of what it sees NaN, also where all its scores are -infinity: one that sees a single key,
    one that sees many chunks with a hole; scores that wait, scores that do not, calls of many pairs.  What has no page has no sum."""
    C = _crisp()
    _say(f"weights all -infinity counts={counts} sign={sign}")
    lens = [0, 3000, 130]
    full = [a + b for a, b in zip(lens, counts)]
    rng = np.random.default_rng(sum(counts))
    table, n_pages = _table(full, 64, rng)
    c, oracle = _new(C, n_pages, 2, 64, O.E4M3)
    k = _rand(2, sum(full), 1)
    k[:, :, 9] = sign * (0.5 + k[:, :, 9].abs())
    _append(C, c, oracle, table, [0] * 3, full, k, _rand(2, sum(full), 2))
    table[1, 2] = -1
    table[2] = -1  # the third sequence's rows see nothing
    ptr, width = _ptr(counts), table.shape[1] * 64
    q = _rand(4, int(ptr[-1]), 3)
    w, held = rng.random((3, 2, width)).astype(np.float32), lens
    want, tol = R.cache_weights(oracle, table, lens, ptr, to_f64(q), 1 / math.sqrt(128), w.astype(np.float64), held)
    last = counts[1] - 1
    for row, h in ((0, 1), (int(ptr[1]) + last, 2), (int(ptr[2]), 0)):
        q[h, row, 9] = -sign * math.inf
    got = to_f64(C.crisp_cache_weights(c, _ints(table), _ints(lens), _ints(ptr), q.to(DEV), _floats(w), _ints(held),
                                       out=torch.full((3, 2, width), 7.0, device=DEV)))
    nan = np.zeros(want.shape, dtype=bool)
    nan[0, 0, 0] = True
    nan[1, 1, :3000 + counts[1]] = True
    nan[1, 1, 128:192] = False
    assert np.isnan(got[nan]).all()
    live = ~np.isnan(want) & ~nan
    assert (np.abs(got - want)[live] <= tol[live]).all()
    assert (got[1, :, 128:192] == w[1, :, 128:192]).all() and (got[np.isnan(want)] == 7.0).all()


def test_weights_strides_repeat_and_workspaces():
    C = _crisp()
    _say("weights strides, workspaces")
    c, oracle, table, _ = _filled(C, [333], 2, 64, O.E4M3, 2)
    x = _rand(6, 20, 3).to(DEV)
    view = x.transpose(0, 1).contiguous().transpose(0, 1)
    w, held, args = torch.zeros(1, 2, 384, device=DEV), _ints([0]), (_ints(table), _ints([313]), _ints([0, 20]))
    want = C.crisp_cache_weights(c, *args, x, w, held, out=torch.zeros_like(w))
    ws = C.cache_weights_workspace(c, 6, 1, 1000)
    for q in (x, view):
        for space in (None, ws):
            assert torch.equal(C.crisp_cache_weights(c, *args, q, w, held, out=torch.zeros_like(w), ws=space), want)
    one = x[:1].expand(6, 20, 128)
    assert torch.equal(C.crisp_cache_weights(c, *args, one, w, held, out=torch.zeros_like(w)),
                       C.crisp_cache_weights(c, *args, one.contiguous(), w, held, out=torch.zeros_like(w)))


def test_weights_sum_to_the_rows():
    """Every row's weights sum to one: in all the pairs of row and head."""
    C = _crisp()
    _say("weights sum")
    c, oracle, table, _ = _filled(C, [3000, 64], 2, 64, O.E4M3, 5)
    w = torch.zeros(2, 2, 3008, device=DEV)
    C.crisp_cache_weights(c, _ints(table), _ints([2991, 60]), _ints([0, 9, 13]), _rand(8, 13, 1).to(DEV), w, _ints([0, 0]))
    got = w.double().sum(-1).cpu().numpy()
    # a row's sum is off by its weights' errors: (3000 / 16 + 64) 2^-24 + 2^-21 and 2 dS, of scores below 2^5: under 2^-13
    np.testing.assert_allclose(got, [[36.0, 36.0], [16.0, 16.0]], rtol=2.0 ** -13)


# ------------------------------------------------------------------ which tokens stay


def _check_keep(C, w, held, lens, keep, cap, sink, recent):
    kept, count, new, moved = R.cache_keep(w, held, lens, keep, cap, sink, recent)
    out = torch.full(w.shape, 7.0, dtype=torch.float32, device=DEV)
    a, b = C.crisp_cache_keep(_floats(w), _ints(held), _ints(lens), _ints(keep), cap, sink, recent, out)
    np.testing.assert_array_equal(b.cpu().numpy(), count)
    np.testing.assert_array_equal(a.cpu().numpy(), kept)
    y = out.cpu().numpy()
    np.testing.assert_array_equal(y[moved], new[moved])
    assert (y[~moved] == 7.0).all()
    inplace = _floats(w)
    a2, _ = C.crisp_cache_keep(inplace, _ints(held), _ints(lens), _ints(keep), cap, sink, recent, inplace)
    z = inplace.cpu().numpy()
    np.testing.assert_array_equal(z[moved], new[moved])
    np.testing.assert_array_equal(z[~moved], w[~moved])
    a3, _ = C.crisp_cache_keep(_floats(w), _ints(held), _ints(lens), _ints(keep), cap, sink, recent)
    assert torch.equal(a, a2) and torch.equal(a, a3)


@pytest.mark.parametrize("n", [2, 3, 64, 65, 500, 1024, 1025])
def test_keep_every_kind_of_budget(n):
    C = _crisp()
    _say(f"keep n={n}")
    rng = np.random.default_rng(n)
    for m in sorted({1, 2, n // 3 + 1, n - 1}):
        for sink, recent in ((0, 0), (4, 16), (1, 0), (0, 1), (n, n), (3, n), (n, 2)):
            if m < n:
                _check_keep(C, rng.random((1, 2, n + 5)).astype(np.float32), [n], [n], [m], m + 3, sink, recent)


def test_keep_ties_and_special_values():
    """Equal weights go to the lowest positions; 0 and -0 are equal, NaN is below all, what is not held counts as 0."""
    C = _crisp()
    _say("keep ties")
    rng = np.random.default_rng(1)
    n = 3001
    equal = np.full((1, 1, n), 0.25, dtype=np.float32)
    few = rng.integers(0, 3, (1, 1, n)).astype(np.float32)
    zeros = np.where(rng.random((1, 1, n)) < 0.5, 0.0, -0.0).astype(np.float32)
    mixed = rng.choice(np.array([0.0, -0.0, 1.0, -1.0, np.inf, -np.inf, np.nan, 1e-45, -1e-45, 3.4e38], dtype=np.float32), (1, 1, n))
    for w in (equal, few, zeros, mixed):
        for m in (1, 100, 2000, 3000):
            for held in (n, 1500, 0, -3):
                _check_keep(C, w, [held], [n], [m], 3000, 2, 5)


def test_keep_close_weights():
    """Weights that differ in the last bit only, every digit of the selection."""
    C = _crisp()
    _say("keep close weights")
    rng = np.random.default_rng(2)
    bits = np.int32(0x3f000000) + rng.integers(0, 1500, (2, 2, 1400)).astype(np.int32)
    w = bits.view(np.float32)
    _check_keep(C, w, [1400, 1400], [1400, 1300], [700, 333], 1000, 4, 30)
    w = (rng.integers(0, 1 << 31, (1, 3, 5000)).astype(np.uint32) & 0x7f7fffff).view(np.float32)
    _check_keep(C, w, [5000], [4999], [1234], 1234, 0, 0)


def test_keep_batch_of_all_kinds():
    """Sequences that are short enough already, empty, longer than the buffer, budgets above the list or below one."""
    C = _crisp()
    _say("keep batch")
    rng = np.random.default_rng(4)
    lens = [0, 1, 5, 300, 299, 300, 301, 200, 77, -4, 250]
    keep = [3, 1, 5, 100, 299, 300, 100, 0, -1, 2, 151]
    _check_keep(C, rng.random((11, 2, 300)).astype(np.float32), [1000] * 11, lens, keep, 150, 4, 32)


@pytest.mark.parametrize("width", [1, 2, 300, 17000])
def test_keep_lists_longer_than_the_buffer(width):
    """More places in the list than the weights have, budgets above every length among them."""
    C = _crisp()
    _say(f"keep width={width}, longer lists")
    rng = np.random.default_rng(width)
    w = rng.random((3, 2, width)).astype(np.float32)
    lens = [width, max(width // 2, 1), width]
    _check_keep(C, w, [width] * 3, lens, [width - 1, width + 3, width + 70], width + 100, 1, 3)


@pytest.mark.parametrize("n,m", [(16384, 5000), (16385, 16384), (40000, 1), (70001, 30000), (24576, 24575), (33000, 60)])
def test_keep_long_sequences(n, m):
    """About as many tokens as one workgroup takes, and more; also in place."""
    C = _crisp()
    _say(f"keep n={n} m={m}")
    rng = np.random.default_rng(n)
    w = np.exp(3 * rng.standard_normal((1, 2, n))).astype(np.float32)
    _check_keep(C, w, [n], [n], [m], m, 4, 100)
    _check_keep(C, w, [n - 9000], [n], [m], m, 0, 0)


def test_keep_long_sequences_that_share_digits():
    """So many weights alike that the list of those that share the limit's first digit does not hold them: all equal, few values, the last
    bits apart, special values."""
    C = _crisp()
    _say("keep long sequences that share digits")
    rng = np.random.default_rng(11)
    n = 40000
    for w in (np.full((1, 1, n), 0.25), rng.integers(0, 3, (1, 1, n)), (np.int32(0x3f000000) + rng.integers(0, 1 << 20, (1, 1, n)).astype(np.int32)).view(np.float32),
              rng.choice(np.array([0.0, -0.0, 1.0, -1.0, np.inf, -np.inf, np.nan], dtype=np.float32), (1, 1, n))):
        for m in (1, 9000, 39999):
            _check_keep(C, w.astype(np.float32), [n], [n], [m], m, 2, 5)


def test_keep_short_and_long_sequences_in_a_wide_buffer():
    C = _crisp()
    _say("keep short and long in a wide buffer")
    rng = np.random.default_rng(12)
    lens = [30000, 5, 16384, 16385, 0, 1, 700, 25000, 30001]
    keep = [10000, 2, 100, 16000, 3, 1, 699, 25000, 5]
    w = np.exp(2 * rng.standard_normal((9, 2, 30000))).astype(np.float32)
    _check_keep(C, w, [1 << 20] * 9, lens, keep, 16000, 4, 64)
    ws = C.cache_keep_workspace(_floats(w), in_place=True)
    ws.fill_(0xff)
    a = C.crisp_cache_keep(_floats(w), _ints(lens), _ints(lens), _ints(keep), 16000, 4, 64, ws=ws)
    b = C.crisp_cache_keep(_floats(w), _ints(lens), _ints(lens), _ints(keep), 16000, 4, 64)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ------------------------------------------------------------------ the move


def _check_gather(C, c, oracle, table, kept, count, new_table):
    C.crisp_cache_gather(c, _ints(table), _ints(kept), _ints(count), _ints(new_table))
    R.cache_gather(oracle, table, kept, count, new_table)
    n_pages = len(oracle.written)
    got = O.decode(c.pages.cpu().numpy(), c.fmt)
    new = sorted({int(p) for s, row in enumerate(new_table) for b, p in enumerate(row)
                  if 0 <= p < n_pages and b * oracle.block < min(count[s], kept.shape[2])})
    np.testing.assert_array_equal(got[new], oracle.codes[new])
    np.testing.assert_array_equal(c.scales.cpu().numpy()[new], np.ldexp(1.0, oracle.exp[new]))
    old = [p for p in range(n_pages) if oracle.written[p].any() and p not in new]
    at = oracle.written[old]
    np.testing.assert_array_equal(got[old].transpose(0, 3, 1, 2, 4)[at], oracle.codes[old].transpose(0, 3, 1, 2, 4)[at])


def _new_pages(table, n_pages, slots):
    free = [p for p in range(n_pages) if p not in set(table[table >= 0].tolist())]
    t = np.array(free[::-1][:table.shape[0] * slots], dtype=np.int32)
    return t.reshape(table.shape[0], slots)


def _some(rng, n, m, heads):
    return np.stack([np.sort(rng.permutation(n)[:m]) for _ in range(heads)])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("block", [64, 128])
@pytest.mark.parametrize("n,m", [(2, 1), (64, 63), (65, 64), (200, 65), (300, 129), (500, 20), (129, 128)])
def test_gather_lengths(n, m, block, fmt):
    C = _crisp()
    _say(f"gather n={n} m={m} block={block} fmt={fmt}")
    rng = np.random.default_rng(n + m)
    slots = -(-m // block)
    c, oracle, table, n_pages = _filled(C, [n], 2, block, fmt, n, spread=6, extra=slots + 2)
    kept = np.full((1, 2, m + 4), -1, dtype=np.int32)
    kept[0, :, :m] = _some(rng, n, m, 2)
    _check_gather(C, c, oracle, table, kept, [m], _new_pages(table, n_pages, slots))


@pytest.mark.parametrize("fmt", FORMATS)
def test_gather_scales_far_apart(fmt):
    """Pages whose exponents differ by up to 120: small values round to 0 beside large ones and come back to full bits without them."""
    C = _crisp()
    _say(f"gather scales fmt={fmt}")
    rng = np.random.default_rng(5)
    c, oracle, table, n_pages = _filled(C, [640, 320], 1, 64, fmt, 5, spread=60, extra=14)
    kept = np.full((2, 1, 300), -1, dtype=np.int32)
    kept[0, 0, :290], kept[1, 0, :150] = _some(rng, 640, 290, 1), _some(rng, 320, 150, 1)
    _check_gather(C, c, oracle, table, kept, [290, 150], _new_pages(table, n_pages, 5))


@pytest.mark.parametrize("fmt", FORMATS)
def test_gather_of_every_code(fmt):
    """Pages that hold every code, NaN among them, under the smallest and largest scales."""
    C = _crisp()
    _say(f"gather codes fmt={fmt}")
    for e in (-64, 0, 100, 119):
        c = C.make_cache(6, 1, 64, fmt, device=DEV)
        oracle = O.Cache(6, 1, 64, fmt)
        c.pages.copy_(torch.arange(256, dtype=torch.uint8, device=DEV).repeat(c.pages.numel() // 256).view(c.pages.shape))
        c.scales.fill_(2.0 ** e)
        oracle.codes[:], oracle.exp[:] = O.decode(c.pages.cpu().numpy(), fmt), e
        kept = np.arange(0, 128, 2, dtype=np.int32)[None, None]
        _check_gather(C, c, oracle, np.array([[0, 1]], dtype=np.int32), kept, [64], np.array([[3]], dtype=np.int32))


def test_gather_largest_values():
    """The largest bf16, whose e4m3 code is rounded past it: the exponent is found without an overflow."""
    C = _crisp()
    _say("gather largest values")
    for fmt in FORMATS:
        c, oracle = _new(C, 5, 1, 64, fmt)
        x = torch.full((1, 100, 128), 3.3895313892515355e38, dtype=torch.bfloat16)
        x[:, 50:] = 1e-30
        x[:, 10] = -x[:, 10]
        table = np.array([[0, 1]], dtype=np.int32)
        _append(C, c, oracle, table, [0], [100], x, -x)
        kept = np.array([[[5, 10, 40, 60, 70, 99]]], dtype=np.int32)
        _check_gather(C, c, oracle, table, kept, [6], np.array([[3]], dtype=np.int32))


def test_gather_bad_places():
    """Kept positions out of range or without a page become zeros; pages of the new table out of range are not written."""
    C = _crisp()
    _say("gather bad places")
    rng = np.random.default_rng(6)
    c, oracle, table, n_pages = _filled(C, [300, 200, 100], 2, 64, O.E4M3, 6, extra=9)
    new = _new_pages(table, n_pages, 3)
    kept = np.full((3, 2, 150), -1, dtype=np.int32)
    for s, n in enumerate((300, 200, 100)):
        kept[s, :, :90] = _some(rng, n, 90, 2)
    kept[0, 0, 5], kept[0, 1, 7], kept[1, 0, 0] = -1, 1 << 30, 320
    table[0, 2] = -1
    table[1, 1] = n_pages + 5
    new[1, 1], new[2, 0] = -1, n_pages
    _check_gather(C, c, oracle, table, kept, [90, 90, 90], new)
    # a count past the list, of none, below none
    _check_gather(C, c, oracle, table, kept, [1000, 0, -7], new)


def test_gather_of_a_batch_equals_appending_the_kept_values():
    """What gather is said to be: the kept tokens' cached values appended to a fresh sequence."""
    C = _crisp()
    _say("gather equals append")
    rng = np.random.default_rng(7)
    lens, m = [777, 130, 400], [300, 100, 65]
    for fmt in FORMATS:
        c, oracle, table, n_pages = _filled(C, lens, 1, 64, fmt, 7, spread=4, extra=2 * 3 * 5)
        new = _new_pages(table, n_pages, 10)
        one, two = np.ascontiguousarray(new[:, :5]), np.ascontiguousarray(new[:, 5:])
        kept = np.full((3, 1, 300), -1, dtype=np.int32)
        rows = []
        for s in range(3):
            kept[s, 0, :m[s]] = _some(rng, lens[s], m[s], 1)[0]
            rows.append([oracle.values(table[s], lens[s], x)[0][:, kept[s, 0, :m[s]]] for x in (0, 1)])
        _check_gather(C, c, oracle, table, kept, m, one)
        k, v = (torch.from_numpy(np.concatenate([r[x] for r in rows], 1)).to(torch.bfloat16) for x in (0, 1))
        _append(C, c, oracle, two, [0, 0, 0], m, k, v)
        a, b = O.decode(c.pages.cpu().numpy(), fmt), c.scales.cpu().numpy()
        for s in range(3):
            for i in range(m[s]):
                assert (a[one[s, i // 64], :, :, i % 64] == a[two[s, i // 64], :, :, i % 64]).all()
            for p in range(-(-m[s] // 64)):
                assert (b[one[s, p]] == b[two[s, p]]).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("block", [64, 128])
def test_gather_in_any_order(block, fmt):
    """Positions that do not ascend, and the same one several times."""
    C = _crisp()
    _say(f"gather in any order block={block} fmt={fmt}")
    rng = np.random.default_rng(21)
    lens = [300, 90]
    c, oracle, table, n_pages = _filled(C, lens, 2, block, fmt, 21, spread=2, extra=8)
    kept = np.stack([np.stack([rng.permutation(n)[:70] if h == 0 else rng.integers(0, n // 10, 70) for h in range(2)]) for n in lens]).astype(np.int32)
    kept[0, 1, 20:40] = kept[0, 1, 20]
    kept[1, 0, ::-1].sort()
    _check_gather(C, c, oracle, table, kept, [70, 65], _new_pages(table, n_pages, 2))


# ------------------------------------------------------------------ far offsets


def test_most_sequences_of_a_call():
    """As many sequences times KV heads as a call takes, each with the same rows over the same pages."""
    C = _crisp()
    _say("2^20 heads")
    n, heads = 1 << 17, 8
    c, oracle = _new(C, 4, heads, 64, O.E4M3)
    table, ones, rp = torch.zeros(n, 1, dtype=torch.int32, device=DEV), torch.ones(n, dtype=torch.int32, device=DEV), torch.arange(n + 1, dtype=torch.int32, device=DEV)
    k = _rand(heads, 3, 1).to(DEV)
    C.crisp_cache_append(c, table[:1], _ints([0]), _ints([0, 3]), k, k)
    q = _rand(heads, 1, 2).to(DEV).expand(heads, n, 128)
    w, held = torch.zeros(n, heads, 3, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV)
    C.crisp_cache_weights(c, table, 2 * ones, rp, q, w, held)
    assert torch.equal(w, w[:1].expand_as(w)) and (w.sum(-1) - 1).abs().max() < 2.0 ** -18
    kept, count = C.crisp_cache_keep(w, 3 * ones, 3 * ones, 2 * ones, 2, 0, 1)
    assert torch.equal(kept, kept[:1].expand_as(kept)) and (count == 2).all() and (kept[0, :, 1] == 2).all()
    new = torch.full((n, 1), -1, dtype=torch.int32, device=DEV)
    new[0], new[n - 1], new[n // 2] = 1, 2, 3
    C.crisp_cache_gather(c, table, kept, count, new)
    assert torch.equal(c.pages[1], c.pages[2]) and torch.equal(c.pages[1], c.pages[3]) and torch.equal(c.scales[1], c.scales[3])


def test_pages_past_32_bits():
    """The same tokens in a small cache and in the last pages of one of more than 2^32 bytes."""
    C = _crisp()
    _say("pages past 32 bits")
    heads, lens, far = 8, [200, 130], 33000
    small, big = C.make_cache(12, heads, 64, C.CACHE_E4M3, DEV), C.make_cache(far + 12, heads, 64, C.CACHE_E4M3, DEV)
    assert big.pages.numel() > 1 << 32
    table, new = _ints([[3, 0, 5, 1], [2, 4, 6, -1]]), _ints([[7, 8], [9, 10]])
    k, v, q = _rand(heads, 330, 1).to(DEV), _rand(heads, 330, 2).to(DEV), _rand(2 * heads, 2, 3).to(DEV)
    got = []
    for c, at in ((small, 0), (big, far)):
        c.pages.zero_()
        c.scales.fill_(1.0)
        t, nt = torch.where(table < 0, table, table + at), new + at
        C.crisp_cache_append(c, t, _ints([0, 0]), _ints([0, 200, 330]), k, v)
        w = C.crisp_cache_weights(c, t, _ints([n - 1 for n in lens]), _ints([0, 1, 2]), q, torch.zeros(2, heads, 256, device=DEV), _ints([0, 0]))
        many = C.crisp_cache_weights(c, t, _ints([100, 100]), _ints([0, 100, 130]), k[:, :130].repeat(2, 1, 1), torch.zeros_like(w), _ints([0, 0]))
        kept, count = C.crisp_cache_keep(w, _ints(lens), _ints(lens), _ints([100, 70]), 128)
        C.crisp_cache_gather(c, t, kept, count, nt)
        got.append((w, many, kept, c.pages[at:at + 11], c.scales[at:at + 11]))
    for a, b in zip(*got):
        assert torch.equal(a, b)
    assert (big.pages[:12] == 0).all()


def test_weights_and_lists_past_32_bits():
    """Buffers of the largest width, whose last head begins behind 2^31 values, against ones of the usual width."""
    C = _crisp()
    _say("weights and lists past 32 bits")
    heads, n, m, wide = 9, 20000, 100, 1 << 28
    rng = np.random.default_rng(1)
    table, n_pages = _table([n], 64, rng, extra=4)
    c = C.make_cache(n_pages, heads, 64, C.CACHE_E4M3, DEV)
    k, q = _rand(heads, n, 1).to(DEV), _rand(heads, 20, 2).to(DEV)
    C.crisp_cache_append(c, _ints(table), _ints([0]), _ints([0, n]), k, k)
    new = _ints(_new_pages(table, n_pages, 2))
    first = torch.from_numpy(np.exp(rng.standard_normal((1, heads, n)))).float().to(DEV)
    got = []
    for width in (n, wide):
        w = torch.empty(1, heads, width, device=DEV)
        w[:, :, :n] = first
        for rows in (1, 20):
            C.crisp_cache_weights(c, _ints(table), _ints([n - rows]), _ints([0, rows]), q[:, :rows], w, _ints([n]))
        before = w[:, :, :n].clone()
        cap = m if width == n else wide
        kept, count = C.crisp_cache_keep(w, _ints([n]), _ints([n]), _ints([m]), cap, 4, 16, w)
        assert (kept[0, heads - 1, m:] == -1).all()
        c.pages[new.long()] = 0
        C.crisp_cache_gather(c, _ints(table), kept, count, new)
        got.append((before, w[:, :, :n].clone(), kept[:, :, :m].clone(), c.pages[new.long()], c.scales[new.long()]))
    for a, b in zip(*got):
        assert torch.equal(a, b)


# ------------------------------------------------------------------ together


def test_long_choices_in_a_graph():
    """The choice from more tokens than one workgroup takes, captured with a workspace: replays follow the device's lengths and budgets."""
    C = _crisp()
    _say("long choices in a graph")
    w = torch.rand(2, 2, 40000, device=DEV)
    n, keep, held = _ints([40000, 300]), _ints([5000, 100]), _ints([40000, 40000])
    ws = C.cache_keep_workspace(w, in_place=True)
    kept_of = []

    def once():
        kept_of[:] = C.crisp_cache_keep(w, held, n, keep, 20000, 4, 64, w, ws)

    once()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        once()
    captured = list(kept_of)
    for i, (lens, budget) in enumerate((([40000, 300], [5000, 100]), ([20000, 17000], [20000, 16999]), ([16384, 40000], [16000, 1]),
                                        ([30001, 39999], [0, 20001]))):
        x = torch.rand(2, 2, 40000, generator=torch.Generator().manual_seed(i)).to(DEV)
        n.copy_(_ints(lens))
        keep.copy_(_ints(budget))
        w.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*captured, w)]
        w.copy_(x)
        once()
        for a, b in zip(got, (*kept_of, w)):
            assert torch.equal(a, b)


def test_evicting_steps_in_a_graph():
    """Rows appended, attended, weighed; then the sequences cut and moved, all captured: replays follow the device's lengths."""
    C = _crisp()
    _say("evict in a graph")
    heads, hq, lens = 2, 4, [300, 190]
    rng = np.random.default_rng(9)
    c, oracle, table, n_pages = _filled(C, lens, heads, 64, O.E4M3, 9, extra=8)
    new = _new_pages(table, n_pages, 3)
    t, nt, held = _ints(table), _ints(new), _ints([0, 0])
    n, keep, ptr = _ints([l - 1 for l in lens]), _ints([100, 150]), _ints([0, 1, 2])
    q, w = _rand(hq, 2, 1).to(DEV), torch.full((2, heads, 320), math.nan, device=DEV)
    out = torch.zeros_like(w)
    ws = C.cache_weights_workspace(c, hq, 2, 2)
    kept_of = []

    def once():
        C.crisp_cache_weights(c, t, n, ptr, q, w, held, out=out, ws=ws)
        kept, count = C.crisp_cache_keep(out, n + 1, n + 1, keep, 160, 4, 16)
        C.crisp_cache_gather(c, t, kept, count, nt)
        kept_of[:] = [kept, count]

    once()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        once()
    captured = list(kept_of)
    for lengths, budget, seed in (([299, 189], [100, 150], 1), ([150, 189], [160, 60], 2), ([250, 101], [64, 99], 3)):
        n.copy_(_ints(lengths))
        keep.copy_(_ints(budget))
        q.copy_(_rand(hq, 2, seed))
        out.zero_()
        c.pages[torch.from_numpy(new.ravel()).long().to(DEV)] = 0
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (*captured, out, c.pages, c.scales)]
        out.zero_()
        c.pages[torch.from_numpy(new.ravel()).long().to(DEV)] = 0
        once()
        for a, b in zip(got, (*kept_of, out, c.pages, c.scales)):
            # scales of pages that no append has written are NaN here
            assert torch.equal(torch.nan_to_num(a.float(), nan=-1.0), torch.nan_to_num(b.float(), nan=-1.0))


def test_two_streams_at_once():
    C = _crisp()
    _say("evict on two streams")
    sides = []
    for i in range(2):
        lens = [900 + 100 * i, 300]
        c, oracle, table, n_pages = _filled(C, lens, 2, 64, O.E4M3, i, extra=12)
        sides.append(dict(c=c, t=_ints(table), nt=_ints(_new_pages(table, n_pages, 4)), n=_ints([x - 1 for x in lens]), q=_rand(4, 2, i).to(DEV),
                          w=torch.zeros(2, 2, 1024, device=DEV), s=torch.cuda.Stream()))
    ptr, keep, held = _ints([0, 1, 2]), _ints([200, 100]), _ints([0, 0])

    def once(d):
        w = C.crisp_cache_weights(d["c"], d["t"], d["n"], ptr, d["q"], d["w"], held, out=torch.zeros_like(d["w"]))
        kept, count = C.crisp_cache_keep(w, d["n"] + 1, d["n"] + 1, keep, 256)
        C.crisp_cache_gather(d["c"], d["t"], kept, count, d["nt"])
        return w, kept

    want = [once(d) for d in sides]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for i, d in enumerate(sides):
            with torch.cuda.stream(d["s"]):
                got.append((i, once(d)))
    torch.cuda.synchronize()
    for i, (w, kept) in got:
        assert torch.equal(w, want[i][0]) and torch.equal(kept, want[i][1])
