"""Attention over the 8-bit cache for queries that are not finite and see few tokens: by the formula a row with a NaN or
an infinity among its elements is NaN as soon as it sees a token, and 0 if it sees none."""
import math

import numpy as np
import pytest
import torch

from tests import cache_oracle as O
from tests.helpers import to_f64
from tests.test_cache import DEV, FORMATS, _append, _crisp, _ints, _new, _ptr, _rand, _say, _table

pytestmark = pytest.mark.gpu

BAD = [math.nan, math.inf, -math.inf]


def _run(fmt, hq, lens, counts, table, n_pages, width, where):
    """Rows of q at `where` = [(head, row, value)] are not finite: NaN where they see a token, the others as the oracle has them."""
    C = _crisp()
    wide = np.full((len(lens), width), -1, dtype=np.int32)
    wide[:, :table.shape[1]] = table
    c, oracle = _new(C, n_pages, 2, 64, fmt)
    _append(C, c, oracle, wide, 0 * lens, lens, _rand(2, lens.sum(), 1), _rand(2, lens.sum(), 2))
    _append(C, c, oracle, wide, lens, counts, _rand(2, counts.sum(), 3), _rand(2, counts.sum(), 4))
    ptr = _ptr(counts)
    seq = np.searchsorted(ptr, np.arange(counts.sum()), side="right") - 1
    sees = np.array([any(wide[s, j] >= 0 for j in range((lens[s] + r - ptr[s]) // 64 + 1)) for r, s in enumerate(seq)])
    q = _rand(hq, counts.sum(), 5)
    bad = np.zeros(q.shape[:2], dtype=bool)
    for h, r, value in where:
        q[h, r, (7 * h + r) % 128] = value
        bad[h, r] = True
    o = to_f64(C.crisp_cache_attn(c, _ints(wide), _ints(lens), _ints(ptr), q.to(DEV)))
    q[torch.from_numpy(bad)] = 0
    want, tol = oracle.attention(wide, lens, ptr, to_f64(q), 1 / math.sqrt(128))
    nan = bad & sees
    assert np.isnan(o[nan]).all(), [(h, r, lens[seq[r]] + r - ptr[seq[r]]) for h, r in np.argwhere(nan & ~np.isnan(o).all(-1))]
    assert (np.abs(o - want)[~nan] <= tol[~nan]).all()
    assert (o[:, ~sees] == 0).all()


# rows a sequence and pages of the table that make units of 16, 32 and 128 rows (4 query heads over 2)
@pytest.mark.parametrize("rows,width", [(1, 17), (12, 17), (60, 900)])
@pytest.mark.parametrize("fmt", FORMATS)
def test_rows_that_see_less_than_a_tile(fmt, rows, width):
    """Histories of no token to one tile, some whole head of every sequence's last row bad, one value each; and one row that sees nothing."""
    _say(f"rows that see less than a tile fmt={fmt} rows={rows}")
    lens = np.array([0, 1, 15, 16, 30, 47, 48, 62, 63, 64, 65, 20])
    counts = np.full(len(lens), rows)
    table, n_pages = _table(lens + counts, 64, np.random.default_rng(rows))
    table[-1] = -1
    ends = _ptr(counts)[1:] - 1
    where = [(h, e, BAD[(h + i) % 3]) for i, e in enumerate(ends) for h in (0, 2, 3)]
    where += [(1, e - rows + 1, BAD[i % 3]) for i, e in enumerate(ends)]
    _run(fmt, 4, lens, counts, table, n_pages, width, where)


@pytest.mark.parametrize("rows,width", [(12, 17), (60, 1300)])
@pytest.mark.parametrize("fmt", FORMATS)
def test_rows_before_the_first_page_stay_zero(fmt, rows, width):
    """Rows of one unit before and behind the first position that has a page: a bad row is 0 there and NaN here."""
    _say(f"rows before the first page fmt={fmt} rows={rows}")
    lens, counts = np.array([64 - rows // 2, 128 - rows // 2, 10]), np.array([rows] * 3)
    table, n_pages = _table(lens + counts, 64, np.random.default_rng(rows))
    table[0, 0] = table[1, 0] = table[1, 1] = -1
    n = int(counts.sum())
    where = [(h, r, BAD[(h + r) % 3]) for r in range(n) for h in (1, 2) if (r + h) % 2]
    _run(fmt, 4, lens, counts, table, n_pages, width, where)
