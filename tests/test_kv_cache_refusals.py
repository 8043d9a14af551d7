"""Reservations that KVCache refuses, in the loop that its documentation gives (reserve, attend, advance by the same counts, nothing
read back): rows of a refused sequence are nowhere stored, get 0 and do not count, other sequences go on, and so does the
refused one once it has pages."""
import copy
import math

import numpy as np
import pytest
import torch

from tests import cache_oracle as O
from tests.helpers import to_f64
from tests.test_kv_cache import DEV, Mirror, _ints, _rand

pytestmark = pytest.mark.gpu

FORMATS = [O.E4M3, O.INT8]


def _kv(n_pages, max_seqs, max_tokens, fmt=O.E4M3, block=64):
    from paper_2609_01925_amd.cache import KVCache
    kv = KVCache(2, n_pages, 2, max_seqs=max_seqs, max_tokens=max_tokens, block=block, fmt=fmt, device=DEV)
    return kv, Mirror(2, 2, block, fmt, -(-max_tokens // block))


def _step(kv, mirror, counts, refused, seed, reserve=True, hq=4):
    """One step as documented; sequences in `refused` are expected to get nothing."""
    counts = np.asarray(counts)
    if reserve:
        got = kv.reserve(_ints(counts))
        assert got.tolist() == [0 if s in refused else c for s, c in enumerate(counts)]
    ptr = np.concatenate([[0], np.cumsum(counts)])
    n = int(ptr[-1])
    for layer in range(len(kv.layers)):
        q, k, v = (_rand(h, n, 100 * seed + 10 * layer + i) for i, h in enumerate((hq, 2, 2)))
        o = to_f64(kv.attend(layer, _ints(ptr), q.to(DEV), k.to(DEV), v.to(DEV)))
        for s, c in enumerate(counts):
            a, b = ptr[s], ptr[s + 1]
            if s in refused:
                assert (o[:, a:b] == 0).all(), f"sequence {s} layer {layer}"
            elif c:
                mirror.append(s, layer, k[:, a:b], v[:, a:b])
                want, tol = mirror.attention(s, layer, q[:, a:b])
                assert (np.abs(o[:, a:b] - want) <= tol).all(), f"sequence {s} layer {layer}"
    kv.advance(_ints(counts))
    for s, c in enumerate(counts):
        if c and s not in refused:
            mirror.len[s] += c
    _held(kv, mirror)


def _held(kv, mirror):
    """Lengths, and every held token's codes and scales, as the mirror has them."""
    lens = [mirror.len.get(s, 0) for s in range(kv.table.shape[0])]
    assert kv.seq_len.tolist() == lens
    table, B = kv.table.cpu().numpy(), kv.block
    for layer, cache in enumerate(kv.layers):
        codes, scales = O.decode(cache.pages.cpu().numpy(), cache.fmt), cache.scales.cpu().numpy()
        for s, n in enumerate(lens):
            for j in range(-(-n // B)):
                t, p = min(n - j * B, B), table[s, j]
                want = mirror.seqs[s][layer]
                np.testing.assert_array_equal(codes[p, :, :, :t], want.codes[j, :, :, :t], err_msg=f"sequence {s} page {j}")
                np.testing.assert_array_equal(scales[p], np.ldexp(1.0, want.exp[j]), err_msg=f"sequence {s} page {j}")


def _forked(mirror, src, dst):
    mirror.seqs[dst], mirror.len[dst] = copy.deepcopy(mirror.seqs[src]), mirror.len[src]


@pytest.mark.parametrize("fmt", FORMATS)
def test_no_pages_left(fmt):
    """Five pages: a sequence that finds none left keeps its length while another decodes, and goes on after a free."""
    print(f"[gpu-case] no pages left fmt={fmt}", flush=True)
    kv, mirror = _kv(5, 4, 640, fmt)
    _step(kv, mirror, [100, 60, 128, 0], (), 1)          # 2 + 1 + 2 pages
    for i in range(3):
        _step(kv, mirror, [1, 5, 1, 7], (1, 2, 3), 2 + i)  # 1: past its page; 2: a new page; 3: a first page
    _step(kv, mirror, [3, 4, 0, 0], (), 5)               # 1 has room for four
    kv.free(_ints([2]))
    del mirror.seqs[2], mirror.len[2]
    _step(kv, mirror, [1, 5, 0, 7], (), 6)
    _step(kv, mirror, [1, 1, 9, 1], (2,), 7)


@pytest.mark.parametrize("fmt,block", [(O.E4M3, 64), (O.INT8, 128)])
def test_tokens_taken_back_into_a_shared_page(fmt, block):
    """A sequence taken back into pages that its fork holds: its rows change nothing of the fork's, with the reservation refused and
    without one; a fork of it goes on."""
    print(f"[gpu-case] taken back into a shared page fmt={fmt} block={block}", flush=True)
    kv, mirror = _kv(20, 4, 640, fmt, block)
    _step(kv, mirror, [2 * block, 10, 0, 0], (), 1)
    assert kv.fork(_ints([0]), _ints([2])).tolist() == [[-1, -1]]
    _forked(mirror, 0, 2)
    kv.advance(_ints([-5, 0, 0, 0]))
    mirror.len[0] -= 5
    _step(kv, mirror, [5, 0, 0, 0], (0,), 2, reserve=False)
    for i in range(2):
        _step(kv, mirror, [2, 1, 3, 0], (0,), 3 + i)
    kv.fork(_ints([0]), _ints([3]))
    _forked(mirror, 0, 3)
    _step(kv, mirror, [1, 1, 1, 4], (0,), 5)
    kv.free(_ints([2, 3]))  # the pages are the sequence's own again
    for s in (2, 3):
        del mirror.seqs[s], mirror.len[s]
    _step(kv, mirror, [4, 1, 0, 0], (), 6)


def test_rows_without_a_reservation():
    """Rows that no reservation covers are not stored; one reservation may cover several steps; fewer rows than reserved may count;
    more taken back than held leaves none."""
    print("[gpu-case] rows without a reservation", flush=True)
    kv, mirror = _kv(8, 3, 320)
    _step(kv, mirror, [70, 0, 3], (), 1)
    _step(kv, mirror, [1, 2, 1], (0, 1, 2), 2, reserve=False)
    assert kv.reserve(_ints([6, 0, 0])).tolist() == [6, 0, 0]
    for i in range(3):
        _step(kv, mirror, [2, 0, 0], (), 3 + i, reserve=False)
    _step(kv, mirror, [2, 0, 0], (0,), 6, reserve=False)
    kv.compact()
    _step(kv, mirror, [1, 0, 1], (), 7)
    kv.advance(_ints([0, 0, -100]))
    mirror.len[2] = 0
    _held(kv, mirror)
    mirror.seqs[2] = mirror.new()
    _step(kv, mirror, [1, 0, 4], (), 8)


@pytest.mark.parametrize("n,pages", [(200, 3), (100, 1)])
def test_prompt_without_pages(n, pages):
    """A prompt whose reservation is refused: its attention is that of the prompt, nothing of it is held."""
    print(f"[gpu-case] prompt without pages n={n}", flush=True)
    from paper_2609_01925_amd import crisp as C
    kv, mirror = _kv(pages, 2, 640)
    before = [c.pages.clone() for c in kv.layers]
    counts = _ints([n, 0])
    assert kv.reserve(counts).tolist() == [0, 0]
    q, k, v = (_rand(h, n, i).to(DEV) for i, h in enumerate((4, 2, 2)))
    for layer in range(2):
        assert torch.equal(kv.prefill(layer, 0, q, k, v), C.crisp_prefill_attn(q, k, v, C.make_params()))
    kv.advance(counts)
    assert kv.seq_len.tolist() == [0, 0] and all(torch.equal(a, c.pages) for a, c in zip(before, kv.layers))
    _step(kv, mirror, [1, 60], () if pages > 1 else (1,), 1)


def test_refusals_in_a_graph():
    """A step captured once and replayed through grants and refusals of both kinds, the bookkeeping between the replays eager."""
    print("[gpu-case] refusals in a graph", flush=True)
    kv, mirror = _kv(6, 3, 320)
    rows, hq = 200, 4
    counts, ptr = _ints([0] * 3), _ints([0] * 4)
    q, k, v = (torch.zeros(2, h, rows, 128, dtype=torch.bfloat16, device=DEV) for h in (hq, 2, 2))
    out = torch.zeros(2, hq, rows, 128, dtype=torch.bfloat16, device=DEV)

    def step():
        kv.reserve(counts)
        for layer in range(2):
            kv.attend(layer, ptr, q[layer], k[layer], v[layer], out=out[layer])
        kv.advance(counts)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()

    def replay(c, refused, seed):
        p = np.concatenate([[0], np.cumsum(c)])
        counts.copy_(_ints(c))
        ptr.copy_(_ints(p))
        for x in (q, k, v):
            x.copy_(torch.stack([_rand(x.shape[1], rows, 10 * seed + j) for j in range(2)]))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for s, m in enumerate(c):
            a, b = p[s], p[s + 1]
            for layer in range(2):
                o = to_f64(out[layer][:, a:b])
                if s in refused:
                    assert (o == 0).all()
                elif m:
                    mirror.append(s, layer, k[layer][:, a:b], v[layer][:, a:b])
                    want, tol = mirror.attention(s, layer, q[layer][:, a:b])
                    assert (np.abs(o - want) <= tol).all()
            if m and s not in refused:
                mirror.len[s] += m
        _held(kv, mirror)

    replay([128, 9, 0], (), 1)
    kv.fork(_ints([0]), _ints([2]))
    _forked(mirror, 0, 2)
    kv.advance(_ints([-1, 0, 0]))
    mirror.len[0] -= 1
    replay([1, 1, 1], (0,), 2)      # 0 would write into 2's page
    replay([1, 190, 1], (0, 1), 3)  # 1 asks for three pages of the two that are left
    replay([0, 60, 2], (), 4)
    kv.free(_ints([2]))
    del mirror.seqs[2], mirror.len[2]
    replay([1, 1, 0], (), 5)


@pytest.mark.parametrize("n", [1, 2, 150])
def test_prompt_of_a_sequence_that_holds_tokens(n):
    """prefill attends to the prompt alone: of a sequence that holds tokens it stores nothing, and its result says so."""
    print(f"[gpu-case] prompt of a sequence that holds tokens n={n}", flush=True)
    from paper_2609_01925_amd import crisp as C
    kv, mirror = _kv(8, 2, 640)
    _step(kv, mirror, [70, 3], (), 1)
    kv.reserve(_ints([n, 0]))
    q, k, v = (_rand(h, n, i).to(DEV) for i, h in enumerate((4, 2, 2)))
    for layer in range(2):
        o = kv.prefill(layer, 0, q, k, v)
        assert o[:, [0, n - 1]].isnan().all()
        assert torch.equal(o[:, 1:n - 1], C.crisp_prefill_attn(q, k, v, C.make_params())[:, 1:n - 1])
    _held(kv, mirror)
    _step(kv, mirror, [2, 1], (), 2)
    kv.free(_ints([0]))
    kv.reserve(_ints([n, 0]))
    assert torch.equal(kv.prefill(0, 0, q, k, v), C.crisp_prefill_attn(q, k, v, C.make_params()))


@pytest.mark.parametrize("seed", range(8))
def test_histories(seed):
    """Steps with and without reservations, forks, ends, tokens taken back and compactions in a random order on few pages: what is
    granted, room, pages, tables, lengths and every held token after each of them."""
    print(f"[gpu-case] KVCache histories seed={seed}", flush=True)
    rng = np.random.default_rng(seed)
    S, block = int(rng.integers(2, 7)), int(rng.choice([64, 128]))
    n_pages = int(rng.integers(3, 16))
    kv, mirror = _kv(n_pages, S, int(rng.integers(2, 6)) * block, int(rng.integers(2)), block)
    pool, room = O.Pool(n_pages, block, kv.table.cpu().numpy(), [0] * S), np.zeros(S, dtype=int)
    for step in range(25):
        pool.seq_len = [mirror.len.get(s, 0) for s in range(S)]
        op = rng.choice(["step"] * 5 + ["fork", "free", "back", "compact"])
        if op == "step":
            counts = rng.integers(0, rng.choice([2, 6, block + 10]), S) * (rng.random(S) < 0.8)
            if rng.random() < 0.85:
                want = np.array(pool.reserve(counts.tolist()))
                assert kv.reserve(_ints(counts)).tolist() == want.tolist(), step
                room = np.where(want < counts, 0, np.maximum(room, want))
            else:
                counts = np.where(room > 0, np.minimum(counts, room), counts)
            refused = [s for s in range(S) if counts[s] and not room[s]]
            if counts.sum():
                _step(kv, mirror, counts, refused, 100 * seed + step, reserve=False)
            room = np.maximum(room - counts, 0)
        elif op == "fork":
            src, dst = rng.integers(0, S, (2, int(rng.integers(1, 4))))
            want, seqs, lens = pool.fork(src.tolist(), dst.tolist()), copy.deepcopy(mirror.seqs), dict(mirror.len)
            assert [tuple(x) for x in kv.fork(_ints(src), _ints(dst)).tolist()] == want, step
            for s, d, pair in zip(src, dst, want):
                if pair != (-2, -2):
                    mirror.seqs[d], mirror.len[d] = copy.deepcopy(seqs.get(s, mirror.new())), lens.get(s, 0)
        elif op == "free":
            ids = rng.integers(-1, S + 1, 2)
            pool.free(ids.tolist())
            kv.free(_ints(ids))
            for s in ids[(ids >= 0) & (ids < S)]:
                mirror.seqs.pop(s, None), mirror.len.pop(s, None)
                room[s] = 0
        elif op == "back":
            back = rng.integers(0, block, S) * (rng.random(S) < 0.4)
            kv.advance(_ints(-back))
            for s in np.nonzero(back)[0]:
                mirror.len[s] = max(0, mirror.len.get(s, 0) - int(back[s]))
                mirror.seqs.setdefault(s, mirror.new())
                room[s] = 0
        else:
            pool.compact()
            kv.compact()
        assert kv.table.tolist() == [list(r) for r in pool.table], (step, op)
        assert kv.pool.tolist() == pool.words().tolist() and kv.room.tolist() == room.tolist(), (step, op)
        _held(kv, mirror)
