"""KVCache after evictions and with rows that do not stay: positions go on as they were, against a second cache that is given turned rows; what
rows that are not taken, or taken back, leave in the weights, against counted sums; what a take-back after an eviction takes,
against the 64-bit mirror."""
import pytest
import torch

from tests import cache_oracle as O
from tests import test_kv_evict as E
from tests.test_kv_cache import _ints

pytestmark = pytest.mark.gpu

DEV = E.DEV


def test_positions_go_on_after_evictions():
    """A cache with rope equals one without that is evicted alike and given q and k turned at positions counted here: through two cuts, a
    fork, tokens taken back and a sequence that begins anew."""
    from paper_2609_01925_amd import crisp as C
    from paper_2609_01925_amd.cache import KVCache
    E._say("KVCache positions after evictions")
    rope = C.make_rope(128, C.ROPE_HALF, 10000.0)
    a, b = (KVCache(1, 60, 2, max_seqs=4, max_tokens=640, device=DEV, rope=r, weights=True) for r in (rope, None))
    pos, lens = [0] * 4, [0] * 4

    def step(counts, seed, call="attend"):
        for kv in (a, b):
            assert kv.reserve(_ints(counts)).tolist() == counts
        q, k, v = E._qkv(sum(counts), seed)
        ptr = E._ptr(counts)
        turned = C.crisp_rope(rope, _ints(pos), ptr, q, k)
        x = getattr(a, call)(0, ptr, q, k, v, weigh=True)
        assert torch.equal(x, getattr(b, call)(0, ptr, *turned, v, weigh=True))
        other = C.crisp_rope(rope, _ints(lens), ptr, q, k)  # with the lengths as positions
        for s, (i, j) in enumerate(zip(ptr.tolist(), ptr.tolist()[1:])):
            assert torch.equal(other[0][:, i:j], turned[0][:, i:j]) == (i == j or lens[s] == pos[s])
        advance(counts, True)

    def advance(counts, weighed=False):
        for kv in (a, b):
            kv.advance(_ints(counts), weighed=weighed)
        for s, c in enumerate(counts):
            pos[s], lens[s] = pos[s] + c, lens[s] + c
        same()

    def evict(keep):
        want = [m if 0 < m < n else 0 for m, n in zip(keep, lens)]
        for kv in (a, b):
            assert kv.evict(_ints(keep), 128, 4, 16).tolist() == want
        lens[:] = [m or n for m, n in zip(want, lens)]
        same()

    def same():
        assert a.pos.tolist() == pos and a.seq_len.tolist() == lens
        assert torch.equal(a.held, b.held)
        for s, n in enumerate(a.held.tolist()):
            assert torch.equal(a.weights[0][s, :, :n], b.weights[0][s, :, :n])
        E._caches(a, b)

    step([300, 150, 0, 90], 1, "prefill_packed")
    step([1, 1, 0, 1], 2)
    evict([100, 64, 50, 0])
    step([1, 3, 0, 1], 3)
    step([70, 1, 0, 0], 4)
    evict([128, 0, 0, 20])
    step([2, 1, 0, 40], 5)
    for kv in (a, b):
        kv.fork(_ints([0]), _ints([2]))
    pos[2], lens[2] = pos[0], lens[0]
    same()
    step([1, 1, 1, 1], 6)
    advance([0, -2, -1, -30])
    step([1, 2, 5, 1], 7)
    for kv in (a, b):
        kv.free(_ints([1]))
    pos[1] = lens[1] = 0
    step([0, 33, 0, 0], 8, "prefill_packed")
    step([1, 1, 1, 1], 9)


def test_rows_that_are_not_taken_keep_what_they_weighed():
    """advance() with fewer rows than were weighed, or negative: the tokens that stay keep the attention of the others.  A step that is weighed
    twice counts twice."""
    from paper_2609_01925_amd.cache import KVCache
    E._say("KVCache rows not taken")
    kv = KVCache(1, 10, 1, max_seqs=1, max_tokens=320, device=DEV, weights=True)
    total = lambda n: kv.weights[0][0, 0, :n].double().sum().item()
    near = lambda x, y: abs(x - y) <= 2.0 ** -13 * y  # as test_weights_sum_to_the_rows
    kv.reserve(_ints([100]))
    kv.prefill(0, 0, *E._qkv(100, 1, 2, 1), weigh=1)
    kv.advance(_ints([100]), weighed=True)
    assert near(total(100), 2)
    kv.reserve(_ints([4]))
    rows = E._qkv(4, 2, 2, 1)
    kv.attend(0, E._ptr([4]), *rows, weigh=True)
    assert near(total(104), 2 + 8)
    left = kv.weights[0][0, 0].clone()
    kv.advance(_ints([1]), weighed=True)  # three of them are not taken
    assert kv.held.tolist() == [101] and torch.equal(kv.weights[0][0, 0, :101], left[:101])
    assert total(101) > 2 + 4  # more than the one row's
    had = total(101)
    kv.reserve(_ints([2]))
    rows = E._qkv(2, 3, 2, 1)
    kv.attend(0, E._ptr([2]), *rows, weigh=True)
    assert near(total(103), had + 4)
    # once more: the tokens held before have it twice, the two rows' own weight, not held yet, starts anew
    kv.attend(0, E._ptr([2]), *rows, weigh=True)
    assert had + 4 < total(103) < had + 8
    kv.advance(_ints([2]), weighed=True)
    left = kv.weights[0][0, 0].clone()
    kv.advance(_ints([-2]))
    assert kv.held.tolist() == [101] and torch.equal(kv.weights[0][0, 0, :101], left[:101])


@pytest.mark.parametrize("fmt,block", [(O.E4M3, 64), (O.INT8, 128)])
def test_rows_taken_back_after_an_eviction(fmt, block):
    """They are the last places of each KV head: the last `recent` tokens, then whatever else stayed."""
    from paper_2609_01925_amd.cache import KVCache
    E._say(f"KVCache rows taken back after an eviction fmt={fmt}")
    kv = KVCache(2, 20, 2, max_seqs=1, max_tokens=640, block=block, fmt=fmt, device=DEV, weights=True)
    mirror = E.Evicting(2, 2, block, fmt, 640 // block)
    E._step(kv, mirror, [200], 1)
    before = E._weights_of(kv)
    assert kv.evict(_ints([80]), 80, 4, 8).tolist() == [80]
    mirror.evict(before, [80], [80], 4, 8)
    kv.advance(_ints([-20]))
    mirror.len[0] -= 20
    assert kv.seq_len.tolist() == [60] and kv.held.tolist() == [60] and kv.pos.tolist() == [180]
    E._step(kv, mirror, [3], 2)
