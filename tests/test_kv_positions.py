"""KVCache after evictions: positions go on as they were, against a second cache that is given turned rows."""
import pytest
import torch

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
