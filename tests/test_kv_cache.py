"""The serving path on the cache (paper_2609_01925_amd/cache.py): prompts by sparse prefill, decoding steps,
drafted tokens taken back, forks, ends of sequences and compaction, on two layers, against one 64-bit
cache a sequence and layer (tests/cache_oracle.py)."""
import copy
import math
import sys

import numpy as np
import pytest
import torch

from tests import cache_oracle as O
from tests.helpers import to_f64

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device=DEV)


def _rand(heads, n, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(heads, n, 128, generator=g) * scale).to(torch.bfloat16)


class Mirror:
    """What each sequence should hold: per layer an oracle cache of its own with its pages in order."""

    def __init__(self, layers, heads, block, fmt, slots):
        self.new = lambda: [O.Cache(slots, heads, block, fmt) for _ in range(layers)]
        self.table = np.arange(slots, dtype=np.int32)[None]
        self.seqs, self.len = {}, {}

    def append(self, s, layer, k, v):
        caches = self.seqs.setdefault(s, self.new())
        n = self.len.setdefault(s, 0)
        caches[layer].append(self.table, [n], [0, k.shape[1]], to_f64(k), to_f64(v))

    def attention(self, s, layer, q):
        return self.seqs[s][layer].attention(self.table, [self.len[s]], [0, q.shape[1]], to_f64(q), 1 / math.sqrt(128))


def _step(kv, mirror, counts, seed, hq=4, hkv=2, scale=1.0):
    """One step of all layers: counts[s] rows of each sequence."""
    got = kv.reserve(_ints(counts))
    assert got.tolist() == counts
    ptr = np.concatenate([[0], np.cumsum(counts)])
    n = int(ptr[-1])
    for layer in range(len(kv.layers)):
        q, k, v = (_rand(h, n, 100 * seed + 10 * layer + i, scale) for i, h in enumerate((hq, hkv, hkv)))
        o = to_f64(kv.attend(layer, _ints(ptr), q.to(DEV), k.to(DEV), v.to(DEV)))
        for s, c in enumerate(counts):
            if c:
                a, b = ptr[s], ptr[s + 1]
                mirror.append(s, layer, k[:, a:b], v[:, a:b])
                want, tol = mirror.attention(s, layer, q[:, a:b])
                assert (np.abs(o[:, a:b] - want) <= tol).all(), f"sequence {s} layer {layer}"
    kv.advance(_ints(counts))
    for s, c in enumerate(counts):
        if c:
            mirror.len[s] += c


@pytest.mark.parametrize("fmt,block", [(O.E4M3, 64), (O.INT8, 128)])
def test_prompts_steps_forks_and_compaction(fmt, block):
    from paper_2609_01925_amd import crisp as C
    from paper_2609_01925_amd.cache import KVCache
    print(f"[gpu-case] KVCache fmt={fmt} block={block}", flush=True)
    sys.stdout.flush()
    kv = KVCache(2, 24, 2, max_seqs=6, max_tokens=640, block=block, fmt=fmt, device=DEV)
    mirror = Mirror(2, 2, block, fmt, 640 // block)
    for s, n in ((0, 300), (3, 131)):  # two prompts
        counts = [0] * 6
        counts[s] = n
        assert kv.reserve(_ints(counts)).tolist() == counts
        for layer in range(2):
            q, k, v = (_rand(h, n, 10 * s + layer + 50 * i).to(DEV) for i, h in enumerate((4, 2, 2)))
            o = kv.prefill(layer, s, q, k, v)
            assert torch.equal(o, C.crisp_prefill_attn(q, k, v, C.make_params()))
            mirror.append(s, layer, k, v)
        kv.advance(_ints(counts))
        mirror.len[s] = n
    for i in range(3):
        _step(kv, mirror, [1, 0, 0, 1, 0, 0], 1 + i)
    assert kv.fork(_ints([0, 0, 3]), _ints([1, 2, 4]))[:, 0].tolist() != [-2] * 3
    for s, d in ((0, 1), (0, 2), (3, 4)):
        mirror.seqs[d], mirror.len[d] = copy.deepcopy(mirror.seqs[s]), mirror.len[s]
    _step(kv, mirror, [1, 1, 1, 1, 1, 0], 5, scale=4.0)  # they part, larger values than before
    _step(kv, mirror, [4, 0, 3, 5, 1, 0], 6)             # drafted tokens ...
    kv.advance(_ints([-3, 0, -1, -5, 0, 0]))             # ... of which some are taken back
    for s, c in ((0, 3), (2, 1), (3, 5)):
        mirror.len[s] -= c
    _step(kv, mirror, [2, 1, 1, 70, 1, 0], 7)
    kv.free(_ints([0, 3]))
    for s in (0, 3):
        del mirror.seqs[s], mirror.len[s]
    assert kv.compact().item() >= 0
    used = (kv.pool[:24] > 0).nonzero()[:, 0].tolist()
    assert used == list(range(len(used)))
    _step(kv, mirror, [0, 1, 2, 0, 1, 0], 8)
    _step(kv, mirror, [90, 0, 1, 0, 1, 200], 9, scale=0.5)  # chunks of new sequences in the freed places
    too_many = [0, 10000, 0, 0, 0, 0]
    assert kv.reserve(_ints(too_many)).tolist() == [0] * 6
    kv.free(_ints([0, 1, 2, 3, 4, 5]))
    assert (kv.pool == 0).all() and (kv.table == -1).all() and (kv.seq_len == 0).all()


def test_serving_loop_in_graphs():
    """A step (reserve, append and attention of two layers, advance) and a turnover (free, fork with its page copies,
    compaction) captured once each and replayed in turn with other counts and ids, beside the same calls made
    eagerly on a second cache: equal outputs, pages, tables and pools after every replay."""
    from paper_2609_01925_amd import crisp as C
    from paper_2609_01925_amd.cache import KVCache
    print("[gpu-case] serving loop in graphs", flush=True)
    n, hq, hkv = 5, 4, 2
    make = lambda: KVCache(2, 40, hkv, max_seqs=n, max_tokens=512, block=64, device=DEV)
    rng = np.random.default_rng(1)
    counts, ptr, rows = torch.zeros(n, dtype=torch.int32, device=DEV), torch.zeros(n + 1, dtype=torch.int32, device=DEV), 90
    ids, src, dst = (torch.full((2,), -1, dtype=torch.int32, device=DEV) for _ in range(3))
    q, k, v = (torch.zeros(2, h, rows, 128, dtype=torch.bfloat16, device=DEV) for h in (hq, hkv, hkv))
    out = [torch.zeros(2, hq, rows, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2)]

    def step(kv, o):
        kv.reserve(counts)
        for layer in range(2):
            kv.attend(layer, ptr, q[layer], k[layer], v[layer], out=o[layer])
        kv.advance(counts)

    def turnover(kv):
        kv.free(ids)
        kv.fork(src, dst)
        kv.compact()

    eager, other = make(), make()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):  # nothing reserved, nothing forked: only what a first call loads
        step(other, out[1])
        turnover(other)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.graph(graphs[0]):
        step(other, out[1])
    with torch.cuda.graph(graphs[1]):
        turnover(other)
    held = np.zeros(n, dtype=np.int64)
    for i in range(8):
        c = rng.integers(0, 18, n)
        counts.copy_(_ints(c))
        ptr.copy_(_ints(np.concatenate([[0], np.cumsum(c)])))
        for x in (q, k, v):
            x.copy_(torch.stack([_rand(x.shape[1], rows, 10 * i + j) for j in range(2)]))
        torch.cuda.synchronize()
        step(eager, out[0])
        graphs[0].replay()
        torch.cuda.synchronize()
        held += c
        assert torch.equal(out[0], out[1]), i
        gone = int(rng.integers(n))
        parent = int(rng.choice([s for s in range(n) if s != gone]))
        ids.copy_(_ints([gone, -1]))
        src.copy_(_ints([parent, n]))
        dst.copy_(_ints([gone, gone]))
        torch.cuda.synchronize()
        turnover(eager)
        graphs[1].replay()
        torch.cuda.synchronize()
        held[gone] = held[parent]
        assert eager.seq_len.tolist() == held.tolist()
        for x, y in ((eager.seq_len, other.seq_len), (eager.table, other.table), (eager.pool, other.pool)):
            assert torch.equal(x, y), i
        used = int((eager.pool[:40] > 0).sum())
        assert 0 < used < 40
        for a, b in zip(eager.layers, other.layers):
            _same_tokens(eager, a, b, used)


def _same_tokens(kv, a, b, used):
    """Codes of the tokens held and scales of the pages in use, equal in two caches of one table."""
    assert torch.equal(a.scales[:used], b.scales[:used])
    table, x, y = kv.table.cpu().numpy(), O.decode(a.pages.cpu().numpy(), a.fmt), O.decode(b.pages.cpu().numpy(), b.fmt)
    for s, n in enumerate(kv.seq_len.tolist()):
        for j in range(-(-n // kv.block)):
            t = min(n - j * kv.block, kv.block)
            np.testing.assert_array_equal(x[table[s, j], :, :, :t], y[table[s, j], :, :, :t])


def test_sequence_index_is_checked():
    from paper_2609_01925_amd.cache import KVCache
    kv = KVCache(1, 4, 1, max_seqs=2, max_tokens=128, device=DEV)
    x = _rand(1, 10, 0).to(DEV)
    for seq in (-1, 2):
        with pytest.raises(ValueError):
            kv.prefill(0, seq, x, x, x)
    with pytest.raises(ValueError):
        KVCache(0, 4, 1, 2, 128, device=DEV)
