"""Rotary positions and attention over packed prompts through the public binding, against the 64-bit oracle (tests/packed_oracle.py)
within counted roundings: layouts, parts of a head, frequency rules, far positions, prompts of none to many tokens at any
place of a block, strides, rows that no sequence covers, values that are not finite, streams and graphs."""
import math
import sys

import numpy as np
import pytest
import torch

from tests import packed_oracle as R
from tests.helpers import to_f64

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


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


def _ptr(counts, lead=0):
    return np.concatenate([[lead], lead + np.cumsum(counts)]).astype(np.int64)


def _worst(got, want, tol):
    live = ~np.isnan(want)
    assert np.isfinite(got[live]).all()
    off = np.abs(got - want)[live]
    return np.max(np.where(off > 0, off / np.maximum(tol[live], 1e-300), 0.0), initial=0.0)


# ------------------------------------------------------------------ rotary positions


def _check_rope(C, counts, start, hq, hkv, dim=128, layout=R.HALF, lead=0, tail=0, base=10000.0, rule=R.PLAIN, rest=(), seed=0):
    ptr = _ptr(counts, lead)
    n = int(ptr[-1]) + tail
    q, k = _rand(hq, n, seed), _rand(max(hkv, 1), n, seed + 1)[:hkv]
    table = C.make_rope(dim, layout, base, rule, *rest)
    f, gain = R.frequencies(dim, base, rule, *rest)
    fill = torch.full((hq, n, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    fill_k = torch.full((max(hkv, 1), n, 128), 7.0, dtype=torch.bfloat16, device=DEV)[:hkv]
    yq, yk = C.crisp_rope(table, _ints(start), _ints(ptr), q.to(DEV), k.to(DEV) if hkv else None, fill, fill_k if hkv else None)
    covered = np.zeros(n, dtype=bool)
    covered[ptr[0]:ptr[-1]] = True
    for x, y in ((q, yq),) + (((k, yk),) if hkv else ()):
        want, tol = R.rope(to_f64(x), start, ptr, f, gain, dim, layout)
        got = to_f64(y)
        worst = _worst(got, want, tol)
        assert worst <= 1.0, f"{worst:.3f} of the tolerance"
        assert (got[:, ~covered] == 7.0).all()


@pytest.mark.parametrize("layout", [R.HALF, R.INTERLEAVED])
@pytest.mark.parametrize("dim", [16, 32, 48, 64, 96, 112, 128])
def test_rope_parts_of_a_head(dim, layout):
    C = _crisp()
    _say(f"rope dim={dim} layout={layout}")
    _check_rope(C, [1, 0, 37, 5], [3, 9, 100, 0], 4, 2, dim, layout, lead=2, tail=3)


@pytest.mark.parametrize("rule,rest", [(R.PLAIN, ()), (R.LINEAR, (4.0,)), (R.BASE, (4.0,)), (R.BANDS, (8.0, 8192.0, 1.0, 4.0)),
                                       (R.RAMP, (16.0, 4096.0, 1.0, 32.0)), (R.RAMP, (1.0, 64.0, 0.5, 100.0))])
@pytest.mark.parametrize("dim", [64, 128])
def test_rope_rules(dim, rule, rest):
    C = _crisp()
    _say(f"rope rule={rule} dim={dim}")
    _check_rope(C, [20, 3], [0, 5000], 3, 1, dim, base=500000.0, rule=rule, rest=rest)


@pytest.mark.parametrize("start", [-(1 << 31), -12345, (1 << 20) + 7, (1 << 30) + 12345, (1 << 31) - 1])
def test_rope_far_positions(start):
    C = _crisp()
    _say(f"rope start={start}")
    _check_rope(C, [5], [start], 2, 1)
    _check_rope(C, [4], [start], 2, 1, layout=R.INTERLEAVED)


@pytest.mark.parametrize("n_seqs,rows", [(1, 1), (63, 1), (64, 1), (65, 1), (300, 2), (5000, 1)])
def test_rope_steps_of_many_sequences(n_seqs, rows):
    """Some sequences without rows, more sequences than one round of the look-up holds."""
    C = _crisp()
    _say(f"rope n_seqs={n_seqs}")
    rng = np.random.default_rng(n_seqs)
    counts = [0 if n_seqs > 1 and rng.random() < 0.2 else rows for _ in range(n_seqs)]
    _check_rope(C, counts, rng.integers(0, 100000, n_seqs), 2, 1, seed=n_seqs)


def test_rope_heads_strides_and_in_place():
    C = _crisp()
    _say("rope strides, in place, without k")
    n, hq, hkv = 50, 7, 2
    both = _rand(hq + 2 * hkv, n, 3).to(DEV)
    packed = both.transpose(0, 1).contiguous()  # [n, heads, 128]
    view = packed.transpose(0, 1)
    start, ptr = _ints([11, 500]), _ints([0, 20, 50])
    t = C.make_rope(96)
    want = C.crisp_rope(t, start, ptr, both[:hq].contiguous(), both[hq:hq + hkv].contiguous())
    got = C.crisp_rope(t, start, ptr, view[:hq], view[hq:hq + hkv])
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    rest = packed[:, hq + hkv:].clone()
    a, b = C.crisp_rope(t, start, ptr, view[:hq], view[hq:hq + hkv], view[:hq], view[hq:hq + hkv])
    assert a.data_ptr() == packed.data_ptr() and torch.equal(a, want[0]) and torch.equal(b, want[1])
    assert torch.equal(packed[:, hq + hkv:], rest)
    only, none = C.crisp_rope(t, start, ptr, both[:hq].contiguous())
    assert none is None and torch.equal(only, want[0])
    # one head for all, and one row for all
    same = both[:1].expand(3, n, 128)
    assert torch.equal(C.crisp_rope(t, start, ptr, same)[0], C.crisp_rope(t, start, ptr, same.contiguous())[0])
    row = both[:2, :1].expand(2, n, 128)
    assert torch.equal(C.crisp_rope(t, start, ptr, row)[0], C.crisp_rope(t, start, ptr, row.contiguous())[0])


def test_rope_many_heads_of_a_long_prompt():
    """Several heads a workgroup, more rows than one; the first and last rows against the oracle, all against a call of a few heads."""
    C = _crisp()
    _say("rope 4000 rows, 32 + 8 heads")
    q, k = _rand(32, 4000, 1).to(DEV), _rand(8, 4000, 2).to(DEV)
    start, ptr = _ints([17]), _ints([0, 4000])
    t = C.make_rope()
    a, b = C.crisp_rope(t, start, ptr, q, k)
    for h in (0, 13, 31):
        assert torch.equal(a[h:h + 1], C.crisp_rope(t, start, ptr, q[h:h + 1])[0])
    assert torch.equal(b[5:6], C.crisp_rope(t, start, ptr, k[5:6])[0])
    f, gain = R.frequencies(128, 10000.0)
    for at in (0, 3990):
        x = to_f64(q[:, at:at + 10])
        want, tol = R.rope(x, [17 + at], [0, 10], f, gain, 128, R.HALF)
        assert _worst(to_f64(a[:, at:at + 10]), want, tol) <= 1.0


# ------------------------------------------------------------------ attention over packed prompts


def _check_packed(C, counts, hq, hkv, lead=0, tail=0, scale=0.0, seed=0, spread=1.0):
    ptr = _ptr(counts, lead)
    n = int(ptr[-1]) + tail
    q, k, v = _rand(hq, n, seed, spread), _rand(hkv, n, seed + 1), _rand(hkv, n, seed + 2)
    out = torch.full((hq, n, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    o = C.crisp_packed_attn(_ints(ptr), q.to(DEV), k.to(DEV), v.to(DEV), scale, out)
    want, tol = R.packed_attention(to_f64(q), to_f64(k), to_f64(v), ptr, scale or 1 / math.sqrt(128))
    got = to_f64(o)
    worst = _worst(got, want, tol)
    assert worst <= 1.0, f"{worst:.3f} of the tolerance"
    covered = np.zeros(n, dtype=bool)
    covered[ptr[0]:ptr[-1]] = True
    assert (got[:, ~covered] == 7.0).all()
    return o


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 192, 193, 257, 400, 777])
def test_packed_one_prompt(n):
    C = _crisp()
    _say(f"packed one prompt n={n}")
    _check_packed(C, [n], 2, 1, seed=n)


@pytest.mark.parametrize("heads", [(1, 1), (7, 1), (6, 2), (4, 4), (9, 3), (8, 8), (16, 16), (32, 8), (10, 5)])
def test_packed_heads(heads):
    C = _crisp()
    _say(f"packed heads={heads}")
    _check_packed(C, [150, 1, 77, 300], *heads, seed=heads[0])


@pytest.mark.parametrize("counts,lead,tail", [
    ([1] * 200, 0, 0), ([0, 5, 0, 0, 130, 0], 0, 7), ([100, 28, 128, 1, 255], 0, 0), ([3, 60, 200, 64, 64, 500], 5, 130),
    ([129], 127, 1), ([64, 64], 200, 300), ([127, 2, 127, 2], 0, 0), ([300, 20, 300, 20], 1, 0), ([5], 0, 1000), ([0, 0], 0, 10)])
def test_packed_ragged(counts, lead, tail):
    """Prompts that begin and end anywhere in a block, empty ones, rows before the first and behind the last."""
    C = _crisp()
    _say(f"packed counts={counts[:6]} lead={lead} tail={tail}")
    _check_packed(C, counts, 4, 2, lead, tail, seed=len(counts))


@pytest.mark.parametrize("n_seqs", [63, 64, 65, 130, 700])
def test_packed_many_short_prompts(n_seqs):
    C = _crisp()
    _say(f"packed n_seqs={n_seqs}")
    rng = np.random.default_rng(n_seqs)
    _check_packed(C, rng.integers(0, 9, n_seqs).tolist(), 2, 1, seed=n_seqs)


def test_packed_many_empty_prompts_in_a_block():
    C = _crisp()
    _say("packed 500 empty prompts between two")
    _check_packed(C, [40] + [0] * 500 + [50], 2, 1, tail=3)


@pytest.mark.parametrize("spread,scale", [(30.0, 0.0), (1.0, 1.0), (1e-3, 0.0), (1.0, 1e-6), (4.0, 2.0)])
def test_packed_sharp_and_flat_scores(spread, scale):
    C = _crisp()
    _say(f"packed spread={spread} scale={scale}")
    _check_packed(C, [200, 90, 450], 2, 2, scale=scale, spread=spread)


def test_packed_growing_scores():
    """Each tile's scores far above the ones before: the running reference is raised throughout, also across a block's prompts."""
    C = _crisp()
    _say("packed growing scores")
    n, ptr = 600, np.array([0, 400, 410, 600])
    q, v = _rand(1, n, 1), _rand(1, n, 2)
    k = (torch.sign(q.float().sum((0, 1))) * torch.linspace(0, 4, n)[None, :, None]).to(torch.bfloat16)
    q = q.abs() * torch.sign(q.float().sum((0, 1))).to(torch.bfloat16)
    o = C.crisp_packed_attn(_ints(ptr), q.to(DEV), k.to(DEV), v.to(DEV))
    want, tol = R.packed_attention(to_f64(q), to_f64(k), to_f64(v), ptr, 1 / math.sqrt(128))
    assert _worst(to_f64(o), want, tol) <= 1.0


def test_packed_strides_and_repeats():
    C = _crisp()
    _say("packed strides")
    n, hq, hkv, ptr = 333, 6, 2, _ints([0, 200, 333])
    x = _rand(hq + 2 * hkv, n, 3).to(DEV)
    view = x.transpose(0, 1).contiguous().transpose(0, 1)
    want = C.crisp_packed_attn(ptr, *(t.contiguous() for t in x.split([hq, hkv, hkv])))
    assert torch.equal(C.crisp_packed_attn(ptr, *view.split([hq, hkv, hkv])), want)
    out = torch.zeros(n, hq + 1, 128, dtype=torch.bfloat16, device=DEV)
    got = C.crisp_packed_attn(ptr, *view.split([hq, hkv, hkv]), out=out[:, :hq].transpose(0, 1))
    assert torch.equal(got, want) and (out[:, hq] == 0).all()
    k1 = x[hq:hq + 1].expand(2, n, 128)  # one head for all, then one key for all: v's mean
    assert torch.equal(C.crisp_packed_attn(ptr, x[:hq], k1, x[-2:]), C.crisp_packed_attn(ptr, x[:hq], k1.contiguous(), x[-2:]))
    k2 = x[hq:hq + 2, :1].expand(2, n, 128)
    assert torch.equal(C.crisp_packed_attn(ptr, x[:hq], k2, x[-2:]), C.crisp_packed_attn(ptr, x[:hq], k2.contiguous(), x[-2:]))


def test_packed_equals_the_dense_layer():
    """One prompt against the prefill's dense kernel, to both kernels' roundings."""
    C = _crisp()
    _say("packed against crisp_dense_attn")
    q, k, v = _rand(4, 1500, 1).to(DEV), _rand(2, 1500, 2).to(DEV), _rand(2, 1500, 3).to(DEV)
    a = C.crisp_packed_attn(_ints([0, 1500]), q, k, v).float()
    b = C.crisp_dense_attn(q, k, v).float()
    # each is off by three roundings of 2^-8 of sizes of at most sum p |v| <= max |v|
    assert (a - b).abs().max() <= 6 * 2.0 ** -8 * v.float().abs().max()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("which", ["q", "k", "v"])
def test_packed_not_finite(which, bad):
    """A value that is not finite reaches the rows that see it and no others: not those before it, nor another prompt's in the
    same block."""
    C = _crisp()
    _say(f"packed {which} has {bad}")
    ptr = np.array([0, 70, 150, 430, 440])
    for at in (0, 40, 69, 70, 149, 150, 290, 300, 429, 430, 439):
        q, k, v = _rand(2, 440, 1), _rand(1, 440, 2), _rand(1, 440, 3)
        clean = C.crisp_packed_attn(_ints(ptr), q.to(DEV), k.to(DEV), v.to(DEV))
        x = dict(q=q, k=k, v=v)[which]
        x[0, at, 5] = bad
        got = C.crisp_packed_attn(_ints(ptr), q.to(DEV), k.to(DEV), v.to(DEV))
        s = int(np.searchsorted(ptr, at, side="right")) - 1
        sees = np.zeros(440, dtype=bool)
        sees[at:(at + 1) if which == "q" else ptr[s + 1]] = True
        heads = [0] if which == "q" else [0, 1]
        seen = torch.from_numpy(sees).to(DEV)
        assert torch.equal(got[:, ~seen], clean[:, ~seen]), f"{which} row {at} reached others"
        if which == "v":
            y = got[:, seen]
            want = torch.isnan(y[..., 5]) if math.isnan(bad) else y[..., 5] == bad
            assert want.all(), f"v row {at}: {y[..., 5]}"
            keep = [e for e in range(128) if e != 5]
            assert torch.equal(y[..., keep], clean[:, seen][..., keep])
        elif which == "q" or math.isnan(bad):
            assert torch.isnan(got[heads][:, seen]).all()


def test_packed_infinities_of_both_signs():
    C = _crisp()
    _say("packed v has infinities of both signs")
    q, k, v = _rand(1, 100, 1), _rand(1, 100, 2), _rand(1, 100, 3)
    v[0, 20, 0], v[0, 30, 0], v[0, 99, 1] = math.inf, -math.inf, math.inf
    o = C.crisp_packed_attn(_ints([0, 100]), q.to(DEV), k.to(DEV), v.to(DEV))[0]
    assert torch.isfinite(o[:20]).all() and (o[20:30, 0] == math.inf).all() and torch.isnan(o[30:, 0]).all()
    assert torch.isfinite(o[:99, 1:]).all() and o[99, 1] == math.inf


def test_packed_same_bits_every_time():
    C = _crisp()
    _say("packed repeats")
    q, k, v = _rand(8, 3001, 1).to(DEV), _rand(2, 3001, 2).to(DEV), _rand(2, 3001, 3).to(DEV)
    ptr = _ints([0, 1700, 1701, 3001])
    first = C.crisp_packed_attn(ptr, q, k, v)
    for _ in range(5):
        assert torch.equal(C.crisp_packed_attn(ptr, q, k, v), first)


def test_packed_long_prompt():
    """Some rows of a long prompt behind a short one against the oracle."""
    C = _crisp()
    _say("packed 9000 behind 100")
    n, ptr = 9100, np.array([0, 100, 9100])
    q, k, v = _rand(2, n, 1), _rand(1, n, 2), _rand(1, n, 3)
    got = to_f64(C.crisp_packed_attn(_ints(ptr), q.to(DEV), k.to(DEV), v.to(DEV)))
    Q, K, V = to_f64(q), to_f64(k), to_f64(v)
    for r in (100, 128, 5000, 8191, 9099):
        for h in range(2):
            x = Q[h, r] @ K[0, 100:r + 1].T / math.sqrt(128)
            p = np.exp(x - x.max())
            p /= p.sum()
            want = p @ V[0, 100:r + 1]
            tol = 2 * 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 1e-4) * (p @ np.abs(V[0, 100:r + 1]))
            assert (np.abs(got[h, r] - want) <= tol).all()


def test_most_rows_and_sequences_of_a_call():
    """2^24 prompts of one token each: attention gives v, turned rows are those of a call of the last few alone."""
    C = _crisp()
    _say("2^24 prompts")
    n = 1 << 24
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randint(0, 1 << 16, (1, n, 128), generator=g, device=DEV, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = torch.where(x.isfinite() & (x.abs() < 2.0 ** 40), x, 1.0)
    q = _rand(1, 1, 2).to(DEV).expand(1, n, 128)
    ptr, start = torch.arange(n + 1, dtype=torch.int32, device=DEV), torch.arange(n, dtype=torch.int32, device=DEV)
    assert torch.equal(C.crisp_packed_attn(ptr, q, q, x), x)
    table = C.make_rope()
    last = 1000
    whole, _ = C.crisp_rope(table, start, ptr, x)
    few, _ = C.crisp_rope(table, start[-last:], ptr[:last + 1], x[:, -last:])
    assert torch.equal(whole[:, -last:], few)


def test_packed_rows_past_32_bits():
    """Rows whose elements lie further apart than 2^31 from the first to the last."""
    C = _crisp()
    _say("packed rows past 32 bits")
    n, ptr = 300, _ints([0, 40, 300])
    qkv = [_rand(1, n, seed).to(DEV) for seed in (1, 2, 3)]

    def spread(stride):
        return torch.empty(n * stride, dtype=torch.bfloat16, device=DEV).as_strided((1, n, 128), (128, stride, 1))

    far = [spread((1 << 23) + 8), spread((1 << 23) - 8), spread((1 << 23) - 8)]
    for a, b in zip(far, qkv):
        a.copy_(b)
    out = spread((1 << 23) + 16)
    want = C.crisp_packed_attn(ptr, *qkv)
    assert torch.equal(C.crisp_packed_attn(ptr, *far, out=out), want) and torch.equal(out, want)
    table, start = C.make_rope(), _ints([7, 100])
    turned = C.crisp_rope(table, start, ptr, qkv[0], qkv[1])
    C.crisp_rope(table, start, ptr, far[0], far[1], out, far[1])
    assert torch.equal(out, turned[0]) and torch.equal(far[1], turned[1])


def test_row_ptr_that_does_not_ascend_stays_within_the_buffers():
    C = _crisp()
    _say("packed row_ptr that does not ascend")
    n = 300
    big = torch.full((3, n + 200, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    q, k, v = _rand(1, n, 1).to(DEV), _rand(1, n, 2).to(DEV), _rand(1, n, 3).to(DEV)
    rng = np.random.default_rng(1)
    for ends in ([0, 200, 100, 300], [300, 0], [250, 10, 260, 20, 300], [0, (1 << 31) - 1, -(1 << 31), 150], rng.integers(0, 300, 90).tolist()):
        big.fill_(7.0)
        C.crisp_packed_attn(_ints(ends), q, k, v, out=big[1:2, :n])
        C.crisp_rope(C.make_rope(), _ints([0] * (len(ends) - 1)), _ints(ends), q, q_out=big[2:3, :n])
        assert (big[0] == 7.0).all() and (big[1:, n:] == 7.0).all()


def test_ropes_and_attention_on_another_stream_and_in_a_graph():
    """A captured call follows the device values of its replay: lengths that move within the same rows, other tensors' contents."""
    C = _crisp()
    _say("rope and packed attention captured")
    n = 260
    q, k, v = _rand(4, n, 1).to(DEV), _rand(2, n, 2).to(DEV), _rand(2, n, 3).to(DEV)
    ptr, start, t = _ints([0, 100, 260]), _ints([0, 7]), C.make_rope()

    def both(q, k, v, qo=None, ko=None, o=None):
        a, b = C.crisp_rope(t, start, ptr, q, k, qo, ko)
        return C.crisp_packed_attn(ptr, a, b, v, out=o)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both(q, k, v)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, both(q, k, v))
    qo, ko, o = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(q, k, v, qo, ko, o)
    for ends, begins, seed in (([0, 100, 260], [0, 7], 1), ([0, 3, 260], [50, 90000], 4), ([20, 20, 200], [1, 2], 5)):
        ptr.copy_(_ints(ends))
        start.copy_(_ints(begins))
        q.copy_(_rand(4, n, seed))
        o.zero_()
        graph.replay()
        want = both(q, k, v, o=torch.zeros_like(q))
        covered = slice(ends[0], ends[-1])
        assert torch.equal(o[:, covered], want[:, covered]) and (o[:, :ends[0]] == 0).all() and (o[:, ends[-1]:] == 0).all()


def test_two_streams_at_once():
    C = _crisp()
    _say("rope and packed attention on two streams")
    data = [[_rand(4, 900, 3 * i + j).to(DEV) for j in range(3)] for i in range(2)]
    ptrs = [_ints([0, 500, 900]), _ints([0, 1, 900])]
    t = C.make_rope()
    want = [C.crisp_packed_attn(p, C.crisp_rope(t, p[:2], p, d[0])[0], d[1], d[2]) for p, d in zip(ptrs, data)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(C.crisp_packed_attn(ptrs[i], C.crisp_rope(t, ptrs[i][:2], ptrs[i], data[i][0])[0], *data[i][1:]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(g, want[i]) for g in got[i])


def test_row_ptr_out_of_range_stays_within_the_buffers():
    """Offsets past the rows and below 0 are brought into range; rows on the way are written or left, never others."""
    C = _crisp()
    _say("packed row_ptr out of range")
    n = 200
    big = torch.full((3, n + 200, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    q, k, v = _rand(1, n, 1).to(DEV), _rand(1, n, 2).to(DEV), _rand(1, n, 3).to(DEV)
    for ends in ([0, 1 << 30], [-5, 90, 200], [50, 100, (1 << 31) - 1]):
        big.fill_(7.0)
        C.crisp_packed_attn(_ints(ends), q, k, v, out=big[1:2, :n])
        C.crisp_rope(C.make_rope(), _ints([0] * (len(ends) - 1)), _ints(ends), q, q_out=big[2:3, :n])
        assert (big[0] == 7.0).all() and (big[1:, n:] == 7.0).all()
    got = C.crisp_packed_attn(_ints([0, 1 << 30]), q, k, v)
    assert torch.equal(got, C.crisp_packed_attn(_ints([0, n]), q, k, v))
