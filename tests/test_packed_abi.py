"""The entry points on packed rows and those of the eviction refuse bad arguments on the host, before anything is launched (no GPU
needed: every call below fails validation or has nothing to do); frequencies of rotary positions against the oracle."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2609_01925_amd import crisp as C
from tests import packed_oracle as R

P = ctypes.c_void_p(0x100000)  # never dereferenced
ODD = ctypes.c_void_p(0x100002)
REF = ctypes.byref
TABLE = C.make_rope()


def _packed(seqs=2, rows=3, hq=4, hkv=2, dim=128):
    return C.CrispPackedShape(seqs, rows, hq, hkv, dim)


def _rope(sh=None, t=TABLE, n=P, r=P, q=P, qh=384, qr=128, k=P, kh=384, kr=128, qo=P, qoh=384, qor=128, ko=P, koh=384, kor=128):
    return C.lib.crisp_rope(REF(sh or _packed()), t, n, r, q, qh, qr, k, kh, kr, qo, qoh, qor, ko, koh, kor, None)


def _attn(sh=None, scale=0.0, r=P, q=P, qh=384, qr=128, k=P, kh=384, kr=128, v=P, vh=384, vr=128, o=P, oh=384, orow=128):
    return C.lib.crisp_packed_attn(REF(sh or _packed()), scale, r, q, qh, qr, k, kh, kr, v, vh, vr, o, oh, orow, None)


def _cache(pages=8, heads=2, dim=128, block=64, fmt=0):
    return C.CrispCacheShape(pages, heads, dim, block, fmt)


def _weights(sh=None, b=(2, 4, 3), hq=4, scale=0.0, p=P, s=P, t=P, n=P, r=P, q=P, qh=384, qr=128, w=P, o=P, width=256, h=P, ws=P,
             wsb=1 << 40):
    return C.lib.crisp_cache_weights(REF(sh or _cache()), REF(C.CrispCacheBatch(*b)), hq, scale, p, s, t, n, r, q, qh, qr, w, o, width, h,
                                     ws, wsb, None)


def _keep(seqs=2, heads=2, width=256, w=P, h=P, n=P, m=P, sink=4, recent=8, cap=64, k=P, c=P, o=P, ws=None, wsb=0):
    return C.lib.crisp_cache_keep(seqs, heads, width, w, h, n, m, sink, recent, cap, k, c, o, ws, wsb, None)


def _gather(sh=None, b=(2, 4, 0), p=P, s=P, t=P, k=P, cap=64, c=P, n=P, wide=1):
    return C.lib.crisp_cache_gather(REF(sh or _cache()), REF(C.CrispCacheBatch(*b)), p, s, t, k, cap, c, n, wide, None)


@pytest.mark.parametrize("sh,code", [
    (_packed(seqs=-1), C.CRISP_EINVAL), (_packed(rows=-1), C.CRISP_EINVAL), (_packed(hq=-1), C.CRISP_EINVAL),
    (_packed(hkv=-1), C.CRISP_EINVAL), (_packed(dim=64), C.CRISP_EUNSUPPORTED), (_packed(seqs=(1 << 24) + 1), C.CRISP_EUNSUPPORTED),
    (_packed(rows=(1 << 24) + 1), C.CRISP_EUNSUPPORTED), (_packed(hq=65536), C.CRISP_EUNSUPPORTED),
    (_packed(hkv=65536), C.CRISP_EUNSUPPORTED)])
def test_bad_packed_shapes(sh, code):
    assert _rope(sh) == code and _attn(sh) == code and C.lib.crisp_last_error()


def test_packed_heads_scales_and_sizes():
    assert _attn(_packed(hq=3)) == C.CRISP_EINVAL and _attn(_packed(hkv=0)) == C.CRISP_EINVAL
    for bad in (-1.0, math.nan, math.inf):
        assert _attn(scale=bad) == C.CRISP_EINVAL
    assert _attn(_packed(rows=1 << 24, hq=128), qh=1 << 31, kh=1 << 31, vh=1 << 31, oh=1 << 31) == C.CRISP_EUNSUPPORTED
    assert _attn(kr=1 << 23, kh=1 << 26) == C.CRISP_EUNSUPPORTED and _attn(vr=1 << 23, vh=1 << 26) == C.CRISP_EUNSUPPORTED


def test_packed_pointers_and_strides():
    for name in ("n", "r", "q", "k", "qo", "ko"):
        for bad in (None, ODD):
            assert _rope(**{name: bad}) == C.CRISP_EINVAL, name
    for name in "rqkvo":
        for bad in (None, ODD):
            assert _attn(**{name: bad}) == C.CRISP_EINVAL, name
    for bad in (-8, 4, 129):
        for name in ("qh", "qr", "kh", "kr", "qoh", "qor", "koh", "kor"):
            assert _rope(**{name: bad}) == C.CRISP_EINVAL, name
        for name in ("qh", "qr", "kh", "kr", "vh", "vr", "oh", "orow"):
            assert _attn(**{name: bad}) == C.CRISP_EINVAL, name
    other = ctypes.c_void_p(0x900000)
    assert _rope(qo=other, qoh=120) == C.CRISP_EINVAL and b"overlap" in C.lib.crisp_last_error()
    assert _rope(ko=other, kor=0) == C.CRISP_EINVAL and _attn(oh=64) == C.CRISP_EINVAL
    assert _rope(qr=512, qh=128) == C.CRISP_EINVAL and b"in place" in C.lib.crisp_last_error()
    assert C.lib.crisp_rope(None, TABLE, P, P, P, 0, 0, P, 0, 0, P, 0, 0, P, 0, 0, None) == C.CRISP_EINVAL
    assert _rope(t=None) == C.CRISP_EINVAL


def test_packed_nothing_to_do():
    for sh in (_packed(seqs=0), _packed(rows=0)):
        assert _rope(sh, n=None, r=None, q=None, k=None, qo=None, ko=None) == C.CRISP_OK
        assert _attn(sh, r=None, q=None, k=None, v=None, o=None) == C.CRISP_OK
    assert _rope(_packed(hq=0, hkv=0), n=None, r=None, q=None, k=None, qo=None, ko=None) == C.CRISP_OK
    assert _attn(_packed(hq=0), r=None, q=None, k=None, v=None, o=None) == C.CRISP_OK


@pytest.mark.parametrize("change", [
    dict(rotary_dim=0), dict(rotary_dim=8), dict(rotary_dim=20), dict(rotary_dim=144), dict(rotary_dim=-16), dict(layout=2), dict(layout=-1),
    dict(scaling=5), dict(scaling=-1), dict(base=1.0), dict(base=0.0), dict(base=math.nan), dict(base=math.inf), dict(factor=0.5),
    dict(factor=math.nan), dict(factor=math.inf), dict(original_len=0.0), dict(original_len=math.inf), dict(low=0.0), dict(low=4.0),
    dict(low=5.0), dict(high=math.inf), dict(low=math.nan), dict(scaling=C.ROPE_BASE, rotary_dim=16, base=1e308, factor=1e10)])
def test_rope_init_refusals(change):
    good = dict(rotary_dim=64, layout=0, base=10000.0, scaling=C.ROPE_BANDS, factor=8.0, original_len=8192.0, low=1.0, high=4.0)
    C.make_rope(**good)
    with pytest.raises(C.CrispError):
        C.make_rope(**dict(good, **change))


def test_rope_init_null_and_bad_tables():
    t = C.CrispRopeTable()
    assert C.lib.crisp_rope_init(None, REF(t)) == C.CRISP_EINVAL
    assert C.lib.crisp_rope_init(REF(C.CrispRopeParams(64, 0, 0, 10000.0)), None) == C.CRISP_EINVAL
    for dim, layout in ((0, 0), (24, 0), (256, 0), (64, 7)):
        t.rotary_dim, t.layout = dim, layout
        assert _rope(t=t) != C.CRISP_OK


@pytest.mark.parametrize("dim", [16, 64, 80, 128])
@pytest.mark.parametrize("rule,rest", [(R.PLAIN, ()), (R.LINEAR, (4.0,)), (R.BASE, (2.5,)), (R.BANDS, (8.0, 8192.0, 1.0, 4.0)),
                                       (R.RAMP, (16.0, 4096.0, 1.0, 32.0)), (R.RAMP, (1.0, 64.0, 0.5, 100.0))])
def test_rope_frequencies(dim, rule, rest):
    """The table against the oracle: some 64-bit operations each, powers and logarithms within a few 2^-53."""
    for base in (10000.0, 500000.0, 1.5):
        t = C.make_rope(dim, R.INTERLEAVED, base, rule, *rest)
        f, gain = R.frequencies(dim, base, rule, *rest)
        assert (t.rotary_dim, t.layout) == (dim, R.INTERLEAVED)
        np.testing.assert_allclose(np.array(t.turns[:dim // 2]) * 2 * np.pi, f, rtol=2.0 ** -47)
        assert abs(t.gain - gain) <= 2.0 ** -24 * gain and list(t.turns[dim // 2:]) == [0.0] * (64 - dim // 2)


# ------------------------------------------------------------------ eviction


@pytest.mark.parametrize("sh,code", [(_cache(pages=0), C.CRISP_EINVAL), (_cache(dim=64), C.CRISP_EUNSUPPORTED),
                                     (_cache(block=32), C.CRISP_EUNSUPPORTED), (_cache(fmt=2), C.CRISP_EINVAL)])
def test_bad_cache_shapes(sh, code):
    n = ctypes.c_size_t()
    assert _weights(sh) == code and _gather(sh) == code
    assert C.lib.crisp_cache_weights_workspace_size(REF(sh), REF(C.CrispCacheBatch(2, 4, 3)), 4, REF(n)) == code


@pytest.mark.parametrize("b,code", [
    ((-1, 4, 3), C.CRISP_EINVAL), ((2, -1, 3), C.CRISP_EINVAL), ((2, 4, -1), C.CRISP_EINVAL), ((2, (1 << 24) + 1, 3), C.CRISP_EUNSUPPORTED),
    ((2, 4, (1 << 24) + 1), C.CRISP_EUNSUPPORTED), (((1 << 19) + 1, 1, 3), C.CRISP_EUNSUPPORTED)])
def test_bad_batches(b, code):
    n = ctypes.c_size_t()
    assert _weights(b=b) == code and _gather(b=b) == code
    assert C.lib.crisp_cache_weights_workspace_size(REF(_cache()), REF(C.CrispCacheBatch(*b)), 4, REF(n)) == code


def test_weights_refusals():
    for name in "pstnrqwoh":
        for bad in (None, ODD):
            assert _weights(**{name: bad}) == C.CRISP_EINVAL, name
    assert _weights(ws=None) == C.CRISP_EINVAL and _weights(ws=ctypes.c_void_p(0x100010)) == C.CRISP_EINVAL
    assert _weights(wsb=16) == C.CRISP_EINVAL and b"too small" in C.lib.crisp_last_error()
    assert _weights(hq=3) == C.CRISP_EINVAL and _weights(width=0) == C.CRISP_EINVAL
    assert _weights(width=(1 << 28) + 1) == C.CRISP_EUNSUPPORTED
    for bad in (-1.0, math.nan, math.inf):
        assert _weights(scale=bad) == C.CRISP_EINVAL
    for bad in (-8, 4, 129):
        assert _weights(qh=bad) == C.CRISP_EINVAL and _weights(qr=bad) == C.CRISP_EINVAL
    assert C.lib.crisp_cache_weights_workspace_size(REF(_cache()), REF(C.CrispCacheBatch(2, 4, 3)), 4, None) == C.CRISP_EINVAL


def test_weights_without_rows_need_the_rest():
    """The weights that are held go to out all the same: q and the workspace alone may be missing."""
    for change in (dict(b=(2, 4, 0)), dict(hq=0)):
        for name in "pstnrwoh":
            assert _weights(**change, **{name: None}) == C.CRISP_EINVAL, name


def test_weights_workspace_is_enough_for_fewer_rows():
    sizes = []
    for rows in list(range(0, 2000, 7)) + [1 << k for k in range(11, 25)]:
        n = ctypes.c_size_t()
        assert C.lib.crisp_cache_weights_workspace_size(REF(_cache()), REF(C.CrispCacheBatch(3, 4, rows)), 28, REF(n)) == C.CRISP_OK
        sizes.append(n.value)
    assert sizes == sorted(sizes) and sizes[0] == 0


def test_keep_refusals():
    for name in "whnmkc":
        for bad in (None, ODD):
            assert _keep(**{name: bad}) == C.CRISP_EINVAL, name
    assert _keep(o=ODD) == C.CRISP_EINVAL
    for change in (dict(seqs=-1), dict(heads=0), dict(width=0), dict(cap=0), dict(cap=-1), dict(sink=-1), dict(recent=-1)):
        assert _keep(**change) == C.CRISP_EINVAL, change
    for change in (dict(width=(1 << 28) + 1), dict(cap=(1 << 28) + 1), dict(heads=65536), dict(seqs=(1 << 19) + 1),
                   dict(width=1 << 28, seqs=33)):
        assert _keep(**change) == C.CRISP_EUNSUPPORTED, change
    n = ctypes.c_size_t()
    size = lambda *args: C.lib.crisp_cache_keep_workspace_size(*args, REF(n))  # noqa: E731
    assert size(2, 2, 16384, 1) == C.CRISP_OK and n.value == 0
    assert size(2, 2, 16385, 0) == C.CRISP_OK and n.value > 0
    apart = n.value
    assert size(2, 2, 16385, 1) == C.CRISP_OK and n.value >= apart + 4 * (4 * 16385 - 255)
    assert size(-1, 2, 64, 0) == C.CRISP_EINVAL and size(2, 2, 0, 0) == C.CRISP_EINVAL
    assert C.lib.crisp_cache_keep_workspace_size(2, 2, 64, 0, None) == C.CRISP_EINVAL
    other = ctypes.c_void_p(0x900000)
    for bad in (None, ctypes.c_void_p(0x100010)):
        assert _keep(width=16385, ws=bad, wsb=1 << 40) == C.CRISP_EINVAL
    assert _keep(width=16385, ws=other, wsb=apart - 1, o=other) == C.CRISP_EINVAL and b"too small" in C.lib.crisp_last_error()
    assert _keep(width=16385, ws=other, wsb=apart) == C.CRISP_EINVAL  # in place it needs more


def test_gather_refusals():
    for name in "pstkcn":
        for bad in (None, ODD):
            assert _gather(**{name: bad}) == C.CRISP_EINVAL, name
    assert _gather(cap=0) == C.CRISP_EINVAL and _gather(wide=-1) == C.CRISP_EINVAL
    assert _gather(wide=(1 << 24) + 1) == C.CRISP_EUNSUPPORTED


def test_eviction_nothing_to_do():
    none = dict(p=None, s=None, t=None)
    assert _weights(b=(0, 4, 3), n=None, r=None, q=None, w=None, o=None, h=None, ws=None, wsb=0, **none) == C.CRISP_OK
    assert _keep(seqs=0, w=None, h=None, n=None, m=None, k=None, c=None, o=None) == C.CRISP_OK
    assert _gather(b=(0, 4, 0), k=None, c=None, n=None, **none) == C.CRISP_OK
    assert _gather(wide=0, k=None, c=None, n=None, **none) == C.CRISP_OK


def test_binding_refuses_tensors_that_are_not_on_the_gpu():
    x, i = torch.zeros(2, 3, 128, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        C.crisp_packed_attn(i, x, x, x)
    with pytest.raises(ValueError):
        C.crisp_rope(TABLE, i[:2], i, x, x)
    with pytest.raises(ValueError):
        C.crisp_cache_keep(torch.zeros(2, 3, 4), i[:2], i[:2], i[:2], 4)
