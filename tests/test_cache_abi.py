"""The cache's entry points refuse bad arguments on the host, before anything is launched (no GPU needed:
every call below fails validation or has nothing to do)."""
import ctypes
import math

import pytest
import torch

from paper_2609_01925_amd import crisp as C

P = ctypes.c_void_p(0x100000)  # never dereferenced
ODD = ctypes.c_void_p(0x100002)
REF = ctypes.byref


def _shape(pages=8, heads=2, dim=128, block=64, fmt=0):
    return C.CrispCacheShape(pages, heads, dim, block, fmt)


def _append(sh=None, b=(2, 4, 3), p=P, s=P, t=P, n=P, r=P, k=P, kh=384, kr=128, v=P, vh=384, vr=128):
    return C.lib.crisp_cache_append(REF(sh or _shape()), REF(C.CrispCacheBatch(*b)), p, s, t, n, r, k, kh, kr, v, vh, vr, None)


def _attn(sh=None, b=(2, 4, 3), hq=4, scale=0.0, p=P, s=P, t=P, n=P, r=P, q=P, qh=384, qr=128, o=P, oh=384, orow=128,
          ws=P, wsb=1 << 40):
    return C.lib.crisp_cache_attn(REF(sh or _shape()), REF(C.CrispCacheBatch(*b)), hq, scale, p, s, t, n, r, q, qh, qr, o, oh,
                                  orow, ws, wsb, None)


@pytest.mark.parametrize("sh,code", [
    (_shape(pages=0), C.CRISP_EINVAL), (_shape(heads=0), C.CRISP_EINVAL), (_shape(dim=64), C.CRISP_EUNSUPPORTED),
    (_shape(block=32), C.CRISP_EUNSUPPORTED), (_shape(fmt=2), C.CRISP_EINVAL), (_shape(fmt=-1), C.CRISP_EINVAL),
    (_shape(pages=(1 << 24) + 1), C.CRISP_EUNSUPPORTED), (_shape(heads=65536), C.CRISP_EUNSUPPORTED)])
def test_bad_cache_shapes(sh, code):
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    assert C.lib.crisp_cache_bytes(REF(sh), REF(a), REF(b)) == code
    assert _append(sh) == code and _attn(sh) == code
    assert C.lib.crisp_cache_copy(REF(sh), P, P, P, 1, None, None) == code
    assert C.lib.crisp_last_error()


@pytest.mark.parametrize("b,code", [
    ((-1, 4, 3), C.CRISP_EINVAL), ((2, -1, 3), C.CRISP_EINVAL), ((2, 4, -1), C.CRISP_EINVAL),
    ((2, (1 << 24) + 1, 3), C.CRISP_EUNSUPPORTED), ((1 << 20, 1 << 12, 3), C.CRISP_EUNSUPPORTED),
    ((2, 4, (1 << 24) + 1), C.CRISP_EUNSUPPORTED)])
def test_bad_batches(b, code):
    n = ctypes.c_size_t()
    assert _append(b=b) == code and _attn(b=b) == code
    assert C.lib.crisp_cache_attn_workspace_size(REF(_shape()), REF(C.CrispCacheBatch(*b)), 4, REF(n)) == code


def test_null_and_misaligned_pointers():
    for name in "pstnrkv":
        assert _append(**{name: None}) == C.CRISP_EINVAL, name
        assert _append(**{name: ODD}) == C.CRISP_EINVAL, name
    for name in "pstnrqo":
        assert _attn(**{name: None}) == C.CRISP_EINVAL, name
        assert _attn(**{name: ODD}) == C.CRISP_EINVAL, name
    assert _attn(ws=None) == C.CRISP_EINVAL and _attn(ws=ctypes.c_void_p(0x100010)) == C.CRISP_EINVAL
    assert _attn(wsb=16) == C.CRISP_EINVAL and b"too small" in C.lib.crisp_last_error()
    assert C.lib.crisp_cache_append(None, None, P, P, P, P, P, P, 0, 0, P, 0, 0, None) == C.CRISP_EINVAL
    assert C.lib.crisp_cache_append(REF(_shape()), None, P, P, P, P, P, P, 0, 0, P, 0, 0, None) == C.CRISP_EINVAL


def test_bad_strides_heads_and_scales():
    for bad in (-8, 4, 129):
        assert _append(kh=bad) == C.CRISP_EINVAL and _append(vr=bad) == C.CRISP_EINVAL
        assert _attn(qr=bad) == C.CRISP_EINVAL and _attn(oh=bad) == C.CRISP_EINVAL
    assert _attn(oh=64) == C.CRISP_EINVAL and _attn(orow=0) == C.CRISP_EINVAL and b"overlap" in C.lib.crisp_last_error()
    assert _attn(hq=3) == C.CRISP_EINVAL and _attn(hq=-2) == C.CRISP_EINVAL
    assert _attn(hq=2 << 20, b=(1, 1, 1 << 20)) == C.CRISP_EUNSUPPORTED
    for bad in (-1.0, math.nan, math.inf):
        assert _attn(scale=bad) == C.CRISP_EINVAL


@pytest.mark.parametrize("head,row,apart", [(384, 128, True), (128, 512, True), (128, 128, False), (376, 128, False),
                                            (128, 504, False), (200, 136, False), (400, 136, True), (136, 536, True)])
def test_output_rows_must_be_apart(head, row, apart):
    """Four heads of three rows: one stride covers the extent that the other makes."""
    assert _attn(oh=head, orow=row, wsb=16) == C.CRISP_EINVAL
    assert (b"too small" if apart else b"overlap") in C.lib.crisp_last_error()


def test_nothing_to_do_needs_no_buffers():
    none = dict(p=None, s=None, t=None, n=None, r=None)
    for b in ((0, 4, 3), (2, 4, 0)):
        assert _append(b=b, k=None, v=None, **none) == C.CRISP_OK
        assert _attn(b=b, q=None, o=None, ws=None, wsb=0, **none) == C.CRISP_OK
    assert _append(b=(2, 0, 3), k=None, v=None, **none) == C.CRISP_OK
    assert _attn(hq=0, q=None, o=None, ws=None, wsb=0, **none) == C.CRISP_OK
    assert C.lib.crisp_cache_copy(REF(_shape()), None, None, None, 0, None, None) == C.CRISP_OK
    assert C.lib.crisp_pool_free(8, 2, 2, P, P, None, None, 0, None) == C.CRISP_OK
    assert C.lib.crisp_pool_fork(8, 64, 2, 2, P, P, None, None, None, 0, None, None) == C.CRISP_OK
    assert C.lib.crisp_pool_reserve(8, 64, 0, 2, P, None, None, None, None, None) == C.CRISP_OK


def test_copy_refusals():
    sh = _shape()
    assert C.lib.crisp_cache_copy(REF(sh), P, P, P, -1, None, None) == C.CRISP_EINVAL
    assert C.lib.crisp_cache_copy(REF(sh), None, P, P, 1, None, None) == C.CRISP_EINVAL
    assert C.lib.crisp_cache_copy(REF(sh), P, P, None, 1, None, None) == C.CRISP_EINVAL
    assert C.lib.crisp_cache_copy(REF(sh), P, P, P, 1, ctypes.c_void_p(0x100001), None) == C.CRISP_EINVAL


def test_pool_sizes_and_refusals():
    assert [C.crisp_pool_words(n) for n in (1, 31, 32, 33, 64, 65)] == [2, 32, 33, 35, 66, 68]
    for n in list(range(1, 300)) + [1 << 24]:
        assert C.pool_pages(torch.empty(C.crisp_pool_words(n), dtype=torch.int32, device="meta")) == n
    for words in (0, 1, 34, 67):
        with pytest.raises(ValueError):
            C.pool_pages(torch.empty(words, dtype=torch.int32, device="meta"))
    for n in (0, -1, (1 << 24) + 1):
        assert C.lib.crisp_pool_words(n) == -1
        with pytest.raises(C.CrispError):
            C.crisp_pool_words(n)
        assert C.lib.crisp_pool_init(n, P, None) != C.CRISP_OK
    assert C.lib.crisp_pool_init(8, None, None) == C.CRISP_EINVAL
    with pytest.raises(ValueError):
        C.crisp_pool_init(8, "cpu")
    reserve = lambda n=8, block=64, s=2, m=2, pool=P, t=P, l=P, c=P, g=P: C.lib.crisp_pool_reserve(n, block, s, m, pool, t, l, c, g, None)
    fork = lambda n=8, block=64, s=2, m=2, pool=P, t=P, l=P, a=P, b=P, k=1, c=P: C.lib.crisp_pool_fork(n, block, s, m, pool, t, l, a, b, k, c, None)
    free = lambda n=8, s=2, m=2, pool=P, t=P, l=P, i=P, k=1: C.lib.crisp_pool_free(n, s, m, pool, t, l, i, k, None)
    compact = lambda n=8, s=2, m=2, pool=P, t=P, mv=P, c=P: C.lib.crisp_pool_compact(n, s, m, pool, t, mv, c, None)
    for call, pointers in ((reserve, ("pool", "t", "l", "c", "g")), (fork, ("pool", "t", "l", "a", "b", "c")),
                           (free, ("pool", "t", "l", "i")), (compact, ("pool", "t", "mv", "c"))):
        for name in pointers:
            assert call(**{name: None}) == C.CRISP_EINVAL and call(**{name: ODD}) == C.CRISP_EINVAL, name
        assert call(n=0) == C.CRISP_EINVAL and call(s=-1) == C.CRISP_EINVAL and call(m=-1) == C.CRISP_EINVAL
        assert call(m=1 << 25) == C.CRISP_EUNSUPPORTED and call(s=1 << 16, m=1 << 16) == C.CRISP_EUNSUPPORTED
    for call in (reserve, fork):
        assert call(block=96) == C.CRISP_EUNSUPPORTED and call(s=4097) == C.CRISP_EUNSUPPORTED
    assert fork(k=-1) == C.CRISP_EINVAL and fork(k=4097) == C.CRISP_EUNSUPPORTED and free(k=-1) == C.CRISP_EINVAL


def test_binding_refuses_tensors_that_do_not_fit():
    """Python checks that the C side cannot make; a cache of host tensors is refused at once."""
    with pytest.raises(ValueError):
        C.Cache(torch.zeros(2, 1, 1, 2, 8192, dtype=torch.uint8), torch.zeros(2, 1, 2))
    with pytest.raises(C.CrispError):
        C.make_cache(4, 1, block=32, device="cpu")
    with pytest.raises(C.CrispError):
        C.make_cache(4, 1, fmt=5, device="cpu")


def test_byte_sizes():
    assert C.crisp_cache_bytes(_shape(pages=10, heads=3, block=128)) == (10 * 3 * 2 * 128 * 128, 10 * 3 * 2 * 4)
