"""The cache's entry points at the largest sizes that they take, and their refusals beyond."""
import ctypes

import pytest
import torch

from paper_2609_01925_amd import crisp as C
from tests.test_cache_abi import REF, _append, _attn, _shape


@pytest.mark.parametrize("n_seqs,code", [(1 << 24, C.CRISP_OK), ((1 << 24) + 1, C.CRISP_EUNSUPPORTED), (2 ** 31 - 1, C.CRISP_EUNSUPPORTED)])
def test_sequences_of_a_call(n_seqs, code):
    """A search for a row's sequence steps through the sequences in 64 parts: past 2^31 - 64 of them the step left 32 bits."""
    n = ctypes.c_size_t()
    for wide in (0, 1, 100):
        b = (n_seqs, wide, 3)
        assert C.lib.crisp_cache_attn_workspace_size(REF(_shape()), REF(C.CrispCacheBatch(*b)), 4, REF(n)) == code
        if code:
            assert _append(b=b) == code and _attn(b=b) == code


@pytest.mark.gpu
def test_reservation_over_a_table_of_2_31_entries():
    """2^31 - 2 slots are asked for, of which the pages cover the first sequence's."""
    print("[gpu-case] reservation over 2^31 - 2 slots", flush=True)
    n_seqs, wide, n_pages = 3641, 589806, 600_000
    assert n_seqs * wide == 2 ** 31 - 2
    pool = C.crisp_pool_init(n_pages, "cuda:0")
    table = torch.full((n_seqs, wide), -1, dtype=torch.int32, device="cuda:0")
    lens = torch.zeros(n_seqs, dtype=torch.int32, device="cuda:0")
    granted = C.crisp_pool_reserve(pool, 64, table, lens, lens + 64 * wide)
    assert granted[0].item() == 64 * wide and (granted[1:] == 0).all()
    assert torch.equal(table[0], torch.arange(wide, dtype=torch.int32, device="cuda:0"))
    assert (table[1:] == -1).all()
    assert (pool[:wide] == 1).all() and (pool[wide:n_pages] == 0).all()


def test_workspace_of_a_batch_is_enough_for_less():
    """What cache_workspace gives for a batch serves the same sequences with fewer rows and in a narrower table."""
    def size(hq, hkv, fmt, seqs, wide, rows):
        n = ctypes.c_size_t()
        b = C.CrispCacheBatch(seqs, wide, rows)
        assert C.lib.crisp_cache_attn_workspace_size(REF(_shape(heads=hkv, fmt=fmt)), REF(b), hq, REF(n)) == C.CRISP_OK
        return n.value

    for hq, hkv in ((32, 8), (28, 4), (7, 1), (4, 4)):
        for fmt in (0, 1):
            for seqs in (1, 2, 3, 7, 32, 64, 100):
                before = None
                for wide in (1, 10, 16, 17, 40, 200, 700, 2048, 20000):
                    at = [size(hq, hkv, fmt, seqs, wide, rows) for rows in range(1, 40 * seqs, 1 + seqs // 4)]
                    assert at == sorted(at), (hq, hkv, fmt, seqs, wide)
                    assert before is None or all(a <= b for a, b in zip(before, at)), (hq, hkv, fmt, seqs, wide)
                    before = at
