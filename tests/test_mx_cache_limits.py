"""What a 4-bit cache says about rows that have no place, and what it does with calls that it refuses."""
import ctypes
import os

import pytest

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(os.path.join(ROOT, "paper_2511_16786_amd", "libflashcache.so")),
                                reason="libflashcache.so not built")


def _rows(shape, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(torch.bfloat16).cuda()


# ---- rows without a place -------------------------------------------------------------------------
def test_missing_counts_pages_that_no_table_has_room_for():
    """Pages from max_pages on are not taken from the pool, so the cursor does not tell of them."""
    import paper_2511_16786_amd as fc
    cache = fc.MxCache(2, 3, 2, 64, 16, 4, 1000, device="cpu")
    assert cache.missing() == 0
    cache.rows.copy_(torch.tensor([[64, 65, 0], [80, 81, 1000]], dtype=torch.int32))
    # 4, 5 and 0 pages, 5, 6 and 63 of four each: 1 + 1 + 2 + 59 too many, of two heads
    assert cache.missing() == 2 * 63
    cache.cursor.fill_(1003)                             # three that the pool did not have
    assert cache.missing() == 2 * 63 + 3
    cache.rows.fill_((1 << 25) - 1)                      # as many rows as are counted
    assert cache.missing() == 12 * ((1 << 21) - 4) + 3


@pytest.mark.gpu
def test_rows_beyond_a_units_table_are_reported_as_missing():
    import paper_2511_16786_amd as fc
    B, L, H, d, ps = 1, 2, 2, 64, 16
    cache = fc.MxCache(B, L, H, d, ps, 2, 64, device="cuda")             # tables of 32 rows, pages in plenty
    for turn in range(40):
        k, v = _rows((B, L, H, d), turn), _rows((B, L, H, d), 100 + turn)
        cache.append(k, v)
        assert cache.missing() == (0 if turn < 32 else L * H)
        if turn == 31:
            q = _rows((B, L, H, d), 999)
            full = cache.attend(q, 0.1)
    assert int(cache.cursor) == 2 * L * H
    assert torch.equal(cache.attend(q, 0.1), full)                       # the rows that have no place are not attended to
    # a compression that keeps more rows than the tables hold
    K, V = _rows((B, L, H, 300, d), 7), _rows((B, L, H, 300, d), 8)
    comp = fc.Compressor(K, 40, fc.total_budget(L, 300, 0.5))
    comp.run_score(K, V)
    comp.run_allocate()
    cache.reset()
    cache.fill(comp, K, V)
    assert cache.missing() == H * int((-(-comp.budgets // ps) - 2).clamp(min=0).sum()) > 0
