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


# ---- refused calls --------------------------------------------------------------------------------
def _filled_state(cache):
    return cache.rows.clone(), cache.cursor.clone(), cache.block_table.clone()


def _compression(B, L, H, N, d, seed):
    import paper_2511_16786_amd as fc
    K, V = _rows((B, L, H, N, d), seed), _rows((B, L, H, N, d), seed + 1)
    comp = fc.Compressor(K, 30, fc.total_budget(L, N, 0.3))
    comp.run(K, V)
    return comp, K, V


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["K", "V", "in the call"])
def test_a_refused_fill_leaves_the_cache_empty(which, monkeypatch):
    """Rows at addresses off by 8 bytes have the descriptor's strides, and what the library refuses of its own comes after the pages."""
    import paper_2511_16786_amd as fc
    from paper_2511_16786_amd import binding
    B, L, H, N, d, ps = 1, 2, 2, 200, 64, 16
    comp, K, V = _compression(B, L, H, N, d, 40)
    cache = fc.MxCache(B, L, H, d, ps, -(-N // ps), 64)
    held = _filled_state(cache)
    if which == "in the call":
        def refuse(*args, **kwargs):
            raise fc.FlashCacheError(binding.FC_EUNSUPPORTED, "flashcache_select_gather_mx")
        with monkeypatch.context() as m:
            m.setattr(binding, "select_gather_mx", refuse)
            with pytest.raises(fc.FlashCacheError):
                cache.fill(comp, K, V)
    else:
        odd = torch.zeros(K.numel() + 4, dtype=K.dtype, device="cuda")[4:].view(K.shape)
        with pytest.raises(ValueError):
            cache.fill(comp, odd if which == "K" else K, odd if which == "V" else V)
    for t, s in zip((cache.rows, cache.cursor, cache.block_table), held):
        assert torch.equal(t, s)
    cache.fill(comp, K, V)                               # (refused too, if the cache took itself for filled)
    assert torch.equal(cache.rows, comp.budgets) and cache.missing() == 0
    # row 0 of the first unit, as the packed copy has it in four bits
    Ko, Vo = (torch.empty((1, 1, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    same, Kw, Vw = torch.zeros_like(cache.pages[:1]), torch.empty_like(Ko), torch.empty_like(Vo)
    fc.mx_load(cache.block_table[:1, 0, 0, :1].long() * ps, cache.pages, ps, Ko, Vo)
    first = torch.zeros((1, 1), dtype=torch.int64, device="cuda")
    fc.mx_store(comp.K_out[:1, :1].contiguous(), comp.V_out[:1, :1].contiguous(), first, same, ps)
    fc.mx_load(first, same, ps, Kw, Vw)
    assert torch.equal(Ko, Kw) and torch.equal(Vo, Vw)


@pytest.mark.gpu
def test_a_query_on_the_host_is_refused_and_no_more_than_that():
    """The workspace is the cache's: a refused query of other whereabouts does not leave one behind that the next call cannot use."""
    import paper_2511_16786_amd as fc
    B, L, H, d, ps = 1, 2, 1, 64, 16
    cache = fc.MxCache(B, L, H, d, ps, 2, 4)
    k, v, q = _rows((B, L, H, d), 50), _rows((B, L, H, d), 51), _rows((B, L, 4 * H, d), 52)
    cache.append(k, v)
    with pytest.raises(ValueError):
        cache.attend(q.cpu(), 0.1)
    out = cache.attend(q, 0.1)
    assert torch.equal(out, cache.attend(q, 0.1)) and bool(out.isfinite().all()) and bool(out.any())


@pytest.mark.parametrize("max_pages,num_pages", [(1, 0), (0, 1), (1, -1), (-1, 1)])
def test_a_cache_without_pages_or_tables_is_refused(max_pages, num_pages):
    """(It would count the first row and only then find that the store refuses a cache without pages.)"""
    import paper_2511_16786_amd as fc
    with pytest.raises(ValueError):
        fc.MxCache(1, 1, 1, 64, 16, max_pages, num_pages, device="cpu")


@pytest.mark.parametrize("rows", [(1 << 29) - 31, (1 << 29) - 1])
def test_rows_whose_launch_would_have_two_to_the_32_threads_are_refused(rows):
    """256 threads for each 32 rows, begun ones too: nothing is launched, on no machine."""
    from paper_2511_16786_amd import binding as b
    for d in (64, 128):
        desc = b.FcRowsDesc(1, d, b.FC_BF16, 0, rows, rows * d, d)
        assert b._lib.flashcache_mx_store(32, 32, ctypes.byref(desc), 32, 16, 4, 32, None) == b.FC_EUNSUPPORTED
        assert b._lib.flashcache_mx_load(32, 32, 16, 4, ctypes.byref(desc), 32, 32, None) == b.FC_EUNSUPPORTED


@pytest.mark.gpu
def test_a_batch_of_no_sequences_is_appended_and_attended_to():
    import paper_2511_16786_amd as fc
    L, H, d, ps = 2, 2, 64, 16
    cache = fc.MxCache(0, L, H, d, ps, 2, 4)
    none = torch.empty((0, L, H, d), dtype=torch.bfloat16, device="cuda")
    cache.append(none, none)
    assert cache.attend(torch.empty((0, L, 3 * H, d), dtype=torch.bfloat16, device="cuda"), 0.1).shape == (0, L, 3 * H, d)
    assert cache.missing() == 0
    with pytest.raises(ValueError):                      # a map of another batch
        fc.assign_pages(cache.rows, 1, ps, cache.block_table, cache.cursor, num_free=4,
                        slots=torch.empty((1, 4), dtype=torch.int64, device="cuda"))


@pytest.mark.gpu
def test_a_number_of_rows_beyond_32_bits_is_refused():
    """(It was cut to its lower half: 2^32 + 1 rows were one.)  What 32 bits hold is cut to the most rows that are counted."""
    import paper_2511_16786_amd as fc
    rows, cursor = torch.zeros((1, 2), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    table = torch.full((1, 2, 1, 3), -1, dtype=torch.int32, device="cuda")
    for add in (2 ** 32 + 1, 2 ** 31, -2 ** 31 - 1):
        with pytest.raises(ValueError):
            fc.assign_pages(rows, add, 16, table, cursor, num_free=9)
    assert not bool(rows.any()) and int(cursor) == 0
    fc.assign_pages(rows, 2 ** 31 - 1, 16, table, cursor, num_free=9)
    assert bool((rows == 2 ** 25 - 1).all()) and int(cursor) == 6 and table.view(-1).tolist() == list(range(6))
