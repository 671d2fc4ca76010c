"""Host checks of the decode steps over the paged cache: nothing is launched, no GPU is touched."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(os.path.join(ROOT, "paper_2511_16786_amd", "libflashcache.so")),
                                reason="libflashcache.so not built")
ref = ctypes.byref
EINVAL, EUNSUPPORTED, EWORKSPACE = 1, 2, 3


def _kv(**over):
    from paper_2511_16786_amd import binding as b
    v = dict(batch=2, layers=3, kv_heads=2, head_dim=64, dtype=1, page_size=16, max_pages=8, reserved=0, num_pages=100, rows_stride_b=3,
             table_stride_b=48, K=16, V=16, rows=4, block_table=4)
    v.update(over)
    return b.FcPagedKv(**v)


BAD_CACHES = [
    (dict(batch=-1), EINVAL), (dict(layers=0), EINVAL), (dict(kv_heads=0), EINVAL), (dict(head_dim=0), EINVAL), (dict(page_size=0), EINVAL),
    (dict(max_pages=0), EINVAL), (dict(num_pages=0), EINVAL), (dict(dtype=2), EINVAL), (dict(rows_stride_b=-1), EINVAL),
    (dict(table_stride_b=-1), EINVAL), (dict(head_dim=4), EINVAL), (dict(batch=32768, layers=1, kv_heads=1), EUNSUPPORTED),
    (dict(page_size=(1 << 25) + 1), EUNSUPPORTED), (dict(num_pages=1 << 31), EUNSUPPORTED), (dict(num_pages=1 << 28), EUNSUPPORTED),
    (dict(head_dim=(1 << 31) - 8), EUNSUPPORTED), (dict(rows=None), EINVAL), (dict(block_table=None), EINVAL), (dict(rows=2), EINVAL),
    (dict(block_table=6), EINVAL), (dict(K=None), EINVAL), (dict(K=8), EINVAL),
]
ATTENDED = [(dict(V=None), EINVAL), (dict(V=24), EINVAL), (dict(head_dim=80), EUNSUPPORTED), (dict(head_dim=256), EUNSUPPORTED)]


@pytest.mark.parametrize("over,status", BAD_CACHES + [(dict(head_dim=520), EUNSUPPORTED), (dict(head_dim=260, dtype=0), EUNSUPPORTED)])
def test_bounds_refuse_caches(over, status):
    from paper_2511_16786_amd import binding as b
    assert b._lib.flashcache_page_bounds(ref(_kv(**over)), 16, None) == status


def test_bounds_refuse_pointers():
    from paper_2511_16786_amd import binding as b
    assert b._lib.flashcache_page_bounds(None, 16, None) == EINVAL
    assert b._lib.flashcache_page_bounds(ref(_kv()), None, None) == EINVAL
    assert b._lib.flashcache_page_bounds(ref(_kv()), 8, None) == EINVAL
    assert b._lib.flashcache_page_bounds(ref(_kv(batch=0, rows=None, K=None)), None, None) == 0


@pytest.mark.parametrize("over,status", [x for x in BAD_CACHES if "K" not in x[0]] + ATTENDED[2:])
def test_choice_refuses_caches(over, status):
    from paper_2511_16786_amd import binding as b
    assert b._lib.flashcache_choose_pages(16, 4, ref(_kv(**over)), 16, 4, 1, 1, 4, 16, 1 << 40, None) == status


def test_choice_refuses_arguments():
    from paper_2511_16786_amd import binding as b
    kv = _kv()
    need = b._lib.flashcache_choose_pages_workspace_bytes(ref(kv))
    assert need > 0 and b._lib.flashcache_choose_pages_workspace_bytes(ref(_kv(layers=0))) == 0

    def call(Q=16, heads=4, kv=kv, bounds=16, count=4, first=1, last=1, chosen=4, ws=16, size=need):
        return b._lib.flashcache_choose_pages(Q, heads, ref(kv), bounds, count, first, last, chosen, ws, size, None)
    assert call(count=0) == EINVAL and call(first=-1) == EINVAL and call(last=-1) == EINVAL and call(first=3, last=2) == EINVAL
    assert call(first=2 ** 31 - 1, last=2 ** 31 - 1) == EINVAL
    assert call(heads=3) == EINVAL and call(heads=0) == EINVAL and call(heads=1) == EINVAL and call(heads=34) == EUNSUPPORTED
    assert call(Q=None) == EINVAL and call(Q=8) == EINVAL and call(bounds=None) == EINVAL and call(bounds=4) == EINVAL
    assert call(chosen=None) == EINVAL and call(chosen=6) == EINVAL
    assert call(ws=None) == EWORKSPACE and call(ws=8) == EWORKSPACE and call(size=need - 1) == EWORKSPACE
    assert call(kv=_kv(batch=0), Q=None, ws=None, size=0) == 0


def test_choice_refuses_counts_beyond_31_bits():
    # (the places behind the last page are written in steps of up to 1024: below 2^30 no step passes 31 bits)
    from paper_2511_16786_amd import binding as b
    for count in (1 << 30, 2 ** 31 - 1):
        assert b._lib.flashcache_choose_pages(16, 4, ref(_kv()), 16, count, 1, 1, 4, 16, 1 << 40, None) == EUNSUPPORTED


@pytest.mark.parametrize("over,status", BAD_CACHES + ATTENDED)
def test_attention_refuses_caches(over, status):
    from paper_2511_16786_amd import binding as b
    bad, good = _kv(**over), _kv()
    assert b._lib.flashcache_decode_attention_chosen(16, 4, ref(bad), 4, 4, 0.1, 16, 16, 1 << 40, None) == status
    for common, own in ((bad, good), (good, bad)):
        assert b._lib.flashcache_decode_attention_shared(16, 4, ref(common), 4, ref(own), 0.1, 16, 16, 1 << 40, None) == status


def test_attention_refuses_arguments():
    from paper_2511_16786_amd import binding as b
    kv = _kv()
    need = b._lib.flashcache_decode_chosen_workspace_bytes(ref(_kv(page_size=128)), 4, 64)
    assert need > 0

    def chosen(Q=16, heads=4, kv=_kv(page_size=128), places=4, count=64, scale=0.1, out=16, ws=16, size=need):
        return b._lib.flashcache_decode_attention_chosen(Q, heads, ref(kv), places, count, scale, out, ws, size, None)
    assert chosen(count=0) == EINVAL and chosen(scale=float("nan")) == EINVAL and chosen(heads=5) == EINVAL and chosen(heads=34) == EUNSUPPORTED
    assert chosen(Q=None) == EINVAL and chosen(Q=4) == EINVAL and chosen(places=None) == EINVAL and chosen(places=2) == EINVAL
    assert chosen(out=None) == EINVAL and chosen(out=4) == EINVAL and chosen(count=1 << 23) == EUNSUPPORTED
    assert chosen(ws=None) == EWORKSPACE and chosen(ws=8) == EWORKSPACE and chosen(size=need - 1) == EWORKSPACE
    assert chosen(kv=_kv(batch=0), Q=None, ws=None, size=0) == 0
    assert b._lib.flashcache_decode_chosen_workspace_bytes(ref(_kv(batch=0)), 4, 64) == 0
    assert b._lib.flashcache_decode_chosen_workspace_bytes(ref(_kv()), 5, 64) == 0

    need = b._lib.flashcache_decode_shared_workspace_bytes(2, 2, 3, 2, 4, 64, 1)
    assert need > 0
    for bad in ((-1, 2, 3, 2, 4, 64, 1), (2, 2, 0, 2, 4, 64, 1), (2, 2, 3, 2, 5, 64, 1), (2, 2, 3, 2, 4, 80, 1), (2, 2, 3, 2, 4, 64, 2),
                (2, 2, 3, 2, 34, 64, 1), (2, 32768, 1, 1, 1, 64, 1), (32768, 2, 1, 1, 1, 64, 1)):
        assert b._lib.flashcache_decode_shared_workspace_bytes(*bad) == 0

    def shared(Q=16, heads=4, common=kv, starts=4, own=kv, scale=0.1, out=16, ws=16, size=need):
        return b._lib.flashcache_decode_attention_shared(Q, heads, ref(common), starts, ref(own), scale, out, ws, size, None)
    for over in (dict(layers=2), dict(kv_heads=4), dict(head_dim=128), dict(dtype=0)):
        assert shared(common=_kv(**over)) == EINVAL
    assert shared(scale=float("nan")) == EINVAL and shared(heads=3) == EINVAL and shared(heads=34) == EUNSUPPORTED
    assert shared(Q=None) == EINVAL and shared(starts=None) == EINVAL and shared(starts=2) == EINVAL and shared(out=None) == EINVAL
    assert shared(out=8) == EINVAL and shared(ws=None) == EWORKSPACE and shared(ws=24) == EWORKSPACE and shared(size=need - 1) == EWORKSPACE
    assert shared(own=_kv(batch=0), Q=None, ws=None, size=0) == 0


def test_append_refuses_arguments():
    import paper_2511_16786_amd as fc
    from paper_2511_16786_amd import binding as b
    plan = fc.rotary_plan(64)

    def heads(batch=2, tokens=3, heads=4, d=64, dtype=1, strides=(768, 256, 64), out=(768, 256, 64)):
        return b.FcHeadsDesc(batch, tokens, heads, d, dtype, 0, *strides, *out)

    def call(plan=plan, pos=4, Q=2, Q_out=16, q=None, K=32, k=None, V=64, v=None, slots=8, sb=6, sh=3, ps=16, pages=100, Kp=256, Vp=512, lim=1024):
        q, k, v = q or heads(), k or heads(heads=2), v or heads(heads=2)
        return b._lib.flashcache_append_paged(ref(plan), pos, Q, Q_out, ref(q), K, ref(k), V, ref(v), slots, sb, sh, ps, pages, Kp, Vp, lim, None)
    assert call(pos=None) == EINVAL and call(pos=2) == EINVAL and call(Q=None) == EINVAL and call(Q_out=None) == EINVAL and call(Q=3) == EINVAL
    assert call(K=None) == EINVAL and call(V=None) == EINVAL and call(K=33) == EINVAL and call(Kp=None) == EINVAL and call(Vp=None) == EINVAL
    assert call(Kp=257) == EINVAL and call(slots=None) == EINVAL and call(slots=4) == EINVAL and call(lim=1025) == EINVAL
    assert call(Kp=512) == EINVAL and call(K=256) == EINVAL and call(V=512) == EINVAL and call(sb=-1) == EINVAL and call(sh=-1) == EINVAL
    assert call(ps=0) == EINVAL and call(pages=0) == EINVAL and call(ps=(1 << 25) + 1) == EUNSUPPORTED and call(pages=1 << 31) == EUNSUPPORTED
    assert call(ps=1 << 20, pages=1 << 12) == EUNSUPPORTED
    assert call(plan=b.FcRotaryPlan()) == EINVAL
    for bad in (dict(d=62), dict(d=32), dict(dtype=3), dict(batch=-1), dict(tokens=-1), dict(heads=-1), dict(strides=(-1, 256, 64))):
        assert call(q=heads(**bad)) == EINVAL and call(k=heads(**{"heads": 2, **bad})) == EINVAL and call(v=heads(**{"heads": 2, **bad})) == EINVAL
    for other in (dict(batch=1), dict(tokens=2), dict(d=128), dict(dtype=0), dict(heads=3)):
        assert call(k=heads(**{"heads": 2, **other})) == EINVAL and call(v=heads(**{"heads": 2, **other})) == EINVAL
    assert call(q=heads(out=(768, 32, 64))) == EINVAL
    wide = dict(d=514)
    assert call(q=heads(**wide), k=heads(heads=2, **wide), v=heads(heads=2, **wide)) == EUNSUPPORTED
    many = dict(batch=1, tokens=1 << 24)
    assert call(q=heads(**many), k=heads(heads=2, **many), v=heads(heads=2, **many)) == EUNSUPPORTED
    most = dict(heads=30000)
    assert call(q=heads(**most), k=heads(**most), v=heads(**most)) == EUNSUPPORTED
    # 2^32 threads and more
    big = dict(batch=1 << 12, tokens=1 << 11, d=512, strides=(1 << 27, 1 << 16, 512), out=(1 << 27, 1 << 16, 512))
    assert call(q=heads(heads=64, **big), k=heads(heads=2, **big), v=heads(heads=2, **big)) == EUNSUPPORTED
    # nothing to do
    none = dict(batch=0)
    assert call(q=heads(**none), k=heads(heads=2, **none), v=heads(heads=2, **none), pos=None, Q=None, K=None, slots=None) == 0


def test_tensors_off_the_gpu_are_refused():
    torch = pytest.importorskip("torch")
    import paper_2511_16786_amd as fc
    K = torch.zeros((4, 16, 64), dtype=torch.bfloat16)
    rows, table = torch.zeros((1, 1), dtype=torch.int32), torch.zeros((1, 1, 1, 2), dtype=torch.int32)
    with pytest.raises(ValueError):
        fc.PagedKV(K, K, rows, table)
    x = torch.zeros((1, 1, 1, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        fc.append_paged(fc.rotary_plan(64), torch.zeros((1, 1), dtype=torch.int32), x, x, x, torch.zeros((1, 1, 1), dtype=torch.int64), K, K)
