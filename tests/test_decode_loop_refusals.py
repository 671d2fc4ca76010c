"""Host checks of the decode loop's entry points and the rotary plan: nothing is launched, no GPU is touched."""
import ctypes
import math
import os

import numpy as np
import pytest

from oracle import decode_loop_ref as dr

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(os.path.join(ROOT, "paper_2511_16786_amd", "libflashcache.so")),
                                reason="libflashcache.so not built")
ref = ctypes.byref


@pytest.mark.parametrize("kw", [
    dict(rotary_dim=128), dict(rotary_dim=2), dict(rotary_dim=20, theta=5e5), dict(rotary_dim=64, scaling="linear", factor=4.0),
    dict(rotary_dim=64, scaling="base", factor=8.0), dict(rotary_dim=128, theta=1e6, scaling="parts", factor=4.0, original_tokens=32768),
    dict(rotary_dim=256, scaling="parts", factor=16.0, original_tokens=4096, beta_fast=20.0, beta_slow=2.0),
])
def test_plan_holds_the_turns_of_each_pair(kw):
    import paper_2511_16786_amd as fc
    plan = fc.rotary_plan(**kw)
    f, m = dr.frequencies(kw["rotary_dim"], **{k: v for k, v in kw.items() if k != "rotary_dim"})
    assert abs(plan.magnitude - m) <= m * 2.0 ** -24
    for i, x in enumerate(f):
        want = math.modf(x / (2 * math.pi))[0] * 2.0 ** 64
        # the frequency and its turns in 64-bit floating point, a few roundings (pow: 1e-15)
        assert abs(plan.turns[i] - want) <= 2.0 ** 64 * x * 1e-14 + 1, i
    assert list(plan.stream_end) == [kw["rotary_dim"] // 2] * 4


def test_plan_takes_given_frequencies_sections_and_magnitude():
    import paper_2511_16786_amd as fc
    plan = fc.rotary_plan(8, frequencies=[2 * math.pi * 0.25, -2 * math.pi * 0.25, 0.0, 2 * math.pi * 3.5], sections=(1, 2, 1),
                          magnitude=1.5)
    # (a quarter of 2^64 to the last bits of a double; a negative one is what it lacks to a whole turn; whole turns vanish)
    assert [round(plan.turns[i] / 2.0 ** 60) for i in range(4)] == [4, 12, 0, 8]
    assert list(plan.stream_end) == [1, 3, 4, 4] and plan.streams == 3 and plan.magnitude == 1.5


@pytest.mark.parametrize("kw,status", [
    (dict(rotary_dim=7), 1), (dict(rotary_dim=0), 1), (dict(rotary_dim=-4), 1), (dict(rotary_dim=258), 2), (dict(rotary_dim=8, theta=0.0), 1),
    (dict(rotary_dim=8, theta=float("nan")), 1), (dict(rotary_dim=8, theta=float("inf")), 1),
    (dict(rotary_dim=8, scaling="linear", factor=0.5), 1), (dict(rotary_dim=8, scaling="base", factor=float("inf")), 1),
    (dict(rotary_dim=8, scaling="parts", factor=2.0), 1),
    (dict(rotary_dim=8, scaling="parts", factor=2.0, original_tokens=64, beta_fast=1.0, beta_slow=1.0), 1),
    (dict(rotary_dim=8, magnitude=-1.0), 1), (dict(rotary_dim=8, sections=(1, 1)), 1), (dict(rotary_dim=8, sections=(5, -1)), 1),
    (dict(rotary_dim=8, frequencies=[1.0, float("nan"), 0.0, 0.0]), 1),
])
def test_plan_refusals(kw, status):
    import paper_2511_16786_amd as fc
    with pytest.raises(fc.FlashCacheError) as e:
        fc.rotary_plan(**kw)
    assert e.value.status == status


def test_plan_argument_errors():
    import paper_2511_16786_amd as fc
    with pytest.raises(ValueError):
        fc.rotary_plan(8, frequencies=[1.0])
    with pytest.raises(ValueError):
        fc.rotary_plan(8, sections=(3,))
    with pytest.raises(ValueError):
        fc.rotary_plan(8, sections=(1, 1, 1, 1, 0))
    with pytest.raises(KeyError):
        fc.rotary_plan(8, scaling="other")


def _heads(b, B=2, T=3, H=4, d=64, dtype=1, **over):
    v = dict(batch=B, tokens=T, heads=H, head_dim=d, dtype=dtype, reserved=0, stride_b=T * H * d, stride_t=H * d, stride_h=d,
             out_stride_b=T * H * d, out_stride_t=H * d, out_stride_h=d)
    v.update(over)
    return b.FcHeadsDesc(**v)


def test_rotary_refusals():
    import paper_2511_16786_amd as fc
    from paper_2511_16786_amd import binding as b
    plan = fc.rotary_plan(64)

    def call(q=None, k=None, plan=plan, pos=16, Q=32, Qo=64, K=32, Ko=64):
        q = _heads(b) if q is None else q
        return b._lib.flashcache_rotary(ref(plan) if plan else None, pos, Q, Qo, ref(q), K, Ko, ref(k) if k else None, 0, None)
    assert call(plan=None) == b.FC_EINVAL
    assert call(plan=b.FcRotaryPlan()) == b.FC_EINVAL                              # not prepared
    assert call(pos=None) == b.FC_EINVAL and call(pos=17) == b.FC_EINVAL
    assert call(Q=None) == b.FC_EINVAL and call(Qo=None) == b.FC_EINVAL and call(Q=33) == b.FC_EINVAL
    assert call(_heads(b, dtype=2)) == b.FC_EINVAL
    assert call(_heads(b, d=32)) == b.FC_EINVAL and call(_heads(b, d=65)) == b.FC_EINVAL and call(_heads(b, d=514)) == b.FC_EUNSUPPORTED
    assert call(_heads(b, stride_t=-64)) == b.FC_EINVAL
    assert call(_heads(b, out_stride_h=32)) == b.FC_EINVAL                         # heads of the output on one another
    assert call(_heads(b, out_stride_t=512), Q=64, Qo=64) == b.FC_EINVAL           # in place with other strides
    assert call(_heads(b, B=1 << 20, T=1 << 20)) == b.FC_EUNSUPPORTED
    assert call(_heads(b, B=1 << 12, T=1 << 12)) == b.FC_EUNSUPPORTED               # 2^24 tokens
    odd = b.FcRotaryPlan()
    ctypes.pointer(odd)[0] = plan
    odd.rotary_dim = 63
    assert call(plan=odd) == b.FC_EINVAL
    assert call(k=_heads(b, T=2)) == b.FC_EINVAL and call(k=_heads(b, dtype=0)) == b.FC_EINVAL and call(k=_heads(b), K=None) == b.FC_EINVAL
    assert call(_heads(b, B=0), Q=None, Qo=None, pos=None) == b.FC_OK
    assert call(_heads(b, T=0), Q=None, Qo=None, pos=None) == b.FC_OK


def test_assign_pages_refusals():
    from paper_2511_16786_amd import binding as b

    def call(rows=48, add=16, B=1, L=2, H=2, ps=16, most=4, free=64, n=8, cur=16, table=80, slots=16, per=8, ro=32, co=32):
        return b._lib.flashcache_assign_pages(rows, add, 0, B, L, H, ps, most, free, n, cur, table, slots, per, ro, co, None)
    for bad in (dict(L=0), dict(H=0), dict(B=-1), dict(ps=0), dict(most=0), dict(n=-1), dict(per=-1), dict(rows=None), dict(cur=None),
                dict(table=None), dict(ro=None), dict(co=None), dict(slots=None), dict(rows=18), dict(add=18), dict(free=18), dict(table=18),
                dict(ro=18), dict(cur=20), dict(co=20), dict(slots=20)):
        assert call(**bad) == b.FC_EINVAL, bad
    for bad in (dict(ro=16), dict(table=16), dict(free=16, ro=16)):                # outputs on inputs other than their own
        assert call(**{**dict(rows=48, add=16, free=64, table=80), **bad}) == b.FC_EINVAL, bad
    for bad in (dict(L=1025), dict(ps=(1 << 25) + 1), dict(B=1024, L=33), dict(H=32768)):
        assert call(**bad) == b.FC_EUNSUPPORTED, bad
    assert call(B=0, rows=None, table=None) == b.FC_OK


def test_mx_page_bytes():
    import paper_2511_16786_amd as fc
    assert fc.mx_page_bytes(64, 128) == 4 * 17 * 128 and fc.mx_page_bytes(16, 64) == 17 * 64 and fc.mx_page_bytes(48, 128) == 3 * 17 * 128
    for ps, d in ((0, 128), (-16, 128), (24, 128), (16, 96), (16, 256), (16, 0), (1 << 26, 128)):
        assert fc.mx_page_bytes(ps, d) == 0


def test_mx_store_and_load_refusals():
    from paper_2511_16786_amd import binding as b

    def desc(**over):
        v = dict(batch=1, head_dim=128, dtype=1, reserved=0, rows=4, stride_b=512, stride_r=128)
        v.update(over)
        return b.FcRowsDesc(**v)
    for name in ("store", "load"):
        def call(d=None, K=32, V=32, slots=32, ps=16, n=4, pages=32):
            d = desc() if d is None else d
            if name == "store":
                return b._lib.flashcache_mx_store(K, V, ref(d), slots, ps, n, pages, None)
            return b._lib.flashcache_mx_load(slots, pages, ps, n, ref(d), K, V, None)
        for kw in (dict(K=None), dict(V=None), dict(slots=None), dict(pages=None), dict(K=40), dict(pages=40), dict(slots=36), dict(n=0), dict(ps=0)):
            assert call(**kw) == b.FC_EINVAL, (name, kw)
        for over in (dict(batch=-1), dict(rows=-1), dict(dtype=3), dict(stride_r=132), dict(stride_b=-8), dict(head_dim=0)):
            assert call(desc(**over)) == b.FC_EINVAL, (name, over)
        assert call(ps=24) == b.FC_EUNSUPPORTED and call(desc(head_dim=96)) == b.FC_EUNSUPPORTED
        assert call(desc(rows=1 << 29)) == b.FC_EUNSUPPORTED
        assert call(desc(batch=65536)) == b.FC_EUNSUPPORTED and call(n=1 << 31) == b.FC_EUNSUPPORTED
        assert call(desc(rows=0), K=None, slots=None) == b.FC_OK and call(desc(batch=0), K=None) == b.FC_OK
    assert call(desc(stride_r=64)) == b.FC_EINVAL                                  # rows of the output on one another


def test_select_gather_mx_refusals():
    import paper_2511_16786_amd as fc
    from paper_2511_16786_amd import binding as b

    def call(d=128, K=32, table=32, ps=16, most=4, n=4, pages=32, rows=8, B=1, idx=32):
        desc = fc.FcKvDesc(B, 2, 2, 64, d, 1, 256 * d, 128 * d, 64 * d, d)
        return b._lib.flashcache_select_gather_mx(K, 32, ref(desc), 32, 32, 32, rows, 0, idx, table, ps, most, n, pages, None)
    for kw in (dict(K=None), dict(table=None), dict(pages=None), dict(table=33), dict(pages=40), dict(most=0), dict(n=0), dict(rows=-1),
               dict(rows=257), dict(idx=None), dict(d=12)):
        assert call(**kw) == b.FC_EINVAL, kw
    assert call(rows=1 << 29) == b.FC_EUNSUPPORTED
    assert call(d=96) == b.FC_EUNSUPPORTED and call(ps=20) == b.FC_EUNSUPPORTED
    assert call(rows=0, K=None, pages=None) == b.FC_OK and call(B=0, K=None) == b.FC_OK


def test_mx_decode_refusals_and_workspace():
    from paper_2511_16786_amd import binding as b
    size = b._lib.flashcache_mx_decode_workspace_bytes

    def call(Q=32, pages=32, table=32, ps=16, most=4, n=4, B=1, L=2, H=2, Hq=8, d=128, dtype=1, rows=32, scale=1.0, out=32, ws=32, wsb=1 << 34):
        return b._lib.flashcache_mx_decode_attention(Q, pages, table, ps, most, n, B, L, H, Hq, d, dtype, rows, ctypes.c_float(scale), out,
                                                     ws, wsb, None)
    for kw in (dict(Q=None), dict(pages=None), dict(table=None), dict(rows=None), dict(out=None), dict(Q=40), dict(pages=40), dict(out=40),
               dict(rows=33), dict(table=34), dict(most=0), dict(n=0), dict(ps=0), dict(Hq=7), dict(Hq=0), dict(dtype=2), dict(B=-1), dict(L=0),
               dict(scale=float("nan"))):
        assert call(**kw) == b.FC_EINVAL, kw
    for kw in (dict(Hq=34), dict(d=96), dict(d=256), dict(ps=40), dict(B=8192, L=4), dict(ps=1 << 25, most=1 << 10, B=1, L=2048, H=1, Hq=1),
               dict(ps=64, n=1 << 30)):
        assert call(**kw) == b.FC_EUNSUPPORTED, kw
    need = size(1, 2, 2, 8, 128)
    assert need > 0 and call(ws=None) == b.FC_EWORKSPACE and call(ws=40) == b.FC_EWORKSPACE and call(wsb=need - 1) == b.FC_EWORKSPACE
    assert call(B=0, Q=None, ws=None) == b.FC_OK
    assert size(1, 2, 2, 34, 128) == 0 and size(1, 2, 2, 7, 128) == 0 and size(1, 2, 2, 8, 96) == 0 and size(0, 2, 2, 8, 128) == 0


def test_binding_refuses_tensors_that_are_not_on_the_current_gpu():
    import torch
    import paper_2511_16786_amd as fc
    x = torch.zeros((1, 1, 2, 64), dtype=torch.bfloat16)
    i32, i64 = torch.zeros((1, 1), dtype=torch.int32), torch.zeros((1, 1), dtype=torch.int64)
    pages = torch.zeros((2, fc.mx_page_bytes(16, 64)), dtype=torch.uint8)
    table = torch.zeros((1, 1, 1, 1), dtype=torch.int32)
    with pytest.raises(ValueError):
        fc.rotary(fc.rotary_plan(64), i32, x)
    with pytest.raises(ValueError):
        fc.assign_pages(i32, 1, 16, table, i64.view(1), num_free=2)
    with pytest.raises(ValueError):
        fc.mx_store(x[0], x[0], i64, pages, 16)
    with pytest.raises(ValueError):
        fc.mx_decode_attention(x, pages, 16, 1, i32, table, 1.0)


# ---- the oracle against itself: facts that need no kernel -----------------------------------------
def test_oracle_grid_holds_its_own_values_and_rounds_by_half_a_step():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((64, 128)).astype(np.float32) * np.exp2(rng.integers(-20, 20, (64, 1))).astype(np.float32)
    codes, E = dr.encode(x)
    y = dr.decode(codes, E)
    assert np.array_equal(dr.decode(*dr.encode(y.astype(np.float32))), y)
    top = np.abs(x).reshape(64, 4, 32).max(-1)
    unit = np.exp2(E.astype(np.float64) - 127)
    assert np.all(top < 7 * unit) and np.all(top >= 3.5 * unit)
    # half the widest gap (4 to 6) in units, and 6 to 7 at the top
    assert np.all(np.abs(y - x).reshape(64, 4, 32) <= unit[..., None])


def test_oracle_layout_places_every_byte_once():
    for d in (64, 128):
        seen = np.zeros(2 * 17 * d, int)
        for slot in range(32):
            for at in dr._places(d, slot):
                seen[at] += 1
        assert np.all(seen == 1)
