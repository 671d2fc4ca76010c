"""Decode steps over the paged cache of bf16 or fp32 rows on the GPU, against float64 (oracle/paged_steps_ref.py, oracle/decode_loop_ref.py).

Places of a cache that hold no rows are NaN throughout, so that a read of one shows.
Tolerances.  u = 2^-24, half a step of fp32.
  append     queries and keys as the rotation by itself: 8 u (|x0| + |x1|) m and the angle's 2^-50; bf16: half a step more, 2^-8 of the
             result.  Values, other slots and bounds of what was stored: equal.
  choice     equal (scores are summed in 64 bits).
  attention  a logit is a sum of d products in fp32: off by at most d u sum |q k| scale, its scaling and exponential by 4 u (|logit| + 1), twice
             (its own and the reference's); the sums over n rows go at least 16 at a time, then pieces: n / 16 + 64 roundings.  All of it
             relative to sum p |v|.
"""
import math

import numpy as np
import pytest

from oracle import decode_loop_ref as dr
from oracle import paged_steps_ref as pr

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
U = 2.0 ** -24


def _fc():
    import paper_2511_16786_amd as fc
    return fc


def _dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _rand(rng, shape, dtype, sigma=1.0):
    return torch.from_numpy((sigma * rng.standard_normal(shape)).astype(np.float32)).to(dtype).cuda()


def _f64(t):
    return t.detach().double().cpu().numpy()


def _int(x, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(x).astype(dtype)).cuda()


class Cache:
    """Rows [B, L] of each layer in pages at random places, NaN everywhere else; `lost`: share of table entries without a page."""

    def __init__(self, rng, rows, H, d, ps, dtype, most=None, lost=0.0, spare=3, sigma=1.0):
        rows = np.asarray(rows)
        B, L = rows.shape
        blocks = -(-np.maximum(rows, 0) // ps)
        self.most = max(1, int(blocks.max())) if most is None else most
        self.ps, self.rows_np = ps, rows
        total = int(blocks.sum()) * H
        free = rng.permutation(total + spare)
        table = np.full((B, L, H, self.most), -1, np.int64)
        K, V = (np.full((total + spare, ps, d), np.nan, np.float32) for _ in "KV")
        at = 0
        for b in range(B):
            for l in range(L):
                for h in range(H):
                    for i in range(min(self.most, int(blocks[b, l]))):
                        page, at = free[at], at + 1
                        n = min(ps, int(rows[b, l]) - i * ps)
                        K[page, :n] = sigma * rng.standard_normal((n, d)) + rng.standard_normal(d)
                        V[page, :n] = rng.standard_normal((n, d))
                        table[b, l, h, i] = page
                        if rng.random() < lost:
                            table[b, l, h, i] = (-1, total + spare, 2 ** 31 - 1)[rng.integers(3)]
        self.table_np = table
        self.K, self.V = (torch.from_numpy(x).to(_dt(dtype)).cuda() for x in (K, V))
        self.rows, self.table = _int(rows), _int(table)
        self.K64, self.V64 = _f64(self.K), _f64(self.V)
        self.kv = _fc().PagedKV(self.K, self.V, self.rows, self.table)

    def unit(self, b, l, h, places=None):
        places = range(self.most) if places is None else places
        return pr.rows_at(self.K64, self.V64, self.rows_np[b, l], self.table_np[b, l, h], self.ps, places)


def _check_attention(got, Q, scale, rows_for, dtype):
    """rows_for(b, l, h): K, V of the unit in float64."""
    got, Q = _f64(got), _f64(Q)
    B, L, Hq, d = Q.shape
    for b in range(B):
        for l in range(L):
            h = 0
            while h * rows_for.group < Hq:
                g = slice(h * rows_for.group, (h + 1) * rows_for.group)
                K, V = rows_for(b, l, h)
                want, size, logit, terms = pr.attend(Q[b, l, g], K, V, scale)
                slip = 2 * (d * U * terms + 4 * U * (logit + 1)) + (K.shape[0] / 16 + 64) * U
                worst = np.max(np.abs(got[b, l, g] - want) - slip * size)
                assert worst <= 0, (b, l, h, K.shape[0], worst)
                h += 1


class _Rows:
    def __init__(self, group, fn):
        self.group, self.fn = group, fn

    def __call__(self, b, l, h):
        return self.fn(b, l, h)


# ---- append -----------------------------------------------------------------------------------
def _slots(rng, B, H, T, held, ps, num_pages, lost=0.0, unit_pages=None):
    """Slots of rows held .. held + T - 1 of B * H units, pages at random places."""
    most = -(-(held + T) // ps)
    free = rng.permutation(num_pages)
    assert B * H * most <= num_pages
    table = free[:B * H * most].reshape(B, H, most).copy()
    row = held + np.arange(T)
    slots = table[:, :, row // ps] * ps + row % ps
    if lost:
        gone = rng.random((B, H, most)) < lost
        slots = np.where(gone[:, :, row // ps], (-1, num_pages * ps, -2 ** 40)[rng.integers(3)], slots)
    return slots, table


@pytest.mark.parametrize("bounds", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,H,G,d,R,ps,held,inter,streams,lost", [
    (1, 1, 1, 1, 64, 64, 16, 0, False, 1, 0.0), (3, 1, 4, 7, 128, 128, 64, 63, False, 3, 0.3), (2, 1, 2, 2, 128, 64, 64, 64, True, 1, 0.0),
    (2, 5, 2, 3, 64, 32, 16, 14, True, 2, 0.0), (1, 130, 3, 1, 80, 20, 48, 7, False, 1, 0.2), (2, 67, 1, 4, 80, 80, 1, 3, True, 1, 0.1),
    (1, 300, 2, 4, 128, 128, 128, 100, False, 4, 0.2), (1, 77, 2, 2, 2, 2, 16, 9, False, 1, 0.0), (1, 33, 1, 1, 512, 64, 7, 5, True, 1, 0.0),
    (2, 19, 5, 0, 6, 4, 3, 0, False, 1, 0.3), (5, 1, 8, 16, 24, 18, 33, 32, True, 1, 0.0), (1, 200, 1, 2, 256, 256, 100, 1, False, 1, 0.0),
])
def test_append(dtype, bounds, B, T, H, G, d, R, ps, held, inter, streams, lost):
    fc = _fc()
    rng = np.random.default_rng(B * 100 + T + d + ps)
    dt = _dt(dtype)
    pages = B * H * -(-(held + T) // ps) + 3
    slots, _ = _slots(rng, B, H, T, held, ps, pages, lost)
    x = _rand(rng, (B, T, (G + 2) * H, d), dt)
    Q, K, V = x[:, :, :G * H], x[:, :, G * H:(G + 1) * H], x[:, :, (G + 1) * H:]
    pos = rng.integers(-5, 200000, (streams, B, T)).astype(np.int32)
    half, sections = R // 2, None
    if streams > 1:
        sections = [half // streams] * (streams - 1)
        sections.append(half - sum(sections))
    plan = fc.rotary_plan(R, theta=5e5, interleaved=inter, sections=sections)
    f, m = dr.frequencies(R, theta=5e5)
    old = _rand(rng, (2, pages, ps, d), dt)
    Kp, Vp = old[0].clone(), old[1].clone()
    lim = _rand(rng, (pages, 2, d), dt) if bounds else None
    lim_before = None if lim is None else _f64(lim)
    got = fc.append_paged(plan, _int(pos), Q, K, V, _int(slots, np.int64), Kp, Vp, bounds=lim)
    assert got.shape == Q.shape and got.dtype == dt

    def check(y, x):
        want, size, angle = dr.rotary(_f64(x), pos, f, R, inter, m, sections=sections)
        slip = np.zeros(want.shape)
        slip[..., :R] = 8 * U
        if want.size:
            tol = size * m * (slip + np.abs(angle).max() * 2.0 ** -50) + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0.0)
            assert np.all(np.abs(_f64(y) - want) <= tol)
            assert np.array_equal(_f64(y)[..., R:], _f64(x)[..., R:])
    check(got, Q)
    flat = torch.from_numpy(slots).cuda().transpose(1, 2).reshape(-1)           # [B, T, H], as the rows are
    ok = (flat >= 0) & (flat < pages * ps)
    rows = torch.where(ok, flat, 0)
    stored = Kp.view(-1, d)[rows].view(B, T, H, d)
    keep = ok.view(B, T, H, 1)
    check(torch.where(keep, stored, torch.zeros_like(stored)), torch.where(keep, K, torch.zeros_like(K)))
    assert torch.equal(Vp.view(-1, d)[rows[ok]], V.reshape(-1, d)[ok])
    other = torch.ones(pages * ps, dtype=torch.bool, device="cuda")
    other[rows[ok]] = False
    assert torch.equal(Kp.view(-1, d)[other], old[0].view(-1, d)[other]) and torch.equal(Vp.view(-1, d)[other], old[1].view(-1, d)[other])
    if bounds:
        assert np.array_equal(_f64(lim), pr.append_bounds(lim_before, _f64(Kp), slots, ps))


@pytest.mark.parametrize("dtype,B,T,H,G,d,inter,bounds", [
    ("bf16", 1, 16001, 4, 7, 128, False, False), ("bf16", 1, 16001, 4, 7, 128, True, True), ("f32", 2, 9001, 2, 4, 128, False, True),
    ("bf16", 3, 5001, 8, 4, 64, False, True), ("f32", 1, 20001, 1, 1, 64, True, False),
])
def test_append_of_many_tokens_is_that_of_few(dtype, B, T, H, G, d, inter, bounds):
    fc = _fc()
    dt, ps, held = _dt(dtype), 48, 29
    g = torch.Generator(device="cuda").manual_seed(T)
    Q, K, V = (torch.randn((B, T, n, d), generator=g, device="cuda").to(dt) for n in (G * H, H, H))
    pos = torch.randint(-1000, 200000, (B, T), generator=g, device="cuda", dtype=torch.int32)
    most = -(-(held + T) // ps)
    pages = B * H * most + 2
    table = torch.randperm(pages, generator=g, device="cuda")[:B * H * most].view(B, H, most)
    row = held + torch.arange(T, device="cuda")
    slots = table[:, :, row // ps] * ps + row % ps
    Kp, Vp = (torch.zeros((pages, ps, d), dtype=dt, device="cuda") for _ in "KV")
    lim = torch.zeros((pages, 2, d), dtype=dt, device="cuda") if bounds else None
    plan = fc.rotary_plan(d, theta=1e6, interleaved=inter)
    want, k = torch.empty_like(Q), torch.zeros_like(Kp)
    v = torch.zeros_like(Vp)
    for t in range(0, T, 61):
        p, *few = (x[:, t:t + 61].contiguous() for x in (pos, Q, K, V))
        fc.append_paged(plan, p, *few, slots[:, :, t:t + 61], k, v, Q_out=want[:, t:t + 61])
    # by the rotation alone: either is off by 8 u (|x0| + |x1|), and half a step of bf16, as the compiler may fuse either product of a sum
    for x, y in zip((Q, K), fc.rotary(plan, pos, Q, K)):
        z = want if x is Q else k.view(-1, d)[slots.transpose(1, 2)]
        a = x.float().abs()
        pair = a.unflatten(-1, (-1, 2)).sum(-1).repeat_interleave(2, -1) if inter else (a[..., :d // 2] + a[..., d // 2:]).repeat(1, 1, 1, 2)
        y = y.float()
        assert bool(((z.float() - y).abs() <= 16 * U * pair + (2.0 ** -7 * (y.abs() + 16 * U * pair) if dtype == "bf16" else 0.0)).all())
    Q_in_place = Q.clone()
    out = fc.append_paged(plan, pos, Q_in_place, K, V, slots, Kp, Vp, Q_out=Q_in_place, bounds=lim)
    assert out is Q_in_place and torch.equal(out, want) and torch.equal(Kp, k) and torch.equal(Vp, v)
    k = Kp.view(-1, d)[slots.transpose(1, 2)]
    at = slots.transpose(1, 2)
    assert torch.equal(Kp.view(-1, d)[at], k) and torch.equal(Vp.view(-1, d)[at], V)
    if bounds:
        at_page = (slots // ps).reshape(-1)
        flat = k.transpose(1, 2).reshape(-1, d).float()
        for j, how in ((0, "amin"), (1, "amax")):
            ref = torch.zeros((pages, d), device="cuda")
            began = (slots[slots % ps == 0] // ps)
            ref[began] = math.inf if j == 0 else -math.inf
            ref.scatter_reduce_(0, at_page[:, None].expand(-1, d), flat, how)
            assert torch.equal(lim[:, j].float(), ref)


def test_append_of_strided_and_unaligned_rows():
    fc = _fc()
    rng = np.random.default_rng(5)
    for dtype in (torch.bfloat16, torch.float32):
        for shift in (0, 1, 2, 4):
            x = _rand(rng, (2, 5, 64 * 8 + 8), dtype)
            Q, K, V = (x[..., shift + a:shift + b].unflatten(2, (-1, 64)) for a, b in ((0, 256), (256, 384), (384, 512)))
            slots = _int(rng.permutation(4 * 16).reshape(2, 2, 16)[:, :, :5], np.int64)
            Kp, Vp = torch.zeros((2, 4, 16, 64), dtype=dtype, device="cuda")
            pos = _int(rng.integers(0, 5000, (2, 5)))
            plan = fc.rotary_plan(64)
            at = slots.transpose(1, 2)

            def straight(*x):
                Kc, Vc = torch.zeros((2, 4, 16, 64), dtype=dtype, device="cuda")
                q = fc.append_paged(plan, pos, *(t.contiguous() for t in x), slots, Kc, Vc)
                return q, Kc.view(-1, 64)[at]
            q, k = straight(Q, K, V)
            assert torch.equal(fc.append_paged(plan, pos, Q, K, V, slots, Kp, Vp), q)
            assert torch.equal(Kp.view(-1, 64)[at], k) and torch.equal(Vp.view(-1, 64)[at], V)
            # storage [B, H, T, d], and a layer's slice of a larger map
            Q, K, V = (_rand(rng, (2, n, 5, 64), dtype).transpose(1, 2) for n in (4, 2, 2))
            wide = torch.full((2, 6, 5), -1, dtype=torch.int64, device="cuda")
            wide[:, 2:4] = slots
            Kp.zero_()
            Vp.zero_()
            q, k = straight(Q, K, V)
            assert torch.equal(fc.append_paged(plan, pos, Q, K, V, wide[:, 2:4], Kp, Vp), q)
            assert torch.equal(Kp.view(-1, 64)[at], k) and torch.equal(Vp.view(-1, 64)[at], V)


def test_append_of_nothing():
    fc = _fc()
    plan = fc.rotary_plan(64)
    pages = torch.ones((2, 4, 16, 64), device="cuda")
    lim = torch.ones((4, 2, 64), device="cuda")
    for B, T, Hq, H in ((0, 1, 4, 2), (2, 0, 4, 2), (2, 3, 0, 0), (2, 3, 4, 0)):
        Q, K, V = (torch.ones((B, T, n, 64), device="cuda") for n in (Hq, H, H))
        slots = torch.full((B, H, T), 5, dtype=torch.int64, device="cuda")
        out = fc.append_paged(plan, torch.zeros((B, T), dtype=torch.int32, device="cuda"), Q, K, V, slots, pages[0], pages[1], bounds=lim)
        assert torch.equal(out, Q)
    assert bool((pages == 1).all()) and bool((lim == 1).all())


# ---- bounds -----------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,H,d,ps,lost", [
    ([[1]], 1, 64, 16, 0.0), ([[0, 5], [17, 33]], 2, 128, 16, 0.0), ([[100, 1, 64]], 3, 64, 64, 0.2), ([[700]], 1, 128, 48, 0.1),
    ([[130], [0], [129]], 2, 80, 128, 0.0), ([[9, 3]], 1, 8, 1, 0.0), ([[50]], 4, 256, 7, 0.0), ([[-4, 31]], 1, 24, 33, 0.0),
])
def test_page_bounds(dtype, rows, H, d, ps, lost):
    fc = _fc()
    rng = np.random.default_rng(d + ps)
    c = Cache(rng, rows, H, d, ps, dtype, lost=lost)
    before = _rand(rng, (c.K.shape[0], 2, d), _dt(dtype))
    got = fc.page_bounds(c.kv, before.clone())
    assert np.array_equal(_f64(got), pr.page_bounds(c.K64, c.rows_np, c.table_np, ps, _f64(before)))
    zeros = pr.page_bounds(c.K64, c.rows_np, c.table_np, ps, np.zeros(before.shape))
    assert np.array_equal(_f64(fc.page_bounds(c.kv)), zeros)


def test_page_bounds_of_many_pages_a_short_table_and_nans():
    fc = _fc()
    rng = np.random.default_rng(8)
    c = Cache(rng, rng.integers(0, 3000, (3, 9)), 3, 64, 16, "bf16")
    assert np.array_equal(_f64(fc.page_bounds(c.kv)), pr.page_bounds(c.K64, c.rows_np, c.table_np, 16, np.zeros((c.K.shape[0], 2, 64))))
    c = Cache(rng, [[100]], 2, 64, 16, "f32", most=3)                # rows beyond the table
    c.K[c.table[0, 0, 0, 1].item(), 3, 5] = math.nan
    c.K[c.table[0, 0, 1, 2].item(), :, 7] = math.nan
    c.K[c.table[0, 0, 1, 0].item(), 2, 9] = math.inf
    got = _f64(fc.page_bounds(c.kv))
    assert np.array_equal(got, pr.page_bounds(_f64(c.K), c.rows_np, c.table_np, 16, np.zeros(got.shape)))
    page = c.table[0, 0, 1, 2].item()
    assert got[page, 0, 7] == math.inf and got[page, 1, 7] == -math.inf


# ---- choice -----------------------------------------------------------------------------------
def test_page_bounds_of_a_table_that_reaches_past_31_bits():
    # place 2^26 of a table of pages of 64 rows begins at row 2^32: it holds none of the unit's 5 rows
    fc = _fc()
    rng = np.random.default_rng(29)
    K = _rand(rng, (2, 64, 64), torch.bfloat16)
    table = torch.full((1, 1, 1, (1 << 26) + 1), -1, dtype=torch.int32, device="cuda")
    table[..., 0], table[..., -1] = 0, 1
    bounds = torch.full((2, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    fc.page_bounds(fc.PagedKV(K, K, _int([[5]]), table), bounds)
    assert torch.equal(bounds[0], torch.stack([K[0, :5].amin(0), K[0, :5].amax(0)]))
    assert (bounds[1] == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,H,G,d,ps,count,first,last,lost", [
    ([[1]], 1, 1, 64, 16, 1, 0, 0, 0.0), ([[0, 40], [500, 1000]], 2, 7, 128, 16, 9, 1, 2, 0.0), ([[2000, 300]], 3, 2, 64, 16, 40, 0, 0, 0.2),
    ([[4000]], 1, 16, 128, 16, 250, 2, 4, 0.0), ([[90000]], 1, 4, 64, 16, 100, 1, 1, 0.1), ([[640, 641]], 2, 3, 128, 64, 4, 2, 2, 0.4),
    ([[300]], 1, 8, 64, 16, 33, 40 - 33, 8, 0.0), ([[17]], 2, 1, 64, 16, 8, 3, 3, 0.5), ([[1040]], 2, 1, 64, 16, 64, 0, 1, 0.0),
])
def test_choose_pages(dtype, rows, H, G, d, ps, count, first, last, lost):
    fc = _fc()
    rng = np.random.default_rng(count + ps + d)
    c = Cache(rng, rows, H, d, ps, dtype, lost=lost, spare=5)
    bounds = fc.page_bounds(c.kv)
    B, L = c.rows_np.shape
    Q = _rand(rng, (B, L, G * H, d), _dt(dtype))
    got = fc.choose_pages(Q, c.kv, bounds, count, first=first, last=last)
    want = pr.choose_pages(_f64(Q), _f64(bounds), c.rows_np, c.table_np, ps, count, first, last)
    assert np.array_equal(got.cpu().numpy(), want)
    # what is there already is written over, with a workspace that holds anything
    ws = fc.chosen_workspace(Q, c.kv, count).fill_(255)
    again = fc.choose_pages(Q, c.kv, bounds, count, first=first, last=last, chosen=torch.full_like(got, 77), workspace=ws)
    assert torch.equal(got, again)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,H,G,d,most", [
    ([[0, 1, 403, 800, 1600, 2400]], 1, 4, 128, None), ([[70, 0], [33, 1021]], 2, 3, 64, 900), ([[512]], 3, 2, 128, None), ([[513]], 3, 2, 128, None),
    ([[256, 255]], 1, 7, 128, None), ([[257, 30]], 1, 7, 128, None), ([[0, 5]], 1, 2, 128, 5000),
])
def test_choose_pages_of_few_units(dtype, rows, H, G, d, most):
    # short layers in a long table, and tables around the longest that a workgroup scores and searches by itself
    fc = _fc()
    rng = np.random.default_rng(rows[0][-1])
    c = Cache(rng, rows, H, d, 4, dtype, most=most, lost=0.1)
    bounds = fc.page_bounds(c.kv)
    B, L = c.rows_np.shape
    Q = _rand(rng, (B, L, G * H, d), _dt(dtype))
    for count, first, last in ((1, 0, 0), (9, 1, 2), (150, 0, 1)):
        got = fc.choose_pages(Q, c.kv, bounds, count, first=first, last=last)
        assert np.array_equal(got.cpu().numpy(), pr.choose_pages(_f64(Q), _f64(bounds), c.rows_np, c.table_np, 4, count, first, last)), count


@pytest.mark.parametrize("dtype,B,L,H,G,d,ps,most,count,first,last,lost", [
    ("bf16", 5, 7, 2, 7, 128, 16, 500, 9, 1, 2, 0.1), ("f32", 3, 11, 2, 3, 64, 16, 2000, 70, 0, 0, 0.1), ("bf16", 10, 14, 2, 1, 64, 16, 400, 12, 2, 0, 0.3),
    ("f32", 13, 10, 2, 4, 128, 32, 900, 5, 0, 1, 0.0), ("bf16", 4, 8, 2, 2, 64, 4, 3000, 513, 5, 5, 0.0), ("bf16", 9, 15, 2, 2, 64, 4, 3000, 100, 0, 3, 0.0),
])
def test_choose_pages_of_many_units(dtype, B, L, H, G, d, ps, most, count, first, last, lost):
    fc = _fc()
    rng = np.random.default_rng(most + count)
    rows = rng.integers(0, most + 1, (B, L))
    rows[0, :3] = 0, 1, most
    c = Cache(rng, rows, H, d, ps, dtype, lost=lost)
    bounds = fc.page_bounds(c.kv)
    Q = _rand(rng, (B, L, G * H, d), _dt(dtype))
    got = fc.choose_pages(Q, c.kv, bounds, count, first=first, last=last)
    assert np.array_equal(got.cpu().numpy(), pr.choose_pages(_f64(Q), _f64(bounds), rows, c.table_np, ps, count, first, last))


def test_choice_between_equal_scores_and_without_numbers():
    fc = _fc()
    rng = np.random.default_rng(2)
    c = Cache(rng, [[16 * 700]], 2, 64, 16, "f32")
    bounds = fc.page_bounds(c.kv)
    few = _rand(rng, (3, 2, 64), torch.float32)                      # three different pages alone
    bounds[:] = few[torch.from_numpy(rng.integers(0, 3, bounds.shape[0])).cuda()]
    bounds[c.table[0, 0, 0, 40:60].long()] = math.nan
    bounds[c.table[0, 0, 1, 10].long(), 1] = math.inf
    bounds[c.table[0, 0, 1, 11].long(), 0] = -math.inf
    Q = _rand(rng, (1, 1, 6, 64), torch.float32)
    for count in (1, 5, 300, 690, 700, 900):
        got = fc.choose_pages(Q, c.kv, bounds, count, first=0, last=1).cpu().numpy()
        assert np.array_equal(got, pr.choose_pages(_f64(Q), _f64(bounds), c.rows_np, c.table_np, 16, count, 0, 1)), count
    # queries of zeros: every score is zero, of either sign; the earliest pages
    got = fc.choose_pages(torch.zeros_like(Q), c.kv, torch.sign(torch.nan_to_num(bounds)), 7, first=0, last=0).cpu().numpy()
    assert np.array_equal(got, np.broadcast_to(np.arange(7), got.shape))
    # and none that is a number
    got = fc.choose_pages(torch.full_like(Q, math.nan), c.kv, bounds, 7, first=0, last=2).cpu().numpy()
    assert np.array_equal(got, np.broadcast_to([0, 1, 2, 3, 4, 698, 699], got.shape))


# ---- attention over chosen pages ---------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,H,G,d,ps,count,lost", [
    ([[1]], 1, 1, 64, 16, 1, 0.0), ([[0, 40], [500, 1000]], 2, 7, 128, 16, 9, 0.0), ([[900, 300]], 3, 2, 64, 48, 40, 0.2),
    ([[4000]], 1, 16, 128, 64, 62, 0.0), ([[90]], 1, 4, 64, 1, 33, 0.1), ([[640, 641]], 2, 3, 128, 128, 4, 0.4),
    ([[3000]], 1, 8, 64, 16, 150, 0.0), ([[17]], 2, 1, 128, 7, 8, 0.5), ([[1040, 3, 0]], 4, 5, 64, 33, 20, 0.0),
])
def test_attention_over_chosen_pages(dtype, rows, H, G, d, ps, count, lost):
    fc = _fc()
    rng = np.random.default_rng(count + ps + d)
    c = Cache(rng, rows, H, d, ps, dtype, lost=lost, spare=5)
    B, L = c.rows_np.shape
    Q = _rand(rng, (B, L, G * H, d), _dt(dtype))
    scale = 1.0 / math.sqrt(d)
    # any order, places twice, beyond the table, negative
    chosen = rng.integers(-2, c.most + 2, (B, L, H, count)).astype(np.int32)
    chosen[0, 0, 0, 0] = 0
    ws = fc.chosen_workspace(Q, c.kv, count).fill_(255)
    for s in (scale, -2 * scale):
        got = fc.decode_attention_chosen(Q, c.kv, _int(chosen), s, workspace=ws)
        _check_attention(got, Q, s, _Rows(G, lambda b, l, h: c.unit(b, l, h, chosen[b, l, h])), dtype)
    # all of them, in order: the attention over the whole cache
    every = np.broadcast_to(np.arange(c.most), (B, L, H, c.most))
    got = fc.decode_attention_chosen(Q, c.kv, _int(every), scale)
    _check_attention(got, Q, scale, _Rows(G, c.unit), dtype)
    none = fc.decode_attention_chosen(Q, c.kv, torch.full((B, L, H, count), -1, dtype=torch.int32, device="cuda"), scale)
    assert bool((none == 0).all())


# ---- attention to a shared prompt --------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("common,own,starts,H,G,d,ps,ps_own,lost", [
    ([[1]], [[0]], [0, 1], 1, 1, 64, 16, 16, 0.0),
    ([[300, 20]], [[5, 6], [0, 0], [100, 7]], [0, 3], 2, 7, 128, 64, 16, 0.0),
    ([[700], [64], [0]], [[3], [9], [1], [40], [0], [2], [8]], [1, 3, 3, 6], 2, 3, 64, 16, 48, 0.2),
    ([[2000, 1]], [[i, 2 * i] for i in range(40)], [0, 40], 1, 16, 128, 64, 64, 0.0),
    ([[100]] * 3, [[33]] * 20, [0, 1, 9, 20], 1, 4, 128, 32, 32, 0.4),
    ([[500, 0, 31]], [[0, 0, 0]] * 9, [0, 9], 3, 1, 64, 16, 16, 0.0),
    ([[50]], [[700], [1]], [2, 2], 2, 2, 64, 16, 16, 0.0),
    ([[129]], [[3]] * 19, [0, 19], 2, 7, 128, 128, 7, 0.1),
    ([[40], [41]], [[3]] * 5, [-7, 2, 99], 1, 2, 64, 1, 16, 0.0),
    ([[9000]], [[3000]] * 2, [0, 2], 1, 5, 128, 64, 16, 0.0),
    ([[500, 77]], [[9, 0]] * 30, [0, 30], 1, 4, 128, 4, 4, 0.5),
    ([[500, 77]], [[9, 0]] * 30, [0, 30], 1, 4, 64, 4, 4, 0.5),
    ([[-3, 90], [41, 17]], [[-1, 8]] * 6, [0, 4, 6], 2, 16, 64, 8, 2, 0.0),
])
def test_attention_to_a_shared_prompt(dtype, common, own, starts, H, G, d, ps, ps_own, lost):
    fc = _fc()
    rng = np.random.default_rng(G + ps + d)
    cc, co = Cache(rng, common, H, d, ps, dtype, lost=lost), Cache(rng, own, H, d, ps_own, dtype, lost=lost)
    P, (B, L) = len(common), co.rows_np.shape
    Q = _rand(rng, (B, L, G * H, d), _dt(dtype))
    scale = 1.0 / math.sqrt(d)

    def rows_for(b, l, h):
        K, V = co.unit(b, l, h)
        for p in range(P):
            if max(0, starts[p]) <= b < starts[p + 1]:
                k, v = cc.unit(p, l, h)
                K, V = np.concatenate((k, K)), np.concatenate((v, V))
        return K, V
    ws = fc.shared_workspace(Q, H, P).fill_(255)
    for _ in range(2):
        got = fc.decode_attention_shared(Q, cc.kv, _int(starts), co.kv, scale, workspace=ws)
        _check_attention(got, Q, scale, _Rows(G, rows_for), dtype)
    assert torch.equal(got, fc.decode_attention_shared(Q, cc.kv, _int(starts), co.kv, scale))


def test_attention_without_prompts_and_of_no_sequences():
    fc = _fc()
    rng = np.random.default_rng(1)
    co = Cache(rng, [[40, 3], [0, 9]], 2, 64, 16, "bf16")
    nothing = fc.PagedKV(co.K, co.V, torch.empty((0, 2), dtype=torch.int32, device="cuda"), torch.empty((0, 2, 2, 1), dtype=torch.int32, device="cuda"))
    Q = _rand(rng, (2, 2, 6, 64), torch.bfloat16)
    got = fc.decode_attention_shared(Q, nothing, _int([0]), co.kv, 0.125)
    _check_attention(got, Q, 0.125, _Rows(3, co.unit), "bf16")
    empty = torch.empty((0, 2, 6, 64), dtype=torch.bfloat16, device="cuda")
    assert fc.decode_attention_shared(empty, co.kv, _int([0, 0, 0]), nothing, 0.125).shape == empty.shape
    lim = torch.ones((co.K.shape[0], 2, 64), dtype=torch.bfloat16, device="cuda")
    assert bool((fc.page_bounds(nothing, lim) == 1).all())
    chosen = fc.choose_pages(empty, nothing, lim, 3)
    assert chosen.shape == (0, 2, 2, 3) and fc.decode_attention_chosen(empty, nothing, chosen, 0.125).shape == empty.shape


def test_many_prompts_and_layers():
    """More entries than a wave's lanes, prompts without sequences among them."""
    fc = _fc()
    rng = np.random.default_rng(6)
    P, B, L, H, G, d = 70, 90, 3, 1, 2, 64
    cc = Cache(rng, rng.integers(0, 60, (P, L)), H, d, 16, "bf16")
    co = Cache(rng, rng.integers(0, 40, (B, L)), H, d, 16, "bf16")
    starts = np.sort(rng.integers(0, B + 1, P + 1))
    Q = _rand(rng, (B, L, G * H, d), torch.bfloat16)

    def rows_for(b, l, h):
        K, V = co.unit(b, l, h)
        for p in range(P):
            if starts[p] <= b < starts[p + 1]:
                k, v = cc.unit(p, l, h)
                K, V = np.concatenate((k, K)), np.concatenate((v, V))
        return K, V
    _check_attention(fc.decode_attention_shared(Q, cc.kv, _int(starts), co.kv, 0.125), Q, 0.125, _Rows(G, rows_for), "bf16")


@pytest.mark.parametrize("dtype,d,B,G,rows", [("bf16", 128, 5, 4, 40000), ("bf16", 64, 20, 6, 70001), ("f32", 128, 9, 8, 20001), ("f32", 64, 6, 3, 33000)])
def test_long_pieces_of_a_shared_prompt(dtype, d, B, G, rows):
    """Pieces of more steps than are looked up together (32 units, many rows), against float64 on the GPU."""
    fc = _fc()
    dt, L, H, ps = _dt(dtype), 8, 4, 48
    g = torch.Generator(device="cuda").manual_seed(rows)
    most = -(-rows // ps)
    pages = L * H * most + 2
    K, V = (torch.randn((pages, ps, d), generator=g, device="cuda").to(dt) for _ in "KV")
    table = torch.randperm(pages, generator=g, device="cuda")[:L * H * most].view(1, L, H, most).to(torch.int32)
    held = torch.tensor([[rows - 37 * l for l in range(L)]], dtype=torch.int32, device="cuda")
    own = fc.PagedKV(K, V, torch.zeros((B, L), dtype=torch.int32, device="cuda"), torch.full((B, L, H, 1), -1, dtype=torch.int32, device="cuda"))
    Q = torch.randn((B, L, H * G, d), generator=g, device="cuda").to(dt)
    scale = 1.0 / math.sqrt(d)
    got = fc.decode_attention_shared(Q, fc.PagedKV(K, V, held, table), _int([0, B]), own, scale)
    for l in range(L):
        n = int(held[0, l])
        for h in range(H):
            j = torch.arange(n, device="cuda")
            at = table[0, l, h].long()[j // ps] * ps + j % ps
            k, v = K.view(-1, d)[at].double(), V.view(-1, d)[at].double()
            q = Q[:, l, h * G:(h + 1) * G].double().reshape(-1, d)
            logit = q @ k.t().contiguous() * scale
            p = torch.softmax(logit, 1)
            want, size = p @ v, p @ v.abs()
            terms = (q.abs() @ k.abs().t().contiguous()).max() * scale
            slip = 2 * (d * U * terms + 4 * U * (logit.abs().max() + 1)) + (n / 16 + 64) * U
            assert bool(((got[:, l, h * G:(h + 1) * G].double().reshape(-1, d) - want).abs() <= slip * size).all())


def test_calls_at_once_on_two_streams():
    """Workspaces of their own, rows beyond the table and below zero."""
    fc = _fc()
    rng = np.random.default_rng(51)
    co, cc = Cache(rng, [[300, -2], [64, 9]], 2, 64, 16, "bf16", most=5), Cache(rng, [[400, 3]], 2, 64, 16, "bf16", most=9)
    Q = _rand(rng, (2, 2, 6, 64), torch.bfloat16)
    bounds, starts = fc.page_bounds(co.kv), _int([0, 2])
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for s in streams * 3:
        with torch.cuda.stream(s):
            chosen = fc.choose_pages(Q, co.kv, bounds, 5, first=0, last=0)
            outs.append((fc.decode_attention_chosen(Q, co.kv, chosen, 0.2), fc.decode_attention_shared(Q, cc.kv, starts, co.kv, 0.2)))
    torch.cuda.synchronize()

    def rows_for(b, l, h):
        return tuple(np.concatenate(x) for x in zip(cc.unit(0, l, h), co.unit(b, l, h)))
    for a, b in outs:
        _check_attention(a, Q, 0.2, _Rows(3, co.unit), "bf16")
        _check_attention(b, Q, 0.2, _Rows(3, rows_for), "bf16")


# ---- as they are used -------------------------------------------------------------------------
def test_slices_of_a_layer():
    fc = _fc()
    rng = np.random.default_rng(12)
    B, L, H, G, d, ps = 3, 4, 2, 3, 64, 16
    cc, co = Cache(rng, rng.integers(1, 200, (2, L)), H, d, ps, "bf16"), Cache(rng, rng.integers(1, 90, (B, L)), H, d, ps, "bf16")
    Q = _rand(rng, (B, L, G * H, d), torch.bfloat16)
    starts, scale = _int([0, 2, 3]), 0.2
    bounds = fc.page_bounds(co.kv)
    whole = (fc.decode_attention_shared(Q, cc.kv, starts, co.kv, scale), fc.choose_pages(Q, co.kv, bounds, 3))
    layered = torch.zeros_like(bounds)
    for l in range(L):
        kc, ko = (fc.PagedKV(c.K, c.V, c.rows[:, l:l + 1], c.table[:, l:l + 1]) for c in (cc, co))
        q = Q[:, l:l + 1].contiguous()
        a, b = _f64(fc.decode_attention_shared(q, kc, starts, ko, scale))[:, 0], _f64(whole[0])[:, l]
        assert np.max(np.abs(a - b)) <= 1e-5 * np.abs(b).max()
        chosen = fc.choose_pages(q, ko, bounds, 3)
        assert torch.equal(chosen[:, 0], whole[1][:, l])
        out = fc.decode_attention_chosen(q, ko, chosen, scale)
        _check_attention(out, q, scale, _Rows(G, lambda b, _, h: co.unit(b, l, h, chosen[b, 0, h].tolist())), "bf16")
        fc.page_bounds(ko, layered)
    assert torch.equal(layered, bounds)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_loop_of_answers_to_a_compressed_prompt(dtype):
    """A prompt is compressed into the prompts' cache; two answers to it decode step by step in a cache of their own, layer by layer, with pages
    taken as rows come; then the same rows as one cache, read whole and by its best pages."""
    fc = _fc()
    rng = np.random.default_rng(21)
    L, H, G, d, N, ps, B, steps = 3, 2, 4, 64, 512, 16, 2, 19
    dt, scale = _dt(dtype), 0.125
    K, V = _rand(rng, (1, L, H, N, d), dt), _rand(rng, (1, L, H, N, d), dt)
    comp = fc.Compressor(K, fc.cutoff_r(N, 0.1), fc.total_budget(L, N, 0.3))
    comp.run(K, V)
    pool = 3 * comp.rows_per_seq // ps + 200
    pages = [torch.full((pool, ps, d), math.nan, dtype=dt, device="cuda") for _ in "KV"]
    bounds = torch.zeros((pool, 2, d), dtype=dt, device="cuda")
    cursor = torch.zeros(1, dtype=torch.int64, device="cuda")
    tables = [torch.full((n, L, H, 40), -1, dtype=torch.int32, device="cuda") for n in (1, B)]
    rows = [torch.zeros((n, L), dtype=torch.int32, device="cuda") for n in (1, B)]
    fc.assign_pages(rows[0], comp.budgets, ps, tables[0], cursor, num_free=pool)
    fc.select_gather_paged(K, V, comp.desc, comp.scores, comp.budgets, comp.layer_offsets, comp.rows_per_seq, comp.idx, tables[0], ps, *pages)
    prompt = fc.PagedKV(*pages, rows[0], tables[0])
    fc.page_bounds(prompt, bounds)
    starts = _int([0, B])
    plan = fc.rotary_plan(d, theta=1e6)
    slots = torch.empty((B, L * H), dtype=torch.int64, device="cuda")
    f, m = dr.frequencies(d, theta=1e6)
    kept = {}
    for step in range(steps):
        fc.assign_pages(rows[1], 1, ps, tables[1], cursor, num_free=pool, slots=slots)
        pos = torch.full((B, 1), N + step, dtype=torch.int32, device="cuda")
        for l in range(L):
            x = _rand(rng, (B, 1, (G + 2) * H, d), dt)
            q = fc.append_paged(plan, pos, x[:, :, :G * H], x[:, :, G * H:(G + 1) * H], x[:, :, (G + 1) * H:],
                                slots.view(B, L, H, 1)[:, l], *pages, bounds=bounds)
            own = fc.PagedKV(*pages, rows[1][:, l:l + 1], tables[1][:, l:l + 1])
            common = fc.PagedKV(*pages, rows[0][:, l:l + 1], tables[0][:, l:l + 1])
            out = fc.decode_attention_shared(q, common, starts, own, scale)
            turned, _, _ = dr.rotary(_f64(x[:, :, G * H:(G + 1) * H]), np.full((1, B, 1), N + step), f, d, magnitude=m)
            kept.setdefault(l, []).append((_f64(torch.from_numpy(turned).to(dt)), _f64(x[:, :, (G + 1) * H:])))
        n = int(rows[0][0, l])
        if step % 6 == 0 or step == steps - 1:
            def rows_for(b, _, h):
                p = tables[0][0, l, h].long()[torch.arange(n) // ps]
                at = torch.arange(n, device="cuda") % ps
                mine = [np.stack([z[i][b, 0, h] for z in kept[l]]) for i in (0, 1)]
                return tuple(np.concatenate((_f64(pages[i][p, at]), mine[i])) for i in (0, 1))
            got, Qf = _f64(out), _f64(q)
            for b in range(B):
                for h in range(H):
                    k, v = rows_for(b, 0, h)
                    want, size, logit, terms = pr.attend(Qf[b, 0, h * G:(h + 1) * G], k, v, scale)
                    # (keys turned and rounded to the dtype by either side: a step of its, 2^-7 or 2^-21, in a logit's terms)
                    slip = 2 * terms * (2.0 ** -7 if dtype == "bf16" else 2.0 ** -20) + 200 * U
                    assert np.max(np.abs(got[b, 0, h * G:(h + 1) * G] - want) - slip * size) <= 0
    # bounds that the steps kept are those of the pages
    fresh = bounds.clone()
    both = fc.PagedKV(*pages, torch.cat((rows[0], rows[1])), torch.cat((tables[0], tables[1])))
    fc.page_bounds(both, fresh)
    assert torch.equal(fresh, bounds)
    # all pages chosen: the attention over the cache; half of them: over these
    Q = _rand(rng, (1 + B, L, G * H, d), dt)
    chosen = fc.choose_pages(Q, both, bounds, 40)
    mask = chosen.cpu().numpy()
    blocks = -(-both.rows.cpu().numpy() // ps)
    assert all(np.array_equal(mask[b, l, h], np.where(np.arange(40) < blocks[b, l], np.arange(40), -1))
               for b in range(1 + B) for l in range(L) for h in range(H))
    got = fc.decode_attention_chosen(Q, both, chosen, scale)
    if dtype == "bf16":
        ref = fc.decode_attention_paged(Q, *pages, H, both.rows, both.block_table, scale)
        assert float((got - ref).abs().max()) <= 2e-5 * float(torch.nan_to_num(pages[1].float()).abs().max())


@pytest.mark.parametrize("what", ["append", "bounds", "chosen", "shared"])
def test_captured_into_a_graph_and_on_another_stream(what):
    fc = _fc()
    rng = np.random.default_rng(31)
    B, L, H, G, d, ps = 2, 3, 2, 4, 128, 16
    cc, co = Cache(rng, [[300, 40, 5]], H, d, ps, "bf16"), Cache(rng, rng.integers(20, 90, (B, L)), H, d, ps, "bf16")
    Q = _rand(rng, (B, L, G * H, d), torch.bfloat16)
    starts = _int([0, 2])
    bounds = fc.page_bounds(co.kv)
    plan = fc.rotary_plan(d)
    x = _rand(rng, (B, 1, (G + 2) * H, d), torch.bfloat16)
    pos = _int([[7], [9]])
    slots = co.table[:, 0, :, :1].long() * ps + 3
    out, q_out = torch.zeros(Q.shape, device="cuda"), torch.zeros((B, 1, G * H, d), dtype=torch.bfloat16, device="cuda")
    chosen = torch.zeros((B, L, H, 3), dtype=torch.int32, device="cuda")
    ws = (fc.chosen_workspace(Q, co.kv, 3), fc.shared_workspace(Q, H, 1))

    def call():
        if what == "append":
            fc.append_paged(plan, pos, x[:, :, :G * H], x[:, :, G * H:(G + 1) * H], x[:, :, (G + 1) * H:], slots, co.K, co.V, Q_out=q_out, bounds=bounds)
            return [q_out, co.K, co.V, bounds]
        if what == "bounds":
            return [fc.page_bounds(co.kv, bounds)]
        if what == "chosen":
            fc.choose_pages(Q, co.kv, bounds, 3, chosen=chosen, workspace=ws[0])
            return [chosen, fc.decode_attention_chosen(Q, co.kv, chosen, 0.1, out=out, workspace=ws[0])]
        return [fc.decode_attention_shared(Q, cc.kv, starts, co.kv, 0.1, out=out, workspace=ws[1])]
    same = lambda a, b: torch.equal(torch.nan_to_num(a.float(), nan=12345.0), torch.nan_to_num(b.float(), nan=12345.0))  # noqa: E731
    call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        results = call()
    for turn in range(4):
        # other inputs: the graph reads what the tensors hold now
        Q.copy_(_rand(rng, Q.shape, torch.bfloat16))
        x.copy_(_rand(rng, x.shape, torch.bfloat16))
        co.rows.copy_(_int(rng.integers(0, 60, (B, L))))
        if what == "shared":
            starts.copy_(_int([[0, 2], [1, 2], [0, 1], [2, 2]][turn]))
        held = [t.clone() for t in (co.K, co.V, bounds)]
        for t in (out, q_out):
            t.fill_(-5)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in results]
        for t, v in zip((co.K, co.V, bounds), held):
            t.copy_(v)
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.default_stream())
            want = [t.clone() for t in call()]
        side.synchronize()
        assert all(same(a, b) for a, b in zip(got, want)), turn


def test_places_beyond_32_bits():
    """A cache whose keys take more than 2^32 bytes, rows at its far end."""
    fc = _fc()
    rng = np.random.default_rng(41)
    ps, d, H, G = 128, 128, 2, 4
    pages = (1 << 32) // (ps * d * 2) + 300
    K, V = (torch.empty((pages, ps, d), dtype=torch.bfloat16, device="cuda") for _ in "KV")
    bounds = torch.zeros((pages, 2, d), dtype=torch.bfloat16, device="cuda")
    T, most = 3 * ps + 9, 4
    table = np.array([pages - 1 - 2 * np.arange(most), pages - 2 - 2 * np.arange(most)]).reshape(1, 1, H, most)
    row = np.arange(T)
    slots = table[0, 0][:, row // ps] * ps + row % ps
    x = _rand(rng, (1, T, (G + 2) * H, d), torch.bfloat16)
    pos = torch.arange(T, device="cuda", dtype=torch.int32)[None]
    plan = fc.rotary_plan(d)
    fc.append_paged(plan, pos, x[:, :, :G * H], x[:, :, G * H:(G + 1) * H], x[:, :, (G + 1) * H:], _int(slots[None], np.int64), K, V, bounds=bounds)
    at = torch.from_numpy(slots).cuda()
    near = torch.zeros((2, 10, ps, d), dtype=torch.bfloat16, device="cuda")
    close = _int(np.stack((row, row + 5 * ps))[None], np.int64)
    fc.append_paged(plan, pos, x[:, :, :G * H], x[:, :, G * H:(G + 1) * H], x[:, :, (G + 1) * H:], close, *near)
    assert torch.equal(K.view(-1, d)[at], near[0].view(-1, d)[close[0]]) and torch.equal(V.view(-1, d)[at], x[0, :, (G + 1) * H:].transpose(0, 1))
    kv = fc.PagedKV(K, V, _int([[T]]), _int(table))
    again = torch.zeros_like(bounds)
    assert torch.equal(fc.page_bounds(kv, again), bounds)
    Q = _rand(rng, (1, 1, G * H, d), torch.bfloat16)
    rows_for = _Rows(G, lambda b, l, h: (_f64(K.view(-1, d)[at[h]]), _f64(V.view(-1, d)[at[h]])))
    chosen = fc.choose_pages(Q, kv, bounds, 4)
    assert chosen.flatten().tolist() == [0, 1, 2, 3] * H
    _check_attention(fc.decode_attention_chosen(Q, kv, chosen, 0.1), Q, 0.1, rows_for, "bf16")
    own = fc.PagedKV(K, V, _int([[0]]), _int(table))
    _check_attention(fc.decode_attention_shared(Q, kv, _int([0, 1]), own, 0.1), Q, 0.1, rows_for, "bf16")
