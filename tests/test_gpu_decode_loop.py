"""The decode loop's operators on the GPU against plain float64 statements of them (oracle/decode_loop_ref.py).

Tolerances.  u = 2^-24, half a step of fp32.
  rotary     an element is x0 c - x1 s: sine and cosine are off by the turn's rounding to 2^-32 and to fp32 (u), the series (2 u) and two
             products (2 u); the two products and the sum add 2 u: together below 8 u (|x0| + |x1|) m.  The angle itself is known to
             2^-52 of position * frequency on both sides.  bf16: half a step more, 2^-8 of the result.
  4 bits     equal: what is stored is defined to the bit.
  attention  a logit is a sum of d products (and d more for the terms of fp32 queries), in fp32: off by at most 3 d u sum |q k| scale, and its
             scaling and exponential by 4 u (|logit| + 1), twice (its own and the reference's); the sums over n rows go 32 at a time:
             n / 32 + 64 roundings.  All of it relative to sum p |v|.
"""
import math

import numpy as np
import pytest

from oracle import decode_loop_ref as dr

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


# ---- rotary -----------------------------------------------------------------------------------
def _check_rotary(got, want, size, angle, R, m, dtype, copied):
    got = _f64(got)
    slip = np.zeros(got.shape)
    slip[..., :R] = 8 * U
    pos = np.abs(angle).max() * 2.0 ** -50
    tol = size * m * (slip + pos) + (2.0 ** -8 * np.abs(want) if dtype == torch.bfloat16 else 0.0)
    worst = np.max(np.abs(got - want) - tol)
    assert worst <= 0, worst
    assert np.array_equal(got[..., R:], copied[..., R:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,Hq,Hk,d,R,inter", [
    (1, 1, 1, 1, 2, 2, False), (8, 1, 28, 4, 128, 128, False), (2, 37, 7, 1, 64, 64, True), (1, 300, 4, 2, 80, 20, False),
    (1, 19, 3, 3, 80, 20, True), (2, 5, 2, 1, 256, 256, False), (1, 7, 5, 0, 512, 64, True), (3, 11, 2, 2, 6, 4, False),
    (1, 130, 33, 8, 128, 32, False), (1, 3, 2, 1, 24, 18, True),
])
def test_rotary(dtype, B, T, Hq, Hk, d, R, inter):
    fc = _fc()
    rng = np.random.default_rng(B * 1000 + T + d)
    dt = _dt(dtype)
    Q = _rand(rng, (B, T, Hq, d), dt)
    K = _rand(rng, (B, T, Hk, d), dt) if Hk else None
    pos = torch.from_numpy(rng.integers(0, 200000, (B, T)).astype(np.int32)).cuda()
    plan = fc.rotary_plan(R, theta=5e5, interleaved=inter)
    f, m = dr.frequencies(R, theta=5e5)
    for inverse in (False, True):
        outs = fc.rotary(plan, pos, Q, K, inverse=inverse)
        for x, y in zip((Q, K), outs):
            if x is None:
                assert y is None
                continue
            want, size, angle = dr.rotary(_f64(x), pos.cpu().numpy()[None], f, R, inter, m, inverse=inverse)
            _check_rotary(y, want, size, angle, R, m, dt, _f64(x))


@pytest.mark.parametrize("scaling,kw", [("linear", {}), ("base", {}), ("parts", dict(original_tokens=4096))])
def test_rotary_scalings_sections_and_far_positions(scaling, kw):
    fc = _fc()
    rng = np.random.default_rng(3)
    R = 64
    Q, K = _rand(rng, (2, 9, 6, 64), torch.float32), _rand(rng, (2, 9, 2, 64), torch.float32)
    pos = rng.integers(-(1 << 31), 1 << 31, (3, 2, 9)).astype(np.int32)
    pos[0, 0, :3] = (2 ** 31 - 1, -2 ** 31, 0)
    plan = fc.rotary_plan(R, theta=1e6, scaling=scaling, factor=4.0, sections=(8, 12, 12), **kw)
    f, m = dr.frequencies(R, theta=1e6, scaling=scaling, factor=4.0, **kw)
    q, k = fc.rotary(plan, torch.from_numpy(pos).cuda(), Q, K)
    for x, y in ((Q, q), (K, k)):
        want, size, angle = dr.rotary(_f64(x), pos, f, R, magnitude=m, sections=(8, 12, 12))
        _check_rotary(y, want, size, angle, R, m, torch.float32, _f64(x))


def test_rotary_in_place_strided_and_unaligned():
    fc = _fc()
    rng = np.random.default_rng(4)
    for dtype in (torch.bfloat16, torch.float32):
        for shift in (0, 1, 2, 4):                     # elements that the rows are away from 16-byte places
            qkv = _rand(rng, (2, 5, 3 * 4 * 64 + 8), dtype)
            before = qkv.clone()
            Q, K = (qkv[..., shift + i * 256:shift + (i + 1) * 256].unflatten(2, (4, 64)) for i in (0, 1))
            pos = torch.from_numpy(rng.integers(0, 5000, (2, 5)).astype(np.int32)).cuda()
            plan = fc.rotary_plan(64)
            f, m = dr.frequencies(64)
            want = [dr.rotary(_f64(x), pos.cpu().numpy()[None], f, 64) for x in (Q, K)]
            fc.rotary(plan, pos, Q, K, Q_out=Q, K_out=K)
            for x, (w, size, angle) in zip((Q, K), want):
                _check_rotary(x, w, size, angle, 64, m, dtype, w)
            rest = torch.ones(qkv.shape[-1], dtype=torch.bool)
            rest[shift:shift + 512] = False
            assert torch.equal(qkv[..., rest], before[..., rest])
            # [B, H, T, d] storage into [B, T, H, d]
            X = _rand(rng, (2, 4, 5, 64), dtype).transpose(1, 2)
            y, _ = fc.rotary(plan, pos, X)
            w, size, angle = dr.rotary(_f64(X), pos.cpu().numpy()[None], f, 64)
            _check_rotary(y, w, size, angle, 64, m, dtype, w)


@pytest.mark.parametrize("dtype,T,Hq,Hk,d,R,inter", [
    ("bf16", 16001, 28, 4, 128, 128, False), ("bf16", 16001, 28, 4, 128, 128, True), ("f32", 16001, 9, 2, 128, 96, False),
    ("f32", 9001, 17, 8, 128, 32, True), ("bf16", 60001, 5, 1, 80, 20, True), ("bf16", 13001, 33, 8, 128, 64, False),
    ("bf16", 5001, 70, 3, 64, 64, False), ("bf16", 40001, 0, 8, 128, 128, False),
])
def test_rotary_of_many_tokens_equals_that_of_few(dtype, T, Hq, Hk, d, R, inter):
    """Large calls take several heads a thread and go past the cache; small ones are tested above against the oracle."""
    fc = _fc()
    g = torch.Generator(device="cuda").manual_seed(T)
    heads = [torch.randn((1, T, h, d), generator=g, device="cuda").to(_dt(dtype)) for h in (Hq, Hk)]
    pos = torch.randint(-1000, 200000, (1, T), generator=g, device="cuda", dtype=torch.int32)
    plan = fc.rotary_plan(R, theta=1e6, interleaved=inter)
    got = fc.rotary(plan, pos, *heads)
    want = [torch.empty_like(x) for x in heads]
    for t in range(0, T, 61):
        q, k = (x[:, t:t + 61] for x in heads)
        fc.rotary(plan, pos[:, t:t + 61].contiguous(), q, k, Q_out=want[0][:, t:t + 61], K_out=want[1][:, t:t + 61])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    fc.rotary(plan, pos, *heads, Q_out=heads[0], K_out=heads[1])             # in place
    assert all(torch.equal(a, b) for a, b in zip(heads, want))


def test_rotary_gradient_against_differences():
    """<g, rotary(x)> has the gradient rotary(g, inverse): against the formula's and against differences of the map itself."""
    fc = _fc()
    rng = np.random.default_rng(6)
    R, d = 48, 64
    plan = fc.rotary_plan(R, scaling="parts", factor=2.0, original_tokens=64, interleaved=True)
    pos = torch.from_numpy(rng.integers(0, 1000, (1, 3)).astype(np.int32)).cuda()
    x, g = _rand(rng, (1, 3, 2, d), torch.float32), _rand(rng, (1, 3, 2, d), torch.float32)
    grad = _f64(fc.rotary(plan, pos, g, inverse=True)[0])
    f, m = dr.frequencies(R, scaling="parts", factor=2.0, original_tokens=64)
    want, size, angle = dr.rotary(_f64(g), pos.cpu().numpy()[None], f, R, True, m, inverse=True)
    assert np.all(np.abs(grad - want) <= size * m * (8 * U + np.abs(angle).max() * 2.0 ** -50))
    for at in ((0, 0, 0, 0), (0, 1, 1, 17), (0, 2, 0, 47), (0, 2, 1, 60)):
        step = torch.zeros_like(x)
        step[at] = 0.5                                 # (the map is linear: any step will do)
        up, down = (_f64(fc.rotary(plan, pos, x + s * step)[0]) for s in (1, -1))
        diff = float(np.sum(_f64(g) * (up - down)))
        # two evaluations of at most 64 elements' errors of 8 u of their size
        scale = float(np.sum(np.abs(_f64(g)) * (np.abs(up) + np.abs(down) + 1)))
        assert abs(diff - grad[at]) <= 32 * U * scale * 2


# ---- pages ------------------------------------------------------------------------------------
@pytest.mark.parametrize("B,L,H,ps,most,high", [
    (1, 1, 1, 16, 3, 40), (2, 3, 2, 16, 5, 70), (8, 28, 4, 64, 8, 400), (3, 70, 1, 1, 9, 9), (1, 300, 2, 7, 4, 25), (2, 1024, 1, 32, 2, 40),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_assign_pages(B, L, H, ps, most, high, in_place):
    fc = _fc()
    rng = np.random.default_rng(B + L + ps)
    rows = np.zeros((B, L), np.int32)
    table = np.full((B, L, H, most), -1, np.int32)
    pool = int(B * L * H * most * 0.8) + 1                 # too few at the end
    free = rng.permutation(pool).astype(np.int32)
    cursor = 0
    t_table, t_free = torch.from_numpy(table).cuda(), torch.from_numpy(free).cuda()
    t_rows, t_cursor = torch.from_numpy(rows).cuda(), torch.zeros(1, dtype=torch.int64, device="cuda")
    for turn in range(4):
        add = rng.integers(-3, high if turn == 0 else 4, (B, L)).astype(np.int32)
        if turn == 2:
            add[:] = 1
        n = int(np.maximum(add, 0).sum(1).max()) * H + (5 if turn != 3 else -2)      # padding, and a map that is too short
        n = max(n, 0)
        table, slots, rows, cursor = dr.assign_pages(rows, add, table, ps, cursor, list(free), n)
        t_slots = torch.full((B, n), -7, dtype=torch.int64, device="cuda")
        arg = 1 if turn == 2 else torch.from_numpy(add).cuda()
        if in_place:
            fc.assign_pages(t_rows, arg, ps, t_table, t_cursor, t_free, slots=t_slots)
        else:
            r, c = torch.empty_like(t_rows), torch.empty_like(t_cursor)
            fc.assign_pages(t_rows, arg, ps, t_table, t_cursor, t_free, slots=t_slots, rows_out=r, cursor_out=c)
            t_rows, t_cursor = r, c
        assert np.array_equal(t_table.cpu().numpy(), table), turn
        assert np.array_equal(t_slots.cpu().numpy(), slots), turn
        assert np.array_equal(t_rows.cpu().numpy(), rows) and int(t_cursor) == cursor, turn
    # without a map, from a counted pool
    fresh = np.full((B, L, H, most), -1, np.int32)
    add = rng.integers(0, high, (B, L)).astype(np.int32)
    want, _, _, end = dr.assign_pages(np.zeros((B, L), np.int32), add, fresh, ps, 3, list(range(pool)), 0)
    t_fresh = torch.from_numpy(fresh).cuda()
    z, c = torch.zeros((B, L), dtype=torch.int32, device="cuda"), torch.full((1,), 3, dtype=torch.int64, device="cuda")
    fc.assign_pages(z, torch.from_numpy(add).cuda(), ps, t_fresh, c, num_free=pool)
    assert np.array_equal(t_fresh.cpu().numpy(), want) and int(c) == end and np.array_equal(z.cpu().numpy(), add)


def test_assigned_pages_serve_the_bf16_cache():
    """The tables are those that select_gather_paged and decode_attention_paged take."""
    fc = _fc()
    rng = np.random.default_rng(1)
    B, L, H, N, d, ps = 2, 3, 2, 200, 64, 16
    K, V = _rand(rng, (B, L, H, N, d), torch.bfloat16), _rand(rng, (B, L, H, N, d), torch.bfloat16)
    comp = fc.Compressor(K, 20, fc.total_budget(L, N, 0.3))
    comp.run(K, V)
    most = -(-N // ps)
    table = torch.full((B, L, H, most), -1, dtype=torch.int32, device="cuda")
    rows, cursor = torch.zeros((B, L), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    pool = B * L * H * most
    free = torch.randperm(pool, device="cuda").to(torch.int32)
    slots = torch.empty((B, comp.rows_per_seq), dtype=torch.int64, device="cuda")
    fc.assign_pages(rows, comp.budgets, ps, table, cursor, free, slots=slots)
    assert torch.equal(rows, comp.budgets)
    Kp, Vp = torch.zeros((pool, ps, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((pool, ps, d), dtype=torch.bfloat16, device="cuda")
    fc.select_gather_paged(K, V, comp.desc, comp.scores, comp.budgets, comp.layer_offsets, comp.rows_per_seq, comp.idx, table, ps, Kp, Vp)
    assert torch.equal(Kp.view(-1, d)[slots.view(-1)], comp.K_out.view(-1, d))
    Q = _rand(rng, (B, L, H * 2, d), torch.bfloat16)
    a = fc.decode_attention(Q, comp.K_out, comp.V_out, H, comp.budgets, comp.layer_offsets, comp.rows_per_seq, 0.125)
    b = fc.decode_attention_paged(Q, Kp, Vp, H, rows, table, 0.125)
    # the same rows, cut into pieces in another way: sums of at most 60 rows in fp32
    assert float((a - b).abs().max()) <= 256 * U * float(V.float().abs().max())


# ---- the 4-bit cache ------------------------------------------------------------------------------
def _hard_rows(rng, n, d):
    """Normal rows of many magnitudes; zeros, values half-way between two codes, extremes of fp32, denormals."""
    x = (rng.standard_normal((n, d)) * np.exp2(rng.integers(-30, 30, (n, 1)))).astype(np.float32)
    halves = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 6.5, 7.0, 6.9999995], np.float32)
    for i in range(0, n, 4):
        x[i] = rng.choice(halves, d) * rng.choice([-1, 1], d) * np.float32(2.0 ** rng.integers(-20, 20))
    x[1] = 0
    x[2] = np.where(rng.random(d) < 0.5, np.float32(3.4e38), np.float32(-1e-38))
    x[3] = (1e-41 * rng.standard_normal(d)).astype(np.float32)
    x[5, ::2] = -0.0
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("ps,B,R", [(16, 1, 1), (16, 2, 33), (48, 1, 150), (64, 3, 500)])
def test_mx_store_and_load(dtype, d, ps, B, R):
    fc = _fc()
    rng = np.random.default_rng(R + d)
    dt = _dt(dtype)
    n_pages = -(-B * R // ps) + 2
    K = torch.from_numpy(_hard_rows(rng, max(8, B * R), d)[:B * R].reshape(B, R, d)).to(dt).cuda()
    V = torch.from_numpy(_hard_rows(rng, max(8, B * R), d)[:B * R].reshape(B, R, d)).to(dt).cuda()
    slots = rng.permutation(n_pages * ps)[:B * R].reshape(B, R).astype(np.int64)
    if R > 8:
        slots[0, 3], slots[-1, 7], slots[0, 5] = -1, n_pages * ps, np.iinfo(np.int64).max
    pages = rng.integers(0, 256, (n_pages, fc.mx_page_bytes(ps, d)), dtype=np.uint8)
    t_pages, t_slots = torch.from_numpy(pages.copy()).cuda(), torch.from_numpy(slots).cuda()
    fc.mx_store(K, V, t_slots, t_pages, ps)
    k, v = K.float().cpu().numpy().reshape(-1, d), V.float().cpu().numpy().reshape(-1, d)
    want = dr.store(pages.reshape(-1).copy(), slots.reshape(-1), k, v)
    assert np.array_equal(t_pages.cpu().numpy().reshape(-1), want)     # what was not stored to is as it was
    Ko, Vo = torch.full_like(K, 7.0), torch.full_like(V, 7.0)
    fc.mx_load(t_slots, t_pages, ps, Ko, Vo)
    wk, wv = dr.load(want, slots.reshape(-1), d)
    # (a block of the row of extremes is NaN: 3.4e38 is infinite in bf16)
    assert np.array_equal(_f64(Ko).reshape(-1, d), wk, equal_nan=True) and np.array_equal(_f64(Vo).reshape(-1, d), wv, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,B,R", [(64, 1, 66005), (64, 3, 22011), (128, 1, 33003), (128, 2, 17001)])
def test_mx_store_and_load_of_many_rows_equal_those_of_few(dtype, d, B, R):
    """Large calls take several rows for each group of lanes, small ones (tested above against the oracle) one."""
    fc = _fc()
    g = torch.Generator(device="cuda").manual_seed(R)
    dt, ps = _dt(dtype), 48
    n_pages = -(-B * R // ps) + 1
    K, V = (torch.randn((B, R, d), generator=g, device="cuda").mul_(3.0).to(dt) for _ in range(2))
    slots = torch.randperm(n_pages * ps, generator=g, device="cuda")[:B * R].view(B, R).contiguous()
    slots[:, ::97] = -1
    slots[:, 5::1001] = n_pages * ps
    pages, want = (torch.full((n_pages, fc.mx_page_bytes(ps, d)), 5, dtype=torch.uint8, device="cuda") for _ in range(2))
    Ko, Vo, Kw, Vw = (torch.full((B, R + 1, d), 7.0, dtype=dt, device="cuda") for _ in range(4))     # a row behind the last one
    fc.mx_store(K, V, slots, pages, ps)
    fc.mx_load(slots, pages, ps, Ko[:, :R], Vo[:, :R])
    for b in range(B):
        for r in range(0, R, 3001):
            part = slots[b:b + 1, r:r + 3001].contiguous()
            rows = slice(r, r + part.shape[1])
            fc.mx_store(K[b:b + 1, rows], V[b:b + 1, rows], part, want, ps)
            fc.mx_load(part, want, ps, Kw[b:b + 1, rows], Vw[b:b + 1, rows])
    assert torch.equal(pages, want) and torch.equal(Ko, Kw) and torch.equal(Vo, Vw)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
def test_select_gather_mx_of_many_rows_equals_the_packed_rows_stored(dtype, d):
    fc = _fc()
    rng = np.random.default_rng(d + 5)
    B, L, H, N, ps = 1, 3, 3, 9000, 64
    dt = _dt(dtype)
    K, V = (torch.from_numpy(rng.standard_normal((B, L, H, N, d), dtype=np.float32)).to(dt).cuda() for _ in range(2))
    comp = fc.Compressor(K, 600, fc.total_budget(L, N, 0.83))
    comp.run(K, V)
    assert comp.rows_per_seq > 2048 * 2048 // d                      # (groups of 16 rows of 128 columns, 32 of 64)
    most = -(-N // ps)
    table = torch.full((B, L, H, most), -1, dtype=torch.int32, device="cuda")
    rows, cursor = torch.zeros((B, L), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    pool = B * L * H * most
    slots = torch.empty((B, comp.rows_per_seq), dtype=torch.int64, device="cuda")
    free = torch.from_numpy(rng.permutation(pool).astype(np.int32)).cuda()
    fc.assign_pages(rows, comp.budgets, ps, table, cursor, free_pages=free, slots=slots)
    pages, want = (torch.full((pool, fc.mx_page_bytes(ps, d)), 3, dtype=torch.uint8, device="cuda") for _ in range(2))
    idx = torch.full_like(comp.idx, -5)
    fc.select_gather_mx(K, V, comp.desc, comp.scores, comp.budgets, comp.layer_offsets, comp.rows_per_seq, idx, table, ps, pages)
    assert torch.equal(idx, comp.idx)
    for r in range(0, comp.rows_per_seq, 20011):
        fc.mx_store(comp.K_out[:, r:r + 20011], comp.V_out[:, r:r + 20011], slots[:, r:r + 20011].contiguous(), want, ps)
    assert torch.equal(pages, want)


def test_mx_blocks_with_values_that_are_not_finite():
    fc = _fc()
    x = torch.ones((1, 4, 128), device="cuda")
    x[0, 0, 5], x[0, 1, 40], x[0, 2, 127] = float("nan"), float("inf"), float("-inf")
    pages = torch.zeros((1, fc.mx_page_bytes(16, 128)), dtype=torch.uint8, device="cuda")
    slots = torch.arange(4, device="cuda").view(1, 4)
    for dt in (torch.float32, torch.bfloat16):
        K = x.to(dt)
        fc.mx_store(K, K, slots, pages, 16)
        k, v = torch.empty_like(K), torch.empty_like(K)
        fc.mx_load(slots, pages, 16, k, v)
        for y in (k, v):
            bad = y.isnan()[0]
            want = torch.zeros_like(bad)
            want[0, :32], want[1, 32:64], want[2, 96:] = True, True, True
            assert torch.equal(bad, want) and bool((y[0][~want] == 1).all())


def test_mx_store_takes_strided_rows_and_load_leaves_gaps():
    fc = _fc()
    rng = np.random.default_rng(9)
    B, R, d, ps = 2, 21, 128, 32
    big = _rand(rng, (2, B, R, 3, d), torch.bfloat16)
    K, V = big[0, :, :, 1], big[1, :, :, 1]
    slots = torch.from_numpy(rng.permutation(64)[:B * R].reshape(B, R)).cuda()
    pages, same = (torch.zeros((2, fc.mx_page_bytes(ps, d)), dtype=torch.uint8, device="cuda") for _ in range(2))
    fc.mx_store(K, V, slots, pages, ps)
    fc.mx_store(K.contiguous(), V.contiguous(), slots, same, ps)
    assert torch.equal(pages, same)
    out = torch.full((2, B, R, 3, d), 9.0, dtype=torch.float32, device="cuda")
    fc.mx_load(slots, pages, ps, out[0, :, :, 1], out[1, :, :, 1])
    assert np.array_equal(_f64(out[0, :, :, 1]), dr.grid(K.float().cpu().numpy()))
    assert bool((out[:, :, :, 0] == 9).all()) and bool((out[:, :, :, 2] == 9).all())


@pytest.mark.parametrize("dtype,d,shared", [("bf16", 128, False), ("bf16", 64, True), ("f32", 128, True), ("f32", 64, False)])
def test_select_gather_mx(dtype, d, shared):
    fc = _fc()
    rng = np.random.default_rng(d + shared)
    B, L, H, N, ps = 2, 3, 2, 700, 48
    dt = _dt(dtype)
    # heads that are not next to each other
    K, V = (_rand(rng, (B, L, H + 1, N, d), dt)[:, :, :H] for _ in range(2))
    comp = fc.Compressor(K, 60, fc.total_budget(L, N, 0.23), shared=shared)
    comp.run(K, V)
    most = -(-N // ps)
    table = torch.full((B, L, H, most), -1, dtype=torch.int32, device="cuda")
    rows, cursor = torch.zeros((B, L), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    pool = B * L * H * most
    slots = torch.empty((B, comp.rows_per_seq), dtype=torch.int64, device="cuda")
    fc.assign_pages(rows, comp.budgets, ps, table, cursor, num_free=pool, slots=slots)
    table[0, 1, 1, 2] = -1                                          # a page that is gone, one beyond the cache
    table[1, 2, 0, 0] = pool
    pages, want = (torch.full((pool, fc.mx_page_bytes(ps, d)), 3, dtype=torch.uint8, device="cuda") for _ in range(2))
    idx = torch.full_like(comp.idx, -5)
    fc.select_gather_mx(K, V, comp.desc, comp.scores, comp.budgets, comp.layer_offsets, comp.rows_per_seq, idx, table, ps, pages,
                        shared=shared)
    assert torch.equal(idx, comp.idx)
    # the same rows as the packed copy, stored by their slots
    b = comp.budgets.cpu().numpy()
    for (bb, l, h, p) in ((0, 1, 1, 2), (1, 2, 0, 0)):
        first = int(comp.layer_offsets[bb, l]) + h * int(b[bb, l])
        slots[bb, first + p * ps:first + min(int(b[bb, l]), (p + 1) * ps)] = -1
    fc.mx_store(comp.K_out, comp.V_out, slots, want, ps)
    assert torch.equal(pages, want)


def test_select_gather_mx_leaves_out_layers_of_bad_budgets():
    """A budget beyond the tokens selects and stores nothing, however large it is; the other layers are as they should be."""
    fc = _fc()
    rng = np.random.default_rng(77)
    B, L, H, N, d, ps = 1, 3, 2, 100, 64, 16
    K, V = _rand(rng, (B, L, H, N, d), torch.bfloat16), _rand(rng, (B, L, H, N, d), torch.bfloat16)
    scores = torch.rand((B, L, H, N), device="cuda")
    for wrong in (N + 1, 2 ** 31 - 1, -3):
        budgets = torch.tensor([[20, wrong, 30]], dtype=torch.int32, device="cuda")
        offs = torch.tensor([[0, 40, 60, 120]], dtype=torch.int64, device="cuda")
        table = torch.arange(L * H * 7, dtype=torch.int32, device="cuda").view(B, L, H, 7)
        pages = torch.full((L * H * 7, fc.mx_page_bytes(ps, d)), 3, dtype=torch.uint8, device="cuda")
        idx = torch.full((1, 120), 5, dtype=torch.int32, device="cuda")
        fc.select_gather_mx(K, V, fc.describe(K), scores, budgets, offs, 120, idx, table, ps, pages)
        assert bool((pages[14:28] == 3).all()) and bool((idx[0, 40:60] == 5).all())
        for l, k in ((0, 20), (2, 30)):
            for h in range(H):
                o = int(offs[0, l]) + h * k
                want = torch.topk(scores[0, l, h], k).indices.sort().values.to(torch.int32)
                assert torch.equal(idx[0, o:o + k], want)
                slots = (int(table[0, l, h, 0]) * ps + torch.arange(k, device="cuda")).view(1, k)
                Ko, Vo = torch.empty((1, k, d), device="cuda"), torch.empty((1, k, d), device="cuda")
                fc.mx_load(slots, pages, ps, Ko, Vo)
                assert np.array_equal(_f64(Ko)[0], dr.grid(K[0, l, h].float().cpu().numpy()[want.cpu().numpy()]))
                assert np.array_equal(_f64(Vo)[0], dr.grid(V[0, l, h].float().cpu().numpy()[want.cpu().numpy()]))


# ---- attention ------------------------------------------------------------------------------------
def _cache(fc, rng, B, L, H, d, ps, rows, pool=None, sigma=1.0, dtype=torch.float32):
    """A cache whose units hold rows[b][l] rows in pages in any order; (pages, table, K, V [unit] in float64)."""
    need = -(-rows // ps)
    most = max(1, int(need.max()))
    total = int(need.sum()) * H
    pool = total + 3 if pool is None else pool
    order = rng.permutation(pool)[:total]
    table = np.full((B, L, H, most), -1, np.int32)
    pages = torch.from_numpy(rng.integers(0, 256, (pool, fc.mx_page_bytes(ps, d)), dtype=np.uint8)).cuda()      # (NaN scales too)
    at, Ks, Vs, slots, kr, vr = 0, [], [], [], [], []
    for b in range(B):
        for l in range(L):
            for h in range(H):
                n = int(need[b, l])
                table[b, l, h, :n] = order[at:at + n]
                at += n
                r = np.arange(rows[b, l])
                slots.append(table[b, l, h, r // ps].astype(np.int64) * ps + r % ps)
                k = (sigma * rng.standard_normal((rows[b, l], d))).astype(np.float32)
                v = (rng.standard_normal((rows[b, l], d)) + 0.25).astype(np.float32)
                kr.append(k)
                vr.append(v)
                Ks.append(dr.grid(k))
                Vs.append(dr.grid(v))
    if sum(map(len, slots)):
        fc.mx_store(torch.from_numpy(np.concatenate(kr)[None]).cuda(), torch.from_numpy(np.concatenate(vr)[None]).cuda(),
                    torch.from_numpy(np.concatenate(slots)[None]).cuda(), pages, ps)
    return pages, table, Ks, Vs


def _check_attend(got, Q, Ks, Vs, B, L, H, G, scale, keep=None):
    got, q = _f64(got), _f64(Q)
    d = q.shape[-1]
    for u in range(B * L * H):
        b, l, h = u // (L * H), u // H % L, u % H
        K, V = Ks[u], Vs[u]
        if keep is not None:
            K, V = K[keep[u]], V[keep[u]]
        want, size, qk, top = dr.attend(q[b, l, h * G:(h + 1) * G], K, V, scale)
        slip = 2 * (3 * d * U * qk + 4 * U * (top + 1)) + (len(K) / 32 + 64) * U
        err = np.abs(got[b, l, h * G:(h + 1) * G] - want)
        assert np.all(err <= size * slip[:, None] + 1e-37), (u, np.max(err / np.maximum(size, 1e-30)), slip)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,L,H,G,d,ps,rows", [
    (1, 1, 1, 1, 64, 16, [1]), (1, 1, 1, 1, 128, 16, [16]), (1, 1, 2, 7, 128, 16, [17]), (1, 1, 1, 16, 64, 32, [31]), (1, 2, 2, 4, 128, 48, [33, 47]),
    (2, 3, 2, 3, 64, 64, [0, 5, 129, 1000, 0, 64]), (1, 1, 4, 7, 128, 64, [5000]), (1, 5, 1, 8, 128, 16, [1, 0, 0, 777, 15]),
    (3, 1, 1, 5, 64, 128, [200, 0, 4097]), (1, 70, 1, 2, 64, 16, list(range(70))),
])
def test_mx_decode_attention(dtype, B, L, H, G, d, ps, rows):
    fc = _fc()
    rng = np.random.default_rng(sum(rows) + G)
    rows = np.array(rows, np.int32).reshape(B, L)
    pages, table, Ks, Vs = _cache(fc, rng, B, L, H, d, ps, rows)
    Q = _rand(rng, (B, L, H * G, d), _dt(dtype))
    scale = 1.0 / math.sqrt(d)
    out = torch.full((B, L, H * G, d), float("nan"), device="cuda")
    got = fc.mx_decode_attention(Q, pages, ps, H, torch.from_numpy(rows).cuda(), torch.from_numpy(table).cuda(), scale, out=out)
    assert got is out
    _check_attend(got, Q, Ks, Vs, B, L, H, G, scale)
    again = fc.mx_decode_attention(Q, pages, ps, H, torch.from_numpy(rows).cuda(), torch.from_numpy(table).cuda(), scale)
    assert torch.equal(got, again)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", range(1, 17))
def test_mx_decode_attention_of_every_group(dtype, d, G):
    fc = _fc()
    rng = np.random.default_rng(100 * G + d)
    B, L, H, ps = 1, 2, 2, 16
    rows = np.array([[1500, 40 + G]], np.int32)
    pages, table, Ks, Vs = _cache(fc, rng, B, L, H, d, ps, rows)
    Q = _rand(rng, (B, L, H * G, d), _dt(dtype))
    guarded = torch.full((L * H * G + 1, d), 5.0, device="cuda")
    got = fc.mx_decode_attention(Q, pages, ps, H, torch.from_numpy(rows).cuda(), torch.from_numpy(table).cuda(), -0.2,
                                 out=guarded[:-1].view(B, L, H * G, d))
    _check_attend(got, Q, Ks, Vs, B, L, H, G, -0.2)
    assert bool((guarded[-1] == 5).all())


@pytest.mark.parametrize("d", [64, 128])
def test_mx_decode_attention_missing_pages_and_rows_beyond_the_table(d):
    fc = _fc()
    rng = np.random.default_rng(d)
    B, L, H, G, ps = 1, 4, 2, 7, 16
    rows = np.array([[90, 40, 33, 700]], np.int32)
    pages, table, Ks, Vs = _cache(fc, rng, B, L, H, d, ps, rows)
    keep = [np.ones(len(k), bool) for k in Ks]
    for u, p, bad in ((0, 1, -1), (1, 5, 10 ** 6), (2, 0, -2 ** 31), (2, 1, -1), (2, 2, -1), (7, 20, len(pages)), (7, 21, -5), (6, 43, -1)):
        table.reshape(B * L * H, -1)[u, p] = bad
        keep[u][p * ps:(p + 1) * ps] = False
    Q = _rand(rng, (B, L, H * G, d), torch.bfloat16)
    claimed = rows.copy()
    claimed[0, 3] = 2 ** 31 - 1                          # all that the table has room for: the last page is partly stale there
    short = table.shape[3] * ps
    got = fc.mx_decode_attention(Q, pages, ps, H, torch.from_numpy(rows).cuda(), torch.from_numpy(table).cuda(), 0.125)
    _check_attend(got, Q, Ks, Vs, B, L, H, G, 0.125, keep)
    assert bool((got[0, 1, :G] == 0).all())              # every page of the unit is gone
    # rows that exceed the table are cut to it, negative ones are none
    table[0, 3, :, -1] = -1
    for h in range(H):
        keep[6 + h][(table.shape[3] - 1) * ps:] = False
    claimed[0, 2] = -4
    got = fc.mx_decode_attention(Q, pages, ps, H, torch.from_numpy(claimed).cuda(), torch.from_numpy(table).cuda(), 0.125)
    keep[4][:] = keep[5][:] = False
    assert short == 44 * ps
    _check_attend(got, Q, Ks, Vs, B, L, H, G, 0.125, keep)


def test_mx_decode_attention_shared_pages_large_logits_and_nan():
    fc = _fc()
    rng = np.random.default_rng(21)
    B, L, H, G, d, ps = 2, 1, 1, 8, 128, 32
    rows = np.array([[640], [640]], np.int32)
    pages, table, Ks, Vs = _cache(fc, rng, B, L, H, d, ps, rows, sigma=20.0)      # one row takes nearly all
    table[1, 0, 0, :10] = table[0, 0, 0, :10]            # a prefix in common
    Ks[1][:320], Vs[1][:320] = Ks[0][:320], Vs[0][:320]
    Q = _rand(rng, (B, L, H * G, d), torch.float32, 4.0)
    r, t = torch.from_numpy(rows).cuda(), torch.from_numpy(table).cuda()
    for scale in (1.0 / math.sqrt(d), -0.3, 0.0):
        got = fc.mx_decode_attention(Q, pages, ps, H, r, t, scale)
        _check_attend(got, Q, Ks, Vs, B, L, H, G, scale)
    # a stored NaN reaches every head that attends to it, and no other sequence
    x = torch.full((1, 1, d), float("nan"), device="cuda")
    slot = torch.tensor([[int(table[1, 0, 0, 15]) * ps + 3]], device="cuda")
    fc.mx_store(x, x, slot, pages, ps)
    got = fc.mx_decode_attention(Q, pages, ps, H, r, t, 0.1)
    assert bool(got[1].isnan().all()) and not bool(got[0].isnan().any())


def test_mx_decode_attention_many_units_and_long_caches():
    fc = _fc()
    rng = np.random.default_rng(2)
    # (units beyond the workgroups; a single unit of many; more layers than a wave's registers hold, one far longer than the others;
    # tables that reach 1024 rows and a page more)
    long = rng.integers(0, 40, 700)
    long[613] = 9000
    for B, L, H, G, d, ps, rows in ((4, 200, 2, 2, 64, 16, rng.integers(0, 60, 800)), (1, 1, 1, 7, 128, 64, np.array([70001])),
                                    (1, 700, 1, 1, 64, 16, long), (1, 3, 2, 4, 128, 16, np.array([1024, 1000, 0])),
                                    (1, 3, 2, 4, 128, 16, np.array([1025, 7, 0]))):
        rows = rows.astype(np.int32).reshape(B, L)
        pages, table, Ks, Vs = _cache(fc, rng, B, L, H, d, ps, rows)
        Q = _rand(rng, (B, L, H * G, d), torch.bfloat16)
        got = fc.mx_decode_attention(Q, pages, ps, H, torch.from_numpy(rows).cuda(), torch.from_numpy(table).cuda(), 0.1)
        _check_attend(got, Q, Ks, Vs, B, L, H, G, 0.1)


def test_mx_cache_beyond_four_gigabytes():
    """Slots whose bytes lie past 2^32."""
    fc = _fc()
    ps, d, n_pages = 4096, 128, 8192                     # 4.56 GB
    pages = torch.empty((n_pages, fc.mx_page_bytes(ps, d)), dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(8)
    K, V = _rand(rng, (1, 300, d), torch.bfloat16), _rand(rng, (1, 300, d), torch.bfloat16)
    slots = (n_pages - 1) * ps + 3900 + torch.arange(300, device="cuda").view(1, 300)      # (the last 104 are behind the cache's end)
    fc.mx_store(K, V, slots, pages, ps)
    k, v = torch.empty_like(K), torch.empty_like(V)
    fc.mx_load(slots, pages, ps, k, v)
    for x, y in ((K, k), (V, v)):
        assert np.array_equal(_f64(y)[0, :196], dr.grid(x.float().cpu().numpy())[0, :196]) and not bool(y[0, 196:].any())
    fc.mx_store(K[:, :200], V[:, :200], slots[:, :200] - 3900, pages, ps)
    table = torch.full((1, 1, 1, 1), n_pages - 1, dtype=torch.int32, device="cuda")
    Q = _rand(rng, (1, 1, 4, d), torch.bfloat16)
    got = fc.mx_decode_attention(Q, pages, ps, 1, torch.full((1, 1), 200, dtype=torch.int32, device="cuda"), table, 0.1)
    _check_attend(got, Q, [dr.grid(K[0, :200].float().cpu().numpy())], [dr.grid(V[0, :200].float().cpu().numpy())], 1, 1, 1, 4, 0.1)


# ---- together -------------------------------------------------------------------------------------
def _compressed(fc, rng, B, L, H, N, d):
    K, V = _rand(rng, (B, L, H, N, d), torch.bfloat16), _rand(rng, (B, L, H, N, d), torch.bfloat16)
    comp = fc.Compressor(K, 40, fc.total_budget(L, N, 0.25))
    comp.run_score(K, V)
    comp.run_allocate()
    return comp, K, V


def _history(comp, K, V, B, L, H, d):
    """Rows of each unit that the compression kept, as the 4-bit cache holds them."""
    budgets, offs, idx = comp.budgets.cpu().numpy(), comp.layer_offsets.cpu().numpy(), comp.idx.cpu().numpy()
    Ks, Vs = [], []
    for b in range(B):
        for l in range(L):
            for h in range(H):
                k = int(budgets[b, l])
                o = int(offs[b, l]) + h * k
                rows = idx[b, o:o + k]
                Ks.append(dr.grid(K[b, l, h].float().cpu().numpy()[rows]))
                Vs.append(dr.grid(V[b, l, h].float().cpu().numpy()[rows]))
    return Ks, Vs


@pytest.mark.parametrize("captured", [False, True])
def test_decode_loop_over_a_compacted_cache(captured):
    """Compress, fill, then steps of rotary, append and attend; a captured step is replayed with eager work between the replays."""
    fc = _fc()
    rng = np.random.default_rng(31)
    B, L, H, G, N, d, ps = 2, 3, 2, 4, 500, 64, 16
    comp, K, V = _compressed(fc, rng, B, L, H, N, d)
    pool = B * L * H * (-(-N // ps))
    cache = fc.MxCache(B, L, H, d, ps, -(-N // ps), pool)
    cache.fill(comp, K, V)
    Ks, Vs = _history(comp, K, V, B, L, H, d)
    plan = fc.rotary_plan(d, theta=1e6)
    # every layer's heads of a token side by side: [B, 1, L * heads, d]
    q, k, v = (torch.zeros((B, 1, L * n, d), dtype=torch.bfloat16, device="cuda") for n in (H * G, H, H))
    pos = torch.zeros((B, 1), dtype=torch.int32, device="cuda")
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    out = torch.empty((B, L, H * G, d), dtype=torch.float32, device="cuda")

    def step():
        fc.rotary(plan, pos, q, k, Q_out=q_out, K_out=k_out)
        cache.append(k_out.view(B, L, H, d), v.view(B, L, H, d))
        cache.attend(q_out.view(B, L, H * G, d), 0.125, out=out)
    graph = None
    held = cache.rows.clone(), cache.cursor.clone(), cache.block_table.clone(), cache.pages.clone()
    if captured:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()                                       # (buffers)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for t, s in zip((cache.rows, cache.cursor, cache.block_table, cache.pages), held):
            t.copy_(s)
    for turn in range(20):                               # over a page's end
        q.copy_(_rand(rng, q.shape, torch.bfloat16))
        k.copy_(_rand(rng, k.shape, torch.bfloat16))
        v.copy_(_rand(rng, v.shape, torch.bfloat16))
        pos.fill_(N + turn)
        if captured:
            graph.replay()
            torch.cuda.synchronize()
            float(torch.randn(1000, device="cuda").sum())            # the program's own work
        else:
            step()
        kn, vn = k_out.view(B * L * H, 1, d).float().cpu().numpy(), v.view(B * L * H, 1, d).float().cpu().numpy()
        Ks = [np.concatenate((a, dr.grid(b))) for a, b in zip(Ks, kn)]
        Vs = [np.concatenate((a, dr.grid(b))) for a, b in zip(Vs, vn)]
        if turn in (0, 1, 7, 19):
            _check_attend(out, q_out.view(B, L, H * G, d), Ks, Vs, B, L, H, G, 0.125)
    assert torch.equal(cache.rows, comp.budgets + 20) and cache.missing() == 0


def test_cache_without_pages_left_keeps_what_it_has():
    fc = _fc()
    rng = np.random.default_rng(32)
    B, L, H, G, d, ps = 1, 2, 1, 2, 128, 16
    cache = fc.MxCache(B, L, H, d, ps, 4, 3)             # three pages for two units
    Ks, Vs = [np.zeros((0, d))] * 2, [np.zeros((0, d))] * 2
    keep = [np.zeros(0, bool)] * 2
    for turn in range(40):
        k, v = _rand(rng, (B, L, H, d), torch.bfloat16), _rand(rng, (B, L, H, d), torch.bfloat16)
        cache.append(k, v)
        for u in range(2):
            Ks[u] = np.concatenate((Ks[u], dr.grid(k[0, u].float().cpu().numpy())))
            Vs[u] = np.concatenate((Vs[u], dr.grid(v[0, u].float().cpu().numpy())))
            # pages 0 and 1, then 2 for the first unit; the others are not there
            keep[u] = np.append(keep[u], turn < 16 or (turn < 32 and u == 0))
    Q = _rand(rng, (B, L, H * G, d), torch.bfloat16)
    _check_attend(cache.attend(Q, 0.1), Q, Ks, Vs, B, L, H, G, 0.1, keep)
    assert cache.missing() == 3


def test_cache_is_filled_again_after_a_reset_and_takes_any_group():
    fc = _fc()
    rng = np.random.default_rng(34)
    B, L, H, N, d, ps = 1, 2, 2, 300, 128, 16
    cache = fc.MxCache(B, L, H, d, ps, -(-N // ps), B * L * H * (-(-N // ps)))
    for turn in range(2):
        comp, K, V = _compressed(fc, rng, B, L, H, N, d)
        cache.fill(comp, K, V)
        Ks, Vs = _history(comp, K, V, B, L, H, d)
        for G in (1, 16, 5):
            Q = _rand(rng, (B, L, H * G, d), torch.bfloat16)
            _check_attend(cache.attend(Q, 0.1), Q, Ks, Vs, B, L, H, G, 0.1)
        with pytest.raises(ValueError):
            cache.fill(comp, K, V)
        cache.reset()
    other, K, V = _compressed(fc, rng, B, L, H, N, 64)
    with pytest.raises(ValueError):
        cache.fill(other, K, V)
    with pytest.raises(ValueError):
        cache.attend(_rand(rng, (B, L, H, 64), torch.bfloat16), 0.1)
    with pytest.raises(ValueError):
        cache.append(_rand(rng, (B, L, H + 1, d), torch.bfloat16), _rand(rng, (B, L, H + 1, d), torch.bfloat16))


def test_refused_rows_are_not_counted():
    """What fill and append refuse leaves the cache as it was."""
    fc = _fc()
    rng = np.random.default_rng(36)
    B, L, H, N, d, ps = 1, 2, 2, 200, 64, 16
    comp, K, V = _compressed(fc, rng, B, L, H, N, d)
    cache = fc.MxCache(B, L, H, d, ps, -(-N // ps) + 1, 64)
    held = cache.rows.clone(), cache.cursor.clone(), cache.block_table.clone()
    odd = torch.zeros(B * L * H * d + 4, dtype=torch.bfloat16, device="cuda")[4:].view(B, L, H, d)     # off by 8 bytes
    k = odd.clone()
    with pytest.raises(ValueError):
        cache.fill(comp, K[:, :, :, :N - 8], V[:, :, :, :N - 8])             # fewer tokens than the descriptor has
    with pytest.raises(ValueError):
        cache.fill(comp, K, V.transpose(1, 2).contiguous().transpose(1, 2))  # other strides
    with pytest.raises(ValueError):
        cache.fill(comp, K.float(), V.float())
    for bad in ((k.half(), k.half()), (odd, k), (k, odd), (k, k.float()), (k.cpu(), k.cpu())):
        with pytest.raises(ValueError):
            cache.append(*bad)
    for t, s in zip((cache.rows, cache.cursor, cache.block_table), held):
        assert torch.equal(t, s)
    cache.fill(comp, K, V)
    cache.append(k, k)
    assert torch.equal(cache.rows, comp.budgets + 1)


def test_strides_of_axes_of_one_do_not_matter():
    fc = _fc()
    rng = np.random.default_rng(35)
    d, ps = 64, 16
    wide = _rand(rng, (3, 7, 5 * d + 1), torch.bfloat16)
    K, V = wide[:1, 2:3, :d], _rand(rng, (1, 1, d), torch.bfloat16)          # (strides of 321 and 2247 elements)
    slots = torch.tensor([[9]], device="cuda")
    pages = torch.zeros((1, fc.mx_page_bytes(ps, d)), dtype=torch.uint8, device="cuda")
    if K.data_ptr() % 16:
        K = K.clone().as_strided((1, 1, d), (2247, 321, 1))
    fc.mx_store(K, V, slots, pages, ps)
    Ko, Vo = torch.empty((1, 1, d), device="cuda"), torch.empty((1, 1, d), device="cuda").as_strided((1, 1, d), (77, 33, 1))
    fc.mx_load(slots, pages, ps, Ko, Vo)
    assert np.array_equal(_f64(Ko), dr.grid(K.float().cpu().numpy())) and np.array_equal(_f64(Vo), dr.grid(V.float().cpu().numpy()))


def test_operators_on_two_streams_at_once():
    """Work of two streams with workspaces of their own, as two sequences' programs would enqueue it."""
    fc = _fc()
    rng = np.random.default_rng(33)
    B, L, H, G, d, ps = 1, 2, 2, 7, 128, 64
    sets = []
    for n in (3000, 900):
        rows = np.array([[n, n // 2]], np.int32)
        pages, table, Ks, Vs = _cache(fc, rng, B, L, H, d, ps, rows)
        Q = _rand(rng, (B, L, H * G, d), torch.bfloat16)
        sets.append((Q, pages, torch.from_numpy(rows).cuda(), torch.from_numpy(table).cuda(), Ks, Vs, torch.cuda.Stream(), []))
    torch.cuda.synchronize()
    for _ in range(8):
        for Q, pages, rows, table, _, _, stream, outs in sets:
            with torch.cuda.stream(stream):
                outs.append(fc.mx_decode_attention(Q, pages, ps, H, rows, table, 0.1))
    torch.cuda.synchronize()
    for Q, _, _, _, Ks, Vs, _, outs in sets:
        _check_attend(outs[0], Q, Ks, Vs, B, L, H, G, 0.1)
        assert all(torch.equal(outs[0], o) for o in outs[1:])
