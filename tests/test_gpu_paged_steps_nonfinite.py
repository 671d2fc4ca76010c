"""Decode steps over the paged cache on the GPU where inputs are not finite, against float64 (oracle/paged_steps_ref.py): a NaN in a query or in an
attended key makes all of that query's result NaN, one in an attended value its column, and neither anything else.

What is finite has the tolerance of attention: a logit is off by at most d u sum |q k| scale, its scaling and exponential by 4 u (|logit| + 1), twice; the
sums over n rows by n / 16 + 64 roundings, u = 2^-24, all of it relative to sum p |v|.
"""
import math

import numpy as np
import pytest

from oracle import paged_steps_ref as pr
from test_gpu_paged_steps import U, Cache, _dt, _f64, _fc, _int, _rand

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _plant(c, which, b, l, h, row, col, value=math.nan):
    """`value` into K or V of one row of a unit."""
    pages = c.K if which == "K" else c.V
    pages[int(c.table_np[b, l, h, row // c.ps]), row % c.ps, col] = value
    c.K64, c.V64 = _f64(c.K), _f64(c.V)


def _check(got, Q, scale, G, rows_for):
    """Returns how many heads of the result are NaN as a whole, and how many in part."""
    got, Q = _f64(got), _f64(Q)
    B, L, Hq, d = Q.shape
    whole = part = 0
    for b in range(B):
        for l in range(L):
            for g in range(Hq):
                K, V = rows_for(b, l, g // G)
                want, size, logit, terms = pr.attend(Q[b, l, g:g + 1], K, V, scale)
                bad = np.isnan(want[0])
                assert np.array_equal(np.isnan(got[b, l, g]), bad), (b, l, g, int(bad.sum()), int(np.isnan(got[b, l, g]).sum()))
                whole += bad.all()
                part += bad.any() and not bad.all()
                if not bad.all():
                    slip = 2 * (d * U * terms + 4 * U * (logit + 1)) + (K.shape[0] / 16 + 64) * U
                    assert np.max((np.abs(got[b, l, g] - want[0]) - slip * size[0])[~bad]) <= 0, (b, l, g)
    return whole, part


# (one workgroup a unit; several; pages of which a NaN row is alone in its step; a unit of a single row)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,H,G,d,ps", [([[40, 5]], 2, 3, 64, 16), ([[2000, 1]], 1, 7, 128, 16), ([[1], [513]], 2, 16, 64, 32), ([[33, 400]], 1, 1, 128, 1)])
def test_nan_in_attention_over_chosen_pages(dtype, rows, H, G, d, ps):
    fc = _fc()
    B, L = np.array(rows).shape
    scale = 1.0 / math.sqrt(d)
    for what in ("query", "first key", "last key", "value"):
        rng = np.random.default_rng(d + ps)
        c = Cache(rng, rows, H, d, ps, dtype)
        Q = _rand(rng, (B, L, G * H, d), _dt(dtype))
        if what == "query":
            Q[0, 0, G - 1, 5] = math.nan
        for b in range(B):
            for l in range(L):
                n = rows[b][l]
                if what == "first key":
                    _plant(c, "K", b, l, H - 1, 0, 7)
                elif what == "last key":
                    _plant(c, "K", b, l, H - 1, n - 1, d - 1)
                elif what == "value":
                    _plant(c, "V", b, l, 0, n // 2, 3)
        chosen = np.broadcast_to(np.arange(c.most), (B, L, H, c.most))
        got = fc.decode_attention_chosen(Q, c.kv, _int(chosen), scale)
        found = _check(got, Q, scale, G, c.unit)
        assert found == {"query": (1, 0), "value": (0, B * L * G)}.get(what, (B * L * G, 0)), what


# (up to 16 queries a prompt, up to 64, more, two tiles of them; own rows alone, in one part and in many)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("common,own,G,H,d", [
    (300, [1, 40], 7, 1, 128), (1, [1, 1], 2, 2, 64), (200, [1] * 9, 4, 1, 64), (129, [3] * 19, 7, 1, 128), (2000, [700, 1], 3, 2, 64), (0, [1, 700], 2, 2, 64),
])
def test_nan_in_attention_to_a_shared_prompt(dtype, common, own, G, H, d):
    fc = _fc()
    B, ps, scale = len(own), 16, 1.0 / math.sqrt(d)
    for what in ("query", "first own key", "last own key", "prompt's key", "prompt's keys", "own value", "prompt's value"):
        if common == 0 and what.startswith("prompt"):
            continue
        rng = np.random.default_rng(d + B)
        cc, co = Cache(rng, [[common]], H, d, ps, dtype), Cache(rng, [[n] for n in own], H, d, ps, dtype)
        Q = _rand(rng, (B, 1, G * H, d), _dt(dtype))
        if what == "query":
            Q[1, 0, 1, 0] = math.nan
        elif what == "first own key":
            _plant(co, "K", 0, 0, 0, 0, 1)
        elif what == "last own key":
            _plant(co, "K", B - 1, 0, 0, own[-1] - 1, 1)
        elif what == "prompt's key":
            _plant(cc, "K", 0, 0, H - 1, common // 2, 2)
        elif what == "prompt's keys":
            for row in range(common):
                _plant(cc, "K", 0, 0, H - 1, row, 2)
        elif what == "own value":
            _plant(co, "V", 0, 0, 0, 0, 1)
        else:
            _plant(cc, "V", 0, 0, 0, common - 1, 1)
        ws = fc.shared_workspace(Q, H, 1).fill_(255)
        got = fc.decode_attention_shared(Q, cc.kv, _int([0, B]), co.kv, scale, workspace=ws)
        found = _check(got, Q, scale, G, lambda b, l, h: tuple(np.concatenate(x) for x in zip(cc.unit(0, 0, h), co.unit(b, 0, h))))
        assert found == {"query": (1, 0), "first own key": (G, 0), "last own key": (G, 0), "own value": (0, G),
                         "prompt's value": (0, B * G)}.get(what, (B * G, 0)), what


def test_a_nan_behind_a_units_rows_changes_nothing():
    """Pages that a unit's rows or list do not reach, and a prompt that is another's."""
    fc = _fc()
    rng = np.random.default_rng(3)
    G, d, ps = 3, 64, 16
    cc, co = Cache(rng, [[90], [50]], 1, d, ps, "bf16"), Cache(rng, [[20]] * 4, 1, d, ps, "bf16")
    for row in range(50):
        _plant(cc, "K", 1, 0, 0, row, 0)
    Q = _rand(rng, (4, 1, G, d), torch.bfloat16)
    got = fc.decode_attention_shared(Q, cc.kv, _int([0, 2, 3]), co.kv, 0.125)

    def rows_for(b, l, h):
        return tuple(np.concatenate(x) for x in zip(cc.unit(0 if b < 2 else 1, 0, 0), co.unit(b, 0, 0))) if b < 3 else co.unit(b, 0, 0)
    assert _check(got, Q, 0.125, G, rows_for) == (G, 0)
    _plant(co, "K", 0, 0, 0, 3, 0)
    chosen = _int([[[[1, -1]]], [[[0, 1]]], [[[1, 0]]], [[[-1, -1]]]])
    got = fc.decode_attention_chosen(Q, co.kv, chosen, 0.125)
    assert _check(got, Q, 0.125, G, lambda b, l, h: co.unit(b, 0, 0, ([1], [0, 1], [1, 0], [])[b])) == (0, 0)
    assert bool((got[3] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("common,own,G,H,d", [(90, [1, 40], 7, 1, 128), (200, [5] * 9, 4, 1, 64), (129, [3] * 19, 7, 1, 128), (0, [300, 20], 2, 2, 64)])
def test_infinite_keys_and_values(dtype, common, own, G, H, d):
    """Keys whose scores are -infinity have no weight; where there are no others the result is zeros.  An infinite value shows in its column alone."""
    fc = _fc()
    rng = np.random.default_rng(d + len(own))
    B, ps, scale = len(own), 16, 1.0 / math.sqrt(d)
    cc, co = Cache(rng, [[common]], H, d, ps, dtype), Cache(rng, [[n] for n in own], H, d, ps, dtype)
    Q = _rand(rng, (B, 1, G * H, d), _dt(dtype))
    Q[..., 4] = Q[..., 4].abs() + 1
    for row in range(0, common, 3):
        _plant(cc, "K", 0, 0, H - 1, row, 4, -math.inf)
    for b in range(B):
        for row in range(1, own[b], 2):
            _plant(co, "K", b, 0, 0, row, 4, -math.inf)

    def rows_for(b, l, h):
        K, V = (np.concatenate(x) for x in zip(cc.unit(0, 0, h), co.unit(b, 0, h)))
        there = np.isfinite(K).all(1)
        return K[there], V[there]

    def shared():
        return fc.decode_attention_shared(Q, cc.kv, _int([0, B]), co.kv, scale)
    assert _check(shared(), Q, scale, G, rows_for) == (0, 0)
    every = _int(np.broadcast_to(np.arange(co.most), (B, 1, H, co.most)))

    def own_rows(b, l, h):
        K, V = co.unit(b, 0, h)
        there = np.isfinite(K).all(1)
        return K[there], V[there]
    assert _check(fc.decode_attention_chosen(Q, co.kv, every, scale), Q, scale, G, own_rows) == (0, 0)
    # a value of infinity, of the first sequence's first row of head 0
    _plant(co, "V", 0, 0, 0, 0, 6, math.inf)
    for got, clean in ((shared(), rows_for), (fc.decode_attention_chosen(Q, co.kv, every, scale), own_rows)):
        assert not bool(torch.isfinite(got[0, 0, :G, 6]).any())
        got[0, 0, :G, 6] = 0
        co.V64 = np.where(np.isinf(co.V64), 0.0, co.V64)
        for b in range(B):
            for g in range(G * H):
                K, V = clean(b, 0, g // G)
                if b == 0 and g < G:
                    V = V.copy()
                    V[:, 6] = 0
                want, size, logit, terms = pr.attend(_f64(Q)[b, 0, g:g + 1], K, V, scale)
                slip = 2 * (d * U * terms + 4 * U * (logit + 1)) + (K.shape[0] / 16 + 64) * U
                assert np.max(np.abs(_f64(got)[b, 0, g] - want[0]) - slip * size[0]) <= 0, (b, g)
    # no other scores
    co.K[..., 4] = torch.where(torch.isnan(co.K[..., 4]), co.K[..., 4], -math.inf)
    cc.K[..., 4] = torch.where(torch.isnan(cc.K[..., 4]), cc.K[..., 4], -math.inf)
    co.V.copy_(torch.where(torch.isinf(co.V), torch.zeros_like(co.V), co.V))
    assert bool((shared() == 0).all()) and bool((fc.decode_attention_chosen(Q, co.kv, every, scale) == 0).all())


# ---- choice ---------------------------------------------------------------------------------------
# (one workgroup for scores and choice of a unit; scores shared out; columns of both widths, lane groups of 8, 16 and 32 lanes)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,H,G,d", [([[4 * 90, 4 * 61]], 2, 3, 64), ([[4 * 300]], 2, 7, 128), ([[4 * 700]], 1, 1, 64)])
def test_choice_where_bounds_are_infinite(dtype, rows, H, G, d):
    """Pages with keys of either infinity, and with columns of NaNs alone, whose bounds are +infinity and -infinity: the score is what the keys' largest
    products make it, however many queries have one sign."""
    fc = _fc()
    rng = np.random.default_rng(d + G)
    c = Cache(rng, rows, H, d, 4, dtype)
    B, L = np.array(rows).shape
    Q = _rand(rng, (B, L, G * H, d), _dt(dtype)).abs()              # every column's queries of one sign ...
    Q[..., 1::4] *= -1
    Q[..., 2::4] *= torch.from_numpy(rng.choice([-1.0, 1.0], Q[..., 2::4].shape)).to(Q)      # ... or of both
    Q[..., 3] = 0
    for l in range(L):
        for h in range(H):
            at = rng.permutation(rows[0][l])[:40]
            for i, row in enumerate(at):
                _plant(c, "K", 0, l, h, row, i % 4 if i < 20 else rng.integers(d), (math.inf, -math.inf)[i // 4 % 2])
            for row in range(8, 12):
                _plant(c, "K", 0, l, h, row, 5)                     # place 2
            for row in range(20, 24):
                _plant(c, "K", 0, l, h, row, 3)                     # place 5: where the queries are 0
    bounds = fc.page_bounds(c.kv)
    found = _f64(bounds)
    assert np.isposinf(found[:, 0]).any() and np.isposinf(found[:, 1]).any() and np.isneginf(found[:, 0]).any() and np.isneginf(found[:, 1]).any()
    scores = [pr.page_score(_f64(Q)[0, 0, :G], *found[p]) for p in c.table_np[0, 0, 0][:rows[0][0] // 4]]
    assert sum(map(math.isinf, scores)) > 5 and sum(map(math.isfinite, scores)) > 20
    for count, first, last in ((1, 0, 0), (12, 0, 0), (33, 1, 2)):
        got = fc.choose_pages(Q, c.kv, bounds, count, first=first, last=last)
        assert np.array_equal(got.cpu().numpy(), pr.choose_pages(_f64(Q), found, c.rows_np, c.table_np, 4, count, first, last)), count


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_choice_where_queries_are_infinite_or_nan(dtype):
    fc = _fc()
    rng = np.random.default_rng(7)
    H, G, d = 3, 2, 64
    c = Cache(rng, [[4 * 200]], H, d, 4, dtype)
    bounds = fc.page_bounds(c.kv)
    bounds[c.table[0, 0, :, 30].long(), 1, 9] = 0
    Q = _rand(rng, (1, 1, G * H, d), _dt(dtype))
    # a query of +infinity: pages that it can score +infinity in, then those of other scores, then -infinity
    Q[0, 0, 0, 9], Q[0, 0, 2, 9], Q[0, 0, 4, 9] = math.inf, -math.inf, math.nan
    found = _f64(bounds)
    kinds = {(h, "nan" if math.isnan(s) else "inf" if s == math.inf else "-inf" if s == -math.inf else "")
             for h in range(H) for s in (pr.page_score(_f64(Q)[0, 0, h * G:(h + 1) * G], *found[p]) for p in c.table_np[0, 0, h])}
    assert kinds >= {(0, "inf"), (0, "-inf"), (1, "inf"), (1, "-inf"), (2, "nan")}, kinds
    for count in (1, 50, 150, 199):
        got = fc.choose_pages(Q, c.kv, bounds, count, first=0, last=1)
        assert np.array_equal(got.cpu().numpy(), pr.choose_pages(_f64(Q), found, c.rows_np, c.table_np, 4, count, 0, 1)), count


def test_choice_between_queries_of_very_different_sizes():
    """A column's queries of either sign, 2^60 apart: the small one's product counts where the large one's is 0."""
    fc = _fc()
    rng = np.random.default_rng(9)
    c = Cache(rng, [[4 * 60]], 1, 64, 4, "f32")
    bounds = fc.page_bounds(c.kv)
    bounds[:, 1] = 0                                                # max(2^60 low, 0) = 0, max(-q low, 0) = -q low
    bounds[:, 0] = -bounds[:, 0].abs() - 1
    Q = torch.zeros((1, 1, 2, 64), device="cuda")
    Q[0, 0, 0], Q[0, 0, 1] = 2.0 ** 60, -0.75
    got = fc.choose_pages(Q, c.kv, bounds, 7, first=0, last=0)
    assert np.array_equal(got.cpu().numpy(), pr.choose_pages(_f64(Q), _f64(bounds), c.rows_np, c.table_np, 4, 7, 0, 0))
