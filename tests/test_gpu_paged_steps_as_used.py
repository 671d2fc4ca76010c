"""Decode steps over the paged cache on the GPU in the calls that programs make of them together, against float64 (oracle/paged_steps_ref.py); tolerances as
in test_gpu_paged_steps.py: a logit is off by at most d u sum |q k| scale, its scaling and exponential by 4 u (|logit| + 1), twice; sums over n rows by
n / 16 + 64 roundings, u = 2^-24, all of it relative to sum p |v|."""
import math

import numpy as np
import pytest

from oracle import paged_steps_ref as pr
from test_gpu_paged_steps import Cache, _check_attention, _dt, _f64, _fc, _int, _rand, _Rows

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_steps_that_rank_pages_by_bounds_kept_as_rows_came(dtype):
    """A prompt of many tokens and then single ones appended with bounds, layer by layer; each step reads some of the pages that there are, then all."""
    fc = _fc()
    rng = np.random.default_rng(23)
    B, L, H, G, d, ps, T, steps, most = 2, 2, 2, 3, 64, 16, 333, 21, 30
    dt, scale = _dt(dtype), 0.125
    pool = B * L * H * most + 1
    K, V = (torch.full((pool, ps, d), math.nan, dtype=dt, device="cuda") for _ in "KV")
    bounds = torch.full((pool, 2, d), math.nan, dtype=dt, device="cuda")
    table = torch.from_numpy(rng.permutation(pool)[:B * L * H * most].reshape(B, L, H, most).astype(np.int32)).cuda()
    rows = torch.zeros((B, L), dtype=torch.int32, device="cuda")
    plan = fc.rotary_plan(d, theta=1e6)
    held = 0
    for tokens in [T] + [1] * steps:
        at = torch.arange(held, held + tokens, device="cuda")
        pos = at.to(torch.int32).expand(B, tokens).contiguous()
        held += tokens
        rows.fill_(held)
        for l in range(L):
            x = _rand(rng, (B, tokens, (G + 2) * H, d), dt)
            x[:, :, G * H:(G + 1) * H] += _rand(rng, (d,), dt) * (pos[..., None, None] // 40 % 3)     # keys that differ from page to page
            slots = table[:, l].long()[:, :, at // ps] * ps + at % ps
            q = fc.append_paged(plan, pos, x[:, :, :G * H], x[:, :, G * H:(G + 1) * H], x[:, :, (G + 1) * H:], slots, K, V, bounds=bounds)
            if held % 5 and held != T + steps:
                continue
            Q = q[:, -1:].contiguous()
            kv = fc.PagedKV(K, V, rows[:, l:l + 1], table[:, l:l + 1])
            K64, V64, table_np = _f64(K), _f64(V), table[:, l:l + 1].cpu().numpy()
            fresh = pr.page_bounds(K64, np.full((B, 1), held), table_np, ps, _f64(bounds))
            assert np.array_equal(fresh, _f64(bounds), equal_nan=True)
            for count, first, last in ((5, 1, 2), (11, 0, 0), (most, 1, 1)):
                chosen = fc.choose_pages(Q, kv, bounds, count, first=first, last=last)
                want = pr.choose_pages(_f64(Q), fresh, np.full((B, 1), held), table_np, ps, count, first, last)
                assert np.array_equal(chosen.cpu().numpy(), want)
                assert count == most or (want[..., :count - last] != np.arange(count - last)).any()      # (not the first ones)
                got = fc.decode_attention_chosen(Q, kv, chosen, scale)
                _check_attention(got, Q, scale, _Rows(G, lambda b, _, h: pr.rows_at(K64, V64, held, table_np[b, 0, h], ps, want[b, 0, h])), dtype)


@pytest.mark.parametrize("dtype,d,B,G", [("bf16", 128, 9, 4), ("bf16", 64, 20, 4), ("f32", 128, 40, 4), ("f32", 64, 5, 7)])
def test_many_queries_of_a_prompt_beyond_32_bits(dtype, d, B, G):
    """A cache of more than 2^32 bytes of keys and as many of values, a prompt at its far end that up to 128 queries read together."""
    fc = _fc()
    rng = np.random.default_rng(d + B)
    dt, ps, H, n = _dt(dtype), 128, 2, 900
    pages = (1 << 32) // (ps * d * (2 if dtype == "bf16" else 4)) + 50
    K, V = (torch.empty((pages, ps, d), dtype=dt, device="cuda") for _ in "KV")
    most = -(-n // ps)
    table = (pages - 1 - rng.permutation(H * most)).reshape(1, 1, H, most)
    at = [torch.from_numpy(table[0, 0, h][np.arange(n) // ps] * ps + np.arange(n) % ps).cuda() for h in range(H)]
    for h in range(H):
        K.view(-1, d)[at[h]], V.view(-1, d)[at[h]] = _rand(rng, (n, d), dt), _rand(rng, (n, d), dt)
    near = [(_f64(K.view(-1, d)[at[h]]), _f64(V.view(-1, d)[at[h]])) for h in range(H)]
    Q = _rand(rng, (B, 1, G * H, d), dt)
    own = fc.PagedKV(K, V, torch.zeros((B, 1), dtype=torch.int32, device="cuda"), torch.full((B, 1, H, 1), -1, dtype=torch.int32, device="cuda"))
    got = fc.decode_attention_shared(Q, fc.PagedKV(K, V, _int([[n]]), _int(table)), _int([0, B]), own, 0.1)
    _check_attention(got, Q, 0.1, _Rows(G, lambda b, l, h: near[h]), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,G,most", [(3, 2, 4000), (30, 4, 700), (1, 1, 20000)])
def test_few_rows_in_tables_as_wide_as_the_longest_answer(dtype, B, G, most):
    fc = _fc()
    rng = np.random.default_rng(most)
    H, d, ps, P = 2, 64, 16, 2
    cc = Cache(rng, rng.integers(0, 150, (P, 1)), H, d, ps, dtype, most=most)
    co = Cache(rng, rng.integers(0, 50, (B, 1)), H, d, ps, dtype, most=most)
    starts = [0, B // 2, B]
    Q = _rand(rng, (B, 1, G * H, d), _dt(dtype))

    def rows_for(b, l, h):
        return tuple(np.concatenate(x) for x in zip(cc.unit(0 if b < B // 2 else 1, 0, h, range(12)), co.unit(b, 0, h, range(12))))
    _check_attention(fc.decode_attention_shared(Q, cc.kv, _int(starts), co.kv, 0.125), Q, 0.125, _Rows(G, rows_for), dtype)
    bounds = fc.page_bounds(co.kv)
    chosen = fc.choose_pages(Q, co.kv, bounds, 3, first=0, last=1)
    want = pr.choose_pages(_f64(Q), _f64(bounds), co.rows_np, co.table_np, ps, 3, 0, 1)
    assert np.array_equal(chosen.cpu().numpy(), want)
    _check_attention(fc.decode_attention_chosen(Q, co.kv, chosen, 0.125), Q, 0.125, _Rows(G, lambda b, l, h: co.unit(b, l, h, want[b, l, h])), dtype)
