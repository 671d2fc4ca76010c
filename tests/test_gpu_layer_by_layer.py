"""A decode loop as a model runs it: a layer's queries and rows are there only after the layer before."""
import numpy as np
import pytest

from oracle import decode_loop_ref as dr
from test_gpu_decode_loop import _check_attend, _compressed, _history, _rand

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("B", [1, 3])
def test_a_step_goes_layer_by_layer_over_the_caches_tensors(B):
    import paper_2511_16786_amd as fc
    rng = np.random.default_rng(50 + B)
    L, H, G, N, d, ps = 3, 2, 4, 300, 64, 16
    comp, K, V = _compressed(fc, rng, B, L, H, N, d)
    cache = fc.MxCache(B, L, H, d, ps, -(-N // ps), B * L * H * -(-N // ps))
    cache.fill(comp, K, V)
    Ks, Vs = _history(comp, K, V, B, L, H, d)
    plan = fc.rotary_plan(d, theta=1e6)
    for turn in range(18):                               # over a page's end
        pos = torch.full((B, 1), N + turn, dtype=torch.int32, device="cuda")
        fc.assign_pages(cache.rows, 1, ps, cache.block_table, cache.cursor, num_free=cache.num_pages, slots=cache.slots)
        for l in range(L):
            q, k, v = (_rand(rng, (B, 1, n, d), torch.bfloat16) for n in (H * G, H, H))
            q, k = fc.rotary(plan, pos, q, k)
            # (a layer's slices of one sequence are contiguous as they are)
            slots, rows, table = cache.slots[:, l * H:(l + 1) * H], cache.rows[:, l:l + 1], cache.block_table[:, l:l + 1]
            assert B > 1 or (slots.is_contiguous() and rows.is_contiguous() and table.is_contiguous())
            fc.mx_store(k.view(B, H, d), v.view(B, H, d), slots.contiguous(), cache.pages, ps)
            out = fc.mx_decode_attention(q, cache.pages, ps, H, rows.contiguous(), table.contiguous(), 0.125)
            mine = [(b * L + l) * H + h for b in range(B) for h in range(H)]
            for u, kn, vn in zip(mine, k.view(B * H, 1, d), v.view(B * H, 1, d)):
                Ks[u] = np.concatenate((Ks[u], dr.grid(kn.float().cpu().numpy())))
                Vs[u] = np.concatenate((Vs[u], dr.grid(vn.float().cpu().numpy())))
            if turn in (0, 7, 17):
                _check_attend(out, q, [Ks[u] for u in mine], [Vs[u] for u in mine], B, 1, H, G, 0.125)
    assert torch.equal(cache.rows, comp.budgets + 18) and cache.missing() == 0
