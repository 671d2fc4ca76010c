"""The 4-bit attention where a wave has many steps: pieces of more than a hundred, waves whose pages exceed the 64 that they look up at
a time, and launches of a workgroup for each of thousands of units, some of them long.  Many units share rows, tables and queries, and
so have to be equal to the bit; one of each kind is compared with 64 bits, within the tolerance that test_gpu_decode_loop.py derives."""
import numpy as np
import pytest

from oracle import decode_loop_ref as dr

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
U = 2.0 ** -24


def _wave_steps(d, dtype, units, rows_of_units, max_pages, ps):
    """Most steps of 32 rows that a wave has, and whether a unit is a workgroup's, by the kernel's rule."""
    groups = 256 * (4 if d == 64 else 3 if dtype == "bf16" else 2)
    steps = -(-np.asarray(rows_of_units) // 32)
    if -(-max_pages * ps // 32) <= 32 or units >= 4 * groups:
        return -(-int(steps.max()) // 4), True
    each = max(4, -(-int(steps.sum()) // (max(groups, units + units // 2) - units)))
    return max(-(-(-(-int(s) // -(-int(s) // each))) // 4) for s in steps if s), False


def _kinds(rng, fc, kinds, H, G, d, ps, sigma=1.0):
    """A pool of pages and, for each kind (a number of rows) and head, a table of its pages in any order, some of them missing."""
    pool, most = 97, -(-max(kinds) // ps)
    k, v = ((s * rng.standard_normal((pool * ps, d)) + 0.25).astype(np.float32) for s in (sigma, 1.0))
    pages = torch.zeros((pool, fc.mx_page_bytes(ps, d)), dtype=torch.uint8, device="cuda")
    fc.mx_store(torch.from_numpy(k[None]).cuda(), torch.from_numpy(v[None]).cuda(), torch.arange(pool * ps, device="cuda")[None], pages, ps)
    table = rng.integers(0, pool, (len(kinds), H, most)).astype(np.int32)
    for i, n in enumerate(kinds):
        if i % 2:                                        # on both sides of where a wave looks its pages up again, and here and there
            gone = rng.random((H, most)) < 0.03
            for wave in range(4):
                start = -(-n // 32) * wave // 4 * 32 // ps
                gone[:, start + 62:start + 66] = True
            gone[:, 0] = False
            table[i][gone] = rng.choice([-1, pool, -2 ** 31, 2 ** 31 - 1], int(gone.sum()))
        table[i, :, -(-n // ps):] = -1
    return pages, table, dr.grid(k), dr.grid(v)


@pytest.mark.parametrize("dtype,B,L,H,G,d,ps,kinds,whole", [
    # a piece for each unit but the longest, which have several
    ("bf16", 1, 250, 2, 2, 128, 16, (4300, 5001, 0, 4225, 6011, 20011, 5555, 33, 4700, 12345), False),
    ("bf16", 5, 100, 1, 9, 64, 16, (4300, 5001, 0, 4225, 6011, 1, 5555, 4703, 20011), False),
    ("f32", 2, 200, 1, 3, 128, 16, (4450, 4999, 4225, 17, 4737, 9001, 4400), False),
    ("f32", 1, 130, 3, 16, 128, 48, (4450, 4999, 0, 4225, 4737, 40003, 4400), False),
    # a workgroup for each of thousands
    ("bf16", 4, 200, 4, 7, 128, 16, (0, 3, 1, 4500, 17, 9001, 0, 33, 2, 1100), True),
    ("f32", 1, 700, 3, 4, 128, 48, (0, 5, 20011, 1, 31, 0, 13001), True),
    ("bf16", 5, 205, 4, 16, 64, 48, (1, 0, 2, 15000, 4, 14003, 90), True),
    ("f32", 5, 205, 4, 1, 64, 16, (1, 2, 0, 4096, 4097, 4129, 5000), True),
])
def test_long_units_among_many(dtype, B, L, H, G, d, ps, kinds, whole):
    import paper_2511_16786_amd as fc
    rng = np.random.default_rng(sum(kinds) + d)
    pages, table, K, V = _kinds(rng, fc, kinds, H, G, d, ps)
    # the first layers are of one kind each, and long kinds are rare among thousands of units
    kind = np.concatenate((np.arange(len(kinds)), rng.choice(len(kinds), B * L - len(kinds), p=[
        (0.002 if n > 1000 else 1.0) / sum(0.002 if m > 1000 else 1.0 for m in kinds) for n in kinds] if whole else None)))
    kind = kind[rng.permutation(B * L)]
    rows = np.array(kinds, np.int32)[kind].reshape(B, L)
    steps, alone = _wave_steps(d, dtype, B * L * H, np.repeat(rows, H), table.shape[2], ps)
    assert alone == whole and 2 * steps * 16 > 64 * ps    # (more tiles than 64 pages have)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q = torch.from_numpy(rng.standard_normal((len(kinds), H * G, d)).astype(np.float32)).to(dt).cuda()
    at = torch.from_numpy(kind).cuda()
    tables = torch.from_numpy(table).cuda()[at].view(B, L, H, -1).contiguous()
    out = torch.full((B, L, H * G, d), float("nan"), device="cuda")
    scale = 0.11
    fc.mx_decode_attention(q[at].view(B, L, H * G, d), pages, ps, H, torch.from_numpy(rows).cuda(), tables, scale, out=out)
    out = out.view(B * L, H * G, d)
    first = np.array([np.flatnonzero(kind == i)[0] for i in range(len(kinds))])
    one = out[torch.from_numpy(first).cuda()]
    assert torch.equal(out, one[at])                     # (cut by the number of rows alone)
    got, Q = one.double().cpu().numpy(), q.double().cpu().numpy()
    for i, n in enumerate(kinds):
        for h in range(H):
            r = np.arange(n)
            page = table[i, h, r // ps].astype(np.int64)
            slot = (page * ps + r % ps)[(page >= 0) & (page < len(pages))]
            mine = slice(h * G, (h + 1) * G)
            want, size, qk, top = dr.attend(Q[i, mine], K[slot], V[slot], scale)
            slip = 2 * (3 * d * U * qk + 4 * U * (top + 1)) + (len(slot) / 32 + 64) * U
            err = np.abs(got[i, mine] - want)
            assert np.all(err <= size * slip[:, None] + 1e-37), (i, h, np.max(err / np.maximum(size, 1e-30)), slip)
