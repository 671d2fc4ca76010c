"""The 24 bits that the 4-bit attention gives to fp32 queries and to all probabilities, each as three bf16 terms.

The general tolerance of test_gpu_decode_loop.py covers any order of a score's sums and is too wide to tell whether the last eight bits
are there.  Here few products are not zero, so that few roundings can occur, and the results depend on the last bits.  u = 2^-24, half a step of fp32.

queries        Unit l has two rows: K is 1 in column l and in the next one, V is 1 and -1.  The query has x and x without its last eight bits
               there: the result is tanh((x scale - x' scale) / 2), and 0 without the last term.  |x scale| < 16, and each score is one
               product of three terms: off by 3 u at most, 48 u of the result for both; scale and reference are the same for both rows;
               exponentials 2 u each, six products' sums 6 u, the sum of both 2 u, the weights' terms 1 u, division and product 2 u: 64 u.
               The last term is 96 steps of 2^-17 and more, 46e-6 of the result, 768 u.
probabilities  Unit l has two rows of any weight, one with 1, row l with p; V is 1 everywhere, so that the result is 1: sums of six products
               6 u, the last term's rounding 1 u, the sum of both and its exchanges 3 u, the merge of the waves 2 u, division and product 2 u:
               14 u.  The last term of p is 96 u and more, which is 48 u of the result.

In both, values are taken of which the last eight bits are neither few (cut off) nor many (rounded up) and the eight before begin with a one,
so that the second term ends where they begin.
"""
import numpy as np
import pytest

U = 2.0 ** -24
SCALE = 0.125
QUERY_SLIP, PROBABILITY_SLIP = 64 * U, 14 * U


def _cut(x):
    """fp32 to its first eight bits."""
    return (np.asarray(x, np.float32).view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)


def _near(x):
    """fp32 to bf16, to nearest (ties do not occur here)."""
    return _cut((np.asarray(x, np.float32).view(np.uint32) + np.uint32(0x8000)).view(np.float32))


def _terms(x, how):
    """Sum of the bf16 terms of fp32 values, as fp32 (exact): three, or two of which the second is cut off or rounded."""
    x = np.asarray(x, np.float32)
    first = _cut(x)
    rest = x - first
    if how == "two, cut off":
        return first + _cut(rest)
    if how == "two, rounded":
        return first + _near(rest)
    second = _cut(rest)
    return (first.astype(np.float64) + second + _near(rest - second)).astype(np.float32)


def _telling(x):
    bits = np.asarray(x, np.float32).view(np.uint32)
    last = bits & 255
    return ((bits >> 15) & 1 == 1) & (last >= 96) & (last <= 160)


def _query_case(d, G, seed, sign):
    """q [d, G, d], K and V rows [d, 2, d]; the scale is SCALE times the sign."""
    rng = np.random.default_rng(seed)
    q = rng.standard_normal((d, G, d)).astype(np.float32)
    K, V = np.zeros((d, 2, d), np.float32), np.ones((d, 2, d), np.float32)
    V[:, 1] = -1
    for l in range(d):
        bits = (np.float32(64).view(np.uint32) + (rng.integers(0, 128, G) << 16) + (rng.integers(128, 256, G) << 8) + rng.integers(96, 161, G)).astype(np.uint32)
        K[l, 0, l] = K[l, 1, (l + 1) % d] = 1
        q[l, :, l] = sign * bits.view(np.float32)
        q[l, :, (l + 1) % d] = sign * (bits & np.uint32(0xFFFFFF00)).view(np.float32)
    assert _telling(q[np.arange(d), :, np.arange(d)]).all()
    return q, K, V


def _queries_answer(q, how=None):
    """[d, G] of every column of the output, in 64 bits."""
    d = q.shape[0]
    held = (q if how is None else _terms(q, how)).astype(np.float64)
    x, y = (held[np.arange(d), :, (np.arange(d) + k) % d] for k in (0, 1))
    return np.tanh(np.abs(x * SCALE) / 2 - np.abs(y * SCALE) / 2)


def _probability_case(d, G, seed):
    """q [32, G, d] (exact in bf16), K and V rows [32, 32, d]."""
    rng = np.random.default_rng(seed)
    grid = _cut(-np.exp2(rng.uniform(-6, 2.4, 20000)).astype(np.float32))
    grid = grid[_telling(_weight(grid))]
    assert len(np.unique(grid)) >= 32
    q = np.full((32, G, d), -4000, np.float32)           # rows of other columns: e^-500
    K, V = np.zeros((32, 32, d), np.float32), np.ones((32, 32, d), np.float32)
    for l in range(32):
        one, some, others = rng.permutation(d)[:3]
        K[l, :, others] = 1
        for row, column in (((l + rng.integers(1, 32)) % 32, one), (l, some)):
            K[l, row, others], K[l, row, column] = 0, 1
        q[l, :, one], q[l, :, some] = 0, rng.choice(grid, G)
    return q, K, V


def _weight(x):
    """p of a score, as fp32 has it but for a step or two."""
    return np.exp2((np.asarray(x, np.float32) * (np.float32(SCALE) * np.float32(1.4426950408889634))).astype(np.float64)).astype(np.float32)


@pytest.mark.parametrize("d", [64, 128])
def test_without_the_last_term_the_results_are_out_of_tolerance(d):
    """What the GPU tests below would find: the tolerances tell three terms from two, whichever way the second ends."""
    for sign in (1, -1):
        q, K, V = _query_case(d, 16, d, sign)
        want = _queries_answer(q)
        assert np.all(np.abs(_queries_answer(q, "three") - want) == 0)
        for how in ("two, cut off", "two, rounded"):
            assert np.all(np.abs(_queries_answer(q, how) - want) > 4 * QUERY_SLIP), how
    q, K, V = _probability_case(d, 16, d)
    lone = np.argmax(K[np.arange(32), np.arange(32)], 1)
    p = _weight(q[np.arange(32), :, lone])
    assert p.min() >= 0.5 and p.max() < 1
    for step in (-2, 0, 2):                              # (an exponential that is off by so many steps)
        near = (p.view(np.uint32) + np.int32(step).astype(np.uint32)).view(np.float32)
        loss = {how: np.abs(_terms(near, how).astype(np.float64) - near) / (1.0 + near) for how in ("three", "two, cut off", "two, rounded")}
        assert loss["three"].max() <= U
        assert min(loss["two, cut off"].min(), loss["two, rounded"].min()) > 3 * PROBABILITY_SLIP


def _attend(fc, torch, q, K, V, dtype, scale):
    L, G, d = q.shape
    n, ps = K.shape[1], 32
    pages = torch.full((L, fc.mx_page_bytes(ps, d)), 255, dtype=torch.uint8, device="cuda")
    slots = (torch.arange(L, device="cuda")[:, None] * ps + torch.arange(n, device="cuda")).view(1, L * n)
    fc.mx_store(torch.from_numpy(K.reshape(1, L * n, d)).cuda(), torch.from_numpy(V.reshape(1, L * n, d)).cuda(), slots, pages, ps)
    back = torch.empty((2, 1, L * n, d), device="cuda")
    fc.mx_load(slots, pages, ps, back[0], back[1])
    assert np.array_equal(back[0].cpu().numpy().ravel(), K.ravel()) and np.array_equal(back[1].cpu().numpy().ravel(), V.ravel())
    Q = torch.from_numpy(q).to(dtype).cuda()[None]
    assert np.array_equal(Q.float().cpu().numpy()[0], q)
    rows = torch.full((1, L), n, dtype=torch.int32, device="cuda")
    table = torch.arange(L, dtype=torch.int32, device="cuda").view(1, L, 1, 1)
    return fc.mx_decode_attention(Q, pages, ps, 1, rows, table, scale)[0].double().cpu().numpy()


@pytest.mark.gpu
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 7, 8, 9, 16])
def test_fp32_queries_count_to_their_last_bit(G, d, sign):
    torch = pytest.importorskip("torch")
    import paper_2511_16786_amd as fc
    q, K, V = _query_case(d, G, d, sign)
    got = _attend(fc, torch, q, K, V, torch.float32, sign * SCALE)
    worst = np.abs(got - _queries_answer(q)[..., None]).max()
    assert worst <= QUERY_SLIP, worst / U


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 7, 8, 9, 16])
def test_probabilities_count_to_their_last_bit(G, d, dtype):
    torch = pytest.importorskip("torch")
    import paper_2511_16786_amd as fc
    q, K, V = _probability_case(d, G, d)
    got = _attend(fc, torch, q, K, V, torch.bfloat16 if dtype == "bf16" else torch.float32, SCALE)
    worst = np.abs(got - 1.0).max()
    assert worst <= PROBABILITY_SLIP, worst / U
