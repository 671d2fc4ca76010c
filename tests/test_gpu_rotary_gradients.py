"""Rotary positions in programs that train: what is refused, and the two calls that make a function with gradients."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_rotary_does_not_drop_gradients():
    """Inputs that want gradients are refused, since none would be recorded; without recording they are as good as any."""
    import paper_2511_16786_amd as fc
    plan = fc.rotary_plan(64)
    pos = torch.arange(3, dtype=torch.int32, device="cuda").view(1, 3)
    Q, K = (torch.randn((1, 3, 2, 64), device="cuda") for _ in range(2))
    want = fc.rotary(plan, pos, Q, K)
    wants = Q.clone().requires_grad_()
    for args, kw in (((wants, K), {}), ((Q, wants), {}), ((wants * 1.0, K), {}), ((Q, K), {"Q_out": wants * 1.0}),
                     ((Q, K), {"K_out": wants * 1.0})):
        with pytest.raises(ValueError):
            fc.rotary(plan, pos, *args, **kw)
    with torch.no_grad():
        got = fc.rotary(plan, pos, wants, K)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and not got[0].requires_grad
    got = fc.rotary(plan, pos, wants.detach(), K)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_rotary_and_its_transpose_make_a_function_with_gradients():
    """As a program that trains would use the two: gradients of Q and K against those of the same turn in torch's operators."""
    import paper_2511_16786_amd as fc
    T, d, theta = 5, 64, 1e4
    plan = fc.rotary_plan(d, theta=theta)
    pos = torch.arange(11, 11 + T, dtype=torch.int32, device="cuda").view(1, T)

    class Turn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k):
            return fc.rotary(plan, pos, q, k)

        @staticmethod
        def backward(ctx, gq, gk):
            return fc.rotary(plan, pos, gq.contiguous(), gk.contiguous(), inverse=True)

    g = torch.Generator(device="cuda").manual_seed(3)
    Q, K = (torch.randn((1, T, h, d), generator=g, device="cuda").requires_grad_() for h in (4, 2))
    q, k = Turn.apply(Q, K)
    gq, gk = torch.randn(q.shape, generator=g, device="cuda"), torch.randn(k.shape, generator=g, device="cuda")
    torch.autograd.backward((q, k), (gq, gk))
    angle = (pos.double()[..., None] * theta ** (-torch.arange(0, d, 2, device="cuda").double() / d))[:, :, None]
    for x, grad in ((Q, gq), (K, gk)):
        y = x.detach().double().requires_grad_()
        a, b = y[..., :d // 2], y[..., d // 2:]
        out = torch.cat((a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()), -1)
        out.backward(grad.double())
        # eight half steps of fp32 of both of a pair's magnitudes, the angle to 2^-50 of itself
        size = grad.double().abs()
        size = (size[..., :d // 2] + size[..., d // 2:]).repeat(1, 1, 1, 2)
        assert bool(((x.grad.double() - y.grad).abs() <= size * (8 * 2.0 ** -24 + 16 * 2.0 ** -50)).all())
