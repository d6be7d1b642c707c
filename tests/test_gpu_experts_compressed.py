"""The experts' weight gradients through the compressor and AdamW, straight from the stack that
the backward pass writes: what matrices of their own give, and nothing from an expert without
rows."""

import pytest

torch = pytest.importorskip("torch")

from paper_2301_09830_amd import optcc  # noqa: E402

pytestmark = pytest.mark.gpu

RANK = 4


class Keep:
    """What the compressor and the optimizer keep for a stack of matrices; a list of single
    ones (own) or slices of one tensor."""

    def __init__(self, e, rows, cols, own):
        g = torch.Generator(device="cuda").manual_seed(2)

        def stack(t):
            return [x.clone() for x in t] if own else t

        def randn(*shape):
            return torch.randn(*shape, generator=g, device="cuda")

        self.W = stack(randn(e, rows, cols))
        self.W16 = stack(torch.zeros(e, rows, cols, dtype=torch.bfloat16, device="cuda"))
        self.err, self.m, self.v, self.M_hat = (stack(torch.zeros(e, rows, cols, device="cuda"))
                                                for _ in range(4))
        self.Q, self.P = stack(randn(e, cols, RANK)), stack(torch.zeros(e, rows, RANK, device="cuda"))

    def step(self, grads, step):
        flags = torch.zeros(1, dtype=torch.int32, device="cuda")
        n = len(grads)
        optcc.occ_step_batched_noalloc([(grads[i], self.err[i], self.Q[i], self.P[i], self.M_hat[i])
                                        for i in range(n)], RANK, 1, flags_out=flags)
        params = optcc.make_params([optcc.make_param(self.W[i], self.m[i], self.v[i], P=self.P[i],
                                                     Q=self.Q[i], W16=self.W16[i]) for i in range(n)])
        optcc.occ_adamw_step(params, lr=1e-2, step=step)
        assert not int(flags) & optcc.OCC_F_NONFINITE


@pytest.mark.parametrize("dw", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("gated", [False, True])
def test_gradients_of_a_stack(gated, dw):
    sizes, n_in, out = [70, 0, 50, 130], 128, 96
    e, m, wide = len(sizes), sum(sizes), 2 * out if gated else out
    g = torch.Generator(device="cuda").manual_seed(1)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)

    at = torch.tensor([0] + sizes).cumsum(0).to(torch.int32).cuda()
    X, Z = randn(m, n_in), randn(m, wide)
    dW = torch.empty(e, wide, n_in, dtype=dw, device="cuda")
    f = optcc.occ_experts_gated_bwd if gated else optcc.occ_experts_linear_bwd
    stack, single = Keep(e, wide, n_in, False), Keep(e, wide, n_in, True)
    first = stack.W.clone()
    for step in (1, 2, 3):
        dY = randn(m, out)
        f(dY, at, X=X, Z=Z, act=optcc.OCC_ACT_SILU, dW=dW)
        before = stack.err.clone()
        stack.step(dW, step)
        single.step([x.clone() for x in dW], step)
        for name in ("W", "W16", "err", "Q", "P", "M_hat", "m", "v"):
            a, b = getattr(stack, name), getattr(single, name)
            assert all(torch.equal(x, y) for x, y in zip(a, b)), name
        # what is sent and what is kept are the gradient and what was kept, within the
        # subtraction's rounding and the sum's
        total = dW.double() + before.double()
        off = (stack.M_hat.double() + stack.err.double() - total).abs()
        size = dW.double().abs() + before.double().abs() + stack.M_hat.double().abs()
        assert (off <= 4 * 2.0 ** -24 * size).all()
    # the expert without rows: nothing to send or to move
    assert not stack.M_hat[1].any() and not stack.err[1].any()
    assert torch.equal(stack.W[1], first[1])
    assert all((stack.W[i] != first[i]).any() for i in (0, 2, 3))
