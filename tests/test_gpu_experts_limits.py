"""Matrices of more than 2^31 elements: the exchange of rows, the distillation loss and
the experts' layers at their far ends, against the same rows in a small call."""

import pytest

torch = pytest.importorskip("torch")

from paper_2301_09830_amd import optcc  # noqa: E402

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def test_distillation():
    t, v, k = 43000, 51200, 4
    S = torch.zeros(t, v, dtype=torch.bfloat16, device="cuda")
    last = torch.randn(400, v, generator=gen(1), device="cuda").to(torch.bfloat16)
    S[-400:] = last
    index = torch.randint(0, v, (t, k), generator=gen(2), device="cuda", dtype=torch.int32)
    teacher = torch.randn(t, k, generator=gen(3), device="cuda")
    loss = optcc.occ_distill_fwd(S, index, teacher, dS=S)
    small = torch.empty_like(last)
    want = optcc.occ_distill_fwd(last, index[-400:], teacher[-400:], dS=small)
    assert torch.equal(loss[-400:], want) and torch.equal(S[-400:], small)
    assert torch.isfinite(loss).all()


def test_exchange():
    t, h = 530000, 4100
    X = torch.zeros(t, h, dtype=torch.bfloat16, device="cuda")
    X[-300:] = torch.randn(300, h, generator=gen(1), device="cuda").to(torch.bfloat16)
    X[:300] = 1.0
    logits = torch.zeros(t, 2, device="cuda")
    logits[-300:, 1] = 1.0                   # the last tokens go to the last expert
    r = optcc.occ_route_fwd(logits, 1)
    assert r.offsets.tolist() == [0, t - 300, t]
    Xs = optcc.occ_dispatch(X, r)
    assert torch.equal(Xs[-300:], X[-300:]) and torch.equal(Xs[:300], X[:300])
    Y = optcc.occ_combine(Xs, r, weights=r.weights, Y=torch.empty_like(X))
    assert torch.equal(Y[-300:], X[-300:]) and torch.equal(Y[:300], X[:300])
    Y.fill_(0.0)
    dYs, dw = optcc.occ_combine_bwd(X, Xs, r, weights=r.weights, dYs=Y)
    assert torch.equal(dYs[-300:], X[-300:])
    want = (X[-300:].double() ** 2).sum(1)
    assert ((dw[-300:, 0].double() - want).abs() <= want * 80 * 2.0 ** -24).all()


@pytest.mark.parametrize("rows", [3, 700])
def test_experts(rows):
    e, n, k = 35, 8192, 8192
    W = torch.zeros(e, n, k, dtype=torch.bfloat16, device="cuda")
    W[-1] = torch.randn(n, k, generator=gen(1), device="cuda").to(torch.bfloat16) / 64
    X = torch.randn(rows, k, generator=gen(2), device="cuda").to(torch.bfloat16)
    at = torch.tensor([0] * e + [rows], dtype=torch.int32, device="cuda")
    Y = optcc.occ_experts_linear_fwd(X, W, at).float()
    want = X.float() @ W[-1].float().t()
    assert float((Y - want).norm() / want.norm()) <= 2.0 ** -8
    dY = torch.randn(rows, n, generator=gen(3), device="cuda").to(torch.bfloat16)
    dX, dW = torch.empty_like(X), torch.full_like(W, 7.0)
    optcc.occ_experts_linear_bwd(dY, at, X=X, W=W, dX=dX, dW=dW)
    for got, ref in ((dX, dY.float() @ W[-1].float()), (dW[-1], dY.float().t() @ X.float())):
        assert float((got.float() - ref).norm() / ref.norm()) <= 2.0 ** -8
    assert not dW[:-1].any()
