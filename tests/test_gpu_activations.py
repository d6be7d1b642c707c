"""GELU of the fp32 layers over its whole range, relative to the value itself.

A layer of one weight 1 makes z = x exactly, its backward pass of dY = 1 the
derivative.  The bound counts roundings, u = 2^-24 each: the argument of the
exponential is rounded twice and its constant once, which weighs 1.5 z^2 u in
the result; the exponential and the reciprocal are good to 2 u, the reciprocal's
argument and constant to 2 u; the polynomial's terms sum to 1.8 times its value
and its coefficients and fit are good to 2 u, 8 steps of which the leading ones
count: 14 u in all; products and sums behind it 4 u.  Doubled for the powers of t:
(30 + 2 z^2) u."""

import math

import pytest

torch = pytest.importorskip("torch")

from paper_2301_09830_amd import optcc  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [3, 60, 20011], ids=["by rows", "few", "tiled"])
def test_gelu_is_as_good_as_its_roundings(tokens):
    z = torch.linspace(-12.5, 12.5, tokens, device="cuda").view(-1, 1)
    one = torch.ones(1, 1, device="cuda")
    y = optcc.occ_linear_fwd(z, one, act=optcc.OCC_ACT_GELU)
    d = torch.empty_like(z)
    optcc.occ_linear_bwd(torch.ones_like(z), W=one, Z=z, act=optcc.OCC_ACT_GELU, dX=d)
    x = z.double().cpu()
    phi = torch.erfc(-x * math.sqrt(0.5)) / 2      # (torch.special.ndtr cancels below -6)
    slope = x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    u = (30 + 2 * x * x) * 2.0 ** -24
    for got, want, size in ((y, x * phi, (x * phi).abs()), (d, phi + slope, phi + slope.abs())):
        off = (got.double().cpu() - want).abs() / (u * size).clamp_min(2.0 ** -126)
        assert float(off.max()) <= 1, (float(off.max()), float(x[off.argmax()]))


@pytest.mark.parametrize("act", range(1, 5))
@pytest.mark.parametrize("tokens", [40, 3000], ids=["direct", "made first"])
def test_derivatives_of_nan_are_nan(act, tokens):
    """A pre-activation that is not a number is not one in the gradients either:
    none of them hides it behind a zero."""
    g = torch.Generator(device="cuda").manual_seed(act)
    for gated in (False, True):
        n, wide = 72, 144 if gated else 72
        dY, X = (torch.randn(tokens, c, generator=g, device="cuda") for c in (n, 56))
        W, Z = torch.randn(wide, 56, generator=g, device="cuda"), torch.randn(tokens, wide, generator=g, device="cuda")
        Z[3, 5] = float("nan")
        dX, dW, db = torch.empty_like(X), torch.empty_like(W), torch.empty(wide, device="cuda")
        (optcc.occ_gated_bwd if gated else optcc.occ_linear_bwd)(dY, X, W, Z=Z, act=act, dX=dX,
                                                                 dW=dW, dbias=db)
        assert torch.isnan(dX[3]).all() and torch.isnan(dW[5]).all() and torch.isnan(db[5])
        assert torch.isnan(dX).any(1).sum() == 1
        # with a gate, u act'(z) and act(z) are both not a number
        assert int(torch.isnan(db).sum()) == (2 if gated else 1)
