"""Every form of the layers' products that the plan chooses (tests/stage_forms.py;
tests/test_layer_plans.py checks on the host that these layers take them), with
all parts of the epilogue, against float64."""

import pytest

torch = pytest.importorskip("torch")

from paper_2301_09830_amd import optcc  # noqa: E402
from stage_forms import ALONE, FORMS, SINGLE, STREAMS  # noqa: E402
from stage_ref import backward64, within  # noqa: E402
from test_gpu_layers import gen, rand, run_backward, run_forward  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", FORMS, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_forms(case):
    kind, dtype, gated, _, _, _, size = case
    act = 4 if gated else 2
    if kind == "fwd":
        run_forward(*size, dtype, act, gated, seed=sum(size))
        run_forward(*size, dtype, act, gated, bias=False, residual=False, save=False)
    else:
        run_backward(*size, dtype, act, gated, seed=sum(size))
        run_backward(*size, dtype, act, gated, dw="f32", accumulate=True)


@pytest.mark.parametrize("case", STREAMS, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_results_past_the_caches(case):
    kind, dtype, gated, size = case
    if kind == "fwd":
        run_forward(*size, dtype, 4 if gated else 2, gated)
    else:
        run_backward(*size, dtype, 4 if gated else 0, gated, accumulate=not gated)


@pytest.mark.parametrize("dtype,act,gated,form,tile,size,output", ALONE)
def test_forms_of_a_gradient_alone(dtype, act, gated, form, tile, size, output):
    g = gen(7)
    t, k, n = size
    wide, dt = 2 * n if gated else n, torch.float32
    dY = rand(g, t, n, dt)
    X, W = (rand(g, t, k, dt), None) if output == "dW" else (None, rand(g, n, k, dt, n ** -0.5))
    Z = rand(g, t, wide, dt) if act else None
    got = torch.empty((wide, k) if output == "dW" else (t, k), device="cuda")
    (optcc.occ_gated_bwd if gated else optcc.occ_linear_bwd)(dY, X, W, Z=Z, act=act, **{output: got})
    within(got, *backward64(dY, X, W, Z, act, gated)[output], output)


@pytest.mark.parametrize("dtype,act,size,single,what", SINGLE)
def test_single_outputs_whose_plan_differs(dtype, act, size, single, what):
    """The requested outputs enter the plan, so the bits may differ from those
    of a call for both; each is right by itself, and repeats bit by bit."""
    g = gen(5)
    t, k, n = size
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    dY, X, W = rand(g, t, n, dt), rand(g, t, k, dt), rand(g, n, k, dt, n ** -0.5)
    Z = rand(g, t, n, dt) if act else None
    ref = backward64(dY, X, W, Z, act, False)
    out = {"dX": torch.empty_like(X), "dW": torch.empty_like(W)}
    optcc.occ_linear_bwd(dY, X, W, Z=Z, act=act, **out)
    for name, got in out.items():
        within(got, *ref[name], name)
    once = torch.empty_like(out[single])
    again = torch.empty_like(once)
    for got in (once, again):
        optcc.occ_linear_bwd(dY, X, W, Z=Z, act=act, **{single: got})
    within(once, *ref[single], single)
    assert torch.equal(once, again)


# The bounds above grow with K and hold for products of far fewer bits.  In
# norm, over independent normal values, errors average out: each rounding to
# fp32 is off by at most 2^-24 of a running sum whose square averages K / 2 of K
# in the end, uniformly (1 / sqrt 3).  The fp32 matrix instruction rounds after
# each product (1 + 3 x 0.75 2^-24, four products, gives 1): sqrt(K / 6) 2^-24 of
# the result.  The one of the planes sums four products or more before it rounds:
# sqrt(K / 24) 2^-24.  And 2^-24 for the operands' planes and the store.  A
# product of planes that is left out costs 2.4e-6 or more (l h, h l and m m; the
# others 1.6e-3).
NORMS = [("fwd", (4096, 256, 4096), "planes"), ("fwd", (4096, 520, 4096), "planes"),
         ("fwd", (1546, 409, 2596), "planes"), ("fwd", (1500, 2304, 2200), "planes"),
         ("bwd", (520, 4096, 4096), "planes"), ("bwd", (4096, 4096, 520), "planes"),
         ("fwd", (200, 520, 130), "fp32"), ("fwd", (1003, 1023, 2047), "fp32"),
         ("fwd", (3, 700, 900), "fp32"), ("fwd", (30, 700, 900), "fp32"),
         ("bwd", (517, 1000, 1500), "fp32"), ("bwd", (300, 200, 100), "fp32")]


@pytest.mark.parametrize("kind,size,units", NORMS)
def test_fp32_layers_are_fp32_in_norm(kind, size, units):
    t, k, n = size
    g = gen(31)
    f32 = torch.float32
    X, W = rand(g, t, k, f32), rand(g, n, k, f32)
    x, w = X.double(), W.double()

    def near(got, want, length):
        error = float((got.double() - want).norm() / want.norm())
        bound = ((length / (24 if units == "planes" else 6)) ** 0.5 + 1) * 2.0 ** -24
        print(f"{kind} {size} K {length}: {error:.2e} of {bound:.2e}", flush=True)
        assert error <= bound

    if kind == "fwd":
        near(optcc.occ_linear_fwd(X, W), x @ w.t(), k)
        return
    dY = rand(g, t, n, f32)
    dX, dW = torch.empty_like(X), torch.empty_like(W)
    optcc.occ_linear_bwd(dY, X, W, dX=dX, dW=dW)
    near(dX, dY.double() @ w, n)
    near(dW, dY.double().t() @ x, t)


def test_planes_of_the_smallest_operands():
    """Operands of 2^-99 keep their 2^-25: their planes end above 2^-126."""
    g = gen(41)
    X, W = rand(g, 4096, 520, torch.float32), rand(g, 4096, 520, torch.float32, 2.0 ** 40)
    X.copy_(torch.copysign(X.abs().frac() + 1, X) * 2.0 ** -99)
    want = X.double() @ W.double().t()
    error = float((optcc.occ_linear_fwd(X, W).double() - want).norm() / want.norm())
    assert error <= ((520 / 24) ** 0.5 + 1) * 2.0 ** -24


def test_planes_of_infinities():
    """A non-finite operand makes every result that it enters NaN, and no other."""
    g = gen(42)
    X, W = rand(g, 4096, 520, torch.float32), rand(g, 4096, 520, torch.float32)
    X[9, 100], X[77, 519], W[5, 3] = float("inf"), float("nan"), float("-inf")
    Y = optcc.occ_linear_fwd(X, W)
    rows = torch.ones(4096, dtype=torch.bool, device="cuda")
    cols = rows.clone()
    rows[[9, 77]], cols[5] = False, False
    assert torch.isnan(Y[~rows]).all() and torch.isnan(Y[:, ~cols]).all()
    assert torch.isfinite(Y[rows][:, cols]).all()
