"""What the Python binding of the router, the exchange, the experts' layers and the
distillation loss refuses before a kernel sees it.  Host checks: no GPU."""

import os

import pytest

torch = pytest.importorskip("torch")

from paper_2301_09830_amd import build as buildmod  # noqa: E402
from paper_2301_09830_amd import optcc  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def built():
    if not (os.path.exists(buildmod.LIB) and os.path.exists(buildmod.LAYERS)):
        buildmod.build()


def ints(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


X, W, AT = torch.zeros(9, 16), torch.zeros(3, 6, 16), ints(4)
ROUTE = optcc.Route(ints(9, 2), torch.zeros(9, 2), ints(4), ints(18), ints(9, 2))


def refused(kind, text, call, *a, **k):
    with pytest.raises(kind, match=text):
        call(*a, **k)


@pytest.mark.parametrize("args,change,kind,text", [
    ((X.half(), W, AT), {}, TypeError, "X must be float32 or bfloat16"),
    ((X, W.bfloat16(), AT), {}, TypeError, "W must be"),
    ((X, W[0], AT), {"Y": torch.zeros(9, 6)}, ValueError, "W must be 3-D"),
    ((X, W[0], AT), {}, ValueError, "W 3-D"),
    ((X[0], W, AT), {"Y": torch.zeros(9, 6)}, ValueError, "X must be 2-D"),
    ((X, W, AT.long()), {}, TypeError, "offsets must be"),
    ((X, W, ints(3)), {}, ValueError, "W must be 2 x 6 x 16"),
    ((X, W, ints(1)), {}, ValueError, "offsets must hold one more value"),
    ((X, W, ints(2, 2)), {}, ValueError, "offsets must hold one more value"),
    ((X, W, None), {}, ValueError, "offsets must be given"),
    ((X, W, ints(8)[::2]), {}, ValueError, "offsets must hold"),
    ((X, W[:, :, :15], AT), {}, ValueError, "W must be 3 x 6 x 16"),
    ((X, W.transpose(1, 2).contiguous().transpose(1, 2), AT), {}, ValueError, "unit column stride"),
    ((X, W, AT), {"bias": torch.zeros(3, 5)}, ValueError, "bias must hold 18"),
    ((X, W, AT), {"bias": torch.zeros(3, 6).bfloat16()}, TypeError, "bias must be"),
    ((X, W, AT), {"R": torch.zeros(9, 5)}, ValueError, "R must be 9 x 6"),
    ((X, W, AT), {"Y": torch.zeros(8, 6)}, ValueError, "Y must be 9 x 6"),
    ((X, W, AT), {"Z": torch.zeros(9, 7)}, ValueError, "Z must be 9 x 6"),
    ((X, W, AT), {"flags": ints(2)}, ValueError, "flags must hold 1"),
    ((X, W, AT), {"flags": torch.zeros(1)}, TypeError, "flags must be"),
    ((X, W, AT), {"ws": 4096}, TypeError, "ws must be a tensor"),
    ((X, W.to("meta"), AT), {}, ValueError, "W lies on another device"),
], ids=lambda v: None)
def test_forward(args, change, kind, text):
    refused(kind, text, optcc.occ_experts_linear_fwd, *args, **change)


def test_gated_weights_hold_both_projections():
    refused(ValueError, "rows of both projections", optcc.occ_experts_gated_fwd, X,
            torch.zeros(3, 7, 16), AT, Y=torch.zeros(9, 3))


@pytest.mark.parametrize("change,kind,text", [
    ({"dW": torch.zeros(3, 6, 15)}, ValueError, "dW must be 3 x 6 x 16"),
    ({"dW": torch.zeros(2, 6, 16)}, ValueError, "dW must be 3 x 6 x 16"),
    ({"dX": torch.zeros(9, 15)}, ValueError, "dX must be 9 x 16"),
    ({"dbias": torch.zeros(6)}, ValueError, "dbias must hold 18"),
    ({"Z": torch.zeros(8, 6)}, ValueError, "Z must be 9 x 6"),
    ({"X": torch.zeros(8, 16)}, ValueError, "X must be 9 x 16"),
    ({"dX": torch.zeros(9, 16).to("meta")}, ValueError, "dX lies on another device"),
], ids=lambda v: None)
def test_backward(change, kind, text):
    args = dict({"X": X, "W": W}, **change)
    refused(kind, text, optcc.occ_experts_linear_bwd, torch.zeros(9, 6), AT, **args)


def test_router():
    logits = torch.zeros(9, 8)
    for k in (0, 33, -1, 1 << 40):
        refused(ValueError, "k is out of range", optcc.occ_route_fwd, logits, k)
    refused(TypeError, "int", optcc.occ_route_fwd, logits, "two")
    refused(TypeError, "logits must be float32 or bfloat16", optcc.occ_route_fwd, logits.double(), 2)
    refused(ValueError, "logits must be 2-D", optcc.occ_route_fwd, logits[0], 2)
    refused(ValueError, "unit column stride", optcc.occ_route_fwd, torch.zeros(8, 9).t(), 2)
    back = torch.zeros(9, 2)
    refused(ValueError, "dweights must hold 18", optcc.occ_route_bwd, back[:8], logits, ROUTE)
    refused(TypeError, "dweights must be", optcc.occ_route_bwd, back.bfloat16(), logits, ROUTE)
    refused(ValueError, "index must be 2-D", optcc.occ_route_bwd, back, logits,
            ROUTE._replace(index=ints(18)))
    refused(ValueError, "weights must hold 18", optcc.occ_route_bwd, back, logits,
            ROUTE._replace(weights=torch.zeros(9, 3)))


def test_exchange():
    Ys, w = torch.zeros(18, 16), torch.zeros(9, 2)
    refused(ValueError, "slots must have a row for each token", optcc.occ_dispatch, X[:8], ROUTE)
    refused(TypeError, "order must be", optcc.occ_dispatch, X, ROUTE._replace(order=torch.zeros(18)))
    refused(ValueError, "order must be given", optcc.occ_dispatch, X, ROUTE._replace(order=None))
    refused(ValueError, "slots must be 2-D", optcc.occ_dispatch, X, ROUTE._replace(slots=ints(18)))
    refused(ValueError, "weights must hold 18", optcc.occ_combine, Ys, ROUTE, weights=w[:, :1])
    refused(ValueError, "flags must hold 1", optcc.occ_combine, Ys, ROUTE, flags=ints(3))
    refused(ValueError, "slots must have a row", optcc.occ_combine_bwd, X[:8], Ys, ROUTE)
    refused(ValueError, "dweights needs Ys", optcc.occ_combine_bwd, X, None, ROUTE, dweights=w)


def test_distillation():
    S, i, t = torch.zeros(5, 40), ints(5, 3), torch.zeros(5, 3)
    refused(TypeError, "S must be float32 or bfloat16", optcc.occ_distill_fwd, S.half(), i, t)
    refused(TypeError, "index must be", optcc.occ_distill_fwd, S, i.long(), t)
    refused(TypeError, "teacher must be float32 or bfloat16", optcc.occ_distill_fwd, S, i, t.half())
    refused(ValueError, "teacher must be 5 x 3", optcc.occ_distill_fwd, S, i, t[:, :2])
    refused(ValueError, "go together", optcc.occ_distill_fwd, S, i, None)
    refused(ValueError, "too many entries", optcc.occ_distill_fwd, S, ints(5, 1025),
            torch.zeros(5, 1025))
    refused(ValueError, "labels must hold 5", optcc.occ_distill_fwd, S, i, t, alpha=0.5, labels=ints(4))
    refused(TypeError, "labels must be", optcc.occ_distill_fwd, S, i, t, alpha=0.5,
            labels=torch.zeros(5, dtype=torch.long))
    refused(ValueError, "scale must hold 5", optcc.occ_distill_fwd, S, i, t, scale=torch.ones(1))
    refused(ValueError, "lse must hold 10", optcc.occ_distill_bwd, S, i, t, torch.zeros(5))


def test_tensors_lie_on_a_gpu():
    S, i, t = torch.zeros(5, 40), ints(5, 3), torch.zeros(5, 3)
    text = "must lie on a GPU"
    refused(ValueError, text, optcc.occ_experts_linear_fwd, X, W, AT)
    refused(ValueError, text, optcc.occ_experts_linear_bwd, torch.zeros(9, 6), AT, X=X,
            dW=torch.zeros(3, 6, 16))
    refused(ValueError, text, optcc.occ_route_fwd, torch.zeros(9, 8), 2)
    refused(ValueError, text, optcc.occ_route_bwd, torch.zeros(9, 2), torch.zeros(9, 8), ROUTE)
    refused(ValueError, text, optcc.occ_dispatch, X, ROUTE)
    refused(ValueError, text, optcc.occ_combine, torch.zeros(18, 16), ROUTE)
    refused(ValueError, text, optcc.occ_combine_bwd, X, torch.zeros(18, 16), ROUTE)
    refused(ValueError, text, optcc.occ_distill_fwd, S, i, t)
    refused(ValueError, text, optcc.occ_distill_bwd, S, i, t, torch.zeros(5, 2))
