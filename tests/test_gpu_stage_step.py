"""The stage example: the operators and the compressor together, and each
gradient of the stage against autograd in fp32."""

import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "stage_step.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("stage_step", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_the_stage_learns(example):
    """Forty steps from a random start: the loss more than halves and stays
    finite (an optimizer that did not move, or moved the wrong way, would not)."""
    losses = example.run(steps=40, hidden=128, tokens=256, rank=8, lr=2e-3)
    assert all(x == x for x in losses)
    assert losses[-1] < 0.5 * losses[0], losses[::8]


def test_gradients_of_the_whole_stage(example):
    """Backward through both blocks against autograd in fp32 on the same bf16
    weights.  Along the way activations and gradients are rounded to bf16 a
    few times, each by at most 2^-8 of a value, independently: 2-norms agree
    within 2^-8 times the square root of about ten roundings."""
    s = example.Stage(96, 200, 8)
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(200, 96, generator=gen, device="cuda").to(torch.bfloat16)
    dz = torch.randn(200, 96, generator=gen, device="cuda").to(torch.bfloat16)
    z = s.forward(x)
    dx = s.backward(dz.clone())
    torch.cuda.synchronize()
    w = [t.bf16.float().requires_grad_() for t in s.weights]
    b = [t.value.clone().requires_grad_() for t in (s.b1, s.b2)]
    xf = x.float().requires_grad_()
    y = torch.nn.functional.gelu(xf @ w[0].t() + b[0]) @ w[1].t() + b[1] + xf
    g, u = (y @ w[2].t()).chunk(2, 1)
    ref = (torch.nn.functional.silu(g) * u) @ w[3].t() + y
    ref.backward(dz.float())
    bound = 2.0 ** -8 * 10 ** 0.5

    def near(got, want):
        return float((got.float() - want).norm() / want.norm()) <= bound

    assert near(z, ref.detach()) and near(dx, xf.grad)
    for t, v in zip(s.weights + [s.b1, s.b2], w + b):
        assert near(t.grad, v.grad)


def test_a_gradient_that_is_not_finite_leaves_the_weights(example):
    s = example.Stage(64, 64, 4)
    x = torch.randn(64, 64, device="cuda").to(torch.bfloat16)
    s.forward(x)
    s.backward(torch.ones_like(x))
    s.W2.grad[3, 5] = float("nan")
    before = [w.value.clone() for w in s.weights] + [s.b1.value.clone()]
    s.update(4, 1, 1e-3)
    after = [w.value for w in s.weights] + [s.b1.value]
    assert int(s.flags) & 1 and all(torch.equal(p, q) for p, q in zip(before, after))
