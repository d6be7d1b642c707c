"""Two steps of the experts' layers and the loss at once, each on a stream of its own, make what
each makes alone."""

import pytest

torch = pytest.importorskip("torch")

from test_gpu_experts_step import Step  # noqa: E402

pytestmark = pytest.mark.gpu


def outputs(s):
    return [s.loss, s.dS, *s.grads.values()]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
def test_two_steps_at_once(dtype):
    sizes = [(700, 128, 96, 8, 2, 3000), (300, 256, 64, 20, 4, 9001)]
    steps = [Step(*size, dtype, seed=i) for i, size in enumerate(sizes)]
    want = []
    for s in steps:
        s.run()
        want.append([x.clone() for x in outputs(s)])
    streams = [torch.cuda.Stream() for _ in steps]
    torch.cuda.synchronize()
    for _ in range(5):
        for s in steps:
            for x in outputs(s):
                x.fill_(7.0)
        torch.cuda.synchronize()
        for _ in range(3):
            for s, stream in zip(steps, streams):
                with torch.cuda.stream(stream):
                    s.run()
        torch.cuda.synchronize()
        for s, w in zip(steps, want):
            assert all(torch.equal(a, b) for a, b in zip(outputs(s), w))
