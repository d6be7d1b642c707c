"""The distillation loss at the ends of the types' ranges: logits and a teacher's list whose
quotients by the temperature 32 bits do not hold, against float64."""

import math

import pytest

torch = pytest.importorskip("torch")

from experts_ref import distill64  # noqa: E402
from paper_2301_09830_amd import optcc  # noqa: E402
from stage_ref import within  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [0.25, 0.7, 1.0, 3.0])
def test_teachers_of_extreme_values(T, dtype):
    """A finite logit is an entry whatever its quotient by the temperature: only -inf is
    masked.  Lists of the lowest value alone, of the largest, of both beside others."""
    t, v, k = 8, 500, 6
    dt, low, high = DT[dtype], torch.finfo(DT[dtype]).min, torch.finfo(DT[dtype]).max
    S = torch.randn(t, v, generator=gen(1), device="cuda").to(dt)
    index = torch.rand(t, v, generator=gen(2), device="cuda").argsort(1)[:, :k].to(torch.int32)
    index = index.contiguous()
    teacher = torch.randn(t, k, generator=gen(3), device="cuda").to(dt)
    teacher[0] = low                       # even over the list
    teacher[1, 2:] = low                   # nothing but for the first two
    teacher[2] = high
    teacher[3, 1] = high
    teacher[4, :3], teacher[4, 3:] = low, -math.inf
    teacher[5, 0], teacher[5, 1] = high, low
    labels = torch.randint(0, v, (t,), generator=gen(4), device="cuda", dtype=torch.int32)
    for alpha in (1.0, 0.5):
        lse, dS = torch.empty(t, 2, device="cuda"), torch.empty_like(S)
        loss = optcc.occ_distill_fwd(S, index, teacher, T, alpha, labels, lse=lse, dS=dS)
        want = distill64(S, index, teacher, T, alpha, labels, None)
        within(loss, *want["loss"], "loss")
        within(dS, *want["dS"], "dS")
        within(lse, *want["lse"], "lse")
        within(optcc.occ_distill_bwd(S, index, teacher, lse, T, alpha, labels), *want["dS_lse"],
               "dS from lse")
