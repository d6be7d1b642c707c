"""The router on either side of every number of experts, choices and tokens at which
it takes another way."""

import math

import pytest

torch = pytest.importorskip("torch")

from paper_2301_09830_amd import optcc  # noqa: E402
from experts_ref import route_bwd64  # noqa: E402
from stage_ref import within  # noqa: E402
from test_gpu_route import check_route, gen, rand  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("e", [2, 8, 31, 32, 33, 64, 65, 127, 128, 129, 256, 257, 512, 513, 1023, 1024])
def test_experts_and_choices(e, dtype):
    for k in (1, 2, 7, 8, 9, 16, 17, 32):
        if k <= e:
            for t in (70, 300):
                check_route(rand(gen(e + k), t, e, DT[dtype]), k, (k + t) % 4 == 0, seed=k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("e", [24, 60, 128, 250, 500, 1000])
def test_ties_masks_and_signs(e, dtype):
    """Few distinct values of both signs, zeros of both signs, masked experts, tokens with
    fewer experts than choices, the type's lowest and largest values, infinities."""
    for k in (3, 8, 12):
        x = torch.randint(-2, 3, (290, e), generator=gen(e), device="cuda").float()
        x = torch.where(torch.rand(290, e, generator=gen(k), device="cuda") < 0.3, -x * 0.0, x)
        x[:, ::5] = -math.inf
        x[3, 2:] = -math.inf
        x[4] = -math.inf
        x[5] = torch.finfo(DT[dtype]).min
        x[6, e // 2] = torch.finfo(DT[dtype]).max
        x[7] = -x[7].abs() - 1e-30
        for renorm in (False, True):
            check_route(x.to(DT[dtype]), k, renorm)


def test_a_negative_nan_is_not_chosen():
    """NaN of both signs: the others are chosen as without it, their weights are NaN."""
    for dtype in DT.values():
        for t in (20, 400):
            for k in (2, 9):
                x = rand(gen(1), t, 30, dtype)
                y = x.clone()
                for row, bits in ((1, -1), (2, 0x7fff if dtype == torch.bfloat16 else 0x7fffffff)):
                    whole = torch.int16 if dtype == torch.bfloat16 else torch.int32
                    y.view(whole)[row, 4] = bits
                    x[row, 4] = -math.inf
                assert torch.isnan(y[1, 4]) and torch.isnan(y[2, 4])
                a, b = (optcc.occ_route_fwd(v, k, renorm=False) for v in (x, y))
                assert torch.equal(a.index, b.index) and torch.equal(a.slots, b.slots)
                assert torch.isnan(b.weights[1:3]).all()
                rest = [i for i in range(t) if i not in (1, 2)]
                assert torch.equal(a.weights[rest], b.weights[rest])


@pytest.mark.parametrize("t", [255, 256, 257, 511, 512, 513, 65535, 65536, 65537, 140001])
def test_tokens_of_a_block(t):
    """Chunks of 256 tokens, blocks of several chunks."""
    check_route(rand(gen(t), t, 10, torch.bfloat16), 3, True)


def test_every_token_chooses_the_same_experts():
    x = torch.zeros(3000, 40, device="cuda")
    x[:, 7], x[:, 30] = 2.0, 1.0
    r = check_route(x, 2, True)
    assert r.offsets[8] - r.offsets[7] == 3000 and r.offsets[31] - r.offsets[30] == 3000


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("e,k", [(10, 2), (10, 7), (200, 16), (700, 32)])
def test_gradient_of_an_expert_chosen_twice(e, k, dtype):
    """A plan of the caller's own: the parts of equal choices add up, in order."""
    x = rand(gen(e), 70, e, DT[dtype])
    r = optcc.occ_route_fwd(x, k)
    index = r.index.clone()
    index[::3, 1] = index[::3, 0]
    index[5] = 3
    index[6, k // 2:] = -1
    r = r._replace(index=index)
    dw = torch.randn(70, k, generator=gen(k), device="cuda")
    for renorm in (True, False):
        got = optcc.occ_route_bwd(dw, x, r, renorm=renorm)
        within(got, *route_bwd64(x, index, r.weights, dw, renorm), "dlogits")
        assert torch.equal(got, optcc.occ_route_bwd(dw, x, r, renorm=renorm))
