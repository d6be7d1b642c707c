"""The router's gradient for more tokens than one launch holds, at both ends of every
launch, against the same tokens in a small call."""

import pytest

torch = pytest.importorskip("torch")

from paper_2301_09830_amd import optcc  # noqa: E402

pytestmark = pytest.mark.gpu

PART = ((1 << 32) - 1) // 256 * 16     # tokens of a launch, 16 lanes each


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_of_more_tokens_than_a_launch(renorm):
    t, e, k = PART + 1037, 4, 1
    at = torch.cat([torch.arange(i, i + 64) for i in (0, PART - 64, PART, t - 64)]).cuda()
    print(f"route_bwd {t} x {e} k {k}", flush=True)
    logits = torch.zeros(t, e, dtype=torch.bfloat16, device="cuda")
    logits[at] = torch.randn(len(at), e, generator=gen(1), device="cuda").to(torch.bfloat16)
    weights, dw = torch.ones(t, k, device="cuda"), torch.ones(t, k, device="cuda")
    weights[at] = torch.rand(len(at), k, generator=gen(2), device="cuda")
    dw[at] = torch.randn(len(at), k, generator=gen(3), device="cuda")
    index = torch.zeros(t, k, dtype=torch.int32, device="cuda")
    index[at] = torch.randint(0, e, (len(at), k), generator=gen(4), device="cuda", dtype=torch.int32)

    def route(i, w):
        return optcc.Route(i, w, None, None, None)

    small = optcc.occ_route_bwd(dw[at], logits[at], route(index[at], weights[at]), renorm=renorm)
    got = optcc.occ_route_bwd(dw, logits, route(index, weights), renorm=renorm,
                              dlogits=torch.full_like(logits, 7.0))
    assert torch.equal(got[at], small)
    # between them: logits 0, weight and gradient 1, the first expert chosen
    p = torch.zeros(e) if renorm else torch.full((e,), -1 / e)
    p[0] += 0.0 if renorm else 1.0
    rest = torch.ones(t, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert (got[rest] == p.to(torch.bfloat16).cuda()).all()
