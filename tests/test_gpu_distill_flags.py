"""A column out of the vocabulary raises OCC_F_BAD_ROWS of any token, also of one that has
no part in the loss; lists and labels that alpha leaves out do not."""

import pytest

torch = pytest.importorskip("torch")

from paper_2301_09830_amd import optcc  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("alpha", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("what", ["label", "list", "neither"])
@pytest.mark.parametrize("t,v", [(5, 100), (300, 600), (3, 230000)])
def test_token_without_a_part(t, v, what, alpha):
    g = torch.Generator(device="cuda").manual_seed(v)
    S = torch.randn(t, v, generator=g, device="cuda")
    index = torch.randint(0, v, (t, 70), generator=g, device="cuda", dtype=torch.int32)
    teacher = torch.randn(t, 70, generator=g, device="cuda")
    labels = torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32)
    scale = torch.rand(t, generator=g, device="cuda") + 0.5
    scale[1] = 0.0
    S[1] = float("nan")
    if what == "label":
        labels[1] = v
    elif what == "list":
        index[1, 69] = v
    raised = (what == "label" and alpha < 1) or (what == "list" and alpha > 0)
    how = dict(temperature=2.0, alpha=alpha, labels=labels, scale=scale)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    lse, dS = torch.full((t, 2), 7.0, device="cuda"), torch.full_like(S, 7.0)
    loss = optcc.occ_distill_fwd(S, index, teacher, **how, lse=lse, dS=dS, flags=flags)
    assert flags.item() == (optcc.OCC_F_BAD_ROWS if raised else 0)
    assert loss[1] == 0 and not lse[1].any() and not dS[1].any()
    assert torch.isfinite(loss).all() and torch.isfinite(dS).all()
    # without a word for it, the same
    again = torch.full_like(S, 7.0)
    assert torch.equal(optcc.occ_distill_fwd(S, index, teacher, **how, dS=again), loss)
    assert torch.equal(again, dS)
    flags.zero_()
    back = optcc.occ_distill_bwd(S, index, teacher, lse, **how, flags=flags)
    assert flags.item() == (optcc.OCC_F_BAD_ROWS if raised else 0)
    assert not back[1].any() and torch.isfinite(back).all()
