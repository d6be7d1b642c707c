"""Refusals of the layers' binding that only tensors on a GPU reach."""

import pytest

torch = pytest.importorskip("torch")

from paper_2301_09830_amd import optcc  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", [-1, 5, 1 << 31, 1 << 32, (1 << 32) + 2, -(1 << 32)])
def test_activations_outside_the_list(act):
    """Also numbers whose low 32 bits are an activation's."""
    X, W, dY = torch.ones(8, 16).cuda(), torch.ones(6, 16).cuda(), torch.ones(8, 6).cuda()
    with pytest.raises(optcc.OccError, match="OCC_E_VALUE"):
        optcc.occ_linear_fwd(X, W, act=act)
    with pytest.raises(optcc.OccError, match="OCC_E_VALUE"):
        optcc.occ_linear_bwd(dY, X, W, Z=dY, act=act, dX=torch.empty_like(X))
