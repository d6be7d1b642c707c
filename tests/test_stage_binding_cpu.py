"""What the Python binding of the stage operators refuses before a kernel sees
it, and what it keeps alive.  Host checks: no GPU."""

import pytest

torch = pytest.importorskip("torch")

from paper_2301_09830_amd import optcc  # noqa: E402


# --- a workspace given by the caller -----------------------------------------
def layer_calls(ws):
    X, W, dY = torch.zeros(8, 16), torch.zeros(6, 16), torch.zeros(8, 6)
    yield lambda: optcc.occ_linear_fwd(X, W, ws=ws)
    yield lambda: optcc.occ_gated_fwd(X, W, ws=ws)
    yield lambda: optcc.occ_linear_bwd(dY, X, W, dX=torch.zeros(8, 16), ws=ws)
    yield lambda: optcc.occ_gated_bwd(dY, X, torch.zeros(12, 16), Z=torch.zeros(8, 12),
                                      dW=torch.zeros(12, 16), ws=ws)


@pytest.mark.parametrize("ws,what", [
    (torch.empty(4096, dtype=torch.uint8, device="meta"), "ws lies on another device"),
    (torch.empty(8192, dtype=torch.uint8)[::2], "ws must be contiguous"),
    (torch.empty(64, 64).t()[:, 1:], "ws must be contiguous")], ids=["device", "step", "turned"])
def test_workspace_is_checked(ws, what):
    for call in layer_calls(ws):
        with pytest.raises(ValueError, match=what):
            call()


def test_workspace_must_be_a_tensor():
    for call in layer_calls(4096):
        with pytest.raises(TypeError, match="ws must be a tensor"):
            call()
