"""Layers at the ends of what the interface admits, against float64."""

import pytest

torch = pytest.importorskip("torch")

from paper_2301_09830_amd import optcc  # noqa: E402
from stage_ref import backward64, forward64, within  # noqa: E402

pytestmark = pytest.mark.gpu


def test_more_tokens_than_small_tiles_have_blocks():
    """2^29 tokens and some: in 64 x 64 tiles that would be 2^32 threads.  All
    rows but the first and last few are zero, so float64 results of those are the
    whole layer's."""
    tokens, n, k = (1 << 29) + 77, 8, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    X = torch.zeros(tokens, k, dtype=torch.bfloat16, device="cuda")
    ends = [slice(0, 70), slice(tokens - 70, tokens)]
    for rows in ends:
        X[rows] = torch.randn(70, k, generator=g, device="cuda").to(torch.bfloat16)
    W = torch.randn(n, k, generator=g, device="cuda").to(torch.bfloat16)
    print(f"layer of {tokens} tokens", flush=True)
    Y = optcc.occ_linear_fwd(X, W)
    for rows in ends:
        y, _, by, _ = forward64(X[rows], W, None, 0, None, False)
        within(Y[rows], y, by, "Y")
    middle = torch.arange(70, tokens - 70, 1000003, device="cuda")
    assert not Y[middle].any()
    dX, dW, db = torch.empty_like(X), torch.empty_like(W), torch.empty(n, device="cuda")
    optcc.occ_linear_bwd(Y, X, W, dX=dX, dW=dW, dbias=db)
    cat = torch.cat([Y[r] for r in ends]), torch.cat([X[r] for r in ends])
    ref = backward64(*cat, W, None, 0, False)
    within(torch.cat([dX[r] for r in ends]), *ref["dX"], "dX")
    within(dW, *ref["dW"], "dW")
    within(db, *ref["dbias"], "dbias")
    assert not dX[middle].any()
