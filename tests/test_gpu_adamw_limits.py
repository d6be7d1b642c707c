"""AdamW at the ends of what the interface admits (tests/test_gpu_adamw.py)."""

import pytest

torch = pytest.importorskip("torch")

from paper_2301_09830_amd import optcc  # noqa: E402
from test_gpu_adamw import B1, B2, EPS, LR, State, check  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 32])
def test_more_blocks_than_a_launch_holds(bits):
    """2^27 rows of one column with 8-bit moments are 2^24 blocks of 256 threads
    (32-bit moments: 2^27 elements, few blocks).  Between two small tensors of
    the same kind; rows at both ends and around each 2^23 blocks against
    float64, the rest stays zero."""
    rows = (1 << 27) + 1003
    cut = ((1 << 32) - 1) // 512 * 8
    at = torch.cat([torch.arange(16), torch.arange(cut - 8, cut + 8),
                    torch.arange(2 * cut - 8, 2 * cut + 8), torch.arange(rows - 16, rows)]).cuda()
    s = State(64, 1, bits, "f32", seed=1, copy=False)
    small = [State(5, 300, bits, "f32", seed=2, copy=False), State(3, 77, bits, "f32", seed=3, copy=False)]
    names = ["W", "G", "m", "v"] + (["m_scale", "v_scale"] if bits == 8 else [])
    big = {k: torch.zeros(rows, 1, dtype=getattr(s, k).dtype, device="cuda") for k in names}
    for k in names:
        big[k][at] = getattr(s, k)
    refs = [x.reference(4) for x in [s] + small]
    p = optcc.make_param(big["W"], big["m"], big["v"], G=big["G"], m_scale=big.get("m_scale"),
                         v_scale=big.get("v_scale"), decay=s.decay)
    print(f"adamw of {rows} rows, {bits} bits", flush=True)
    optcc.occ_adamw_step([small[0].param(), p, small[1].param()], LR, 4, B1, B2, EPS)
    torch.cuda.synchronize()
    for k in names:
        getattr(s, k).copy_(big[k][at])
        if k in ("W", "m", "v"):
            big[k][at] = 0
            assert not big[k].any(), k
    for x, ref, what in zip([s] + small, refs, ("large", "first", "last")):
        check(x, ref, what)
