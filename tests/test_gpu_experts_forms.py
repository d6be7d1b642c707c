"""Every form of the experts' products that the plan chooses (tests/experts_forms.py;
tests/test_experts_plans.py checks on the host that these layers take them), with
all parts of the epilogue, against float64."""

import pytest

pytest.importorskip("torch")

from experts_forms import FORMS, split  # noqa: E402
from test_gpu_experts import run_backward, run_forward  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", FORMS, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_forms(case):
    kind, dtype, gated, _, _, _, db, (experts, rows, n_in, out) = case
    sizes, act = split(rows, experts), 4 if gated else 2
    if kind == "fwd":
        run_forward(sizes, n_in, out, dtype, act, gated, seed=rows)
        run_forward(sizes[::-1], n_in, out, dtype, act, gated, bias=False, residual=False,
                    save=False)
    else:
        want = "xwb" if db else "xw"
        run_backward(sizes, n_in, out, dtype, act, gated, want=want, seed=rows)
        run_backward(sizes[::-1], n_in, out, dtype, act, gated, want=want, dw_f32=True,
                     accumulate=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gated", [False, True])
def test_last_rows_of_every_count(gated, dtype):
    """Runs that end in each part of a tile of 256 rows, and dW whose rows do."""
    sizes, n = [257, 383, 384, 385, 512, 1, 128, 129, 0, 255, 256], 1096 if gated else 2192
    run_forward(sizes, 192, n, dtype, 4, gated)
    run_backward(sizes, 520, n, dtype, 4, gated)


@pytest.mark.parametrize("gated", [False, True])
def test_experts_without_rows_have_zeros(gated):
    for sizes, n_in, out in (([0, 0, 700, 0], 516, 1025), ([0, 3, 0], 40, 24)):
        for dtype in ("bf16", "f32"):
            run_backward(sizes, n_in, out, dtype, 4, gated, pad=4, gap=8)
            run_backward(sizes, n_in, out, dtype, 4, gated, dw_f32=True)


def test_no_rows_at_all_have_zeros_in_every_expert():
    """With the experts' gradients next to each other, and apart."""
    import torch
    from paper_2301_09830_amd import optcc

    at = torch.zeros(6, dtype=torch.int32, device="cuda")
    for dt in (torch.bfloat16, torch.float32):
        for gap in (0, 3):
            dW = torch.ones(5, 12 + gap, 40, dtype=dt, device="cuda")
            db = torch.ones(5, 12, device="cuda")
            optcc.occ_experts_gated_bwd(torch.empty(0, 6, dtype=dt, device="cuda"), at,
                                        X=torch.empty(0, 40, dtype=dt, device="cuda"),
                                        Z=torch.empty(0, 12, dtype=dt, device="cuda"),
                                        dW=dW[:, :12], dbias=db)
            assert not dW[:, :12].any() and (dW[:, 12:] == 1).all() and not db.any()
