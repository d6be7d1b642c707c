"""A layer of one expert makes the results of the plain layer, bit by bit, where both plans
take the same form, tile and no parts of K."""

import pytest

torch = pytest.importorskip("torch")

import experts_plans  # noqa: E402
import layer_plans  # noqa: E402
from paper_2301_09830_amd import optcc  # noqa: E402

DT = {"bf16": torch.bfloat16, "f32": torch.float32}

# kind, type, gated, (rows, in, out), form, tile
SAME = [
    ("fwd", "bf16", False, (512, 256, 256), "tiled", 64),
    ("fwd", "bf16", False, (2000, 203, 517), "tiled", 64),      # copied first
    ("fwd", "bf16", False, (4096, 1024, 1024), "tiled", 128),
    ("fwd", "bf16", False, (8192, 1024, 4096), "tiled", 256),
    ("fwd", "bf16", True, (2000, 520, 512), "tiled", 64),
    ("fwd", "bf16", True, (2000, 203, 517), "tiled", 128),
    ("fwd", "bf16", True, (8192, 1024, 4096), "tiled", 256),
    ("fwd", "f32", False, (2000, 520, 512), "tiled", 64),
    ("fwd", "f32", False, (2000, 203, 517), "direct", 64),
    ("fwd", "f32", False, (8192, 1024, 4096), "planes", 256),
    ("fwd", "f32", True, (2000, 203, 517), "tiled", 128),
    ("fwd", "f32", True, (8192, 1024, 4096), "planes", 256),
    ("bwd", "bf16", False, (1000, 1024, 1024), "tiled", 64),
    ("bwd", "bf16", True, (2000, 520, 512), "tiled", 64),
    ("bwd", "bf16", True, (4096, 2048, 2048), "tiled", 256),
    ("bwd", "f32", False, (1000, 1024, 1024), "tiled", 64),
    ("bwd", "f32", True, (4096, 2048, 2048), "planes", 256),
]


def act(gated):
    return optcc.OCC_ACT_SILU if gated else optcc.OCC_ACT_GELU


@pytest.mark.skipif(not layer_plans.AVAILABLE, reason="g++ or the HIP headers not available")
def test_the_forms_are_the_same(tmp_path):
    (tmp_path / "layers").mkdir()
    (tmp_path / "experts").mkdir()
    layers = layer_plans.compile_plans(tmp_path / "layers")
    experts = experts_plans.compile_plans(tmp_path / "experts")
    how = [dict(act=act(gated), gated=gated) for _, _, gated, _, _, _ in SAME]
    a = layer_plans.plans(layers, [layer_plans.case(kind, dt, *size, **h)
                                   for (kind, dt, _, size, _, _), h in zip(SAME, how)])
    b = layer_plans.plans(experts, [experts_plans.case(kind, dt, 1, *size, **h)
                                    for (kind, dt, _, size, _, _), h in zip(SAME, how)])
    for (kind, _, _, _, form, tile), p, q in zip(SAME, a, b):
        assert (p["form"], p["tile"]) == (q["form"], q["tile"]) == (form, tile)
        assert p["x_splits"] == 1 and (kind == "fwd" or p["w_splits"] == 1)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dtype,gated,size,form,tile", SAME, ids=str)
def test_one_expert(kind, dtype, gated, size, form, tile):
    (m, k, n), dt, a = size, DT[dtype], act(gated)
    wide = 2 * n if gated else n
    g = torch.Generator(device="cuda").manual_seed(m + k)

    def rand(*shape, scale=1.0, dt=dt):
        return torch.randn(*shape, generator=g, device="cuda").mul_(scale).to(dt)

    print(f"one expert {kind} {dtype} gated {gated} {m}x{k}x{n}", flush=True)
    X, W, at = rand(m, k), rand(wide, k, scale=k ** -0.5), torch.tensor([0, m]).to(torch.int32).cuda()
    if kind == "fwd":
        b, R = rand(wide, dt=torch.float32), rand(m, n)
        Z = [torch.empty(m, wide, dtype=dt, device="cuda") for _ in "ab"]
        f, h = ((optcc.occ_gated_fwd, optcc.occ_experts_gated_fwd) if gated else
                (optcc.occ_linear_fwd, optcc.occ_experts_linear_fwd))
        want = f(X, W, bias=b, act=a, R=R, Z=Z[0])
        got = h(X, W[None], at, bias=b[None], act=a, R=R, Z=Z[1])
        assert torch.equal(got, want) and torch.equal(*Z)
        return
    dY, Z = rand(m, n), rand(m, wide)
    dX, dW = [torch.empty_like(X) for _ in "ab"], [torch.empty_like(W) for _ in "ab"]
    db = [torch.empty(wide, device="cuda") for _ in "ab"]
    f, h = ((optcc.occ_gated_bwd, optcc.occ_experts_gated_bwd) if gated else
            (optcc.occ_linear_bwd, optcc.occ_experts_linear_bwd))
    f(dY, X=X, W=W, Z=Z, act=a, dX=dX[0], dW=dW[0], dbias=db[0])
    h(dY, at, X=X, W=W[None], Z=Z, act=a, dX=dX[1], dW=dW[1][None], dbias=db[1][None])
    assert torch.equal(*dX) and torch.equal(*dW)
