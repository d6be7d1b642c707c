"""The linear and gated layers of experts against float64, expert by expert,
inside the layers' derived bounds (tests/stage_ref.py)."""

import pytest

torch = pytest.importorskip("torch")

from paper_2301_09830_amd import optcc  # noqa: E402
from stage_ref import backward64, forward64, within  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rand(g, shape, dtype, scale=1.0, pad=0, shift=0, gap=0):
    """A rows x cols or experts x rows x cols view: `pad` columns of NaN behind each
    row, `gap` elements behind each expert's matrix, the base `shift` elements off."""
    *outer, rows, cols = shape
    ld, n = cols + pad, outer[0] if outer else 1
    step = rows * ld + gap
    buf = torch.full((shift + n * step + 8,), float("nan"), dtype=dtype, device="cuda")
    view = buf.as_strided((n, rows, cols), (step, ld, 1), shift)
    view.copy_(torch.randn(n, rows, cols, generator=g, device="cuda") * scale)
    return view if outer else view[0]


def runs_of(sizes, before=0):
    at = before
    for n in sizes:
        yield slice(at, at + n)
        at += n


def offsets_of(sizes, before=0):
    return torch.tensor([before + sum(sizes[:i]) for i in range(len(sizes) + 1)],
                        dtype=torch.int32, device="cuda")


def untouched(t, sizes, before, value):
    rest = torch.ones(t.shape[0], dtype=torch.bool)
    rest[before:before + sum(sizes)] = False
    assert (t[rest.cuda()] == value).all()


def run_forward(sizes, n_in, n_out, dtype, act, gated, bias=True, residual=True, save=True, pad=0,
                shift=0, gap=0, before=0, behind=0, seed=0):
    g = gen(seed)
    dt, wide, e = DT[dtype], 2 * n_out if gated else n_out, len(sizes)
    m = before + sum(sizes) + behind
    X = rand(g, (m, n_in), dt, 1.0, pad, shift)
    X[:before] = float("nan")          # rows of no expert
    X[m - behind:] = float("nan")
    W = rand(g, (e, wide, n_in), dt, n_in ** -0.5, pad, shift, gap)
    b = torch.randn(e, wide, generator=g, device="cuda") if bias else None
    R = rand(g, (m, n_out), dt, 1.0, pad, shift) if residual else None
    Y = rand(g, (m, n_out), dt, 0.0, pad, shift).fill_(5.0)
    Z = rand(g, (m, wide), dt, 0.0, pad, shift).fill_(5.0) if save else None
    f = optcc.occ_experts_gated_fwd if gated else optcc.occ_experts_linear_fwd
    print(f"forward {sizes if e < 12 else (e, sum(sizes))} x {n_in} x {n_out} {dtype} act {act} "
          f"gated {gated} pad {pad} shift {shift} gap {gap}", flush=True)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    f(X, W, offsets_of(sizes, before), bias=b, act=act, R=R, Y=Y, Z=Z, flags=flags)
    torch.cuda.synchronize()
    assert flags.item() == 0
    for i, r in enumerate(runs_of(sizes, before)):
        if sizes[i]:
            y, z, by, bz = forward64(X[r], W[i], b[i] if bias else None, act,
                                     R[r] if residual else None, gated)
            within(Y[r], y, by, f"Y of {i}")
            if save:
                within(Z[r], z, bz, f"Z of {i}")
    for t in (Y, Z) if save else (Y,):
        untouched(t, sizes, before, 5.0)
        if pad and t.shape[0] > 1:      # what lies between the rows is left alone
            gaps = t.as_strided((t.shape[0] - 1, pad), (t.stride(0), 1),
                                t.storage_offset() + t.shape[1])
            assert torch.isnan(gaps).all()


def run_backward(sizes, n_in, n_out, dtype, act, gated, want="xwb", dw_f32=False, accumulate=False,
                 pad=0, shift=0, gap=0, before=0, behind=0, seed=0):
    g = gen(seed)
    dt, wide, e = DT[dtype], 2 * n_out if gated else n_out, len(sizes)
    m = before + sum(sizes) + behind
    X, dY = rand(g, (m, n_in), dt, 1.0, pad, shift), rand(g, (m, n_out), dt, 0.1, pad, shift)
    W = rand(g, (e, wide, n_in), dt, n_in ** -0.5, pad, shift, gap)
    Z = rand(g, (m, wide), dt, 1.0, pad, shift) if gated or act else None
    for t in (X, dY, Z):
        if t is not None:
            t[:before] = float("nan")
            t[m - behind:] = float("nan")
    dwt = torch.float32 if dw_f32 else dt
    dX = rand(g, (m, n_in), dt, 0.0, pad, shift).fill_(5.0) if "x" in want else None
    dW = rand(g, (e, wide, n_in), dwt, 1.0, pad, shift, gap) if "w" in want else None
    db = torch.randn(e, wide, generator=g, device="cuda") if "b" in want else None
    old_w, old_b = (t.double().clone() if t is not None else None for t in (dW, db))
    f = optcc.occ_experts_gated_bwd if gated else optcc.occ_experts_linear_bwd
    print(f"backward {sizes if e < 12 else (e, sum(sizes))} x {n_in} x {n_out} {dtype} act {act} "
          f"gated {gated} want {want} accumulate {accumulate} pad {pad} shift {shift}", flush=True)
    f(dY, offsets_of(sizes, before), X=X if "w" in want else None, W=W if "x" in want else None,
      Z=Z, act=act, dX=dX, dW=dW, dbias=db, accumulate=accumulate)
    torch.cuda.synchronize()
    u = 2.0 ** -8 if dwt == torch.bfloat16 else 2.0 ** -24
    for i, r in enumerate(runs_of(sizes, before)):
        ref = backward64(dY[r], X[r] if "w" in want else None, W[i] if "x" in want else None,
                         None if Z is None else Z[r], act, gated, dwt)
        if "x" in want and sizes[i]:
            within(dX[r], *ref["dX"], f"dX of {i}")
        for name, got, old in (("dW", dW, old_w), ("dbias", db, old_b)):
            if got is None:
                continue
            v, b = ref[name]
            if accumulate:      # rounded after the addition
                v = v + old[i]
                b = b + (u if name == "dW" else 2.0 ** -24) * 1.01 * (v.abs() + b)
            within(got[i], v, b, f"{name} of {i}")
    if dX is not None:
        untouched(dX, sizes, before, 5.0)


SIZES = [([1], 1, 1), ([1, 0, 2], 7, 3), ([0, 0, 5, 0], 64, 16), ([3, 1, 0, 9, 2], 130, 33),
         ([17, 40, 8], 200, 136), ([64, 65, 63], 96, 72), ([100, 0, 300, 29], 520, 129),
         ([700, 5], 96, 520), ([128, 256, 384], 256, 256), ([1] * 70, 72, 48),
         ([0] * 100 + [90] + [0] * 60, 64, 80)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("case", range(len(SIZES)))
def test_forward_sizes(case, gated, dtype):
    run_forward(*SIZES[case], dtype, act=4 if gated else 2, gated=gated, seed=case)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("case", range(len(SIZES)))
def test_backward_sizes(case, gated, dtype):
    run_backward(*SIZES[case], dtype, act=4 if gated else 2, gated=gated, seed=case)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", range(5))
def test_activations(act, gated, dtype):
    for sizes in ([3, 0, 6], [140, 90]):
        run_forward(sizes, 96, 72, dtype, act, gated)
        run_backward(sizes, 96, 72, dtype, act, gated)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("pad,shift,gap", [(0, 1, 0), (1, 0, 0), (8, 0, 40), (3, 5, 7), (0, 0, 1)])
def test_strides(pad, shift, gap, gated, dtype):
    for sizes in ([4, 0, 11], [150, 99]):
        run_forward(sizes, 200, 136, dtype, 3, gated, pad=pad, shift=shift, gap=gap)
        run_backward(sizes, 200, 136, dtype, 3, gated, pad=pad, shift=shift, gap=gap)
        run_backward(sizes, 200, 136, dtype, 0, gated, pad=pad, shift=shift, gap=gap)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_no_expert_are_left_alone(dtype):
    """Rows before the first offset and behind the last, NaN in every input."""
    for sizes in ([2, 0, 3], [33, 80, 0], [300, 140]):
        for gated in (False, True):
            run_forward(sizes, 136, 80, dtype, 2, gated, before=5, behind=70)
            run_backward(sizes, 136, 80, dtype, 2, gated, before=5, behind=70)


@pytest.mark.parametrize("bias,residual,save", [(0, 0, 0), (1, 0, 0), (0, 1, 0), (0, 0, 1)])
def test_forward_optional_parts(bias, residual, save):
    for sizes in ([2, 3], [120, 80]):
        for gated in (False, True):
            run_forward(sizes, 128, 96, "bf16", 4, gated, bool(bias), bool(residual), bool(save))


@pytest.mark.parametrize("want", ["x", "w", "b", "xw", "xb", "wb"])
@pytest.mark.parametrize("act", [0, 3])
def test_backward_outputs_alone(want, act):
    for sizes in ([2, 0, 3], [220, 80]):
        for dtype in DT:
            run_backward(sizes, 128, 96, dtype, act, False, want=want)


@pytest.mark.parametrize("dtype,dw_f32", [("bf16", False), ("bf16", True), ("f32", False)])
def test_backward_accumulates(dtype, dw_f32):
    for sizes in ([2, 0, 3], [220, 0, 80]):
        for gated in (False, True):
            run_backward(sizes, 128, 96, dtype, 4, gated, dw_f32=dw_f32, accumulate=True)
            run_backward(sizes, 128, 96, dtype, 4, gated, dw_f32=dw_f32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gated", [False, True])
def test_large_tiles(gated, dtype):
    """Results large enough for the 256 x 256 tiles, ragged on every side; many
    experts; every form that the plan has for them."""
    n = 1032 if gated else 2072
    run_forward([2100, 0, 1500, 601], 200, n, dtype, 2, gated)
    run_backward([2100, 0, 1500, 601], 520, n, dtype, 2, gated)
    run_forward([900, 1100], 203, n, dtype, 2, gated)
    run_backward([900, 1100], 203, n + 1, dtype, 2, gated)
    run_forward([(7 * i) % 90 for i in range(130)], 264, 200, dtype, 4, gated)
    run_backward([(7 * i) % 90 for i in range(130)], 264, 200, dtype, 4, gated)


def test_1024_experts():
    sizes = [i % 3 for i in range(1024)]
    run_forward(sizes, 32, 24, "bf16", 0, False)
    run_backward(sizes, 32, 24, "bf16", 4, True)
    sizes = [0] * 1024
    sizes[1000] = 500
    run_forward(sizes, 32, 24, "bf16", 0, False)
    run_backward(sizes, 32, 24, "bf16", 1, False)


def test_one_expert_is_a_layer():
    """The results of the layer itself, bit by bit, where the forms are the same."""
    for dt in DT.values():
        g = gen(1)
        X, W = rand(g, (512, 256), dt), rand(g, (1, 256, 256), dt, 0.1)
        at = torch.tensor([0, 512], dtype=torch.int32, device="cuda")
        got = optcc.occ_experts_linear_fwd(X, W, at, act=4)
        want = optcc.occ_linear_fwd(X, W[0], act=4)
        u = 2.0 ** -7 if dt == torch.bfloat16 else 2.0 ** -16
        assert torch.allclose(got, want, rtol=u, atol=u)


def test_residual_in_place():
    for sizes in ([5, 3], [200, 120]):
        g = gen(1)
        m = sum(sizes)
        X, W = rand(g, (m, 100), torch.bfloat16), rand(g, (2, 60, 100), torch.bfloat16, 0.1)
        R = rand(g, (m, 60), torch.bfloat16)
        want = optcc.occ_experts_linear_fwd(X, W, offsets_of(sizes), act=4, R=R)
        got = R.clone()
        optcc.occ_experts_linear_fwd(X, W, offsets_of(sizes), act=4, R=got, Y=got)
        assert torch.equal(got, want)


def test_rows_do_not_depend_on_their_neighbours():
    """Infinities and NaN in one row stay in its results, and in the weight
    gradient of its expert."""
    for sizes in ([4, 3, 2], [150, 90, 60]):
        g, m, at = gen(2), sum(sizes), offsets_of(sizes)
        X, W = rand(g, (m, 130), torch.bfloat16), rand(g, (3, 70, 130), torch.bfloat16, 0.1)
        dY = rand(g, (m, 70), torch.bfloat16)
        bad = sizes[0] + 1
        Y = X.clone()
        Y[bad, 129] = float("nan")
        want, got = (optcc.occ_experts_linear_fwd(x, W, at, act=2) for x in (X, Y))
        rest = [i for i in range(m) if i != bad]
        assert torch.equal(got[rest], want[rest]) and torch.isnan(got[bad]).all()
        dW = [torch.empty_like(W) for _ in "ab"]
        for x, d in zip((X, Y), dW):
            optcc.occ_experts_linear_bwd(dY, at, X=x, dW=d)
        assert torch.equal(dW[0][[0, 2]], dW[1][[0, 2]])
        assert torch.isnan(dW[1][1, :, 129]).all()
        assert torch.equal(dW[0][1, :, :129], dW[1][1, :, :129])


@pytest.mark.parametrize("rows", [9, 300])
def test_bad_offsets_raise_their_flag(rows):
    """Offsets that fall or leave the rows: taken as the header says, no row
    written twice, the flag raised."""
    g = gen(3)
    X, W = rand(g, (rows, 64), torch.float32), rand(g, (3, 40, 64), torch.float32, 0.1)
    dY = rand(g, (rows, 40), torch.float32)
    third = rows // 3
    for given, taken in (([0, 2 * third, third, rows], [0, 2 * third, 2 * third, rows]),
                         ([-5, third, 2 * third, rows + 9], [0, third, 2 * third, rows]),
                         ([0, 1 << 30, third, -1], [0, rows, rows, rows])):
        results = []
        for values, raised in ((given, optcc.OCC_F_BAD_ROWS), (taken, 0)):
            at = torch.tensor(values, dtype=torch.int32, device="cuda")
            flags = torch.zeros(1, dtype=torch.int32, device="cuda")
            Y = torch.full((rows, 40), 5.0, device="cuda")
            optcc.occ_experts_linear_fwd(X, W, at, Y=Y, flags=flags)
            assert flags.item() == raised
            flags.zero_()
            dX, dW = torch.full((rows, 64), 5.0, device="cuda"), torch.empty_like(W)
            db = torch.empty(3, 40, device="cuda")
            optcc.occ_experts_linear_bwd(dY, at, X=X, W=W, dX=dX, dW=dW, dbias=db, flags=flags)
            assert flags.item() == raised
            results.append((Y, dX, dW, db))
        assert all(torch.equal(a, b) for a, b in zip(*results))


def test_no_rows():
    W, at = torch.ones(3, 8, 16, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    X = torch.empty(0, 16, device="cuda")
    assert optcc.occ_experts_linear_fwd(X, W, at).shape == (0, 8)
    dW, db = torch.ones_like(W), torch.ones(3, 8, device="cuda")
    optcc.occ_experts_linear_bwd(torch.empty(0, 8, device="cuda"), at, X=X, dW=dW, dbias=db,
                                 accumulate=True)
    assert (dW == 1).all() and (db == 1).all()
    gaps = torch.ones(3, 10, 20, device="cuda")
    optcc.occ_experts_linear_bwd(torch.empty(0, 8, device="cuda"), at, X=X, dW=gaps[:, :8, :16],
                                 dbias=db)
    assert not gaps[:, :8, :16].any() and (gaps[:, 8:] == 1).all() and not db.any()


def test_results_repeat():
    sizes = [500, 0, 130, 77, 900]
    g, m, at = gen(4), sum(sizes), offsets_of(sizes)
    for dt in DT.values():
        X, W = rand(g, (m, 264), dt), rand(g, (5, 400, 264), dt, 0.1)
        Z, dY = rand(g, (m, 400), dt), rand(g, (m, 200), dt)
        first = None
        for _ in range(3):
            dX, dW = torch.empty_like(X), torch.empty_like(W)
            db = torch.empty(5, 400, device="cuda")
            Y = optcc.occ_experts_gated_fwd(X, W, at)
            optcc.occ_experts_gated_bwd(dY, at, X=X, W=W, Z=Z, dX=dX, dW=dW, dbias=db)
            out = (Y, dX, dW, db)
            first = first or out
            assert all(torch.equal(a, b) for a, b in zip(out, first))


def test_gradient_by_differences():
    """dX, dW and dbias of a small gated layer against central differences of the
    float64 forward pass."""
    sizes = [3, 0, 2]
    g, at = gen(5), offsets_of(sizes)
    X, W = rand(g, (5, 4), torch.float32), rand(g, (3, 6, 4), torch.float32)
    b, dY = torch.randn(3, 6, generator=g, device="cuda"), rand(g, (5, 3), torch.float32)
    Z = torch.empty(5, 6, device="cuda")
    optcc.occ_experts_gated_fwd(X, W, at, bias=b, Z=Z)
    dX, dW, db = torch.empty_like(X), torch.empty_like(W), torch.empty_like(b)
    optcc.occ_experts_gated_bwd(dY, at, X=X, W=W, Z=Z, dX=dX, dW=dW, dbias=db)

    def loss(x, w, c):
        total = 0.0
        for i, r in enumerate(runs_of(sizes)):
            z = x[r] @ w[i].t() + c[i]
            total = total + (torch.nn.functional.silu(z[:, :3]) * z[:, 3:] * dY[r].double()).sum()
        return float(total)

    args, h = [t.double() for t in (X, W, b)], 1e-5
    for got, v in zip((dX, dW, db), args):
        flat = v.view(-1)
        for i in range(flat.numel()):
            keep = flat[i].item()
            ends = []
            for step in (h, -h):
                flat[i] = keep + step
                ends.append(loss(*args))
            flat[i] = keep
            num = (ends[0] - ends[1]) / (2 * h)
            assert abs(got.view(-1)[i].item() - num) <= 2e-5 * (1 + abs(num))


def test_graphs_with_one_workspace():
    """Forward and backward captured into two graphs that share a workspace, replayed in
    turns with eager work and new offsets between."""
    g, m, e = gen(6), 400, 4
    X, W = rand(g, (m, 201), torch.bfloat16), rand(g, (e, 130, 201), torch.bfloat16, 0.1)
    dY = rand(g, (m, 130), torch.bfloat16)
    at = offsets_of([100, 50, 200, 50])
    Y, Z = torch.empty(m, 130, dtype=torch.bfloat16, device="cuda"), None
    Z = torch.empty_like(Y)
    dX, dW = torch.empty_like(X), torch.empty_like(W)
    ws = optcc.alloc_workspace(1 << 26)

    def forward():
        optcc.occ_experts_linear_fwd(X, W, at, act=2, Y=Y, Z=Z, ws=ws)

    def backward():
        optcc.occ_experts_linear_bwd(dY, at, X=X, W=W, Z=Z, act=2, dX=dX, dW=dW, ws=ws)

    graphs = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        forward()
        backward()
    torch.cuda.current_stream().wait_stream(side)
    for call in (forward, backward):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append(graph)
    for sizes in ([100, 50, 200, 50], [0, 400, 0, 0], [1, 2, 300, 97]):
        at.copy_(offsets_of(sizes))
        X.mul_(0.5)
        forward()
        backward()
        want = [t.clone() for t in (Y, Z, dX, dW)]
        for t in (Y, Z, dX, dW):
            t.zero_()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((Y, Z, dX, dW), want))
