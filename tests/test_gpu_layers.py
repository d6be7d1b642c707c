"""The linear and gated layers against float64, element by element, inside
derived bounds (tests/stage_ref.py)."""

import pytest

torch = pytest.importorskip("torch")

from paper_2301_09830_amd import optcc  # noqa: E402
from stage_ref import backward64, forward64, within  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rand(g, rows, cols, dtype, scale=1.0, pad=0, shift=0):
    """A rows x cols view with `pad` columns of NaN behind each row, whose base
    is `shift` elements off its allocation."""
    ld = cols + pad
    buf = torch.full((shift + rows * ld + 8,), float("nan"), dtype=dtype, device="cuda")
    view = buf[shift:shift + rows * ld].view(rows, ld)[:, :cols]
    view.copy_(torch.randn(rows, cols, generator=g, device="cuda") * scale)
    return view


def run_forward(tokens, n_in, n_out, dtype, act, gated, bias=True, residual=True, save=True,
                pad=0, shift=0, seed=0):
    g = gen(seed)
    dt, wide = DT[dtype], 2 * n_out if gated else n_out
    X = rand(g, tokens, n_in, dt, 1.0, pad, shift)
    W = rand(g, wide, n_in, dt, n_in ** -0.5, pad, shift)
    b = torch.randn(wide, generator=g, device="cuda") if bias else None
    R = rand(g, tokens, n_out, dt, 1.0, pad, shift) if residual else None
    Y = rand(g, tokens, n_out, dt, 0.0, pad, shift)
    Z = rand(g, tokens, wide, dt, 0.0, pad, shift) if save else None
    f = optcc.occ_gated_fwd if gated else optcc.occ_linear_fwd
    print(f"forward {tokens}x{n_in}x{n_out} {dtype} act {act} gated {gated} pad {pad} shift {shift}",
          flush=True)
    f(X, W, bias=b, act=act, R=R, Y=Y, Z=Z)
    torch.cuda.synchronize()
    y, z, by, bz = forward64(X, W, b, act, R, gated)
    within(Y, y, by, "Y")
    if save:
        within(Z, z, bz, "Z")
    if pad and tokens > 1:      # what lies between the rows is left alone
        for t in (Y, Z) if save else (Y,):
            gap = t.as_strided((t.shape[0] - 1, pad), (t.stride(0), 1),
                               t.storage_offset() + t.shape[1])
            assert torch.isnan(gap).all()


# a tile is 128 or 256 rows and columns and 64 (bf16) or 32 (fp32) of K; up to
# 64 tokens go another way, in groups of 16
SIZES = [(1, 1, 1), (1, 64, 16), (1, 4096, 256), (2, 7, 3), (15, 31, 17), (16, 128, 33),
         (17, 1000, 16), (33, 65, 130), (64, 520, 48), (65, 64, 128), (65, 1, 1), (100, 63, 127),
         (128, 8, 129), (129, 72, 256), (257, 200, 257), (300, 1023, 513), (700, 96, 1100),
         (128, 8192, 130)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_forward_sizes(size, gated, dtype):
    run_forward(*size, dtype, act=4 if gated else 2, gated=gated, seed=sum(size))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", range(5))
def test_forward_activations(act, gated, dtype):
    run_forward(130, 96, 72, dtype, act, gated)
    run_forward(9, 96, 72, dtype, act, gated)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (8, 0), (3, 5), (40, 8)])
def test_forward_strides(pad, shift, gated, dtype):
    run_forward(150, 200, 136, dtype, 3, gated, pad=pad, shift=shift)
    run_forward(19, 200, 136, dtype, 3, gated, pad=pad, shift=shift)


@pytest.mark.parametrize("bias,residual,save", [(0, 0, 0), (1, 0, 0), (0, 1, 0), (0, 0, 1)])
def test_forward_optional_parts(bias, residual, save):
    for tokens in (5, 200):
        for gated in (False, True):
            run_forward(tokens, 128, 96, "bf16", 4, gated, bool(bias), bool(residual), bool(save))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gated", [False, True])
def test_forward_large_tiles(gated, dtype):
    """Results large enough for the 256 x 256 tiles, ragged on every side."""
    run_forward(4100, 200, 2060 if gated else 4150, dtype, 2, gated)


def test_residual_in_place():
    for tokens in (5, 200):
        g = gen(1)
        X, W = rand(g, tokens, 100, torch.bfloat16), rand(g, 60, 100, torch.bfloat16, 0.1)
        R = rand(g, tokens, 60, torch.bfloat16)
        want = optcc.occ_linear_fwd(X, W, act=4, R=R)
        got = R.clone()
        optcc.occ_linear_fwd(X, W, act=4, R=got, Y=got)
        assert torch.equal(got, want)


def test_rows_do_not_depend_on_their_neighbours():
    """Infinities and NaN in one token's input stay in that token's output."""
    for tokens in (7, 200):
        g = gen(2)
        X, W = rand(g, tokens, 130, torch.bfloat16), rand(g, 70, 130, torch.bfloat16, 0.1)
        want = optcc.occ_linear_fwd(X, W, act=2)
        X[3, 129] = float("inf")
        X[5, 0] = float("nan")
        got = optcc.occ_linear_fwd(X, W, act=2)
        rest = [t for t in range(tokens) if t not in (3, 5)]
        assert torch.equal(got[rest], want[rest])
        assert torch.isnan(got[5]).all() and not torch.isfinite(got[3]).all()


@pytest.mark.parametrize("act", range(5))
def test_extreme_preactivations(act):
    """Pre-activations far outside the exponential's range: act and act' end at
    their limits (0 or z; 0 or 1)."""
    far = [-3e38, -1e30, -1e20, -1e10, -500.0, -100.0, 100.0, 500.0, 1e10, 1e20, 1e30]
    for tokens in (11, 66):
        z = torch.tensor((far * 6)[:tokens], device="cuda").view(-1, 1)
        one = torch.ones(1, 1, device="cuda")
        y = optcc.occ_linear_fwd(z, one, act=act)
        want = z if act == 0 else z.clamp_min(0)
        assert torch.isfinite(y).all() and torch.allclose(y, want, rtol=1e-6, atol=1e-30)
        dX = torch.empty_like(z)
        optcc.occ_linear_bwd(torch.ones_like(z), W=one, Z=z, act=act, dX=dX)
        d = torch.ones_like(z) if act == 0 else (z > 0).float()
        assert torch.allclose(dX, d, rtol=1e-5, atol=1e-30)


def run_backward(tokens, n_in, n_out, dtype, act, gated, pad=0, shift=0, dw=None, seed=0,
                 accumulate=False):
    g = gen(seed)
    dt, wide = DT[dtype], 2 * n_out if gated else n_out
    dw_dt = DT[dw or dtype]
    dY = rand(g, tokens, n_out, dt, 1.0, pad, shift)
    X = rand(g, tokens, n_in, dt, 1.0, pad, shift)
    W = rand(g, wide, n_in, dt, n_in ** -0.5, pad, shift)
    Z = rand(g, tokens, wide, dt, 1.5, pad, shift) if gated or act else None
    dX = rand(g, tokens, n_in, dt, 0.0, pad, shift)
    dW = rand(g, wide, n_in, dw_dt, 1.0, pad, shift)
    db = torch.randn(wide, generator=g, device="cuda")
    dW0, db0 = dW.double(), db.double()
    f = optcc.occ_gated_bwd if gated else optcc.occ_linear_bwd
    print(f"backward {tokens}x{n_in}x{n_out} {dtype} act {act} gated {gated} pad {pad} {shift}",
          flush=True)
    f(dY, X, W, Z=Z, act=act, dX=dX, dW=dW, dbias=db, accumulate=accumulate)
    torch.cuda.synchronize()
    ref = backward64(dY, X, W, Z, act, gated, dw_dt)
    within(dX, *ref["dX"], "dX")
    for name, got, old in (("dW", dW, dW0), ("dbias", db, db0)):
        v, b = ref[name]
        if accumulate:
            u = 2.0 ** -8 * 1.01 if got.dtype == torch.bfloat16 else 2.0 ** -22
            v, b = v + old, b + u * (v.abs() + old.abs())
        within(got, v, b, name)
    return dX, dW, db


BWD_SIZES = [(1, 1, 1), (1, 64, 64), (2, 7, 3), (31, 33, 55), (64, 128, 128), (65, 100, 129),
             (200, 257, 70), (513, 136, 264), (1000, 63, 500), (8000, 72, 40), (33, 4096, 24)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("size", BWD_SIZES, ids=lambda s: "x".join(map(str, s)))
def test_backward_sizes(size, gated, dtype):
    run_backward(*size, dtype, act=4 if gated else 2, gated=gated, seed=sum(size))
    if not gated:
        run_backward(*size, dtype, act=0, gated=False, seed=sum(size))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", range(5))
def test_backward_activations(act, gated, dtype):
    run_backward(130, 96, 72, dtype, act, gated)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (8, 0), (3, 5), (40, 8)])
def test_backward_strides(pad, shift, gated):
    for dtype in ("bf16", "f32"):
        run_backward(150, 200, 136, dtype, 3, gated, pad=pad, shift=shift)
        if not gated:
            run_backward(150, 200, 136, dtype, 0, gated, pad=pad, shift=shift)


@pytest.mark.parametrize("gated", [False, True])
def test_backward_large_tiles(gated):
    run_backward(4100, 2056, 1040 if gated else 2090, "bf16", 4, gated)
    run_backward(2100, 2060, 2080, "f32", 4, gated)


@pytest.mark.parametrize("dtype,dw", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_accumulation(dtype, dw):
    for size in ((200, 130, 72), (4096, 64, 64)):      # the second splits K
        for gated in (False, True):
            run_backward(*size, dtype, 4, gated, dw=dw, accumulate=True)


def test_fp32_weight_gradient_of_a_bf16_layer():
    run_backward(300, 130, 72, "bf16", 0, False, dw="f32")


def test_single_outputs_agree_with_all_of_them():
    g = gen(5)
    dY, X = rand(g, 200, 72, torch.bfloat16), rand(g, 200, 130, torch.bfloat16)
    W, Z = rand(g, 72, 130, torch.bfloat16, 0.1), rand(g, 200, 72, torch.bfloat16)
    make = lambda: (torch.empty_like(X), torch.empty_like(W), torch.empty(72, device="cuda"))  # noqa: E731
    dX, dW, db = make()
    optcc.occ_linear_bwd(dY, X, W, Z=Z, act=2, dX=dX, dW=dW, dbias=db)
    x, w, b = make()
    optcc.occ_linear_bwd(dY, W=W, Z=Z, act=2, dX=x)
    optcc.occ_linear_bwd(dY, X=X, Z=Z, act=2, dW=w)
    optcc.occ_linear_bwd(dY, Z=Z, X=X, act=2, dbias=b)
    assert torch.equal(x, dX) and torch.equal(w, dW) and torch.equal(b, db)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", range(5))
def test_gradients_against_differences(act, gated):
    """<dW, V>, <dX, V> and <db, v> against central differences of the loss
    sum(C * Y) through the layer's own fp32 forward pass.

    With steps of h in a direction scaled so that z moves by about h, the
    difference is off by h^2 / 6 of the third derivative (below 2 for these
    functions) and by the rounding of Y (2^-23 of its size) over h: for
    h = 2e-2 both are below 2e-4 of sum |C|.  Where relu's argument changes its
    sign within the difference, an element's quotient may be off by the
    argument's whole slope: those elements are counted from Z itself."""
    g = gen(act + 10 * gated)
    t, k, n, h = 96, 64, 40, 2e-2
    wide = 2 * n if gated else n
    f32 = torch.float32
    X, W = rand(g, t, k, f32), rand(g, wide, k, f32, k ** -0.5)
    b = torch.randn(wide, generator=g, device="cuda") * 0.1
    C = torch.randn(t, n, generator=g, device="cuda")
    fwd = optcc.occ_gated_fwd if gated else optcc.occ_linear_fwd
    bwd = optcc.occ_gated_bwd if gated else optcc.occ_linear_bwd
    Z = torch.empty(t, wide, device="cuda")
    fwd(X, W, bias=b, act=act, Z=Z)
    dX, dW, db = torch.empty_like(X), torch.empty_like(W), torch.empty(wide, device="cuda")
    bwd(C, X, W, Z=Z, act=act, dX=dX, dW=dW, dbias=db)

    def loss(x, w, c):
        return float((fwd(x, w, bias=c, act=act).double() * C.double()).sum())

    def kinks(up, down):
        if act != optcc.OCC_ACT_RELU:
            return 0.0
        z = []
        for x, w, c in (up, down):
            z.append(torch.empty(t, wide, device="cuda"))
            fwd(x, w, bias=c, act=act, Z=z[-1])
        hit = (z[0][:, :n] > 0) != (z[1][:, :n] > 0)
        slope = (z[0] - z[1])[:, :n].abs() / (2 * h) * C.abs()
        if gated:
            slope = slope * torch.maximum(z[0][:, n:].abs(), z[1][:, n:].abs())
        return float(slope[hit].sum())

    scale = float(C.abs().sum())
    VX, VW = torch.randn_like(X), torch.randn_like(W) * k ** -0.5
    vb = torch.randn_like(b)
    for grad, v, at in ((dX, VX, lambda s: (X + s * VX, W, b)),
                        (dW, VW, lambda s: (X, W + s * VW, b)),
                        (db, vb, lambda s: (X, W, b + s * vb))):
        want = (loss(*at(h)) - loss(*at(-h))) / (2 * h)
        got = float((grad.double() * v.double()).sum())
        far = 1e-3 * scale * (2 if gated else 1) + kinks(at(h), at(-h))
        assert abs(got - want) <= far, (act, gated, got, want)


def test_no_tokens():
    for dt in (torch.bfloat16, torch.float32):
        X = torch.empty(0, 24, dtype=dt, device="cuda")
        W = torch.randn(10, 24, device="cuda").to(dt)
        assert optcc.occ_linear_fwd(X, W).shape == (0, 10)
        dW, db = torch.full_like(W, 7), torch.full((10,), 7.0, device="cuda")
        dY = torch.empty(0, 10, dtype=dt, device="cuda")
        optcc.occ_linear_bwd(dY, X, W, dX=torch.empty_like(X), dW=dW, dbias=db, accumulate=True)
        assert (dW == 7).all() and (db == 7).all()
        optcc.occ_linear_bwd(dY, X, W, dX=torch.empty_like(X), dW=dW, dbias=db)
        assert (dW == 0).all() and (db == 0).all()


def test_repeats_are_bitwise_equal():
    g = gen(9)
    for t, k, n in ((12, 700, 80), (200, 4096, 136), (2100, 520, 2056)):
        X, W = rand(g, t, k, torch.bfloat16), rand(g, n, k, torch.bfloat16, 0.05)
        Z = rand(g, t, n, torch.bfloat16)
        dY = rand(g, t, n, torch.bfloat16)
        one = None
        for _ in range(3):
            y = optcc.occ_linear_fwd(X, W, act=2)
            dX, dW, db = torch.empty_like(X), torch.empty_like(W), torch.empty(n, device="cuda")
            optcc.occ_linear_bwd(dY, X, W, Z=Z, act=2, dX=dX, dW=dW, dbias=db)
            now = [y, dX, dW, db]
            one = one or now
            assert all(torch.equal(a, c) for a, c in zip(one, now))


def test_offsets_beyond_32_bits():
    """X, W-side gradients and Y whose last rows lie more than 2^32 bytes in."""
    g = gen(11)
    tokens, wide, narrow = 70016, 32768, 64
    big = torch.empty(tokens, wide, dtype=torch.bfloat16, device="cuda")   # 4.6e9 bytes
    W = rand(g, wide, narrow, torch.bfloat16, 0.1)
    X = rand(g, tokens, narrow, torch.bfloat16)
    optcc.occ_linear_fwd(X, W, act=4, Y=big)
    for rows in (slice(0, 40), slice(tokens - 40, tokens)):
        y, _, by, _ = forward64(X[rows], W, None, 4, None, False)
        within(big[rows], y, by, "Y")
    # big as the gradient: dX contracts over its columns, dW over its rows
    dX = torch.empty_like(X)
    optcc.occ_linear_bwd(big, W=W, dX=dX)
    rows = slice(tokens - 40, tokens)
    within(dX[rows], *backward64(big[rows], None, W, None, 0, False)["dX"], "dX")
    dW = torch.empty(narrow, wide, dtype=torch.bfloat16, device="cuda")
    optcc.occ_linear_bwd(X, X=big, dW=dW)
    cols = slice(wide - 32, wide)
    ref = backward64(X, big[:, cols], None, None, 0, False)["dW"]
    within(dW[:, cols], *ref, "dW")


def test_on_another_stream_and_in_a_graph():
    g = gen(12)
    X, W = rand(g, 200, 136, torch.bfloat16), rand(g, 72, 136, torch.bfloat16, 0.1)
    dY, Z = rand(g, 200, 72, torch.bfloat16), torch.empty(200, 72, dtype=torch.bfloat16, device="cuda")
    Y, dX, dW = torch.empty_like(Z), torch.empty_like(X), torch.empty_like(W)
    db = torch.empty(72, device="cuda")
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")

    def work():
        optcc.occ_linear_fwd(X, W, act=2, Y=Y, Z=Z, ws=ws)
        optcc.occ_linear_bwd(dY, X, W, Z=Z, act=2, dX=dX, dW=dW, dbias=db, ws=ws)

    work()
    torch.cuda.synchronize()
    want = [t.clone() for t in (Y, dX, dW, db)]
    side = torch.cuda.Stream()
    for t in (Y, dX, dW, db):
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (Y, dX, dW, db)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        work()
    for i in range(4):
        X.mul_(0.5 if i % 2 else 2.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (Y, dX, dW, db)]
        work()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (Y, dX, dW, db)))


# fp32 products of some size run on the bf16 matrix units, each operand as
# three bf16 planes; the bounds stay those of fp32
PLANES = [(2048, 1030, 3000), (1500, 2304, 2200), (3001, 2047, 1533)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("size", PLANES, ids=lambda s: "x".join(map(str, s)))
def test_fp32_planes(size, gated):
    t, k, n = size
    a = optcc.occ_linear_t(optcc.OCC_F32, 0, t, 2304, 2200, 4096, 2304, 4096, 2304, None, None, 0,
                           None, 0, 4096, 2200)
    assert optcc.lib().occ_linear_fwd_workspace_bytes(a) > 6 * t * 2304     # planes are made
    run_forward(t, k, n, "f32", 4 if gated else 2, gated)
    run_forward(t, k, n, "f32", 0, gated, bias=False, residual=False, pad=3, shift=1)
    run_backward(t, k, n, "f32", 4 if gated else 2, gated, accumulate=True)
    if not gated:
        run_backward(t, k, n, "f32", 0, gated, pad=5, shift=2)


def test_fp32_planes_of_the_largest_values():
    """Values that bf16 would round to infinity, beside ordinary ones; a NaN
    stays in its row."""
    g = gen(21)
    X, W = rand(g, 1500, 2304, torch.float32), rand(g, 2200, 2304, torch.float32, 1e-3)
    X[7, :40] = 3.4028e38
    X[9, 100] = float("nan")
    Y = optcc.occ_linear_fwd(X, W)
    keep = [i for i in range(1500) if i != 9]
    y, _, by, _ = forward64(X[keep], W, None, 0, None, False)
    within(Y[keep], y, by, "Y")
    assert torch.isnan(Y[9]).all()


# Small layers take their operands as they lie (no workspace); larger ones make
# dZ and aligned copies first.  Above 1024 tokens the bias gradient is summed in
# strips.  Both sides at odd widths, where pieces of 16 bytes end inside rows and
# gated ones hold columns of both projections.
FORMS = [(1024, 65, 131), (1025, 65, 131), (1024, 7, 1), (1025, 3, 2), (90, 1531, 37),
         (1300, 1021, 1535), (2500, 517, 1999)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("size", FORMS, ids=lambda s: "x".join(map(str, s)))
def test_forms_of_the_products(size, gated, dtype):
    run_backward(*size, dtype, act=3, gated=gated, seed=sum(size))
    run_backward(*size, dtype, act=1, gated=gated, pad=3, shift=1, accumulate=True)
    if not gated:
        run_backward(*size, dtype, act=0, gated=False, pad=1)
    run_forward(*size, dtype, act=4, gated=gated, pad=1, shift=3)


def test_workspaces_of_both_forms():
    def need(tokens, width):
        a = optcc.occ_linear_grad_t(optcc.OCC_BF16, optcc.OCC_BF16, 2, 0, tokens, width, width, 4096,
                                    width, 4096, width, 4096, width, 4096, width, 4096, width, 4096,
                                    width, None)
        return optcc.lib().occ_linear_bwd_workspace_bytes(a)
    assert need(64, 64) == 0 and need(2500, 2048) >= 2500 * 2048 * 2


@pytest.mark.parametrize("tokens", [40, 1500])
def test_infinities_behind_an_edge_do_not_count(tokens):
    """What lies between the rows of every operand is NaN (rand), and a zero
    gradient times a finite act' is zero: no NaN reaches a result."""
    for gated in (False, True):
        g = gen(9)
        wide = 2 * 37 if gated else 37
        dY = rand(g, tokens, 37, torch.bfloat16, 0.0, pad=5, shift=1)
        X, W = rand(g, tokens, 41, torch.bfloat16, pad=7), rand(g, wide, 41, torch.bfloat16, pad=3)
        Z = rand(g, tokens, wide, torch.bfloat16, 50.0, pad=9, shift=3)
        dX, dW = torch.full_like(X, 7.0), torch.full_like(W, 7.0)
        db = torch.full((wide,), 7.0, device="cuda")
        (optcc.occ_gated_bwd if gated else optcc.occ_linear_bwd)(dY, X, W, Z=Z, act=2, dX=dX, dW=dW, dbias=db)
        assert not dX.any() and not dW.any() and not db.any()
