"""The router and the exchange of rows against float64, whole numbers exactly,
values inside derived bounds (tests/experts_ref.py)."""

import math

import pytest

torch = pytest.importorskip("torch")

from experts_ref import combine64, combine_bwd64, plan64, route_bwd64, weights64  # noqa: E402
from paper_2301_09830_amd import optcc  # noqa: E402
from stage_ref import within  # noqa: E402

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


def check_route(logits, k, renorm, seed=0):
    t, e = logits.shape
    print(f"route {t}x{e} k {k} {logits.dtype} renorm {renorm} ld {logits.stride(0)}", flush=True)
    r = optcc.occ_route_fwd(logits, k, renorm=renorm)
    torch.cuda.synchronize()
    index, offsets, order, slots = plan64(logits, k)
    assert r.offsets.tolist() == offsets
    assert torch.equal(r.index.long(), index)
    assert r.order[:offsets[-1]].tolist() == order
    assert torch.equal(r.slots.cpu().long(), slots)
    w, b = weights64(logits, index, renorm)
    within(r.weights, w, b, "weights")
    dw = torch.randn(t, k, generator=gen(seed + 1), device="cuda")
    got = optcc.occ_route_bwd(dw, logits, r, renorm=renorm)
    within(got, *route_bwd64(logits, index, r.weights, dw, renorm), "dlogits")
    return r


SIZES = [(1, 1, 1), (1, 4, 2), (3, 5, 5), (8, 64, 2), (16, 16, 4), (33, 65, 8), (255, 128, 8),
         (256, 129, 3), (257, 128, 8), (300, 3, 3), (1000, 256, 16), (1025, 257, 6), (40, 1024, 32),
         (700, 1000, 17), (2000, 64, 1), (70000, 12, 2)]


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_route_sizes(size, dtype, renorm):
    t, e, k = size
    check_route(rand(gen(sum(size)), t, e, DT[dtype]), k, renorm, seed=sum(size))


@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 5), (8, 8)])
def test_route_strides(pad, shift):
    for dtype in DT.values():
        for t in (20, 600):
            check_route(rand(gen(pad), t, 61, dtype, 1.0, pad, shift), 4, False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ties_go_to_the_lowest_index(dtype):
    """Few distinct values, zeros of both signs among them."""
    for t, e, k in ((50, 40, 8), (500, 130, 8), (30, 600, 20)):
        x = torch.randint(-2, 3, (t, e), generator=gen(t), device="cuda").float()
        x = torch.where(torch.rand(t, e, generator=gen(e), device="cuda") < 0.5, -x * 0.0, x)
        check_route(x.to(DT[dtype]), k, True)
    check_route(torch.zeros(300, 64, dtype=DT[dtype], device="cuda"), 3, False)


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("tokens", [12, 400])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_experts(dtype, tokens, renorm):
    """-inf masks an expert; rows that leave fewer than k, one, or none."""
    x = rand(gen(5), tokens, 24, DT[dtype])
    x[:, 3] = -math.inf
    x[1, 2:] = -math.inf
    x[2, 1:] = -math.inf
    x[5] = -math.inf
    x[7] = torch.finfo(DT[dtype]).min      # equal, and not masked
    r = check_route(x, 4, renorm)
    assert r.index[5].tolist() == [-1] * 4 and r.slots[5].tolist() == [-1] * 4
    assert r.index[1].tolist()[2:] == [-1, -1] and not r.weights[1, 2:].any()
    assert r.index[7].tolist() == [0, 1, 2, 3]
    dw = torch.full((tokens, 4), float("nan"), device="cuda")
    dw[0] = 1.0
    d = optcc.occ_route_bwd(dw, x, r, renorm=renorm)
    assert not d[5].any() and torch.isfinite(d[0]).all()   # what stands at no choice is not read


@pytest.mark.parametrize("tokens", [9, 300])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nan_and_infinity_stay_in_their_token(dtype, tokens):
    x = rand(gen(6), tokens, 40, DT[dtype])
    want = optcc.occ_route_fwd(x, 3, renorm=False)
    y = x.clone()
    y[2, 7] = float("nan")
    y[4, 9] = math.inf
    r = optcc.occ_route_fwd(y, 3, renorm=False)
    rest = [t for t in range(tokens) if t not in (2, 4)]
    assert torch.equal(r.index[rest], want.index[rest])
    assert torch.equal(r.weights[rest], want.weights[rest])
    assert torch.isnan(r.weights[2]).all() and 7 not in r.index[2].tolist()
    assert r.index[4, 0] == 9 and torch.isnan(r.weights[4, 0])
    assert sorted(r.slots.view(-1).tolist()) == list(range(3 * tokens))


def test_order_behind_the_last_entry_is_left_alone():
    for t in (10, 500):
        x = torch.full((t, 8), -math.inf, device="cuda")
        x[:, 2] = 1.0
        r = optcc.Route(*(torch.full(s, -7, dtype=d, device="cuda") for s, d in (
            ((t, 2), torch.int32), ((t, 2), torch.float32), ((9,), torch.int32),
            ((2 * t,), torch.int32), ((t, 2), torch.int32))))
        got = optcc.occ_route_fwd(x, 2, route=r)
        assert all(a is b for a, b in zip(got, r))
        assert r.offsets.tolist() == [0, 0, 0] + [t] * 6
        assert r.order[:t].tolist() == list(range(0, 2 * t, 2)) and (r.order[t:] == -7).all()


def test_gradient_by_differences():
    """The gradient of sum(weights * dw) against central differences of the
    weights in float64."""
    for renorm in (True, False):
        x = torch.randn(6, 10, generator=gen(9), device="cuda")
        r = optcc.occ_route_fwd(x, 3, renorm=renorm)
        dw = torch.randn(6, 3, generator=gen(10), device="cuda")
        got = optcc.occ_route_bwd(dw, x, r, renorm=renorm)
        h = 1e-5

        def f(y):
            return (weights64(y, r.index.long(), renorm)[0] * dw.double()).sum(1)

        for e in range(10):
            step = torch.zeros(6, 10, dtype=torch.float64, device="cuda")
            step[:, e] = h
            num = (f(x.double() + step) - f(x.double() - step)) / (2 * h)
            # h^2 / 6 times a third derivative of a softmax (below 1), and rounding
            assert torch.allclose(got[:, e].double(), num, rtol=0, atol=1e-5)


def test_dlogits_in_place():
    for t in (5, 300):
        x = rand(gen(4), t, 50, torch.bfloat16)
        r = optcc.occ_route_fwd(x, 4, renorm=False)
        dw = torch.randn(t, 4, generator=gen(3), device="cuda")
        want = optcc.occ_route_bwd(dw, x, r, renorm=False)
        got = x.clone()
        optcc.occ_route_bwd(dw, got, r, renorm=False, dlogits=got)
        assert torch.equal(got, want)


def test_no_tokens():
    x = torch.empty(0, 7, device="cuda")
    r = optcc.occ_route_fwd(x, 2)
    assert r.offsets.tolist() == [0] * 8 and r.index.shape == (0, 2)
    assert optcc.occ_route_bwd(torch.empty(0, 2, device="cuda"), x, r).shape == (0, 7)
    X = torch.empty(0, 16, device="cuda")
    Xs = optcc.occ_dispatch(X, r)
    assert Xs.shape == (0, 16) and optcc.occ_combine(Xs, r).shape == (0, 16)
    dYs, dw = optcc.occ_combine_bwd(X, Xs, r)
    assert dYs.shape == (0, 16) and dw.shape == (0, 2)


# ---------------------------------------------------------------------------
# exchange
# ---------------------------------------------------------------------------
def check_exchange(t, h, e, k, dtype, weighted=True, residual=True, pad=0, shift=0, masked=False):
    print(f"exchange {t}x{h} e {e} k {k} {dtype} pad {pad} shift {shift}", flush=True)
    g, dt = gen(t + h), DT[dtype]
    logits = rand(g, t, e, torch.float32)
    if masked:
        logits[::3, 1:] = -math.inf
        logits[1] = -math.inf
    r = optcc.occ_route_fwd(logits, k)
    n = int(r.offsets[-1])
    X, Ys = rand(g, t, h, dt, 1.0, pad, shift), rand(g, t * k, h, dt, 1.0, pad, shift)
    w = r.weights if weighted else None
    if masked:     # what stands where no entry is
        Ys[n:] = float("nan")
        r.weights[r.index < 0] = float("nan")
    R = rand(g, t, h, dt, 1.0, pad, shift) if residual else None
    Xs = rand(g, t * k, h, dt, 0.0, pad, shift).fill_(5.0)
    optcc.occ_dispatch(X, r, Xs=Xs)
    token = r.order[:n].long() // k
    assert torch.equal(Xs[:n], X[token]) and (Xs[n:] == 5.0).all()
    Y = rand(g, t, h, dt, 0.0, pad, shift)
    optcc.occ_combine(Ys, r, weights=w, R=R, Y=Y)
    within(Y, *combine64(Ys, r.slots, w, R), "Y")
    dY = rand(g, t, h, dt, 1.0, pad, shift)
    dYs = rand(g, t * k, h, dt, 0.0, pad, shift).fill_(7.0)
    _, dw = optcc.occ_combine_bwd(dY, Ys, r, weights=w, dYs=dYs)
    torch.cuda.synchronize()
    v, b, vw, bw = combine_bwd64(dY, Ys, r.slots, w)
    live = r.slots >= 0
    within(dYs[r.slots[live].long()], v[live], b[live], "dYs")
    assert (dYs[n:] == 7.0).all()
    within(dw, vw, bw, "dweights")
    only, none = optcc.occ_combine_bwd(dY, None, r, weights=w)
    assert none is None and torch.equal(only[:n], dYs[:n])
    for m in (Xs, Y, dYs):      # what lies between the rows is left alone
        if pad and m.shape[0] > 1:
            gap = m.as_strided((m.shape[0] - 1, pad), (m.stride(0), 1),
                               m.storage_offset() + m.shape[1])
            assert torch.isnan(gap).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 1, 1, 1), (1, 4096, 8, 2), (7, 3, 5, 5), (64, 1000, 16, 3),
                                  (130, 513, 9, 6), (33, 4097, 4, 1), (1000, 64, 64, 8),
                                  (20, 2048, 40, 32)], ids=str)
def test_exchange_sizes(size, dtype):
    check_exchange(*size, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (8, 0), (3, 5)])
def test_exchange_strides(pad, shift, dtype):
    check_exchange(50, 300, 8, 2, dtype, pad=pad, shift=shift)


def test_exchange_without_weights_and_residual():
    check_exchange(40, 200, 6, 3, "bf16", weighted=False, residual=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_exchange_of_masked_choices(dtype):
    check_exchange(60, 136, 6, 3, dtype, masked=True)


def test_combine_onto_its_residual():
    g = gen(8)
    r = optcc.occ_route_fwd(rand(g, 70, 9, torch.float32), 2)
    Ys, R = rand(g, 140, 264, torch.bfloat16), rand(g, 70, 264, torch.bfloat16)
    want = optcc.occ_combine(Ys, r, weights=r.weights, R=R)
    got = R.clone()
    optcc.occ_combine(Ys, r, weights=r.weights, R=got, Y=got)
    assert torch.equal(got, want)


def test_plans_that_fit_nothing_raise_their_flag():
    """Entries and places out of range, or named twice: the rows concerned are
    left alone, the flag is raised."""
    g = gen(11)
    r = optcc.occ_route_fwd(rand(g, 6, 4, torch.float32), 2)
    X, Ys = rand(g, 6, 32, torch.float32), rand(g, 12, 32, torch.float32)

    def flags():
        return torch.zeros(1, dtype=torch.int32, device="cuda")

    f = flags()
    optcc.occ_dispatch(X, r, flags=f)
    optcc.occ_combine(Ys, r, flags=f)
    optcc.occ_combine_bwd(X, Ys, r, flags=f)
    assert f.item() == 0
    for bad in (-1, 12, 1 << 30):
        order, f = r.order.clone(), flags()
        order[3] = bad
        Xs = torch.full((12, 32), 5.0, device="cuda")
        optcc.occ_dispatch(X, r._replace(order=order), Xs=Xs, flags=f)
        assert f.item() == optcc.OCC_F_BAD_ROWS and (Xs[3] == 5.0).all()
        assert torch.equal(Xs[4:], X[r.order[4:].long() // 2])
    slots, f = r.slots.clone(), flags()
    slots[2, 1] = 12
    want, _ = combine64(Ys, torch.where(slots == 12, -1, slots), None, None)
    got = optcc.occ_combine(Ys, r._replace(slots=slots), flags=f)
    assert f.item() == optcc.OCC_F_BAD_ROWS and torch.allclose(got.double(), want, atol=1e-5)
    slots, f = r.slots.clone(), flags()
    slots[2, 1] = slots[3, 0]           # two entries with one place
    dYs, dw = optcc.occ_combine_bwd(X, Ys, r._replace(slots=slots), flags=f)
    assert f.item() == optcc.OCC_F_BAD_ROWS and dw[2, 1] == 0
    assert torch.equal(dYs[slots[3, 0]], X[3])
    offsets, f = r.offsets.clone(), flags()
    offsets[-1] = 100                   # more rows than there are
    assert torch.equal(optcc.occ_dispatch(X, r._replace(offsets=offsets)), X[r.order.long() // 2])


def test_results_repeat():
    g = gen(12)
    x, Ys = rand(g, 3000, 60, torch.bfloat16), rand(g, 12000, 72, torch.bfloat16)
    dY = rand(g, 3000, 72, torch.bfloat16)
    first = None
    for _ in range(3):
        r = optcc.occ_route_fwd(x, 4, renorm=False)
        out = [*r, optcc.occ_combine(Ys, r, weights=r.weights),
               *optcc.occ_combine_bwd(dY, Ys, r, weights=r.weights)]
        first = first or out
        assert all(torch.equal(a, b) for a, b in zip(out, first))
