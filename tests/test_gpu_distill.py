"""The distillation loss and its gradient against float64, element by element,
inside derived bounds (tests/experts_ref.py)."""

import math

import pytest

torch = pytest.importorskip("torch")

from experts_ref import distill64  # noqa: E402
from paper_2301_09830_amd import optcc  # noqa: E402
from stage_ref import within  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def logits(g, t, v, dtype, scale=2.0, pad=0, shift=0):
    ld = v + pad
    buf = torch.full((shift + t * ld + 8,), float("nan"), dtype=dtype, device="cuda")
    view = buf[shift:shift + t * ld].view(t, ld)[:, :v]
    view.copy_(torch.randn(t, v, generator=g, device="cuda") * scale)
    return view


def inputs(t, v, k, dtype, seed=0, pad=0, shift=0):
    """(S, index, teacher, labels, scale): distinct columns, some labels missing, one
    token without a part."""
    g = gen(seed)
    S = logits(g, t, v, DT[dtype], 2.0, pad, shift)
    index = torch.rand(t, v, generator=g, device="cuda").argsort(1)[:, :k].to(torch.int32)
    teacher = torch.gather(S.float(), 1, index.long())
    teacher = (teacher + torch.randn(t, k, generator=g, device="cuda")).to(DT[dtype])
    labels = torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32)
    labels[::5] = -1
    scale = torch.rand(t, generator=g, device="cuda") / t
    if t > 2:
        scale[2] = 0.0
    return S, index.contiguous(), teacher.contiguous(), labels, scale


def check(S, index, teacher, T=1.0, alpha=1.0, labels=None, scale=None):
    t, v = S.shape
    print(f"distill {t}x{v} {S.dtype} k {None if index is None else index.shape[1]} T {T} "
          f"alpha {alpha} ld {S.stride(0)}", flush=True)
    how = dict(temperature=T, alpha=alpha, labels=labels, scale=scale)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    lse, dS = torch.full((t, 2), 7.0, device="cuda"), torch.full_like(S, 7.0)
    loss = optcc.occ_distill_fwd(S, index, teacher, **how, lse=lse, dS=dS, flags=flags)
    torch.cuda.synchronize()
    assert flags.item() == 0
    want = distill64(S, index, teacher, T, alpha, labels, scale)
    within(loss, *want["loss"], "loss")
    within(lse, *want["lse"], "lse")
    within(dS, *want["dS"], "dS")
    again = optcc.occ_distill_bwd(S, index, teacher, lse, **how)
    within(again, *want["dS_lse"], "dS from lse")
    # without a gradient, and in place
    assert torch.equal(optcc.occ_distill_fwd(S, index, teacher, **how), loss)
    for f in (lambda s: optcc.occ_distill_fwd(s, index, teacher, **how, dS=s),
              lambda s: optcc.occ_distill_bwd(s, index, teacher, lse, **how, dS=s)):
        s = S.clone()
        f(s)
        assert torch.equal(s, dS) or torch.equal(s, again)
    return loss, lse, dS


# rows that 2, 4, 8, 16 and 26 pieces of 4, 8 or 16 waves hold, and longer ones
SIZES = [(1, 1, 1), (1, 5, 3), (3, 64, 64), (5, 1000, 7), (40, 4096, 16), (600, 513, 9),
         (520, 5000, 33), (513, 9001, 64), (515, 17000, 5), (513, 40000, 20), (4, 51200, 16),
         (3, 100003, 100), (2, 250000, 11), (512, 60000, 3), (7, 2049, 1024), (9, 16385, 2)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_sizes(size, dtype):
    S, index, teacher, labels, scale = inputs(*size, dtype, seed=sum(size))
    check(S, index, teacher, T=2.0, alpha=0.5, labels=labels, scale=scale)
    check(S, index, teacher)


@pytest.mark.parametrize("T,alpha", [(1.0, 0.25), (0.5, 1.0), (4.0, 0.0), (1.0, 0.0), (3.0, 0.9)])
def test_temperatures_and_weights(T, alpha):
    for dtype in DT:
        S, index, teacher, labels, scale = inputs(30, 3000, 12, dtype, 3)
        check(S, index, teacher, T, alpha, labels, scale)
        check(S, index, teacher, T, alpha, labels)
        check(S, index, teacher, T, alpha, None, scale)


def test_labels_alone():
    """Without a teacher the loss is the cross entropy."""
    for dtype in DT:
        S, _, _, labels, scale = inputs(50, 777, 1, dtype, 4)
        loss, _, _ = check(S, None, None, 1.0, 0.0, labels, scale)
        want = torch.nn.functional.cross_entropy(S.double(), labels.long(), reduction="none",
                                                 ignore_index=-1) * scale.double()
        assert torch.allclose(loss.double(), want, rtol=1e-5, atol=1e-7)


@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (8, 0), (3, 5)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides(pad, shift, dtype):
    S, index, teacher, labels, scale = inputs(20, 1003, 6, dtype, 5, pad, shift)
    wide = torch.full((20, 9), 3, dtype=torch.int32, device="cuda")
    wide[:, :6] = index
    other = torch.zeros(20, 8, dtype=teacher.dtype, device="cuda")
    other[:, :6] = teacher
    a = check(S, wide[:, :6], other[:, :6], 2.0, 0.5, labels, scale)
    b = check(S.contiguous(), index, teacher, 2.0, 0.5, labels, scale)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    dS = logits(gen(1), 20, 1003, DT[dtype], 0.0, pad, shift)
    optcc.occ_distill_fwd(S, index, teacher, dS=dS)
    if pad:       # what lies between the rows is left alone
        gap = dS.as_strided((19, pad), (dS.stride(0), 1), dS.storage_offset() + 1003)
        assert torch.isnan(gap).all()


@pytest.mark.parametrize("v", [300, 230000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masks(dtype, v):
    """Masked entries, whatever stands there; tokens without entries, label or
    either; masked columns of the vocabulary."""
    S, index, teacher, labels, _ = inputs(12, v, 8, dtype, 6)
    S[:, v - 50:] = -math.inf             # columns that no token can be
    S[4, :40] = torch.finfo(S.dtype).min
    index = index % (v - 50)
    labels = torch.where(labels >= 0, labels % (v - 50), labels)
    index[1, 3:] = -1
    teacher[1, 3:] = float("nan")
    index[2] = -5
    teacher[2] = float("nan")
    teacher[3, 1:] = -math.inf
    teacher[6] = -math.inf
    labels[2], labels[6], labels[7] = -1, 5, -1
    scale = torch.ones(12, device="cuda")
    scale[8] = 0.0
    S[8], teacher[8] = float("nan"), float("nan")
    loss, lse, dS = check(S, index, teacher, 2.0, 0.5, labels, scale)
    assert loss[2] == 0 and not dS[2].any() and loss[8] == 0 and not dS[8].any()
    assert not lse[2].any() and not lse[8].any() and not dS[:, v - 50:].any()
    assert lse[6, 0] == 0 and lse[6, 1] != 0 and lse[7, 1] == 0 and lse[7, 0] != 0
    check(S, index, teacher, 1.0, 1.0, None, scale)


def test_rows_of_the_lowest_value():
    """Every logit at the type's lowest value: the softmax is even."""
    for dtype in DT.values():
        for v in (64, 230000):
            S = torch.full((3, v), torch.finfo(dtype).min, dtype=dtype, device="cuda")
            index = torch.tensor([[1, 5]] * 3, dtype=torch.int32, device="cuda")
            dS = torch.empty_like(S)
            loss = optcc.occ_distill_fwd(S, index, torch.zeros(3, 2, device="cuda"), dS=dS)
            # sum p log p + log v, in a few roundings of log v
            want = math.log(v) - math.log(2)
            assert torch.allclose(loss, torch.full_like(loss, want), rtol=1e-6, atol=0)
            assert torch.allclose(dS[:, 0].double(), torch.tensor(1 / v, dtype=torch.float64),
                                  rtol=2.0 ** -8, atol=0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_columns_listed_twice(dtype):
    """Equal columns add up, the label among them."""
    S, index, teacher, labels, scale = inputs(20, 200, 10, dtype, 7)
    index[:, 4] = index[:, 1]
    index[:, 9] = index[:, 1]
    index[3] = 17
    labels[:] = index[:, 1]
    check(S, index, teacher, 2.0, 0.5, labels, scale)
    check(S, index, teacher, 1.0, 1.0)


def test_mixed_types():
    S, index, teacher, labels, scale = inputs(9, 500, 10, "bf16", 8)
    check(S, index, teacher.float(), 2.0, 0.5, labels, scale)
    check(S.float(), index, teacher, 2.0, 0.5, labels, scale)


@pytest.mark.parametrize("v", [100, 230000])
def test_out_of_the_vocabulary(v):
    """Counts as masked, raises the flag, and touches nothing."""
    S, index, teacher, labels, scale = inputs(6, v, 5, "f32", 9)
    for change in ("index", "label"):
        i, lab = index.clone(), labels.clone()
        if change == "index":
            i[1, 2] = v
            i[3, 0] = (1 << 31) - 1
        else:
            lab[4] = v
        flags = torch.zeros(1, dtype=torch.int32, device="cuda")
        how = dict(temperature=2.0, alpha=0.5, scale=scale)
        dS, lse = torch.empty_like(S), torch.empty(6, 2, device="cuda")
        loss = optcc.occ_distill_fwd(S, i, teacher, labels=lab, dS=dS, lse=lse, flags=flags, **how)
        assert flags.item() == optcc.OCC_F_BAD_ROWS
        i, lab = torch.where(i >= v, -1, i), torch.where(lab >= v, -1, lab)
        want = torch.empty_like(S)
        assert torch.equal(optcc.occ_distill_fwd(S, i, teacher, labels=lab, dS=want, **how), loss)
        assert torch.equal(dS, want)


def test_nan_and_infinity_stay_in_their_token():
    for v in (500, 230000):
        S, index, teacher, _, _ = inputs(6, v, 5, "f32", 10)
        want = torch.empty_like(S)
        a = optcc.occ_distill_fwd(S, index, teacher, dS=want)
        B = S.clone()
        B[1, v - 1] = float("nan")
        B[3, 7] = math.inf
        t = teacher.clone()
        t[4, 0] = float("nan")
        got = torch.empty_like(S)
        b = optcc.occ_distill_fwd(B, index, t, dS=got)
        assert torch.equal(a[[0, 2, 5]], b[[0, 2, 5]])
        assert torch.equal(got[[0, 2, 5]], want[[0, 2, 5]])
        assert torch.isnan(b[[1, 3, 4]]).all() and torch.isnan(got[1]).all()
        # an entry that the student cannot be: the loss is infinite
        C = S.clone()
        C[0, index[0, 0].long()] = -math.inf
        assert optcc.occ_distill_fwd(C, index, teacher)[0] == math.inf


def test_gradient_by_differences():
    S, index, teacher, labels, scale = inputs(5, 12, 4, "f32", 11)
    for T, alpha in ((2.0, 0.5), (1.0, 1.0), (0.5, 0.3)):
        dS = torch.empty_like(S)
        optcc.occ_distill_fwd(S, index, teacher, T, alpha, labels, scale, dS=dS)
        h = 1e-5
        for j in range(12):
            ends = []
            for sign in (1, -1):
                x = S.double()
                x[:, j] += sign * h
                ends.append(distill64(x, index, teacher, T, alpha, labels, scale)["loss"][0])
            num = (ends[0] - ends[1]) / (2 * h)
            # h^2 / 6 times a third derivative (below 1 / T), and rounding
            assert torch.allclose(dS[:, j].double(), num, rtol=0, atol=1e-7)


def test_no_tokens_and_repeats():
    S, index, teacher, labels, scale = inputs(40, 3000, 9, "bf16", 12)
    assert optcc.occ_distill_fwd(S[:0], index[:0], teacher[:0]).shape == (0,)
    lse = torch.empty(0, 2, device="cuda")
    assert optcc.occ_distill_bwd(S[:0], index[:0], teacher[:0], lse).shape == (0, 3000)
    first = None
    for _ in range(3):
        dS = torch.empty_like(S)
        out = (optcc.occ_distill_fwd(S, index, teacher, 2.0, 0.5, labels, scale, dS=dS), dS)
        first = first or out
        assert all(torch.equal(a, b) for a, b in zip(out, first))


def test_captured_with_its_backward():
    """Forward and backward in a graph, replayed on new logits between eager calls."""
    S, index, teacher, labels, scale = inputs(30, 2000, 9, "bf16", 13)
    how = dict(temperature=2.0, alpha=0.5, labels=labels, scale=scale)
    loss, lse = torch.empty(30, device="cuda"), torch.empty(30, 2, device="cuda")
    dS = torch.empty_like(S)

    def call():
        optcc.occ_distill_fwd(S, index, teacher, **how, loss=loss, lse=lse)
        optcc.occ_distill_bwd(S, index, teacher, lse, **how, dS=dS)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        S.mul_(0.75)
        call()
        want = [x.clone() for x in (loss, lse, dS)]
        for x in (loss, lse, dS):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((loss, lse, dS), want))
