"""The router, the exchange of rows, the experts' layers and the distillation loss
refuse bad arguments on the host, before any device work: every call here returns
an error code or is one with nothing to do."""

import ctypes
import os
import re

import pytest

from paper_2301_09830_amd import build as buildmod
from paper_2301_09830_amd import optcc

BASE, STEP = 1 << 32, 1 << 28
WS, WS_BYTES = BASE + 20 * STEP, 1 << 26
NULL, SHAPE, DTYPE, ALIGN, ALIAS, WORKSPACE, FLAGS, VALUE = 1, 2, 5, 6, 7, 8, 10, 11


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(buildmod.LIB):
        buildmod.build()
    return optcc.lib()


def at(i):
    return BASE + i * STEP


def changed(a, change):
    for k, v in change.items():
        setattr(a, k, v)
    return ctypes.byref(a)


def test_limits_are_the_headers():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    header = open(os.path.join(root, "include", "optcc.h")).read()
    for name in ("OCC_MAX_EXPERTS", "OCC_MAX_CHOICES", "OCC_MAX_TEACHER"):
        assert int(re.search(rf"#define {name} (\d+)", header).group(1)) == getattr(optcc, name)


# --- router ---------------------------------------------------------------------
def route(**change):
    r = optcc.occ_route_t()
    r.dtype, r.k, r.renorm, r.tokens, r.experts, r.ldl = optcc.OCC_BF16, 4, 1, 100, 32, 32
    for i, name in enumerate(("logits", "index", "weights", "offsets", "order", "slots")):
        setattr(r, name, at(i))
    return changed(r, change)


ROUTE = [
    (dict(dtype=2), DTYPE), (dict(renorm=2), VALUE), (dict(k=0), SHAPE), (dict(k=33), SHAPE),
    (dict(k=33, experts=64, ldl=64), SHAPE), (dict(experts=3, ldl=3), SHAPE),
    (dict(experts=0), SHAPE), (dict(experts=1025, ldl=1025), SHAPE), (dict(tokens=-1), SHAPE),
    (dict(tokens=1 << 28), SHAPE), (dict(ldl=31), SHAPE), (dict(logits=None), NULL),
    (dict(index=None), NULL), (dict(weights=None), NULL), (dict(offsets=None), NULL),
    (dict(order=None), NULL), (dict(slots=None), NULL), (dict(logits=at(0) + 1), ALIGN),
    (dict(order=at(4) + 2), ALIGN), (dict(index=at(0)), ALIAS), (dict(slots=at(1) + 64), ALIAS),
    (dict(weights=at(3) + 4), ALIAS),
]


@pytest.mark.parametrize("change,code", ROUTE, ids=str)
def test_route_refusals(L, change, code):
    assert L.occ_route_fwd(route(**change), WS, WS_BYTES, None) == code


def test_route_workspace(L):
    assert L.occ_route_fwd_workspace_bytes(route()) == 0        # one launch
    many = dict(tokens=100000)
    need = L.occ_route_fwd_workspace_bytes(route(**many))
    assert need > 0
    for ws, n in ((None, need), (WS, need - 1), (WS + 8, need)):
        assert L.occ_route_fwd(route(**many), ws, n, None) == WORKSPACE
    assert L.occ_route_fwd(route(**many), at(0), need, None) == ALIAS
    assert L.occ_route_fwd_workspace_bytes(route(k=0)) == 0
    assert L.occ_route_fwd(None, WS, WS_BYTES, None) == NULL


ROUTE_BWD = [
    (dict(k=40), at(10), at(11), 32, SHAPE), ({}, at(10), at(11), 31, SHAPE),
    ({}, None, at(11), 32, NULL), ({}, at(10), None, 32, NULL), (dict(index=None), at(10), at(11), 32, NULL),
    (dict(renorm=0, logits=None), at(10), at(11), 32, NULL), ({}, at(10) + 2, at(11), 32, ALIGN),
    ({}, at(10), at(11) + 1, 32, ALIGN), ({}, at(10), at(10), 32, ALIAS),
    ({}, at(10), at(2) + 16, 32, ALIAS), (dict(renorm=0), at(10), at(0), 40, ALIAS),
]


@pytest.mark.parametrize("change,dw,dl,ldd,code", ROUTE_BWD, ids=str)
def test_route_bwd_refusals(L, change, dw, dl, ldd, code):
    assert L.occ_route_bwd(route(**change), dw, dl, ldd, None) == code


def test_no_tokens_to_route(L):
    assert L.occ_route_bwd(route(tokens=0, index=None), None, None, 32, None) == 0


# --- exchange ---------------------------------------------------------------------
def exchange(**change):
    x = optcc.occ_exchange_t()
    x.dtype, x.k, x.tokens, x.experts, x.rows, x.width = optcc.OCC_BF16, 4, 100, 32, 400, 64
    x.offsets, x.order, x.slots, x.flags = at(0), at(1), at(2), at(3)
    return changed(x, change)


EXCHANGE = [(dict(dtype=7), DTYPE), (dict(k=0), SHAPE), (dict(k=33), SHAPE), (dict(experts=0), SHAPE),
            (dict(experts=1025), SHAPE), (dict(tokens=-1), SHAPE), (dict(rows=-1), SHAPE),
            (dict(rows=1 << 30), SHAPE), (dict(width=0), SHAPE), (dict(width=(1 << 24) + 1), SHAPE),
            (dict(tokens=1 << 29), SHAPE), (dict(flags=at(3) + 1), ALIGN)]


@pytest.mark.parametrize("change,code", EXCHANGE, ids=str)
def test_exchange_refusals(L, change, code):
    assert L.occ_dispatch(exchange(**change), at(5), 64, at(6), 64, None) == code
    assert L.occ_combine(exchange(**change), at(4), at(5), 64, at(6), 64, at(7), 64, None) == code
    assert L.occ_combine_bwd(exchange(**change), at(4), at(5), 64, at(6), 64, at(7), 64, at(8),
                             None) == code


def test_dispatch_refusals(L):
    def call(X=at(5), ldx=64, Xs=at(6), ldxs=64, **change):
        return L.occ_dispatch(exchange(**change), X, ldx, Xs, ldxs, None)

    assert call(ldx=63) == call(ldxs=63) == SHAPE
    assert call(X=None) == call(Xs=None) == call(offsets=None) == call(order=None) == NULL
    assert call(X=at(5) + 1) == call(Xs=at(6) + 1) == call(order=at(1) + 2) == ALIGN
    assert call(Xs=at(5) + 128) == call(Xs=at(1)) == call(flags=at(6)) == ALIAS
    assert call(rows=0, X=None, Xs=None) == 0


def test_combine_refusals(L):
    def call(w=at(4), Ys=at(5), ldys=64, R=at(6), ldr=64, Y=at(7), ldy=64, **change):
        return L.occ_combine(exchange(**change), w, Ys, ldys, R, ldr, Y, ldy, None)

    assert call(ldys=63) == call(ldr=63) == call(ldy=63) == SHAPE
    assert call(Ys=None) == call(Y=None) == call(slots=None) == NULL
    assert call(w=at(4) + 2) == call(R=at(6) + 1) == call(Y=at(7) + 1) == ALIGN
    assert call(Y=at(5)) == call(Y=at(4)) == call(Y=at(2)) == call(R=at(7), ldr=65) == ALIAS
    assert call(R=at(7) + 2) == ALIAS          # R = Y from the same place only
    assert call(tokens=0, Y=None, Ys=None) == 0


def test_combine_bwd_refusals(L):
    def call(w=at(4), dY=at(5), lddy=64, Ys=at(6), ldys=64, dYs=at(7), lddys=64, dw=at(8), **change):
        return L.occ_combine_bwd(exchange(**change), w, dY, lddy, Ys, ldys, dYs, lddys, dw, None)

    assert call(lddy=63) == call(ldys=63) == call(lddys=63) == SHAPE
    assert call(dYs=None, dw=None) == call(dY=None) == call(Ys=None) == NULL
    assert call(order=None) == call(slots=None) == NULL
    assert call(dw=at(8) + 2) == call(dYs=at(7) + 1) == ALIGN
    assert call(dYs=at(6)) == call(dYs=at(5) + 64) == call(dw=at(4)) == call(dw=at(1)) == ALIAS
    assert call(tokens=0, dY=None) == 0


# --- layers ---------------------------------------------------------------------
def experts(**change):
    p = optcc.occ_experts_t()
    a = p.l
    a.dtype, a.act, a.tokens, a.in_, a.out = optcc.OCC_BF16, optcc.OCC_ACT_GELU, 100, 64, 32
    for i, (name, ld, n) in enumerate((("X", "ldx", 64), ("W", "ldw", 64), ("R", "ldr", 32),
                                       ("Z", "ldz", 64), ("Y", "ldy", 32))):
        setattr(a, name, at(i))
        setattr(a, ld, n)
    a.bias = at(6)
    p.experts, p.stride_w, p.offsets, p.flags = 8, 64 * 64, at(7), at(8)
    for k in list(change):
        if hasattr(a, k):
            setattr(a, k, change.pop(k))
    return changed(p, change)


FORWARD = [
    (dict(dtype=2), DTYPE), (dict(act=5), VALUE), (dict(tokens=-1), SHAPE), (dict(in_=0), SHAPE),
    (dict(out=0), SHAPE), (dict(ldx=63), SHAPE), (dict(ldw=63), SHAPE), (dict(ldy=31), SHAPE),
    (dict(ldr=31), SHAPE), (dict(ldz=31), SHAPE), (dict(experts=0), SHAPE),
    (dict(experts=1025), SHAPE), (dict(stride_w=31 * 64), SHAPE), (dict(stride_w=-1), SHAPE),
    (dict(stride_w=1 << 44), SHAPE), (dict(X=None), NULL), (dict(W=None), NULL), (dict(Y=None), NULL),
    (dict(offsets=None), NULL), (dict(X=BASE + 1), ALIGN), (dict(offsets=at(7) + 2), ALIGN),
    (dict(flags=at(8) + 1), ALIGN), (dict(bias=at(6) + 2), ALIGN), (dict(Y=BASE + 64), ALIAS),
    (dict(Z=at(4)), ALIAS), (dict(R=at(4) + 2), ALIAS), (dict(R=at(4), ldr=40), ALIAS),
    (dict(Y=at(7)), ALIAS), (dict(Y=at(1) + 7 * 64 * 64 * 2), ALIAS),      # the last expert's weights
    (dict(flags=at(4)), ALIAS), (dict(bias=at(4)), ALIAS),
]


@pytest.mark.parametrize("change,code", FORWARD, ids=str)
def test_forward_refusals(L, change, code):
    for fn in (L.occ_experts_linear_fwd, L.occ_experts_gated_fwd):
        assert fn(experts(**change), WS, WS_BYTES, None) == code


def grads(**change):
    p = optcc.occ_experts_grad_t()
    a = p.l
    a.dtype = a.dw_dtype = optcc.OCC_BF16
    a.act, a.tokens, a.in_, a.out = optcc.OCC_ACT_GELU, 100, 64, 32
    for i, (name, ld, n) in enumerate((("dY", "lddy", 32), ("X", "ldx", 64), ("W", "ldw", 64),
                                       ("Z", "ldz", 64), ("dX", "lddx", 64), ("dW", "lddw", 64))):
        setattr(a, name, at(i))
        setattr(a, ld, n)
    a.dbias = at(6)
    p.experts, p.stride_w, p.stride_dw, p.offsets, p.flags = 8, 64 * 64, 64 * 64, at(7), at(8)
    for k in list(change):
        if hasattr(a, k):
            setattr(a, k, change.pop(k))
    return changed(p, change)


BACKWARD = [
    (dict(dtype=3), DTYPE), (dict(dtype=0, dw_dtype=1), DTYPE), (dict(act=7), VALUE),
    (dict(tokens=-1), SHAPE), (dict(in_=0), SHAPE), (dict(lddy=31), SHAPE), (dict(ldz=31), SHAPE),
    (dict(lddx=63), SHAPE), (dict(lddw=63), SHAPE), (dict(experts=0), SHAPE),
    (dict(experts=1025), SHAPE), (dict(stride_w=64), SHAPE), (dict(stride_dw=64), SHAPE),
    (dict(dY=None), NULL), (dict(Z=None), NULL), (dict(X=None), NULL), (dict(W=None), NULL),
    (dict(offsets=None), NULL), (dict(dX=None, dW=None, dbias=None), NULL), (dict(dY=BASE + 1), ALIGN),
    (dict(dbias=at(6) + 1), ALIGN), (dict(offsets=at(7) + 1), ALIGN), (dict(dX=BASE + 32), ALIAS),
    (dict(dW=at(1)), ALIAS), (dict(dbias=at(2)), ALIAS), (dict(dX=at(5) + 7 * 64 * 64 * 2), ALIAS),
    (dict(dbias=at(7)), ALIAS),
]


@pytest.mark.parametrize("change,code", BACKWARD, ids=str)
def test_backward_refusals(L, change, code):
    for fn in (L.occ_experts_linear_bwd, L.occ_experts_gated_bwd):
        assert fn(grads(**change), 0, WS, WS_BYTES, None) == code


def test_layer_workspaces(L):
    big = dict(tokens=50000)
    need = L.occ_experts_linear_bwd_workspace_bytes(grads(**big))
    assert need > 0 and need % 256 == 0
    assert L.occ_experts_gated_bwd_workspace_bytes(grads(**big)) > need
    for ws, n in ((None, need), (WS, need - 1), (WS + 8, need)):
        assert L.occ_experts_linear_bwd(grads(**big), 0, ws, n, None) == WORKSPACE
    assert L.occ_experts_linear_bwd(grads(**big), 0, BASE, need, None) == ALIAS
    assert L.occ_experts_linear_bwd(grads(**big), 2, WS, WS_BYTES, None) == FLAGS
    assert L.occ_experts_linear_bwd(None, 0, WS, WS_BYTES, None) == NULL
    assert L.occ_experts_gated_fwd(None, WS, WS_BYTES, None) == NULL
    assert L.occ_experts_linear_fwd_workspace_bytes(experts()) == 0
    assert L.occ_experts_linear_fwd_workspace_bytes(experts(out=0)) == 0
    assert L.occ_experts_gated_bwd_workspace_bytes(grads(experts=0)) == 0


def test_layers_without_rows(L):
    assert L.occ_experts_linear_fwd(experts(tokens=0, X=None, Y=None), None, 0, None) == 0
    assert L.occ_experts_gated_bwd(grads(tokens=0, dY=None, Z=None, X=None), 1, None, 0, None) == 0


def test_launches_that_no_grid_holds(L):
    wide = dict(in_=1 << 22, out=1 << 22, ldx=1 << 22, ldw=1 << 22, ldy=1 << 22, ldr=1 << 22,
                ldz=1 << 23, experts=4, stride_w=1 << 41, tokens=1 << 29)
    for change in (wide, dict(wide, tokens=3)):     # tiles of the rows; weights of all experts
        assert L.occ_experts_gated_fwd(experts(**change, bias=None), WS, WS_BYTES, None) != 0


# --- distillation -----------------------------------------------------------------
def distill(**change):
    d = optcc.occ_distill_t()
    d.dtype, d.t_dtype, d.tokens, d.vocab, d.lds, d.k = optcc.OCC_BF16, optcc.OCC_F32, 10, 100, 100, 8
    d.ldi = d.ldt = 8
    d.ldds = 100
    d.temperature, d.alpha = 2.0, 0.5
    for i, name in enumerate(("S", "index", "teacher", "labels", "scale", "loss", "lse", "dS", "flags")):
        setattr(d, name, at(i))
    return changed(d, change)


DISTILL = [
    (dict(dtype=2), DTYPE), (dict(t_dtype=-1), DTYPE), (dict(temperature=0.0), VALUE),
    (dict(temperature=-1.0), VALUE), (dict(temperature=float("nan")), VALUE),
    (dict(temperature=float("inf")), VALUE), (dict(alpha=-0.1), VALUE), (dict(alpha=1.5), VALUE),
    (dict(alpha=float("nan")), VALUE), (dict(tokens=-1), SHAPE), (dict(tokens=1 << 30), SHAPE),
    (dict(vocab=0), SHAPE), (dict(vocab=(1 << 24) + 1, lds=1 << 25, ldds=1 << 25), SHAPE),
    (dict(k=-1), SHAPE), (dict(k=1025, ldi=2000, ldt=2000), SHAPE), (dict(lds=99), SHAPE),
    (dict(ldds=99), SHAPE), (dict(ldi=7), SHAPE), (dict(ldt=7), SHAPE), (dict(S=None), NULL),
    (dict(index=None), NULL), (dict(teacher=None), NULL), (dict(S=at(0) + 1), ALIGN),
    (dict(dS=at(7) + 1), ALIGN), (dict(teacher=at(2) + 2), ALIGN), (dict(labels=at(3) + 1), ALIGN),
    (dict(scale=at(4) + 2), ALIGN), (dict(lse=at(6) + 2), ALIGN), (dict(flags=at(8) + 2), ALIGN),
    (dict(dS=at(0) + 2), ALIAS), (dict(dS=at(0), ldds=101), ALIAS), (dict(dS=at(1)), ALIAS),
    (dict(dS=at(3)), ALIAS), (dict(flags=at(7)), ALIAS),
]


@pytest.mark.parametrize("change,code", DISTILL, ids=str)
def test_distill_refusals(L, change, code):
    assert L.occ_distill_fwd(distill(**change), None) == code
    assert L.occ_distill_bwd(distill(**change), None) == code


def test_distill_outputs(L):
    assert L.occ_distill_fwd(distill(loss=None), None) == NULL
    assert L.occ_distill_bwd(distill(dS=None), None) == NULL
    assert L.occ_distill_bwd(distill(lse=None), None) == NULL
    assert L.occ_distill_fwd(distill(loss=at(4)), None) == ALIAS
    assert L.occ_distill_fwd(distill(lse=at(5)), None) == ALIAS
    assert L.occ_distill_bwd(distill(dS=at(6)), None) == ALIAS
    assert L.occ_distill_fwd(distill(tokens=0, S=None, loss=None), None) == 0
    assert L.occ_distill_bwd(distill(tokens=0, S=None, dS=None), None) == 0
    assert L.occ_distill_fwd(None, None) == NULL
