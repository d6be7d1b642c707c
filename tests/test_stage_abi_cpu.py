"""The stage operators refuse bad arguments on the host, before any device
work: every call here returns an error code or is one with nothing to do."""

import ctypes
import os

import pytest

from paper_2301_09830_amd import build as buildmod
from paper_2301_09830_amd import optcc

BASE = 1 << 32
STEP = 1 << 28


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(buildmod.LIB):
        buildmod.build()
    return optcc.lib()


def layer(**change):
    a = optcc.occ_linear_t()
    a.dtype, a.act = optcc.OCC_BF16, optcc.OCC_ACT_GELU
    a.tokens, a.in_, a.out = 100, 64, 32
    for i, (p, ld, n) in enumerate((("X", "ldx", 64), ("W", "ldw", 64), ("R", "ldr", 32),
                                    ("Z", "ldz", 64), ("Y", "ldy", 32))):
        setattr(a, p, BASE + i * STEP)
        setattr(a, ld, n)
    a.bias = BASE + 6 * STEP
    for k, v in change.items():
        setattr(a, k, v)
    return a


def grad(**change):
    a = optcc.occ_linear_grad_t()
    a.dtype = a.dw_dtype = optcc.OCC_BF16
    a.act = optcc.OCC_ACT_GELU
    a.tokens, a.in_, a.out = 100, 64, 32
    for i, (p, ld, n) in enumerate((("dY", "lddy", 32), ("X", "ldx", 64), ("W", "ldw", 64),
                                    ("Z", "ldz", 64), ("dX", "lddx", 64), ("dW", "lddw", 64))):
        setattr(a, p, BASE + i * STEP)
        setattr(a, ld, n)
    a.dbias = BASE + 7 * STEP
    for k, v in change.items():
        setattr(a, k, v)
    return a


WS, WS_BYTES = BASE + 10 * STEP, 1 << 26

FORWARD = [
    (dict(dtype=2), 5), (dict(act=5), 11), (dict(act=-1), 11), (dict(tokens=-1), 2),
    (dict(tokens=1 << 30), 2), (dict(in_=0), 2), (dict(out=0), 2), (dict(in_=(1 << 24) + 1), 2),
    (dict(ldx=63), 2), (dict(ldw=63), 2), (dict(ldy=31), 2), (dict(ldr=31), 2), (dict(ldz=31), 2),
    (dict(ldx=1 << 31), 2), (dict(X=None), 1), (dict(W=None), 1), (dict(Y=None), 1),
    (dict(X=BASE + 1), 6), (dict(Y=BASE + 4 * STEP + 1), 6), (dict(bias=BASE + 6 * STEP + 2), 6),
    (dict(Y=BASE + 64), 7), (dict(Z=BASE + 4 * STEP), 7), (dict(R=BASE + 4 * STEP + 2), 7),
    (dict(R=BASE + 4 * STEP, ldr=40), 7),      # R = Y only with Y's leading dimension
    (dict(bias=BASE + 4 * STEP), 7),
]


@pytest.mark.parametrize("change,code", FORWARD, ids=str)
def test_forward_refusals(L, change, code):
    for fn in (L.occ_linear_fwd, L.occ_gated_fwd):
        assert fn(ctypes.byref(layer(**change)), WS, WS_BYTES, None) == code


def test_gated_leading_dimension_counts_both_projections(L):
    assert L.occ_gated_fwd(ctypes.byref(layer(ldz=63)), WS, WS_BYTES, None) == 2


BACKWARD = [
    (dict(dtype=3), 5), (dict(dtype=0, dw_dtype=1), 5), (dict(dw_dtype=9), 5), (dict(act=7), 11),
    (dict(tokens=-1), 2), (dict(in_=0), 2), (dict(out=(1 << 24) + 1), 2), (dict(lddy=31), 2),
    (dict(ldz=31), 2), (dict(lddx=63), 2), (dict(lddw=63), 2), (dict(ldx=10), 2),
    (dict(dY=None), 1), (dict(Z=None), 1), (dict(X=None), 1), (dict(W=None), 1),
    (dict(dX=None, dW=None, dbias=None), 1), (dict(dY=BASE + 1), 6),
    (dict(dbias=BASE + 7 * STEP + 1), 6), (dict(dX=BASE + 32), 7), (dict(dW=BASE + STEP), 7),
    (dict(dbias=BASE + 2 * STEP), 7), (dict(dX=BASE + 5 * STEP), 7),
]


@pytest.mark.parametrize("change,code", BACKWARD, ids=str)
def test_backward_refusals(L, change, code):
    for fn in (L.occ_linear_bwd, L.occ_gated_bwd):
        assert fn(ctypes.byref(grad(**change)), 0, WS, WS_BYTES, None) == code


def test_workspaces(L):
    g = grad(tokens=50000)
    need = L.occ_linear_bwd_workspace_bytes(ctypes.byref(g))
    assert need > 0 and need % 256 == 0
    assert L.occ_gated_bwd_workspace_bytes(ctypes.byref(g)) > need
    for ws, n in ((None, need), (WS, need - 1), (WS + 8, need)):
        assert L.occ_linear_bwd(ctypes.byref(g), 0, ws, n, None) == 8
    assert L.occ_linear_bwd(ctypes.byref(g), 0, BASE, need, None) == 7   # the workspace is dY
    assert L.occ_linear_bwd(ctypes.byref(g), 2, WS, WS_BYTES, None) == 10
    assert L.occ_linear_bwd(None, 0, WS, WS_BYTES, None) == 1
    assert L.occ_linear_fwd(None, WS, WS_BYTES, None) == 1
    # invalid arguments have no workspace; few tokens need none
    assert L.occ_linear_bwd_workspace_bytes(ctypes.byref(grad(out=0))) == 0
    assert L.occ_linear_fwd_workspace_bytes(ctypes.byref(layer(tokens=4))) == 0
    # a small layer takes its operands as they lie
    assert L.occ_linear_fwd_workspace_bytes(ctypes.byref(layer(X=BASE + 2))) == 0
    assert L.occ_linear_bwd_workspace_bytes(ctypes.byref(grad())) == 0
    # in a large one, rows off 16 bytes are copied
    large = dict(tokens=8192, in_=2048, out=2048, ldx=2048, ldw=2048, ldr=2048, ldy=2048, ldz=2048)
    a, b = layer(**large), layer(**large, X=BASE + 2)
    assert L.occ_linear_fwd_workspace_bytes(ctypes.byref(b)) > \
        L.occ_linear_fwd_workspace_bytes(ctypes.byref(a))


def test_no_tokens_need_no_pointers(L):
    a = layer(tokens=0, X=None, Y=None)
    assert L.occ_linear_fwd(ctypes.byref(a), None, 0, None) == 0
    g = grad(tokens=0, dY=None, Z=None, X=None)
    assert L.occ_linear_bwd(ctypes.byref(g), 1, None, 0, None) == 0


def param(**change):
    p = optcc.occ_param_t()
    p.rows, p.cols, p.ldg, p.rank = 16, 300, 300, 4
    for i, k in enumerate(("W", "W16", "G", "P", "Q", "m", "v", "m_scale", "v_scale")):
        setattr(p, k, BASE + i * STEP)
    p.state_bits = 8
    for k, v in change.items():
        setattr(p, k, v)
    return p


def hyper(**change):
    h = optcc.occ_adamw_t(1e-3, 0.9, 0.95, 1e-8, 1, 0, 0, None, None)
    for k, v in change.items():
        setattr(h, k, v)
    return h


PARAMS = [
    (dict(rows=0), 2), (dict(cols=0), 2), (dict(cols=1 << 30), 2), (dict(ldg=299), 2),
    (dict(state_bits=16), 11), (dict(decay=float("nan")), 11), (dict(W=None), 1), (dict(m=None), 1),
    (dict(v=None), 1), (dict(m_scale=None), 1), (dict(G=None, P=None), 1), (dict(G=None, Q=None), 1),
    (dict(G=None, rank=0), 3), (dict(G=None, rank=129), 3), (dict(g_dtype=2), 5),
    (dict(W=BASE + 2), 6), (dict(G=BASE + 2 * STEP + 2), 6), (dict(state_bits=32, m=BASE + 5 * STEP + 1), 6),
    (dict(v_scale=BASE + 8 * STEP + 2), 6), (dict(m=BASE + 64), 7), (dict(G=BASE), 7),
    (dict(v=BASE + 5 * STEP), 7), (dict(v_scale=BASE + 7 * STEP), 7), (dict(W16=BASE + STEP * 2), 7),
]


@pytest.mark.parametrize("change,code", PARAMS, ids=str)
def test_adamw_tensor_refusals(L, change, code):
    p = (optcc.occ_param_t * 1)(param(**change))
    assert L.occ_adamw_step(p, 1, ctypes.byref(hyper()), None) == code


HYPER = [(dict(lr=float("inf")), 11), (dict(beta1=1.0), 11), (dict(beta1=-0.1), 11),
         (dict(beta2=1.0), 11), (dict(beta2=float("nan")), 11), (dict(eps=-1e-8), 11),
         (dict(step=0), 11), (dict(grad_scale=BASE + 1), 6), (dict(flags=BASE + 2), 6),
         (dict(grad_scale=BASE), 7), (dict(flags=BASE + 5 * STEP), 7)]


@pytest.mark.parametrize("change,code", HYPER, ids=str)
def test_adamw_hyperparameter_refusals(L, change, code):
    p = (optcc.occ_param_t * 1)(param())
    assert L.occ_adamw_step(p, 1, ctypes.byref(hyper(**change)), None) == code


def test_adamw_lists(L):
    h = hyper()
    p = (optcc.occ_param_t * 2)(param(), param())       # the same tensor twice
    assert L.occ_adamw_step(p, 2, ctypes.byref(h), None) == 7
    assert L.occ_adamw_step(p, 0, ctypes.byref(h), None) == 2
    assert L.occ_adamw_step(None, 1, ctypes.byref(h), None) == 1
    assert L.occ_adamw_step(p, 1, None, None) == 1


def test_value_status_has_a_text():
    assert "range" in optcc.occ_status_str(11)


def test_binding_refusals():
    torch = pytest.importorskip("torch")
    X, W = torch.zeros(4, 8), torch.zeros(6, 8)
    with pytest.raises(TypeError):
        optcc.occ_linear_fwd(X.double(), W)
    with pytest.raises(TypeError):
        optcc.occ_linear_fwd(X, W.bfloat16())
    with pytest.raises(ValueError):
        optcc.occ_linear_fwd(X, torch.zeros(6, 9))
    with pytest.raises(ValueError):
        optcc.occ_linear_fwd(X, W, R=torch.zeros(4, 5))
    with pytest.raises(ValueError):
        optcc.occ_linear_fwd(X, torch.zeros(8, 6).t())          # columns apart
    with pytest.raises(ValueError):
        optcc.occ_linear_fwd(X, W, bias=torch.zeros(5))
    with pytest.raises(TypeError):
        optcc.occ_linear_fwd(X, W, bias=torch.zeros(6, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        optcc.occ_gated_fwd(X, torch.zeros(7, 8))                # not two projections
    w = torch.zeros(4, 300)
    with pytest.raises(ValueError):
        optcc.make_param(w, w.clone(), w.clone())                # no gradient
    with pytest.raises(ValueError):
        optcc.make_param(w, w.clone(), w.clone(), G=w, P=w, Q=w)
    with pytest.raises(ValueError):
        optcc.make_param(w, torch.zeros(4, 300, dtype=torch.uint8),
                         torch.zeros(4, 300, dtype=torch.uint8), G=w)
    with pytest.raises(TypeError):
        optcc.make_param(w, torch.zeros(4, 300, dtype=torch.uint8), w.clone(), G=w,
                         m_scale=torch.zeros(4, 2), v_scale=torch.zeros(4, 2))
    with pytest.raises(ValueError):
        optcc.make_param(w, torch.zeros(4, 301), w.clone(), G=w)
    with pytest.raises(TypeError):
        optcc.make_param(w.bfloat16(), w.clone(), w.clone(), G=w)


def test_layers_need_tensors_on_a_gpu():
    torch = pytest.importorskip("torch")
    X, W, dY = torch.zeros(4, 8), torch.zeros(6, 8), torch.zeros(4, 6)
    with pytest.raises(ValueError):
        optcc.occ_linear_fwd(X, W)
    with pytest.raises(ValueError):
        optcc.occ_linear_bwd(dY, X, W, dX=torch.zeros(4, 8), dW=torch.zeros(6, 8))
    with pytest.raises(TypeError):
        optcc.occ_linear_fwd(X, W, R=1.0)
    with pytest.raises(ValueError):
        optcc.occ_linear_bwd(dY, X, W[0], dX=torch.zeros(4, 8))
    with pytest.raises(TypeError):
        optcc.occ_linear_bwd(dY.half(), X, W, dW=torch.zeros(6, 8))
